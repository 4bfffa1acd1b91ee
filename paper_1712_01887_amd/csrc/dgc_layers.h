// Shared between the host side and the kernels of the layers of recurrent language models with matrix states: argument
// blocks and launchers.  Nothing here is visible through the C ABI.
#ifndef DGC_LAYERS_H_
#define DGC_LAYERS_H_

#include "dgc_operators.h"
#include "dgc_steps.h"

namespace dgc {

struct RotaryArgs {
  dgc_heads x[DGC_ROTARY_MAX], out[DGC_ROTARY_MAX];
  int32_t heads[DGC_ROTARY_MAX];
  int32_t count;
  int32_t rows, head_dim, rotary_dim;
  const int64_t* positions;
  const uint64_t* frequencies;
  float magnitude;
  bool half, inverse;
};

// The one operator that attention and its gradients are made of, for every sequence and head:
//   out_i = out_scale (sum over j <= i of d^(i-j) scale (a_i . b_j) c_j  +  d^(i+1-late) a_i . first)
//   last  = d^n first + sum over j of d^(n-1-j+late) scale b_j c_j^T
// where step i is row i of the sequence, or, reversed, its row n - 1 - i.
struct WalkArgs {
  dgc_heads a, b, c, out;  // out.data null: only `last` is wanted
  const float* log_decay;
  const float* first;  // may be null: element (i, j) of head h of sequence s at (s * heads + h) * da * dc + i * state_a + j * state_c
  float* last;         // the same; may be null
  int32_t state_a, state_c;
  int32_t heads, da, dc;  // elements of a and b, of c and out
  int64_t rows, sequences, max_length;
  const int64_t* row_offsets;  // may be null
  float scale, out_scale;
  float* states;  // workspace of the walk, where sequences are cut: as many states as they have segments
  int32_t late;  // 1: the state comes in and leaves with the decay of the step between done
  bool reverse;
};

struct VocabArgs {
  const void* hidden;
  const void* weight;
  int64_t hidden_stride, weight_stride;
  int32_t rows, vocab, width;
  const int32_t* labels;
  const float* row_weight;  // may be null
  float* loss;              // forward; may be null
  float* lse;               // forward: written, may be null; backward: read
  void* dhidden;            // may be null
  void* dweight;            // may be null
  int64_t dhidden_stride, dweight_stride;
  uint32_t* diag_flags;  // may be null
};

hipError_t launch_rotary(const RotaryArgs& a, int32_t dtype, hipStream_t stream);
constexpr int kWalksMax = 3;
// Up to kWalksMax walks of the same sequences, of which none needs what another one leaves; da and dc may be exchanged.
// Where sequences are cut, launch_walk_states forms the states in front of their segments (of b and c alone), which
// launch_walks reads, from `states`, as they lie with a walk's own state_a and state_c.
hipError_t launch_walk_states(const WalkArgs* w, int count, int32_t dtype, hipStream_t stream);
hipError_t launch_walks(const WalkArgs* w, int count, int32_t dtype, hipStream_t stream);
size_t walk_workspace_bytes(int64_t rows, int64_t sequences, int64_t max_length, int32_t heads, int32_t da, int32_t dc, bool ragged);
int64_t walk_workgroups(int64_t sequences, int32_t heads, int32_t dc);
hipError_t launch_vocab_forward(const VocabArgs& a, void* workspace, int32_t dtype, hipStream_t stream);
hipError_t launch_vocab_backward(const VocabArgs& a, void* workspace, int32_t dtype, hipStream_t stream);
size_t vocab_workspace_bytes(int32_t dtype, int32_t rows, int32_t vocab, int32_t width, bool backward);

}  // namespace dgc
#endif  // DGC_LAYERS_H_
