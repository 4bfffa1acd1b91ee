// Shared between the host side and the kernels of the operators on logits and sequences: argument
// blocks, element types and small device helpers.  Nothing here is visible through the C ABI.
#ifndef DGC_OPERATORS_H_
#define DGC_OPERATORS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dgc.h"
#include "dgc_internal.h"

namespace dgc {

// ---- argument blocks ---------------------------------------------------------
struct TopArgs {
  const void* logits;
  int64_t row_stride;
  int32_t rows, vocab, k;
  float inv_temperature;
  int32_t* out_idx;
  float* out_val;
  float* out_lse;  // may be null
};

struct DistillArgs {
  const void* logits;
  void* grad;  // may be null, may be logits
  int64_t row_stride, grad_stride;
  int32_t rows, vocab, k;
  const int32_t* top_idx;
  const float* top_val;
  const float* top_lse;     // may be null
  const int32_t* labels;    // null: no hard term
  const float* row_weight;  // may be null
  float temperature, hard_weight;
  float* loss;           // may be null
  uint32_t* diag_flags;  // may be null
};

struct ScanArgs {
  const void* gate;
  const void* x;
  int64_t gate_stride, x_stride;
  const float* first;  // forward: h0, backward: dh_last; may be null
  float* last;         // forward: h_last, backward: dh0; may be null
  float* states;       // forward: written, may be null; backward: read
  void* h;             // forward only
  int64_t h_stride;
  const void* dh;  // backward only, from here on
  void* dgate;
  void* dx;
  int64_t dh_stride, dgate_stride, dx_stride;
  const int64_t* row_offsets;  // may be null
  int64_t rows, max_length, channels;
  int64_t sequences;
};

hipError_t launch_top_logits(const TopArgs& a, int32_t dtype, hipStream_t stream);
hipError_t launch_distill(const DistillArgs& a, int32_t dtype, hipStream_t stream);
hipError_t launch_scan(const ScanArgs& a, void* workspace, int32_t dtype, bool free_input, bool backward, hipStream_t stream);
size_t scan_workspace_bytes(const ScanArgs& a);  // of the shape alone
int64_t scan_workgroups(const ScanArgs& a);      // tiles or workgroups, whichever a launch counts

// ---- element types ---------------------------------------------------------------
// An element as it lies in memory, and what it stands for.  To 16 bits: once, to the nearest, ties to even.
template <typename T>
__device__ __forceinline__ float to_float(T x) {
  return static_cast<float>(x);
}
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  return static_cast<T>(x);
}

// N elements that lie behind each other, aligned to the whole of them.
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T e[N];
};

}  // namespace dgc
#endif  // DGC_OPERATORS_H_
