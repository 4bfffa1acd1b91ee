// Host side of the layers of recurrent language models with matrix states: argument checks and launches.
// The layers themselves run in the kernels of dgc_rotary.hip, dgc_attention.hip and dgc_vocab.hip.

#include <cmath>

#include "dgc_layers.h"

using namespace dgc;

namespace {

constexpr int64_t kIntLimit = (int64_t)1 << 31;
constexpr int64_t kOffsetLimit = (int64_t)1 << 60;

bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

size_t element_bytes(int32_t dtype) { return dtype == DGC_F32 ? 4 : 2; }

bool type_known(int32_t dtype) { return dtype == DGC_F32 || dtype == DGC_F16 || dtype == DGC_BF16; }

bool product_fits(int64_t n, int64_t stride) { return n == 0 || stride <= kOffsetLimit / n; }

// An array of heads that a call touches: its address and strides.
dgc_status check_heads(const dgc_heads* x, int64_t rows, int64_t heads, int64_t dim, size_t element, bool written) {
  if (!x || x->row_stride < 0 || x->head_stride < 0) return DGC_ERR_INVALID_ARG;
  if (!product_fits(rows, x->row_stride) || !product_fits(heads, x->head_stride)) return DGC_ERR_CAPACITY;
  if (written && rows > 0) {
    const bool heads_in_rows = (rows == 1 || x->row_stride >= (heads - 1) * x->head_stride + dim) && (heads == 1 || x->head_stride >= dim);
    const bool rows_in_heads = (heads == 1 || x->head_stride >= (rows - 1) * x->row_stride + dim) && (rows == 1 || x->row_stride >= dim);
    if (!heads_in_rows && !rows_in_heads) return DGC_ERR_INVALID_ARG;
  }
  if (rows > 0 && !x->data) return DGC_ERR_INVALID_ARG;
  return aligned_to(x->data, element) ? DGC_OK : DGC_ERR_ALIGNMENT;
}

// Of an attention array also: the rows of a chunk have offsets of 32 bits.
dgc_status check_rows_of_heads(const dgc_heads* x, int64_t rows, int64_t heads, int64_t dim, size_t element, bool written) {
  if (x && x->row_stride >= kWidthLimit) return DGC_ERR_CAPACITY;
  return check_heads(x, rows, heads, dim, element, written);
}

dgc_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need == 0) return DGC_OK;
  if (!workspace) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(workspace, 256)) return DGC_ERR_ALIGNMENT;
  return have < need ? DGC_ERR_CAPACITY : DGC_OK;
}

dgc_status check_attention(const dgc_attention* s) {
  if (!s || !type_known(s->dtype) || s->reserved != 0) return DGC_ERR_INVALID_ARG;
  if (s->heads < 1 || s->key_dim < 1 || s->value_dim < 1 || s->rows < 0 || s->sequences < 0 || s->max_length < 0)
    return DGC_ERR_INVALID_ARG;
  if (s->key_dim > DGC_HEAD_MAX || s->value_dim > DGC_HEAD_MAX || !std::isfinite(s->scale)) return DGC_ERR_INVALID_ARG;
  if (s->heads > 65535 || s->rows >= (int64_t)1 << 40 || s->sequences >= kIntLimit || s->max_length >= kIntLimit)
    return DGC_ERR_CAPACITY;
  if (!s->row_offsets && s->sequences * s->max_length != s->rows) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(s->row_offsets, 8)) return DGC_ERR_ALIGNMENT;
  return (walk_workgroups(s->sequences, s->heads, DGC_HEAD_MAX) + 8) * kWalksMax < kIntLimit ? DGC_OK : DGC_ERR_CAPACITY;
}

dgc_status check_vocab(const dgc_vocab* s) {
  if (!s || !type_known(s->dtype) || s->reserved != 0) return DGC_ERR_INVALID_ARG;
  if (s->rows < 0 || s->vocab < 1 || s->width < 1 || s->hidden_stride < s->width || s->weight_stride < s->width)
    return DGC_ERR_INVALID_ARG;
  if (s->rows >= 1 << 24 || s->vocab >= 1 << 24 || s->width >= 1 << 20 || s->hidden_stride >= 1 << 24 || s->weight_stride >= 1 << 24)
    return DGC_ERR_CAPACITY;
  return s->rows * s->vocab < (int64_t)1 << 46 ? DGC_OK : DGC_ERR_CAPACITY;  // tiles that one launch numbers
}

VocabArgs vocab_args(const dgc_vocab* s, const void* hidden, const void* weight, const int32_t* labels, const float* row_weight,
                     uint32_t* diag) {
  VocabArgs v{};
  v.hidden = hidden;
  v.weight = weight;
  v.hidden_stride = s->hidden_stride;
  v.weight_stride = s->weight_stride;
  v.rows = (int32_t)s->rows;
  v.vocab = (int32_t)s->vocab;
  v.width = (int32_t)s->width;
  v.labels = labels;
  v.row_weight = row_weight;
  v.diag_flags = diag;
  return v;
}

dgc_status check_vocab_inputs(const dgc_vocab* s, const void* hidden, const void* weight, const int32_t* labels,
                              const float* row_weight, const void* diag) {
  if (s->rows > 0 && (!hidden || !weight || !labels)) return DGC_ERR_INVALID_ARG;
  const size_t e = element_bytes(s->dtype);
  return aligned_to(hidden, e) && aligned_to(weight, e) && aligned_to(labels, 4) && aligned_to(row_weight, 4) && aligned_to(diag, 4)
             ? DGC_OK
             : DGC_ERR_ALIGNMENT;
}

}  // namespace

extern "C" {

dgc_status dgc_rotary_frequencies(int32_t rotary_dim, double base, double factor, double context, double low_turns,
                                  double high_turns, uint64_t* out) {
  if (rotary_dim < 0 || rotary_dim > DGC_HEAD_MAX || rotary_dim % 2 != 0) return DGC_ERR_INVALID_ARG;
  if (!std::isfinite(base) || base < 1.0 || !std::isfinite(factor) || factor < 1.0 || !std::isfinite(context) || context < 0.0)
    return DGC_ERR_INVALID_ARG;
  if (!(low_turns >= 0.0) || !(high_turns > low_turns) || !std::isfinite(high_turns)) return DGC_ERR_INVALID_ARG;
  if (rotary_dim > 0 && !out) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(out, 8)) return DGC_ERR_ALIGNMENT;
  constexpr long double kTurn = 6.283185307179586476925286766559L;
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    const long double f = std::exp(-2.0L * i / rotary_dim * std::log((long double)base)) / kTurn;
    long double kept = (f * context - low_turns) / ((long double)high_turns - low_turns);
    kept = kept < 0.0L ? 0.0L : kept > 1.0L ? 1.0L : kept;
    out[i] = (uint64_t)std::nearbyint(std::ldexp(f * kept + f * (1.0L - kept) / factor, 64));
  }
  return DGC_OK;
}

dgc_status dgc_rotary(const dgc_rotary_shape* s, const int64_t* positions, const uint64_t* frequencies, float magnitude,
                      int32_t count, const int32_t* heads, const dgc_heads* x, const dgc_heads* out, void* stream_) {
  if (!s || !type_known(s->dtype) || (s->flags & ~(uint32_t)(DGC_ROTARY_HALF | DGC_ROTARY_INVERSE)) != 0) return DGC_ERR_INVALID_ARG;
  if (s->rows < 0 || s->head_dim < 1 || s->head_dim > DGC_HEAD_MAX || s->rotary_dim < 0 || s->rotary_dim > s->head_dim || s->rotary_dim % 2 != 0)
    return DGC_ERR_INVALID_ARG;
  if (count < 1 || count > DGC_ROTARY_MAX || !heads || !x || !out || !std::isfinite(magnitude)) return DGC_ERR_INVALID_ARG;
  if (s->rows >= kIntLimit) return DGC_ERR_CAPACITY;
  if ((s->rows > 0 && !positions) || (s->rotary_dim > 0 && !frequencies)) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(positions, 8) || !aligned_to(frequencies, 8)) return DGC_ERR_ALIGNMENT;
  const size_t e = element_bytes(s->dtype);
  RotaryArgs a{};
  for (int32_t i = 0; i < count; ++i) {
    if (heads[i] < 1) return DGC_ERR_INVALID_ARG;
    if (heads[i] > 65535) return DGC_ERR_CAPACITY;
    dgc_status st = check_heads(&x[i], s->rows, heads[i], s->head_dim, e, false);
    if (st == DGC_OK) st = check_heads(&out[i], s->rows, heads[i], s->head_dim, e, true);
    if (st != DGC_OK) return st;
    if (s->rows > 0 && out[i].data == x[i].data && (out[i].row_stride != x[i].row_stride || out[i].head_stride != x[i].head_stride))
      return DGC_ERR_INVALID_ARG;
    a.x[i] = x[i];
    a.out[i] = out[i];
    a.heads[i] = heads[i];
  }
  if (s->rows == 0) return DGC_OK;
  for (int32_t i = 0; i < count; ++i)  // an array that is turned twice, or read while it is turned
    for (int32_t j = 0; j < count; ++j)
      if (i != j && (out[i].data == out[j].data || out[i].data == x[j].data)) return DGC_ERR_INVALID_ARG;
  a.count = count;
  a.rows = (int32_t)s->rows;
  a.head_dim = s->head_dim;
  a.rotary_dim = s->rotary_dim;
  a.positions = positions;
  a.frequencies = frequencies;
  a.magnitude = magnitude;
  a.half = (s->flags & DGC_ROTARY_HALF) != 0;
  a.inverse = (s->flags & DGC_ROTARY_INVERSE) != 0;
  return hip_ok(launch_rotary(a, s->dtype, static_cast<hipStream_t>(stream_)), "launch rotary kernel") ? DGC_OK : DGC_ERR_HIP;
}

dgc_status dgc_linear_attention_workspace_bytes(const dgc_attention* shape, int32_t backward, size_t* bytes) {
  const dgc_status st = check_attention(shape);
  if (st != DGC_OK) return st;
  if (!bytes || (backward != 0 && backward != 1)) return DGC_ERR_INVALID_ARG;
  *bytes = walk_workspace_bytes(shape->rows, shape->sequences, shape->max_length, shape->heads, shape->key_dim, shape->value_dim, shape->row_offsets != nullptr) * (backward ? 2 : 1);
  return DGC_OK;
}

dgc_status dgc_linear_attention_forward(const dgc_attention* s, const dgc_heads* q, const dgc_heads* k, const dgc_heads* v,
                                        const float* log_decay, const float* state0, const dgc_heads* o, float* state_last,
                                        void* workspace, size_t workspace_bytes, void* stream_) {
  dgc_status st = check_attention(s);
  if (st != DGC_OK) return st;
  const size_t e = element_bytes(s->dtype);
  for (const dgc_heads* x : {q, k})
    if ((st = check_rows_of_heads(x, s->rows, s->heads, s->key_dim, e, false)) != DGC_OK) return st;
  if ((st = check_rows_of_heads(v, s->rows, s->heads, s->value_dim, e, false)) != DGC_OK) return st;
  if ((st = check_rows_of_heads(o, s->rows, s->heads, s->value_dim, e, true)) != DGC_OK) return st;
  if (!log_decay) return DGC_ERR_INVALID_ARG;
  if (s->rows > 0)
    for (const dgc_heads* x : {q, k, v})
      if (x->data == o->data) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(log_decay, 4) || !aligned_to(state0, 4) || !aligned_to(state_last, 4)) return DGC_ERR_ALIGNMENT;
  size_t need = 0;
  dgc_linear_attention_workspace_bytes(s, 0, &need);
  if ((st = check_workspace(workspace, workspace_bytes, need)) != DGC_OK) return st;
  if (s->sequences == 0) return DGC_OK;
  WalkArgs w{};
  w.a = *q;
  w.b = *k;
  w.c = *v;
  w.out = *o;
  w.log_decay = log_decay;
  w.first = state0;
  w.last = state_last;
  w.state_a = s->value_dim;
  w.state_c = 1;
  w.heads = s->heads;
  w.da = s->key_dim;
  w.dc = s->value_dim;
  w.rows = s->rows;
  w.sequences = s->sequences;
  w.max_length = s->max_length;
  w.row_offsets = s->row_offsets;
  w.scale = 1.0f;
  w.out_scale = s->scale;
  w.states = static_cast<float*>(workspace);
  const hipStream_t stream = static_cast<hipStream_t>(stream_);
  hipError_t err = launch_walk_states(&w, 1, s->dtype, stream);
  if (err == hipSuccess) err = launch_walks(&w, 1, s->dtype, stream);
  return hip_ok(err, "launch attention kernels") ? DGC_OK : DGC_ERR_HIP;
}

dgc_status dgc_linear_attention_backward(const dgc_attention* s, const dgc_heads* q, const dgc_heads* k, const dgc_heads* v,
                                         const float* log_decay, const float* state0, const dgc_heads* d_o,
                                         const float* dstate_last, const dgc_heads* dq, const dgc_heads* dk, const dgc_heads* dv,
                                         float* dstate0, void* workspace, size_t workspace_bytes, void* stream_) {
  dgc_status st = check_attention(s);
  if (st != DGC_OK) return st;
  const size_t e = element_bytes(s->dtype);
  for (const dgc_heads* x : {q, k})
    if ((st = check_rows_of_heads(x, s->rows, s->heads, s->key_dim, e, false)) != DGC_OK) return st;
  for (const dgc_heads* x : {v, d_o})
    if ((st = check_rows_of_heads(x, s->rows, s->heads, s->value_dim, e, false)) != DGC_OK) return st;
  for (const dgc_heads* x : {dq, dk})
    if ((st = check_rows_of_heads(x, s->rows, s->heads, s->key_dim, e, true)) != DGC_OK) return st;
  if ((st = check_rows_of_heads(dv, s->rows, s->heads, s->value_dim, e, true)) != DGC_OK) return st;
  if (!log_decay) return DGC_ERR_INVALID_ARG;
  if (s->rows > 0) {
    for (const dgc_heads* x : {q, k, v, d_o})
      for (const dgc_heads* y : {dq, dk, dv})
        if (x->data == y->data) return DGC_ERR_INVALID_ARG;
    if (dq->data == dk->data || dq->data == dv->data || dk->data == dv->data) return DGC_ERR_INVALID_ARG;
  }
  if (dstate0 && dstate0 == state0) return DGC_ERR_INVALID_ARG;  // which dq's walk reads while dv's leaves dstate0
  if (!aligned_to(log_decay, 4) || !aligned_to(state0, 4) || !aligned_to(dstate_last, 4) || !aligned_to(dstate0, 4)) return DGC_ERR_ALIGNMENT;
  size_t need = 0;
  dgc_linear_attention_workspace_bytes(s, 1, &need);
  if ((st = check_workspace(workspace, workspace_bytes, need)) != DGC_OK) return st;
  if (s->sequences == 0) return DGC_OK;
  const hipStream_t stream = static_cast<hipStream_t>(stream_);
  WalkArgs forward{};  // with k and v: the states as in the forward call
  forward.b = *k;
  forward.c = *v;
  forward.log_decay = log_decay;
  forward.first = state0;
  forward.states = static_cast<float*>(workspace);
  forward.state_a = s->value_dim;
  forward.state_c = 1;
  forward.heads = s->heads;
  forward.da = s->key_dim;
  forward.dc = s->value_dim;
  forward.rows = s->rows;
  forward.sequences = s->sequences;
  forward.max_length = s->max_length;
  forward.row_offsets = s->row_offsets;
  forward.scale = 1.0f;
  WalkArgs w[3] = {forward, forward, forward};
  WalkArgs &walk_dq = w[0], &walk_dk = w[1], &walk_dv = w[2];
  // dv: from the last step to the first, with the state's gradient for a state
  walk_dv.a = *k;
  walk_dv.b = *q;
  walk_dv.c = *d_o;
  walk_dv.out = *dv;
  walk_dv.first = dstate_last;
  walk_dv.last = dstate0;
  walk_dv.states = forward.states + need / 2 / sizeof(float);
  walk_dv.scale = s->scale;
  walk_dv.out_scale = 1.0f;
  walk_dv.late = 1;
  walk_dv.reverse = true;
  // dk: the same with v for k, and q and do changed round, and so the state's rows and columns
  walk_dk = walk_dv;
  walk_dk.a = *v;
  walk_dk.b = *d_o;
  walk_dk.c = *q;
  walk_dk.out = *dk;
  walk_dk.last = nullptr;
  // dq: the forward walk with do for q, and k and v changed round
  walk_dq.a = *d_o;
  walk_dq.b = *v;
  walk_dq.c = *k;
  walk_dq.out = *dq;
  walk_dq.out_scale = s->scale;
  for (WalkArgs* x : {&walk_dq, &walk_dk}) {
    x->state_a = 1;
    x->state_c = s->value_dim;
    x->da = s->value_dim;
    x->dc = s->key_dim;
  }
  const WalkArgs states[2] = {forward, walk_dv};
  hipError_t err = launch_walk_states(states, 2, s->dtype, stream);
  // dk reads dstate_last; dv may leave dstate0 in its place
  const bool in_place = dstate0 && dstate0 == dstate_last;
  if (err == hipSuccess) err = launch_walks(w, in_place ? 2 : 3, s->dtype, stream);
  if (err == hipSuccess && in_place) err = launch_walks(&walk_dv, 1, s->dtype, stream);
  return hip_ok(err, "launch attention kernels") ? DGC_OK : DGC_ERR_HIP;
}

dgc_status dgc_vocab_loss_workspace_bytes(const dgc_vocab* shape, int32_t backward, size_t* bytes) {
  const dgc_status st = check_vocab(shape);
  if (st != DGC_OK) return st;
  if (!bytes || (backward != 0 && backward != 1)) return DGC_ERR_INVALID_ARG;
  *bytes = vocab_workspace_bytes(shape->dtype, (int32_t)shape->rows, (int32_t)shape->vocab, (int32_t)shape->width, backward != 0);
  return DGC_OK;
}

dgc_status dgc_vocab_loss_forward(const dgc_vocab* s, const void* hidden, const void* weight, const int32_t* labels,
                                  const float* row_weight, float* loss, float* lse, uint32_t* diag_flags_dev, void* workspace,
                                  size_t workspace_bytes, void* stream_) {
  dgc_status st = check_vocab(s);
  if (st != DGC_OK) return st;
  if ((st = check_vocab_inputs(s, hidden, weight, labels, row_weight, diag_flags_dev)) != DGC_OK) return st;
  if (s->rows > 0 && !loss && !lse) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(loss, 4) || !aligned_to(lse, 4)) return DGC_ERR_ALIGNMENT;
  VocabArgs v = vocab_args(s, hidden, weight, labels, row_weight, diag_flags_dev);
  if ((st = check_workspace(workspace, workspace_bytes, vocab_workspace_bytes(s->dtype, v.rows, v.vocab, v.width, false))) != DGC_OK) return st;
  if (s->rows == 0) return DGC_OK;
  v.loss = loss;
  v.lse = lse;
  return hip_ok(launch_vocab_forward(v, workspace, s->dtype, static_cast<hipStream_t>(stream_)), "launch vocabulary loss kernels") ? DGC_OK : DGC_ERR_HIP;
}

dgc_status dgc_vocab_loss_backward(const dgc_vocab* s, const void* hidden, const void* weight, const int32_t* labels,
                                   const float* row_weight, const float* lse, void* dhidden, int64_t dhidden_stride, void* dweight,
                                   int64_t dweight_stride, uint32_t* diag_flags_dev, void* workspace, size_t workspace_bytes,
                                   void* stream_) {
  dgc_status st = check_vocab(s);
  if (st != DGC_OK) return st;
  if ((st = check_vocab_inputs(s, hidden, weight, labels, row_weight, diag_flags_dev)) != DGC_OK) return st;
  if (s->rows > 0 && !dhidden && !dweight) return DGC_ERR_INVALID_ARG;
  if ((dhidden && dhidden_stride < s->width) || (dweight && dweight_stride < s->width)) return DGC_ERR_INVALID_ARG;
  if ((dhidden && dhidden_stride >= 1 << 24) || (dweight && dweight_stride >= 1 << 24)) return DGC_ERR_CAPACITY;
  if (s->rows > 0 && !lse) return DGC_ERR_INVALID_ARG;
  for (const void* x : {hidden, weight})
    if (x && (x == dhidden || x == dweight)) return DGC_ERR_INVALID_ARG;
  if (dhidden && dhidden == dweight) return DGC_ERR_INVALID_ARG;
  const size_t e = element_bytes(s->dtype);
  if (!aligned_to(dhidden, e) || !aligned_to(dweight, e) || !aligned_to(lse, 4)) return DGC_ERR_ALIGNMENT;
  VocabArgs v = vocab_args(s, hidden, weight, labels, row_weight, diag_flags_dev);
  if ((st = check_workspace(workspace, workspace_bytes, vocab_workspace_bytes(s->dtype, v.rows, v.vocab, v.width, true))) != DGC_OK) return st;
  if (s->rows == 0 && !dweight) return DGC_OK;
  v.lse = const_cast<float*>(lse);
  v.dhidden = dhidden;
  v.dweight = dweight;
  v.dhidden_stride = dhidden_stride;
  v.dweight_stride = dweight_stride;
  return hip_ok(launch_vocab_backward(v, workspace, s->dtype, static_cast<hipStream_t>(stream_)), "launch vocabulary loss kernels") ? DGC_OK : DGC_ERR_HIP;
}

}  // extern "C"
