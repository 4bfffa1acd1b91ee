// Host side of the operators on logits and sequences: argument checks and launches.
// The operators themselves run in the kernels of dgc_logits.hip and dgc_scan.hip.

#include <cmath>

#include "dgc_operators.h"
#include "dgc_steps.h"

using namespace dgc;

namespace {

constexpr int64_t kIntLimit = (int64_t)1 << 31;

bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

size_t element_bytes(int32_t dtype) { return dtype == DGC_F32 ? 4 : 2; }

bool type_known(int32_t dtype) { return dtype == DGC_F32 || dtype == DGC_F16 || dtype == DGC_BF16; }

// rows * stride elements must have an address
bool addressable(int64_t rows, int64_t stride) { return rows == 0 || stride <= ((int64_t)1 << 60) / rows; }

// The kernels take exponentials as powers of two, of logits times log2(e) / temperature.
bool temperature_fits(float t) { return t > 0.0f && std::isfinite(t) && std::isfinite(1.0f / t * 1.44269504f); }

dgc_status check_logits(const dgc_logits* s) {
  if (!s || !type_known(s->dtype) || s->reserved != 0) return DGC_ERR_INVALID_ARG;
  if (s->rows < 0 || s->vocab < 1 || s->row_stride < s->vocab) return DGC_ERR_INVALID_ARG;
  if (s->rows >= kIntLimit || s->vocab >= kIntLimit || !addressable(s->rows, s->row_stride)) return DGC_ERR_CAPACITY;
  return DGC_OK;
}

dgc_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need == 0) return DGC_OK;
  if (!workspace) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(workspace, 256)) return DGC_ERR_ALIGNMENT;
  return have < need ? DGC_ERR_CAPACITY : DGC_OK;
}

ScanArgs scan_args(const dgc_scan* s) {
  ScanArgs a{};
  a.row_offsets = s->row_offsets;
  a.rows = s->rows;
  a.max_length = s->max_length;
  a.channels = s->channels;
  a.sequences = s->sequences;
  return a;
}

dgc_status check_scan(const dgc_scan* s) {
  if (!s || !type_known(s->dtype) || (s->flags & ~(uint32_t)DGC_SCAN_FREE_INPUT) != 0) return DGC_ERR_INVALID_ARG;
  if (s->rows < 0 || s->sequences < 0 || s->max_length < 0 || s->channels < 1) return DGC_ERR_INVALID_ARG;
  if (s->rows >= (int64_t)1 << 40 || s->channels >= kWidthLimit || s->sequences >= kIntLimit || s->max_length >= kIntLimit)
    return DGC_ERR_CAPACITY;
  if (!s->row_offsets && s->sequences * s->max_length != s->rows) return DGC_ERR_INVALID_ARG;
  if (s->row_offsets && !aligned_to(s->row_offsets, 8)) return DGC_ERR_ALIGNMENT;
  return scan_workgroups(scan_args(s)) < kIntLimit ? DGC_OK : DGC_ERR_CAPACITY;
}

int64_t state_rows(const dgc_scan* s) { return s->rows / DGC_SCAN_STATE_ROWS + s->sequences; }

}  // namespace

extern "C" {

dgc_status dgc_logits_workspace_bytes(const dgc_logits* shape, size_t* bytes) {
  const dgc_status st = check_logits(shape);
  if (st != DGC_OK) return st;
  if (!bytes) return DGC_ERR_INVALID_ARG;
  *bytes = 0;  // all of a row's work is one workgroup's
  return DGC_OK;
}

dgc_status dgc_top_logits(const dgc_logits* shape, const void* logits, float temperature, int32_t k, int32_t* out_idx,
                          float* out_val, float* out_lse, void* /*workspace*/, size_t /*workspace_bytes*/, void* stream_) {
  const dgc_status st = check_logits(shape);
  if (st != DGC_OK) return st;
  if (k < 1 || k > DGC_TOP_MAX || !temperature_fits(temperature)) return DGC_ERR_INVALID_ARG;
  if (shape->rows == 0) return DGC_OK;
  if (!logits || !out_idx || !out_val) return DGC_ERR_INVALID_ARG;
  if (!aligned_to(logits, element_bytes(shape->dtype)) || !aligned_to(out_idx, 4) || !aligned_to(out_val, 4) ||
      !aligned_to(out_lse, 4))
    return DGC_ERR_ALIGNMENT;
  TopArgs a{};
  a.logits = logits;
  a.row_stride = shape->row_stride;
  a.rows = (int32_t)shape->rows;
  a.vocab = (int32_t)shape->vocab;
  a.k = k;
  a.inv_temperature = 1.0f / temperature;
  a.out_idx = out_idx;
  a.out_val = out_val;
  a.out_lse = out_lse;
  if (!hip_ok(launch_top_logits(a, shape->dtype, static_cast<hipStream_t>(stream_)), "launch top-logits kernels"))
    return DGC_ERR_HIP;
  return DGC_OK;
}

dgc_status dgc_distill_loss(const dgc_logits* shape, const void* logits, int32_t k, const int32_t* top_idx,
                            const float* top_val, const float* top_lse, const int32_t* labels,
                            const float* row_weight, float temperature, float hard_weight, float* loss, void* grad,
                            int64_t grad_stride, uint32_t* diag_flags_dev, void* /*workspace*/, size_t /*workspace_bytes*/,
                            void* stream_) {
  const dgc_status st = check_logits(shape);
  if (st != DGC_OK) return st;
  if (k < 0 || k > DGC_TOP_MAX || !temperature_fits(temperature)) return DGC_ERR_INVALID_ARG;
  if (!(hard_weight >= 0.0f) || !(hard_weight <= 1.0f) || (hard_weight > 0.0f && !labels)) return DGC_ERR_INVALID_ARG;
  if (!loss && !grad) return DGC_ERR_INVALID_ARG;
  if (grad && grad_stride < shape->vocab) return DGC_ERR_INVALID_ARG;
  if (grad == logits && grad && grad_stride != shape->row_stride) return DGC_ERR_INVALID_ARG;
  if (grad && !addressable(shape->rows, grad_stride)) return DGC_ERR_CAPACITY;
  if (shape->rows == 0) return DGC_OK;
  if (!logits || (k > 0 && (!top_idx || !top_val))) return DGC_ERR_INVALID_ARG;
  const size_t e = element_bytes(shape->dtype);
  if (!aligned_to(logits, e) || !aligned_to(grad, e) || !aligned_to(top_idx, 4) || !aligned_to(top_val, 4) ||
      !aligned_to(top_lse, 4) || !aligned_to(labels, 4) || !aligned_to(row_weight, 4) || !aligned_to(loss, 4) ||
      !aligned_to(diag_flags_dev, 4))
    return DGC_ERR_ALIGNMENT;
  DistillArgs a{};
  a.logits = logits;
  a.grad = grad;
  a.row_stride = shape->row_stride;
  a.grad_stride = grad_stride;
  a.rows = (int32_t)shape->rows;
  a.vocab = (int32_t)shape->vocab;
  a.k = k;
  a.top_idx = top_idx;
  a.top_val = top_val;
  a.top_lse = top_lse;
  a.labels = hard_weight > 0.0f ? labels : nullptr;
  a.row_weight = row_weight;
  a.temperature = temperature;
  a.hard_weight = hard_weight;
  a.loss = loss;
  a.diag_flags = diag_flags_dev;
  if (!hip_ok(launch_distill(a, shape->dtype, static_cast<hipStream_t>(stream_)), "launch distillation kernels"))
    return DGC_ERR_HIP;
  return DGC_OK;
}

dgc_status dgc_gated_scan_workspace_bytes(const dgc_scan* shape, size_t* bytes) {
  const dgc_status st = check_scan(shape);
  if (st != DGC_OK) return st;
  if (!bytes) return DGC_ERR_INVALID_ARG;
  *bytes = scan_workspace_bytes(scan_args(shape));
  return DGC_OK;
}

dgc_status dgc_gated_scan_state_rows(const dgc_scan* shape, int64_t* rows) {
  const dgc_status st = check_scan(shape);
  if (st != DGC_OK) return st;
  if (!rows) return DGC_ERR_INVALID_ARG;
  *rows = state_rows(shape);
  return DGC_OK;
}

dgc_status dgc_gated_scan_forward(const dgc_scan* shape, const void* gate, int64_t gate_stride, const void* x,
                                  int64_t x_stride, const float* h0, void* h, int64_t h_stride, float* h_last,
                                  float* states, void* workspace, size_t workspace_bytes, void* stream_) {
  dgc_status st = check_scan(shape);
  if (st != DGC_OK) return st;
  if (gate_stride < shape->channels || x_stride < shape->channels || h_stride < shape->channels)
    return DGC_ERR_INVALID_ARG;
  if (gate_stride >= kWidthLimit || x_stride >= kWidthLimit || h_stride >= kWidthLimit) return DGC_ERR_CAPACITY;
  if (shape->sequences == 0) return DGC_OK;
  if (shape->rows > 0 && (!gate || !x || !h)) return DGC_ERR_INVALID_ARG;
  if ((h == gate && h && h_stride != gate_stride) || (h == x && h && h_stride != x_stride)) return DGC_ERR_INVALID_ARG;
  const size_t e = element_bytes(shape->dtype);
  if (!aligned_to(gate, e) || !aligned_to(x, e) || !aligned_to(h, e) || !aligned_to(h0, 4) || !aligned_to(h_last, 4) ||
      !aligned_to(states, 4))
    return DGC_ERR_ALIGNMENT;
  ScanArgs a = scan_args(shape);
  if ((st = check_workspace(workspace, workspace_bytes, scan_workspace_bytes(a))) != DGC_OK) return st;
  a.gate = gate;
  a.x = x;
  a.gate_stride = gate_stride;
  a.x_stride = x_stride;
  a.first = h0;
  a.last = h_last;
  a.states = states;
  a.h = h;
  a.h_stride = h_stride;
  if (!hip_ok(launch_scan(a, workspace, shape->dtype, (shape->flags & DGC_SCAN_FREE_INPUT) != 0, false,
                          static_cast<hipStream_t>(stream_)),
              "launch scan kernels"))
    return DGC_ERR_HIP;
  return DGC_OK;
}

dgc_status dgc_gated_scan_backward(const dgc_scan* shape, const void* gate, int64_t gate_stride, const void* x,
                                   int64_t x_stride, const float* states, const void* dh, int64_t dh_stride,
                                   const float* dh_last, void* dgate, int64_t dgate_stride, void* dx,
                                   int64_t dx_stride, float* dh0, void* workspace, size_t workspace_bytes,
                                   void* stream_) {
  dgc_status st = check_scan(shape);
  if (st != DGC_OK) return st;
  for (int64_t stride : {gate_stride, x_stride, dh_stride, dgate_stride, dx_stride}) {
    if (stride < shape->channels) return DGC_ERR_INVALID_ARG;
    if (stride >= kWidthLimit) return DGC_ERR_CAPACITY;
  }
  if (shape->sequences == 0) return DGC_OK;
  if (shape->rows > 0 && (!gate || !x || !states || !dh || !dgate || !dx)) return DGC_ERR_INVALID_ARG;
  const size_t e = element_bytes(shape->dtype);
  for (const void* p : {gate, x, dh, static_cast<const void*>(dgate), static_cast<const void*>(dx)})
    if (!aligned_to(p, e)) return DGC_ERR_ALIGNMENT;
  if (!aligned_to(states, 4) || !aligned_to(dh_last, 4) || !aligned_to(dh0, 4)) return DGC_ERR_ALIGNMENT;
  const int64_t in_stride[3] = {gate_stride, x_stride, dh_stride};
  const void* in[3] = {gate, x, dh};
  for (int i = 0; i < 3 && shape->rows > 0; ++i)
    if ((dgate == in[i] && dgate_stride != in_stride[i]) || (dx == in[i] && dx_stride != in_stride[i]))
      return DGC_ERR_INVALID_ARG;
  if (shape->rows > 0 && dgate == dx) return DGC_ERR_INVALID_ARG;
  ScanArgs a = scan_args(shape);
  if ((st = check_workspace(workspace, workspace_bytes, scan_workspace_bytes(a))) != DGC_OK) return st;
  a.gate = gate;
  a.x = x;
  a.gate_stride = gate_stride;
  a.x_stride = x_stride;
  a.first = dh_last;
  a.last = dh0;
  a.states = const_cast<float*>(states);
  a.dh = dh;
  a.dgate = dgate;
  a.dx = dx;
  a.dh_stride = dh_stride;
  a.dgate_stride = dgate_stride;
  a.dx_stride = dx_stride;
  if (!hip_ok(launch_scan(a, workspace, shape->dtype, (shape->flags & DGC_SCAN_FREE_INPUT) != 0, true,
                          static_cast<hipStream_t>(stream_)),
              "launch scan kernels"))
    return DGC_ERR_HIP;
  return DGC_OK;
}

}  // extern "C"
