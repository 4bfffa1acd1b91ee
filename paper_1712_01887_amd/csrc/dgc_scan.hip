// The gated linear recurrence: h_t = a_t h_{t-1} + b_t x_t with a = sigmoid(gate), forward and backward.

#include "dgc_operators.h"

namespace dgc {
namespace {

struct Gates {
  float a, b;  // sigmoid(f), sigmoid(-f): neither is formed as one minus the other, so both keep their relative accuracy
};

__device__ __forceinline__ Gates gates_of(float f) {
  const float t = __expf(-fabsf(f));
  const float s = __builtin_amdgcn_rcpf(1.0f + t);
  const float ts = t * s;
  return f < 0.0f ? Gates{ts, s} : Gates{s, ts};
}

// Rows [begin, begin + length) of a sequence, cut to the arrays and to max_length whatever the offsets say.
__device__ __forceinline__ void sequence_rows(const ScanArgs& a, int64_t s, int64_t& begin, int64_t& length) {
  if (!a.row_offsets) {
    begin = s * a.max_length;
    length = a.max_length;
    return;
  }
  const int64_t lo = a.row_offsets[s], hi = a.row_offsets[s + 1];
  begin = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
  length = (hi > a.rows ? a.rows : hi) - begin;
  length = length < 0 ? 0 : length > a.max_length ? a.max_length : length;
}

// Where the state in front of step c * kStateRows of a sequence is kept: no two of them at one place, all below
// rows / kStateRows + sequences.
constexpr int kStateRows = DGC_SCAN_STATE_ROWS;
__device__ __forceinline__ int64_t state_row(int64_t s, int64_t begin, int64_t c) { return begin / kStateRows + s + c; }

// One thread walks one channel of one sequence.
template <typename T, bool FREE>
__global__ __launch_bounds__(64) void scan_forward_kernel(ScanArgs a) {
  const int64_t blocks = (a.channels + 63) / 64;
  const int64_t s = blockIdx.x / blocks;
  const int64_t d = (blockIdx.x - s * blocks) * 64 + threadIdx.x;
  if (d >= a.channels) return;
  int64_t begin, length;
  sequence_rows(a, s, begin, length);
  const T* gate = static_cast<const T*>(a.gate) + begin * a.gate_stride + d;
  const T* x = static_cast<const T*>(a.x) + begin * a.x_stride + d;
  T* h = static_cast<T*>(a.h) + begin * a.h_stride + d;
  float state = a.first ? a.first[s * a.channels + d] : 0.0f;
  for (int64_t t = 0; t < length; ++t) {
    if (a.states && t % kStateRows == 0) a.states[state_row(s, begin, t / kStateRows) * a.channels + d] = state;
    const Gates g = gates_of(to_float(gate[t * a.gate_stride]));
    const float xt = to_float(x[t * a.x_stride]);
    state = fmaf(g.a, state, FREE ? xt : g.b * xt);
    h[t * a.h_stride] = from_float<T>(state);
  }
  if (a.last) a.last[s * a.channels + d] = state;
}

// The same backwards: the states of kStateRows steps are formed again from the kept one, then walked from the last.
template <typename T, bool FREE>
__global__ __launch_bounds__(64) void scan_backward_kernel(ScanArgs a) {
  __shared__ float before[kStateRows][64];
  const int64_t blocks = (a.channels + 63) / 64;
  const int64_t s = blockIdx.x / blocks;
  const int64_t d = (blockIdx.x - s * blocks) * 64 + threadIdx.x;
  if (d >= a.channels) return;
  int64_t begin, length;
  sequence_rows(a, s, begin, length);
  const T* gate = static_cast<const T*>(a.gate) + begin * a.gate_stride + d;
  const T* x = static_cast<const T*>(a.x) + begin * a.x_stride + d;
  const T* dh = static_cast<const T*>(a.dh) + begin * a.dh_stride + d;
  T* dgate = static_cast<T*>(a.dgate) + begin * a.dgate_stride + d;
  T* dx = static_cast<T*>(a.dx) + begin * a.dx_stride + d;
  float flow = a.first ? a.first[s * a.channels + d] : 0.0f;  // a_{t+1} g_{t+1}
  for (int64_t c = (length + kStateRows - 1) / kStateRows - 1; c >= 0; --c) {
    const int64_t t0 = c * kStateRows;
    const int steps = (int)(length - t0 < kStateRows ? length - t0 : kStateRows);
    float state = a.states[state_row(s, begin, c) * a.channels + d];
    for (int i = 0; i < steps; ++i) {
      before[i][threadIdx.x] = state;
      const Gates g = gates_of(to_float(gate[(t0 + i) * a.gate_stride]));
      const float xt = to_float(x[(t0 + i) * a.x_stride]);
      state = fmaf(g.a, state, FREE ? xt : g.b * xt);
    }
    for (int i = steps - 1; i >= 0; --i) {
      const int64_t t = t0 + i;
      const Gates g = gates_of(to_float(gate[t * a.gate_stride]));
      const float xt = to_float(x[t * a.x_stride]);
      const float gt = to_float(dh[t * a.dh_stride]) + flow;
      const float hb = before[i][threadIdx.x];
      dx[t * a.dx_stride] = from_float<T>(FREE ? gt : g.b * gt);
      dgate[t * a.dgate_stride] = from_float<T>(gt * (FREE ? hb : hb - xt) * (g.a * g.b));
      flow = g.a * gt;
    }
  }
  if (a.last) a.last[s * a.channels + d] = flow;
}

template <typename T>
hipError_t launch(const ScanArgs& a, bool free_input, bool backward, hipStream_t stream) {
  const dim3 grid((unsigned)(a.sequences * ceil_div(a.channels, 64)));
  auto kernel = backward ? (free_input ? scan_backward_kernel<T, true> : scan_backward_kernel<T, false>)
                         : (free_input ? scan_forward_kernel<T, true> : scan_forward_kernel<T, false>);
  kernel<<<grid, 64, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan(const ScanArgs& a, int32_t dtype, bool free_input, bool backward, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return launch<float>(a, free_input, backward, stream);
    case DGC_F16: return launch<_Float16>(a, free_input, backward, stream);
    default: return launch<__bf16>(a, free_input, backward, stream);
  }
}

}  // namespace dgc
