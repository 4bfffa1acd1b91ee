// Rotary positions: the pairs of every head turned by their row's position times the pair's frequency.

#include "dgc_layers.h"

namespace dgc {
namespace {

constexpr int kThreads = 256;

// cos and sin of an angle given as a fraction of a turn in 64 bits.  The nearest quarter is taken off in whole numbers; what
// is left, an eighth of a turn at most in size, goes through the first terms of the series of sin and cos, whose next ones
// are below 2e-9 there.
__device__ __forceinline__ void turn(uint64_t fraction, float& cosine, float& sine) {
  const uint32_t quarter = (uint32_t)((fraction + (1ull << 61)) >> 62);
  const int32_t left = (int32_t)((fraction - ((uint64_t)quarter << 62)) >> 32);
  const float x = (float)left * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float y = x * x;
  float s = fmaf(y, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(y, s, 8.33333333e-3f);
  s = fmaf(y, s, -1.66666667e-1f);
  s = fmaf(x * y, s, x);
  float c = fmaf(y, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(y, c, -1.38888889e-3f);
  c = fmaf(y, c, 4.16666667e-2f);
  c = fmaf(y, c, -0.5f);
  c = fmaf(y, c, 1.0f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  cosine = (quarter + 1) & 2 ? -a : a;
  sine = quarter & 2 ? -b : b;
}

// A thread to a pair, or to an element that is only copied.
template <typename T>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  const int which = blockIdx.y;
  const int pairs = a.rotary_dim / 2, units = a.head_dim - pairs, heads = a.heads[which];
  const int64_t total = (int64_t)a.rows * heads * units;
  const T* x = static_cast<const T*>(a.x[which].data);
  T* out = static_cast<T*>(a.out[which].data);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
    const int unit = (int)(i % units);
    const int64_t rest = i / units;
    const int head = (int)(rest % heads);
    const int64_t row = rest / heads;
    const T* from = x + row * a.x[which].row_stride + head * a.x[which].head_stride;
    T* to = out + row * a.out[which].row_stride + head * a.out[which].head_stride;
    if (unit >= pairs) {
      to[unit + pairs] = from[unit + pairs];
      continue;
    }
    uint64_t fraction = (uint64_t)a.positions[row] * a.frequencies[unit];
    if (a.inverse) fraction = 0 - fraction;
    float c, s;
    turn(fraction, c, s);
    c *= a.magnitude;
    s *= a.magnitude;
    const int p = a.half ? unit : 2 * unit, q = a.half ? unit + pairs : 2 * unit + 1;
    const float u = to_float(from[p]), v = to_float(from[q]);
    to[p] = from_float<T>(u * c - v * s);
    to[q] = from_float<T>(u * s + v * c);
  }
}

template <typename T>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  int64_t most = 0;
  for (int i = 0; i < a.count; ++i) most = std::max<int64_t>(most, a.heads[i]);
  const int64_t groups = ((int64_t)a.rows * most * (a.head_dim - a.rotary_dim / 2) + kThreads - 1) / kThreads;
  const dim3 grid((uint32_t)std::min<int64_t>(groups, 1 << 20), (uint32_t)a.count);
  rotary_kernel<T><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return launch<float>(a, stream);
    case DGC_F16: return launch<_Float16>(a, stream);
    default: return launch<__bf16>(a, stream);
  }
}

}  // namespace dgc
