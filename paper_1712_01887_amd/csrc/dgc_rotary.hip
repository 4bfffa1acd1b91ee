// Rotary positions: the pairs of every head turned by their row's position times the pair's frequency.
//
// Bound by memory: every element is read and written once.  65536 rows of 32 heads of 128 in bfloat16, 1074 MB, take 252 to 264
// us, 4.1 to 4.3 TB/s; with a thread to a pair, which forms its angle for every head, they took 552.

#include <algorithm>

#include "dgc_layers.h"

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kWorkgroups = 2048;  // that fill the device

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

// 16 bytes of elements.  Loads and stores of them take any address, so that a head may begin at any element.
typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
constexpr int kElements = 16 / sizeof(T);

// `count` elements from `from` on, or to `to` on.
template <typename T>
__device__ __forceinline__ void read(float (&x)[kElements<T>], const T* from, int count) {
  if (count == kElements<T>) {
    const Loose words = *reinterpret_cast<const Loose*>(from);
    const auto piece = __builtin_bit_cast(Pack<T, kElements<T>>, words);
#pragma unroll
    for (int i = 0; i < kElements<T>; ++i) x[i] = piece.get(i);
  } else {
#pragma unroll
    for (int i = 0; i < kElements<T>; ++i) x[i] = i < count ? to_float(from[i]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void write(T* to, const float (&x)[kElements<T>], int count) {
  if (count == kElements<T>) {
    Pack<T, kElements<T>> piece;
    piece.set(x);
    *reinterpret_cast<Loose*>(to) = __builtin_bit_cast(Loose, piece);
  } else {
#pragma unroll
    for (int i = 0; i < kElements<T>; ++i)
      if (i < count) to[i] = from_float<T>(x[i]);
  }
}

// A thread has a piece of a row's heads (half: two, a half apart), forms the angles of its pairs once and turns the piece of
// every head of its group.  The pieces behind the turned ones are copied.
template <typename T, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, int pieces, int turned, int group) {
  constexpr int N = kElements<T>, kPairs = HALF ? N : N / 2, kAhead = 4;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = id / pieces;
  if (row >= a.rows) return;
  const int piece = (int)(id - row * pieces);
  const bool turns = piece < turned;
  const int half = a.rotary_dim / 2;
  const int at = turns ? piece * N : a.rotary_dim + (piece - turned) * N;
  const int left = turns ? (HALF ? half : a.rotary_dim) - at : a.head_dim - at, count = left < N ? left : N;
  float c[kPairs], s[kPairs];
  if (turns) {
    const uint64_t position = (uint64_t)a.positions[row];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int pair = HALF ? at + i : at / 2 + i;
      uint64_t fraction = pair < half ? position * a.frequencies[pair] : 0;
      if (a.inverse) fraction = 0 - fraction;
      turn(fraction, c[i], s[i]);
      c[i] *= a.magnitude;
      s[i] *= a.magnitude;
    }
  }
  int first = blockIdx.y * group, rest = group;  // heads of this workgroup, of those of all arrays behind each other
  for (int which = 0; which < a.count && rest > 0; ++which) {
    if (first >= a.heads[which]) {
      first -= a.heads[which];
      continue;
    }
    const int heads = a.heads[which] - first < rest ? a.heads[which] - first : rest;
    const int64_t step_x = a.x[which].head_stride, step_out = a.out[which].head_stride;
    const T* x = static_cast<const T*>(a.x[which].data) + row * a.x[which].row_stride + first * step_x + at;
    T* out = static_cast<T*>(a.out[which].data) + row * a.out[which].row_stride + first * step_out + at;
    // a few heads are read before the first of them is written: to the compiler they might overlap
    for (int h = 0; h < heads; h += kAhead, x += kAhead * step_x, out += kAhead * step_out) {
      float u[kAhead][N], v[HALF ? kAhead : 1][N];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (h + j < heads) {
          read(u[j], x + j * step_x, count);
          if constexpr (HALF)
            if (turns) read(v[j], x + j * step_x + half, count);
        }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (h + j >= heads) break;
        if (turns) {
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            float& p = u[j][HALF ? i : 2 * i];
            float& q = HALF ? v[HALF ? j : 0][i] : u[j][HALF ? i : 2 * i + 1];
            const float one = p * c[i] - q * s[i], two = p * s[i] + q * c[i];
            p = one;
            q = two;
          }
          if constexpr (HALF) write(out + j * step_out + half, v[j], count);
        }
        write(out + j * step_out, u[j], count);
      }
    }
    rest -= heads;
    first = 0;
  }
}

template <typename T>
void launch_rows(const RotaryArgs& a, hipStream_t stream) {
  constexpr int N = kElements<T>;
  const int turned = ((a.half ? a.rotary_dim / 2 : a.rotary_dim) + N - 1) / N, pieces = turned + (a.head_dim - a.rotary_dim + N - 1) / N;
  int heads = 0;
  for (int i = 0; i < a.count; ++i) heads += a.heads[i];
  const int64_t groups = ((int64_t)a.rows * pieces + kThreads - 1) / kThreads;
  // all heads to a thread where the rows alone fill the device, fewer where they do not
  const int parts = (int)std::min<int64_t>(std::max<int64_t>(1, kWorkgroups / groups), heads), group = (heads + parts - 1) / parts;
  const dim3 grid((uint32_t)groups, (uint32_t)((heads + group - 1) / group));
  if (a.half) rotary_kernel<T, true><<<grid, kThreads, 0, stream>>>(a, pieces, turned, group);
  else rotary_kernel<T, false><<<grid, kThreads, 0, stream>>>(a, pieces, turned, group);
}

// A launch has less than 2^32 threads, a row up to DGC_HEAD_MAX of them: rows beyond that are launched behind the others.
template <typename T>
hipError_t launch(const RotaryArgs& all, hipStream_t stream) {
  constexpr int32_t kMost = (1 << 24) - 1;
  static_assert((int64_t)kMost * DGC_HEAD_MAX + kThreads - 1 <= UINT32_MAX, "threads of a launch");
  RotaryArgs a = all;
  for (int32_t left = all.rows; left > 0; left -= a.rows) {
    a.rows = std::min(left, kMost);
    launch_rows<T>(a, stream);
    a.positions += a.rows;
    for (int i = 0; i < a.count; ++i) {
      a.x[i].data = static_cast<T*>(a.x[i].data) + a.rows * a.x[i].row_stride;
      a.out[i].data = static_cast<T*>(a.out[i].data) + a.rows * a.out[i].row_stride;
    }
  }
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
