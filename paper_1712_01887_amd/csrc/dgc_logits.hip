// Operators on rows of logits: a teacher's largest ones as pairs, and the loss of a student against such pairs
// with its gradient.

#include "dgc_operators.h"

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2E = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float wave_sum_f(float x) {
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max_f(float x) {
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// The workgroup's sum or maximum, the same in every thread.  `words`: kWaves floats of LDS.
__device__ __forceinline__ float block_sum(float x, float* words) {
  x = wave_sum_f(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = x;
  __syncthreads();
  float s = 0.0f;
  for (int i = 0; i < kWaves; ++i) s += words[i];
  return s;
}
__device__ __forceinline__ float block_max(float x, float* words) {
  x = wave_max_f(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = x;
  __syncthreads();
  float m = words[0];
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, words[i]);
  return m;
}

// A whole number that orders as the logits do, zero for those that are never chosen (NaN, -inf); both zeros are one.
__device__ __forceinline__ uint32_t order_key(float z) {
  if (!(z > -kInf)) return 0u;
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void top_logits_kernel(TopArgs a) {
  __shared__ unsigned long long best[kWaves];
  __shared__ float words[kWaves];
  const int64_t r = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + r * a.row_stride;
  unsigned long long last = ~0ull;  // the pair chosen before: value, then index from the highest
  for (int p = 0; p < a.k; ++p) {
    unsigned long long mine = 0;
    if (last != 0)
      for (int j = threadIdx.x; j < a.vocab; j += kThreads) {
        const uint32_t key = order_key(to_float(z[j]));
        const unsigned long long word = key ? (unsigned long long)key << 32 | (uint32_t)~j : 0ull;
        if (word < last && word > mine) mine = word;
      }
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor(mine, o);
      if (other > mine) mine = other;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) best[threadIdx.x / 64] = mine;
    __syncthreads();
    last = best[0];
    for (int i = 1; i < kWaves; ++i) last = best[i] > last ? best[i] : last;
    if (threadIdx.x == 0) {
      const int j = (int)~(uint32_t)last;
      a.out_idx[r * a.k + p] = last ? j : -1;
      a.out_val[r * a.k + p] = last ? to_float(z[j]) : -kInf;
    }
  }
  if (!a.out_lse) return;
  float m = -kInf;
  for (int j = threadIdx.x; j < a.vocab; j += kThreads) m = fmaxf(m, to_float(z[j]));
  m = block_max(m, words);
  const float shift = m == -kInf ? 0.0f : m;
  float sum = 0.0f;
  const float c = a.inv_temperature * kLog2E;
  for (int j = threadIdx.x; j < a.vocab; j += kThreads) sum += exp2_fast((to_float(z[j]) - shift) * c);
  sum = block_sum(sum, words);
  if (threadIdx.x == 0) a.out_lse[r] = shift * a.inv_temperature + kLn2 * __log2f(sum);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  __shared__ float words[kWaves];
  __shared__ int taken;
  const int64_t r = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + r * a.row_stride;
  T* grad = a.grad ? static_cast<T*>(a.grad) + r * a.grad_stride : nullptr;
  const float w = a.row_weight ? a.row_weight[r] : 1.0f;
  int y = a.labels ? a.labels[r] : -1;
  int at = threadIdx.x < a.k ? a.top_idx[r * a.k + threadIdx.x] : -1;
  if ((y >= a.vocab || at >= a.vocab) && a.diag_flags) atomicOr(a.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
  if (y >= a.vocab) y = -1;
  if (at >= a.vocab) at = -1;
  float m = -kInf;
  if (w != 0.0f)
    for (int j = threadIdx.x; j < a.vocab; j += kThreads) m = fmaxf(m, to_float(z[j]));
  m = block_max(m, words);
  const float shift = m == -kInf ? 0.0f : m;
  const float tau = a.temperature, inv_tau = 1.0f / tau, c = inv_tau * kLog2E;
  const bool second = y >= 0 && tau != 1.0f;
  float sum = 0.0f, sum1 = 0.0f;
  if (w != 0.0f)
    for (int j = threadIdx.x; j < a.vocab; j += kThreads) {
      const float zj = to_float(z[j]) - shift;
      sum += exp2_fast(zj * c);
      if (second) sum1 += exp2_fast(zj * kLog2E);
    }
  sum = block_sum(sum, words);
  sum1 = second ? block_sum(sum1, words) : sum;
  if (w == 0.0f || sum == 0.0f) {
    if (a.loss && threadIdx.x == 0) a.loss[r] = 0.0f;
    if (grad)
      for (int j = threadIdx.x; j < a.vocab; j += kThreads) grad[j] = from_float<T>(0.0f);
    return;
  }
  // the pairs, one to a thread
  const float t = at >= 0 ? a.top_val[r * a.k + threadIdx.x] * inv_tau : -kInf;
  const float z_at = at >= 0 ? to_float(z[at]) - shift : 0.0f;
  const float z_y = y >= 0 ? to_float(z[y]) - shift : 0.0f;
  float log_p;
  if (a.top_lse) {
    log_p = t - a.top_lse[r];
  } else {
    float tm = block_max(t, words);
    tm = tm == -kInf ? 0.0f : tm;
    const float total = block_sum(at >= 0 ? __expf(t - tm) : 0.0f, words);
    log_p = t - tm - (total > 0.0f ? __logf(total) : 0.0f);
  }
  const float p = at >= 0 ? __expf(log_p) : 0.0f;
  const float mass = block_sum(p, words);
  const float kl = block_sum(p != 0.0f ? p * (log_p - z_at * inv_tau + __logf(sum)) : 0.0f, words);
  if (a.loss && threadIdx.x == 0)
    a.loss[r] = w * ((1.0f - a.hard_weight) * tau * tau * kl + (y >= 0 ? a.hard_weight * (__logf(sum1) - z_y) : 0.0f));
  if (!grad) return;
  const float soft = w * (1.0f - a.hard_weight) * tau, hard = y >= 0 ? w * a.hard_weight : 0.0f;
  const float cs = soft * mass / sum, ch = hard / sum1;
  if (threadIdx.x == 0) taken = 0;
  __syncthreads();
  if (at >= 0 && at == y) taken = 1;
  for (int j = threadIdx.x; j < a.vocab; j += kThreads) {
    const float zj = to_float(z[j]) - shift;
    float g = cs * exp2_fast(zj * c);
    if (hard != 0.0f) g += ch * exp2_fast(zj * kLog2E);
    grad[j] = from_float<T>(g);
  }
  __syncthreads();
  // the few elements that a pair or the label names, once more
  if (at >= 0) {
    float g = cs * exp2_fast(z_at * c) - soft * p;
    if (hard != 0.0f) g += ch * exp2_fast(z_at * kLog2E) - (at == y ? hard : 0.0f);
    grad[at] = from_float<T>(g);
  }
  if (threadIdx.x == 0 && y >= 0 && !taken)
    grad[y] = from_float<T>(cs * exp2_fast(z_y * c) + ch * exp2_fast(z_y * kLog2E) - hard);
}

}  // namespace

hipError_t launch_top_logits(const TopArgs& a, int32_t dtype, hipStream_t stream) {
  const dim3 grid((unsigned)a.rows);
  auto kernel = dtype == DGC_F32   ? top_logits_kernel<float>
                : dtype == DGC_F16 ? top_logits_kernel<_Float16>
                                   : top_logits_kernel<__bf16>;
  kernel<<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& a, int32_t dtype, hipStream_t stream) {
  const dim3 grid((unsigned)a.rows);
  auto kernel = dtype == DGC_F32 ? distill_kernel<float> : dtype == DGC_F16 ? distill_kernel<_Float16> : distill_kernel<__bf16>;
  kernel<<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace dgc
