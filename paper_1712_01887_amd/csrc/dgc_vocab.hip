// Softmax cross entropy of an output layer without its logits in memory, and its gradients.
//
// Four products: the logits hidden weight^T, formed once for their statistics and once for the shares P; P weight and
// P^T hidden.  A piece of the vocabulary at a time, P of a piece is all that is kept.  Elements of 16 bits are multiplied as
// they are; those of 32 are taken apart into three parts of bfloat16 (24 bits in three times eight, none lost), of whose products
// the six large ones are summed: 2^-23 of a product is left out at most.  bfloat16 has binary32's exponents, so that this is so
// whatever other rows and columns hold.  Two parts of binary16 take half the products, but need a scale, and however that is
// shared (by an array, by rows), some sum runs over rows of different ones: a row of 1e20 that counts nothing made zeros of
// its neighbours.
//
// Bound by the matrix units: 4096 rows, width 2048, vocabulary 131072 in bfloat16, forward and backward, are 8.8 TFLOP in 7.55 to
// 7.81 ms, 1130 to 1165 TFLOP/s (a library's product of that shape reaches 1293).  Under the profiler, where all takes 7.8: statistics
// 1.85 ms, shares 1.99, dhidden 2.20, dweight 1.70.  The logits are formed twice because dweight needs the log-sum-exp: 8 units of
// rows * vocab * width where 6 would do if logits were kept.

#include <type_traits>

#include "dgc_layers.h"
#include "dgc_product.h"

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kPad = 256;                  // rows and columns of P are whole tiles of the largest shape
constexpr int64_t kShares = 1 << 25;       // elements of P that are kept at a time, if this many rows of kLeast columns fit
constexpr int64_t kPacked = 1 << 26;       // elements of a packed piece of the weight
constexpr int kLeast = 2048;               // columns of a piece at least, unless there are fewer
constexpr int kSplitMax = 32;

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

template <typename T>
struct Inner {  // what an element is multiplied as
  using E = T;
  static constexpr int kParts = 1;
};
template <>
struct Inner<float> {
  using E = __bf16;
  static constexpr int kParts = 3;
};
// The upper 16 bits, a bfloat16 part that is no larger.
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

using Large = Tile<256, 256, 2, 4>;
using Middle = Tile<128, 128, 2, 2>;
using Small = Tile<64, 64, 2, 2>;
// Of operands in three parts, of which LDS holds one workgroup's: with eight wavefronts, two to a SIMD, one multiplies while the
// other reads.  700 x 10000 x 1500 in binary32, forward and backward: 615 us, with four wavefronts 656, with the large tile, whose
// fragments are read half as often, where there is room for it 578.
using Large3 = Tile<256, 128, 4, 2>;
using Middle3 = Tile<128, 128, 2, 4>;

// ---- scale of shares in 16 bits ----------------------------------------------------------------
// w_r P_rj, which both gradients are sums over, is rounded to the 16-bit type, after a scaling by 2^14 over the largest weight:
// where all rows weigh the same, as in a mean, a share is rounded as it is, and what is most of a label's row of dweight, a share
// of nearly -1, hardly at all.  20 x 10000 x 1500 in bfloat16: 1.67e-3 of dhidden's norm away from 64 bits, without the scaling 1.95e-3;
// 104 rows, 119301 x 48 in binary16: 2.1e-4 of dweight's, with a power of two 3.1e-4.  binary16 holds 2^-38 of the largest: rows
// that weigh less are lost in dweight, where the others' terms are that much larger, but not in their own row of dhidden: that is
// formed from P_rj 2^14, and w_r comes in at the end.  bfloat16 holds all weights, and takes the one matrix for both.  A second part
// of the shares would be half as much again of all products; it would change vocabularies of some hundreds, whose shares are neither
// nearly 0 nor nearly -1: 30 x 68 x 107 in bfloat16 is 2.1e-3 from 64 bits, what the rounding of the results alone leaves 1.7e-3.
//
// `largest`: the bits of the largest absolute row weight.
__device__ __forceinline__ int exponent_of(uint32_t largest) {
  const int e = (int)(largest >> 23);
  return e < 28 ? 28 : e;  // scales and their inverses stay normal
}
__device__ __forceinline__ float shares_scale(uint32_t largest) {
  return largest < 0x0d800000u ? __uint_as_float((uint32_t)(268 - exponent_of(largest)) << 23) : 16384.0f / __uint_as_float(largest);
}
__device__ __forceinline__ float shares_unscale(uint32_t largest) {
  return largest < 0x0d800000u ? __uint_as_float((uint32_t)(exponent_of(largest) - 14) << 23) : __uint_as_float(largest) * (1.0f / 16384.0f);
}

// A row's weight, zero where it has no label; `label` is -1 then.
__device__ __forceinline__ float live_weight(const VocabArgs& v, int row, int& label) {
  label = v.labels[row];
  if (label < 0 || label >= v.vocab) {
    label = -1;
    return 0.0f;
  }
  return v.row_weight ? v.row_weight[row] : 1.0f;
}

__device__ __forceinline__ uint32_t finite_size(float x) {
  const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
  return bits < 0x7f800000u ? bits : 0u;
}

// The largest row weight, by one workgroup.
__device__ void largest_weight(const VocabArgs& v, uint32_t* largest) {
  constexpr int kAhead = 4;
  __shared__ uint32_t waves[kThreads / 64];
  uint32_t most = 0;
  for (int r = threadIdx.x; r < v.rows; r += kAhead * kThreads) {
    float w[kAhead];
    int label[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int row = r + i * kThreads < v.rows ? r + i * kThreads : r;
      label[i] = v.labels[row];
      w[i] = v.row_weight ? v.row_weight[row] : 1.0f;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (label[i] >= 0 && label[i] < v.vocab) most = max(most, finite_size(w[i]));
  }
  for (int m = 1; m < 64; m *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, m));
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = most;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int i = 1; i < kThreads / 64; ++i) most = max(most, waves[i]);
  *largest = most;
}

// ---- packed copies ---------------------------------------------------------------------------
// Rows of an array as the products read them: `columns` elements to a row, a multiple of 64, zeros behind `width`; binary32
// in three parts; rows without a weight as zeros if `masked`.  The last workgroup finds the largest row weight, if that is wanted.
template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(const VocabArgs v, const T* x, int64_t stride, int rows, bool masked,
                                                        typename Inner<T>::E* out, int columns, int64_t plane, uint32_t* largest) {
  using E = typename Inner<T>::E;
  const int groups = gridDim.x - (largest != nullptr);
  if ((int)blockIdx.x == groups) return largest_weight(v, largest);
  const int pieces = columns / 8;
  const int64_t total = (int64_t)rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)groups * kThreads) {
    const int row = (int)(i / pieces), column = (int)(i % pieces) * 8;
    int label;
    const bool dead = masked && live_weight(v, row, label) == 0.0f;
    const T* from = x + row * stride + column;
    float value[8];
    if (column + 8 <= v.width) {
#pragma unroll
      for (int w = 0; w < (int)sizeof(T) / 2; ++w) {
        const auto some = __builtin_bit_cast(Pack<T, 16 / sizeof(T)>, reinterpret_cast<const Loose*>(from)[w]);
#pragma unroll
        for (int j = 0; j < (int)(16 / sizeof(T)); ++j) value[w * (16 / sizeof(T)) + j] = some.get(j);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) value[j] = column + j < v.width ? to_float(from[j]) : 0.0f;
    }
#pragma unroll
    for (int p = 0; p < Inner<T>::kParts; ++p) {
      typename Matrix<E>::Fragment part;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (p == 0) value[j] = dead ? 0.0f : value[j];
        part[j] = (E)(p + 1 < Inner<T>::kParts ? cut(value[j]) : value[j]);
        value[j] -= (float)part[j];
      }
      *reinterpret_cast<Words4*>(out + p * plane + (int64_t)row * columns + column) = __builtin_bit_cast(Words4, part);
    }
  }
}

// ---- statistics ------------------------------------------------------------------------------
// What largest logits have to be subtracted in exponents: where there is none, -inf, nothing is.
__device__ __forceinline__ float shift_of(float top) { return top == -INFINITY ? 0.0f : top; }

// The largest logit and the sum of exponentials of every row of a tile, at [tile of columns][row]; a label's logit.  A part
// without a column, a wavefront's behind the vocabulary, has -inf and 0, which change nothing where parts are joined: any
// finite number there would scale rows of very negative logits away.
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void statistics_kernel(const VocabArgs v, Operand hidden, Operand weight, int depth, int first, int columns,
                                                                 float2* parts, float* at_label) {
  __shared__ float2 joined[S::kWavesN][S::kM];
  int tile_m, tile_n;
  tile_of(blockIdx.x, (v.rows + S::kM - 1) / S::kM, (columns + S::kN - 1) / S::kN, tile_m, tile_n);
  const int m0 = tile_m * S::kM, n0 = tile_n * S::kN;
  Sums z[S::kBlocksM][S::kBlocksN];
  multiply_tile<typename Inner<T>::E, S, false, false, Inner<T>::kParts>(z, hidden, weight, m0, n0, 0, depth);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wave_m = wave / S::kWavesN * (S::kBlocksM * 32), wave_n = wave % S::kWavesN * (S::kBlocksN * 32);
#pragma unroll
  for (int i = 0; i < S::kBlocksM; ++i) {
    const int row = wave_m + 32 * i + (lane & 31);
    const int label = m0 + row < v.rows ? v.labels[m0 + row] - first - n0 : -1;
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < S::kBlocksN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int column = wave_n + 32 * j + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
        float x = z[i][j][e];
        if (n0 + column >= columns) x = -INFINITY;
        else if (column == label) at_label[m0 + row] = x;
        top = fmaxf(top, x);
        z[i][j][e] = x;
      }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float shift = shift_of(top);
#pragma unroll
    for (int j = 0; j < S::kBlocksN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f((z[i][j][e] - shift) * 1.44269504f);
    sum += __shfl_xor(sum, 32);
    if (lane < 32) joined[wave % S::kWavesN][row] = make_float2(top, sum);
  }
  __syncthreads();
  for (int row = threadIdx.x; row < S::kM; row += S::kThreads) {
    if (m0 + row >= v.rows) break;
    float top = joined[0][row].x, sum = 0.0f;
#pragma unroll
    for (int i = 1; i < S::kWavesN; ++i) top = fmaxf(top, joined[i][row].x);
    const float shift = shift_of(top);
#pragma unroll
    for (int i = 0; i < S::kWavesN; ++i) sum += joined[i][row].y * __builtin_amdgcn_exp2f((joined[i][row].x - shift) * 1.44269504f);
    parts[(int64_t)(first / S::kN + tile_n) * v.rows + m0 + row] = make_float2(top, sum);
  }
}

// Joins a part's largest logit and sum to those of the parts before it.
__device__ __forceinline__ void join(float& top, float& sum, float2 part) {
  const float larger = fmaxf(top, part.x), shift = shift_of(larger);
  sum = sum * __builtin_amdgcn_exp2f((top - shift) * 1.44269504f) + part.y * __builtin_amdgcn_exp2f((part.x - shift) * 1.44269504f);
  top = larger;
}

// A row to 8 threads, which take its tiles in turn.
__global__ __launch_bounds__(kThreads) void join_kernel(const VocabArgs v, const float2* parts, const float* at_label, int tiles) {
  const int row = blockIdx.x * (kThreads / 8) + threadIdx.x % (kThreads / 8), part = threadIdx.x / (kThreads / 8);
  __shared__ float2 joined[8][kThreads / 8];
  float top = -INFINITY, sum = 0.0f;
  if (row < v.rows)
    for (int i = part; i < tiles; i += 8) join(top, sum, parts[(int64_t)i * v.rows + row]);
  joined[part][threadIdx.x % (kThreads / 8)] = make_float2(top, sum);
  __syncthreads();
  if (part != 0 || row >= v.rows) return;
  const int n = tiles < 8 ? tiles : 8;
  for (int i = 1; i < n; ++i) join(top, sum, joined[i][threadIdx.x]);
  const float lse = top + logf(sum);
  int label;
  const float w = live_weight(v, row, label);
  if (v.lse) v.lse[row] = lse;
  if (v.loss) v.loss[row] = w != 0.0f ? w * (lse - at_label[row]) : 0.0f;
  if (v.diag_flags && v.labels[row] >= v.vocab) atomicOr(v.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
}

// ---- gradients -------------------------------------------------------------------------------
// Shares of a piece, rounded to what they are multiplied as: whole tiles, zeros outside the rows and the vocabulary.  In binary16
// P_rj for dhidden and w_r P_rj for dweight, either of which may be null or the other one; else w_r P_rj, at `weighted`.
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void shares_kernel(const VocabArgs v, Operand hidden, Operand weight, int depth, int first, int columns,
                                                             const uint32_t* largest, typename Inner<T>::E* plain, typename Inner<T>::E* weighted,
                                                             int64_t stride, int64_t plane) {
  using E = typename Inner<T>::E;
  constexpr int kParts = Inner<T>::kParts;
  int tile_m, tile_n;
  tile_of(blockIdx.x, (v.rows + S::kM - 1) / S::kM, (columns + S::kN - 1) / S::kN, tile_m, tile_n);
  const int m0 = tile_m * S::kM, n0 = tile_n * S::kN;
  Sums z[S::kBlocksM][S::kBlocksN];
  multiply_tile<E, S, false, false, kParts>(z, hidden, weight, m0, n0, 0, depth);
  __shared__ __align__(16) E staged[S::kWaves][32 * kBlockPitch];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wave_m = wave / S::kWavesN * (S::kBlocksM * 32), wave_n = wave % S::kWavesN * (S::kBlocksN * 32);
  const float scale = sizeof(T) == 2 ? shares_scale(*largest) : 1.0f;
#pragma unroll
  for (int i = 0; i < S::kBlocksM; ++i) {
    const int row = m0 + wave_m + 32 * i + (lane & 31);
    int label = -1;
    float w = row < v.rows ? live_weight(v, row, label) : 0.0f;
    const float lse = w != 0.0f ? v.lse[row] : 0.0f;
    if (v.diag_flags && first + n0 + wave_n == 0 && lane < 32 && row < v.rows && v.labels[row] >= v.vocab) atomicOr(v.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
    const bool live = w != 0.0f;
    w *= scale;
#pragma unroll
    for (int j = 0; j < S::kBlocksN; ++j) {
      const int64_t corner = (int64_t)(m0 + wave_m + 32 * i) * stride + n0 + wave_n + 32 * j;
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int column = n0 + wave_n + 32 * j + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
        p[e] = __builtin_amdgcn_exp2f((z[i][j][e] - lse) * 1.44269504f);
        if (first + column == label) p[e] -= 1.0f;
        if (!live || column >= columns) p[e] = 0.0f;
      }
      auto store = [&](E* to, const float (&x)[16]) {
        store_block(staged[wave], x, lane, [&](int row, int column, Words4 eight) { *reinterpret_cast<Words4*>(to + corner + row * stride + column) = eight; });
      };
      float x[16];
      if constexpr (__is_same(T, _Float16)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = p[e] * 16384.0f;
        if (plain) store(plain, x);
        if (weighted == plain) continue;
      }
      if (weighted) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = p[e] == 0.0f ? 0.0f : p[e] * w;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          float y[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            y[e] = part + 1 < kParts ? cut(x[e]) : x[e];
            x[e] -= y[e];
          }
          store(weighted + part * plane, y);
        }
      }
    }
  }
}

// Sums over a piece (blockIdx.y: a part of it) of shares weight, added to what earlier pieces have left.
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void dhidden_kernel(const VocabArgs v, Operand shares, Operand weight, int depth, int part, bool add, float* total) {
  int tile_m, tile_n;
  tile_of(blockIdx.x, (v.rows + S::kM - 1) / S::kM, (v.width + S::kN - 1) / S::kN, tile_m, tile_n);
  const int m0 = tile_m * S::kM, n0 = tile_n * S::kN, from = blockIdx.y * part;
  Sums x[S::kBlocksM][S::kBlocksN];
  multiply_tile<typename Inner<T>::E, S, false, true, Inner<T>::kParts>(x, shares, weight, m0, n0, from, depth - from < part ? depth - from : part);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wave_m = wave / S::kWavesN * (S::kBlocksM * 32), wave_n = wave % S::kWavesN * (S::kBlocksN * 32);
  const int64_t pitch = (v.width + 3) / 4 * 4;
  float* out = total + (int64_t)blockIdx.y * v.rows * pitch;
#pragma unroll
  for (int i = 0; i < S::kBlocksM; ++i) {
    const int row = m0 + wave_m + 32 * i + (lane & 31);
    if (row >= v.rows) continue;
#pragma unroll
    for (int j = 0; j < S::kBlocksN; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int column = n0 + wave_n + 32 * j + 2 * e + 4 * (lane >> 5);
        if (column >= v.width) continue;
        float4* to = reinterpret_cast<float4*>(out + row * pitch + column);
        float4 y = make_float4(x[i][j][e], x[i][j][e + 1], x[i][j][e + 2], x[i][j][e + 3]);
        if (add) {
          const float4 before = *to;
          y = make_float4(y.x + before.x, y.y + before.y, y.z + before.z, y.w + before.w);
        }
        *to = y;
      }
  }
}

// dhidden from the parts' sums, in their order.
template <typename T>
__global__ __launch_bounds__(kThreads) void finish_kernel(const VocabArgs v, const float* total, int parts, const uint32_t* largest) {
  const int64_t pitch = (v.width + 3) / 4 * 4, size = v.rows * pitch;
  const float unscale = __is_same(T, _Float16) ? 1.0f / 16384.0f : __is_same(T, __bf16) ? shares_unscale(*largest) : 1.0f;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < size / 4; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / (pitch / 4);
    const int column = (int)(i % (pitch / 4)) * 4;
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < parts; ++p) {
      const float4 y = *reinterpret_cast<const float4*>(total + p * size + i * 4);
      x[0] += y.x, x[1] += y.y, x[2] += y.z, x[3] += y.w;
    }
    int label;
    const float w = __is_same(T, _Float16) ? live_weight(v, (int)row, label) * unscale : unscale;
    T* to = static_cast<T*>(v.dhidden) + row * v.dhidden_stride + column;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (column + j < v.width) to[j] = from_float<T>(x[j] * w);
  }
}

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void dweight_kernel(const VocabArgs v, Operand shares, Operand hidden, int first, int columns, const uint32_t* largest) {
  int tile_m, tile_n;
  tile_of(blockIdx.x, (columns + S::kM - 1) / S::kM, (v.width + S::kN - 1) / S::kN, tile_m, tile_n);
  const int m0 = tile_m * S::kM, n0 = tile_n * S::kN;
  Sums x[S::kBlocksM][S::kBlocksN];
  multiply_tile<typename Inner<T>::E, S, true, true, Inner<T>::kParts>(x, shares, hidden, m0, n0, 0, (v.rows + kDepth - 1) / kDepth * kDepth);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wave_m = wave / S::kWavesN * (S::kBlocksM * 32), wave_n = wave % S::kWavesN * (S::kBlocksN * 32);
  const float unscale = sizeof(T) == 2 && v.rows > 0 ? shares_unscale(*largest) : 1.0f;
  __shared__ __align__(16) T staged[sizeof(T) == 2 ? S::kWaves : 1][sizeof(T) == 2 ? 32 * kBlockPitch : 8];
#pragma unroll
  for (int i = 0; i < S::kBlocksM; ++i)
#pragma unroll
    for (int j = 0; j < S::kBlocksN; ++j) {
      const int row0 = m0 + wave_m + 32 * i, column0 = n0 + wave_n + 32 * j;
      T* to = static_cast<T*>(v.dweight) + (int64_t)(first + row0) * v.dweight_stride + column0;
      float y[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = x[i][j][e] * unscale;
      if constexpr (sizeof(T) == 2) {
        store_block(staged[wave], y, lane, [&](int row, int column, Words4 eight) {
          const int left = v.width - column0 - column;
          if (row0 + row >= columns || left <= 0) return;
          T* at = to + row * v.dweight_stride + column;
          if (left >= 8) {
            *reinterpret_cast<Loose*>(at) = __builtin_bit_cast(Loose, eight);
          } else {
#pragma unroll
            for (int k = 0; k < 7; ++k)
              if (k < left) at[k] = __builtin_bit_cast(T, (uint16_t)(eight[k / 2] >> (k % 2 * 16)));
          }
        });
      } else if (row0 + (lane & 31) < columns) {
        T* at = to + (lane & 31) * v.dweight_stride + 4 * (lane >> 5);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int left = v.width - column0 - 8 * q - 4 * (lane >> 5);
          if (left >= 4) {
            const float4 four = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
            *reinterpret_cast<Loose*>(at + 8 * q) = __builtin_bit_cast(Loose, four);
          } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
              if (k < left) at[8 * q + k] = y[4 * q + k];
          }
        }
      }
    }
}

// ---- host ------------------------------------------------------------------------------------
int parts_of(int32_t dtype) { return dtype == DGC_F32 ? Inner<float>::kParts : 1; }
int planes_of_shares(int32_t dtype) { return dtype == DGC_F16 ? 2 : parts_of(dtype); }

enum Shape { kLarge, kMiddle, kSmall };
constexpr int64_t kTilesLeast = 200;

// Sides of a tile; `parts` of the operands.
constexpr int64_t side_m(Shape s) { return s == kLarge ? 256 : s == kMiddle ? 128 : 64; }
constexpr int64_t side_n(int parts, Shape s) { return parts != 1 && s == kLarge ? 128 : side_m(s); }
int64_t tiles_of(int parts, Shape s, int64_t m, int64_t n) { return (m + side_m(s) - 1) / side_m(s) * ((n + side_n(parts, s) - 1) / side_n(parts, s)); }

// Large tiles of operands in three parts are taken for more than 512 rows only; below, too much of the last one is not there.
// Large and middle, us, of all products of rows x 20000 x 1024: 300 rows 510 and 446, 512: 611 and 604, 640: 744 and 758, 896: 972
// and 1014, 1408: 1446 and 1577.
bool large_fit(int parts, int64_t m) { return parts == 1 || m > 512; }

// The largest shape whose tiles are enough for most of the device's 256 compute units; small ones take four to a unit.  A tile
// of 256 x 256 reads half as much for a product as four of 128 x 128: 4096 x 8192 x 2048 takes 116 to 133 us in large tiles
// (dweight, shares), 4096 x 2048 x 8192, which has only 128 of them, 149 in middle ones (dhidden).
Shape shape_of(int parts, int64_t m, int64_t n) {
  return large_fit(parts, m) && tiles_of(parts, kLarge, m, n) >= kTilesLeast ? kLarge : tiles_of(parts, kMiddle, m, n) >= kTilesLeast ? kMiddle : kSmall;
}

// Pairs of a row and a tile of columns that calls of up to `rows` rows leave statistics of, at most: fewer rows may go by smaller
// tiles, and the most rows of either smaller kind are the other two candidates.  `columns`: that tiles are chosen by.
int64_t pairs_of(int parts, int64_t rows, int64_t vocab, int64_t columns) {
  int64_t most = 0, r = rows;
  for (const Shape now : {kLarge, kMiddle, kSmall}) {
    if (shape_of(parts, r, columns) != now) continue;
    const int64_t side = side_n(parts, now);
    most = std::max(most, r * ((vocab + side - 1) / side));
    r = std::min(r, (kTilesLeast - 1) / ((columns + side - 1) / side) * side_m(now));
  }
  return most;
}

// Where things lie in the workspace; sizes that do not fall when there are more rows.
struct Layout {
  int64_t columns;        // of a packed row
  int64_t shares_elements, piece_packed, pairs = 0;
  size_t largest, parts, at_label, hidden, weight, shares, total, bytes;

  Layout(int32_t dtype, int64_t rows, int64_t vocab, int64_t width, bool backward) {
    const int p = parts_of(dtype);
    columns = up(width, kDepth);
    const int64_t vocab_pad = up(vocab, kPad), rows_pad = up(rows, kPad);
    piece_packed = std::min(vocab_pad, std::max<int64_t>(kLeast, kPacked / columns / kPad * kPad));
    shares_elements = std::min(rows_pad * vocab_pad, std::max(kShares, rows_pad * kLeast));
    size_t at = 0;
    auto take = [&](size_t n) {
      const size_t here = at;
      at += whole(n);
      return here;
    };
    largest = take(4);
    hidden = take((size_t)rows * columns * 2 * p);
    weight = take((size_t)piece_packed * columns * 2 * p);
    if (backward) {
      shares = take((size_t)shares_elements * 2 * planes_of_shares(dtype));
      total = take((size_t)std::min(kSplitMax * rows, std::max(split_rows(p), rows)) * up(width, 4) * 4);
    } else {
      pairs = std::max(pairs_of(p, rows, vocab, vocab), pairs_of(p, rows, vocab, std::min(piece_packed, vocab)));
      parts = take((size_t)pairs * 8);
      at_label = take((size_t)rows * 4);
    }
    bytes = at;
  }
  // Parts of the sums over a piece: more than one only where there are few rows, 4096 rows in all at most, or, of operands in
  // three parts, 8192 (700 x 10000 x 1500: 252 workgroups instead of 180, 546 us instead of 578).
  static int64_t split_rows(int parts) { return parts == 1 ? 4096 : 8192; }
  static int64_t splits_at_most(int parts, int64_t rows) {
    return rows == 0 ? 0 : std::max<int64_t>(1, std::min<int64_t>(kSplitMax, split_rows(parts) / rows));
  }
};

// The same for sums over the vocabulary, which can be split into parts: the largest shape whose tiles fill the device in
// as many parts as there is room for.
Shape dhidden_shape(int parts, int64_t rows, int64_t width) {
  const int64_t splits = Layout::splits_at_most(parts, rows);
  if (rows > 128 && large_fit(parts, rows) && tiles_of(parts, kLarge, rows, width) * splits >= kTilesLeast) return kLarge;
  return rows > 64 && tiles_of(parts, kMiddle, rows, width) * splits >= (parts == 1 ? 300 : kTilesLeast) ? kMiddle : kSmall;
}

// ROOM: whether the kernel leaves LDS to a large tile of operands in three parts.
template <int PARTS, bool ROOM, typename F>
void with_shape(Shape s, F f) {
  using L = std::conditional_t<PARTS == 1, Large, std::conditional_t<ROOM, Large3, Middle3>>;
  if (s == kLarge) f(L{});
  else if (s == kMiddle) f(std::conditional_t<PARTS == 1, Middle, Middle3>{});
  else f(Small{});
}

template <typename S>
uint32_t tiles_of(S, int64_t m, int64_t n) {
  return (uint32_t)(((m + S::kM - 1) / S::kM) * ((n + S::kN - 1) / S::kN));
}

template <typename T>
struct Run {
  using E = typename Inner<T>::E;
  static constexpr int kParts = Inner<T>::kParts;
  const VocabArgs& v;
  const Layout& at;
  char* workspace;
  hipStream_t stream;
  uint32_t* largest = reinterpret_cast<uint32_t*>(workspace + at.largest);

  // Whether an array can be read as it lies: rows of whole 4 bytes at multiples of them, that a buffer's 32 bits span.
  bool direct(const void* x, int64_t stride) const {
    return kParts == 1 && v.width % 2 == 0 && stride % 2 == 0 && stride <= 1 << 22 && reinterpret_cast<uintptr_t>(x) % 4 == 0;
  }
  Operand as_it_lies(const void* x, int64_t stride, int first, int rows) const {
    return {static_cast<const char*>(x) + first * stride * 2, stride * 2, 0, rows, v.width * 2};
  }
  Operand pack(const void* x, int64_t stride, int first, int rows, bool masked, size_t to, uint32_t* largest_weight = nullptr) const {
    E* out = reinterpret_cast<E*>(workspace + to);
    const int64_t plane = (int64_t)rows * at.columns;
    const uint32_t groups = (uint32_t)std::min<int64_t>((rows * at.columns / 8 + kThreads - 1) / kThreads, 8192);
    pack_kernel<T><<<groups + (largest_weight != nullptr), kThreads, 0, stream>>>(v, static_cast<const T*>(x) + first * stride, stride, rows, masked, out, (int)at.columns, plane, largest_weight);
    return {reinterpret_cast<const char*>(out), at.columns * 2, plane * 2, rows, (int32_t)at.columns * 2};
  }
  Operand weight(int first, int rows) const {
    return direct(v.weight, v.weight_stride) ? as_it_lies(v.weight, v.weight_stride, first, rows)
                                             : pack(v.weight, v.weight_stride, first, rows, false, at.weight);
  }

  hipError_t forward() const {
    float2* parts = reinterpret_cast<float2*>(workspace + at.parts);
    float* at_label = reinterpret_cast<float*>(workspace + at.at_label);
    const Operand hidden = direct(v.hidden, v.hidden_stride) ? as_it_lies(v.hidden, v.hidden_stride, 0, v.rows)
                                                             : pack(v.hidden, v.hidden_stride, 0, v.rows, false, at.hidden);
    const int64_t at_once = direct(v.weight, v.weight_stride) ? v.vocab : at.piece_packed;
    int tiles = 0;
    with_shape<kParts, true>(shape_of(kParts, v.rows, std::min<int64_t>(at_once, v.vocab)), [&](auto shape) {
      using S = decltype(shape);
      tiles = (v.vocab + S::kN - 1) / S::kN;
      if ((int64_t)tiles * v.rows > at.pairs) return;  // never: the layout counts them the same way
      // a launch has less than 2^32 threads (shares, a piece at a time, and gradients that fit memory, stay far below)
      const int piece = (int)std::min<int64_t>(at_once, UINT32_MAX / S::kThreads / ((v.rows + S::kM - 1) / S::kM) * S::kN);
      for (int first = 0; first < v.vocab; first += piece) {
        const int columns = std::min(piece, v.vocab - first);
        statistics_kernel<T, S><<<tiles_of(shape, v.rows, columns), S::kThreads, 0, stream>>>(v, hidden, weight(first, columns), v.width, first, columns, parts, at_label);
      }
    });
    if ((int64_t)tiles * v.rows > at.pairs) return hipErrorInvalidValue;
    join_kernel<<<(v.rows + kThreads / 8 - 1) / (kThreads / 8), kThreads, 0, stream>>>(v, parts, at_label, tiles);
    return hipGetLastError();
  }

  hipError_t backward() const {
    E* shares = reinterpret_cast<E*>(workspace + at.shares);
    float* total = reinterpret_cast<float*>(workspace + at.total);
    const Operand hidden = v.rows > 0 ? pack(v.hidden, v.hidden_stride, 0, v.rows, true, at.hidden, sizeof(T) == 2 ? largest : nullptr) : Operand{};
    const int64_t rows_pad = up(v.rows, kPad);
    int64_t piece = up(v.vocab, kPad);
    if (rows_pad > 0) piece = std::min({piece, at.shares_elements / rows_pad / kPad * kPad, (int64_t)1 << 22});  // a tile's rows in a buffer's 32 bits
    if (!direct(v.weight, v.weight_stride)) piece = std::min(piece, at.piece_packed);
    const int64_t plane = rows_pad * piece;
    // what either gradient is formed from: the same, but in binary16 where rows may weigh differently
    const bool apart = __is_same(T, _Float16) && v.row_weight;
    E* const for_dweight = shares + (apart && v.dhidden && v.dweight ? plane : 0);
    E* const plain = apart && !v.dhidden ? nullptr : shares;
    E* const weighted = apart && !v.dweight ? nullptr : for_dweight;
    int parts = 1;
    for (int first = 0; first < v.vocab; first += (int)piece) {
      const int columns = (int)std::min<int64_t>(piece, v.vocab - first);
      const Operand w = v.rows > 0 ? weight(first, columns) : Operand{};
      // whole tiles of shares were written, so that a sum over them may run to the next step's end
      const auto whole_tiles = [&](const E* x) { return Operand{reinterpret_cast<const char*>(x), piece * 2, plane * 2, (int32_t)rows_pad, (int32_t)piece * 2}; };
      if (v.rows > 0)
        with_shape<kParts, false>(shape_of(kParts, v.rows, columns), [&](auto shape) {
          using S = decltype(shape);
          shares_kernel<T, S><<<tiles_of(shape, v.rows, columns), S::kThreads, 0, stream>>>(v, hidden, w, v.width, first, columns, largest, plain, weighted, piece, plane);
        });
      if (v.rows > 0 && v.dhidden)
        with_shape<kParts, true>(dhidden_shape(kParts, v.rows, v.width), [&](auto shape) {
          using S = decltype(shape);
          const uint32_t tiles = tiles_of(shape, v.rows, v.width);
          const int depth = (int)up(columns, kDepth);
          // as many parts of the sum as the device takes workgroups, of 512 terms at least
          constexpr int kResident = S::kM == 256 ? 256 : S::kM == 128 ? (kParts == 1 ? 512 : 256) : kParts == 1 ? 1024 : 768;
          if (first == 0) parts = (int)std::max<int64_t>(1, std::min<int64_t>({Layout::splits_at_most(kParts, v.rows), (int64_t)(kResident / tiles), (int64_t)(depth / 512)}));
          const int part = (int)up((depth + parts - 1) / parts, kDepth);
          if (first == 0) parts = (depth + part - 1) / part;  // none that begins behind the end; a last piece may have some
          dhidden_kernel<T, S><<<dim3(tiles, parts), S::kThreads, 0, stream>>>(v, whole_tiles(shares), w, depth, part, first > 0, total);
        });
      if (v.dweight)
        with_shape<kParts, true>(shape_of(kParts, columns, v.width), [&](auto shape) {
          using S = decltype(shape);
          dweight_kernel<T, S><<<tiles_of(shape, columns, v.width), S::kThreads, 0, stream>>>(v, whole_tiles(for_dweight), hidden, first, columns, largest);
        });
    }
    if (v.rows > 0 && v.dhidden) finish_kernel<T><<<(uint32_t)std::min<int64_t>(((int64_t)v.rows * up(v.width, 4) / 4 + kThreads - 1) / kThreads, 8192), kThreads, 0, stream>>>(v, total, parts, largest);
    return hipGetLastError();
  }
};

template <typename T>
hipError_t run(const VocabArgs& v, void* workspace, int32_t dtype, bool backward, hipStream_t stream) {
  const Layout at(dtype, v.rows, v.vocab, v.width, backward);
  const Run<T> r{v, at, static_cast<char*>(workspace), stream};
  return backward ? r.backward() : r.forward();
}

hipError_t run(const VocabArgs& v, void* workspace, int32_t dtype, bool backward, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return run<float>(v, workspace, dtype, backward, stream);
    case DGC_F16: return run<_Float16>(v, workspace, dtype, backward, stream);
    default: return run<__bf16>(v, workspace, dtype, backward, stream);
  }
}

}  // namespace

size_t vocab_workspace_bytes(int32_t dtype, int32_t rows, int32_t vocab, int32_t width, bool backward) {
  return Layout(dtype, rows, vocab, width, backward).bytes;
}

hipError_t launch_vocab_forward(const VocabArgs& a, void* workspace, int32_t dtype, hipStream_t stream) { return run(a, workspace, dtype, false, stream); }

hipError_t launch_vocab_backward(const VocabArgs& a, void* workspace, int32_t dtype, hipStream_t stream) { return run(a, workspace, dtype, true, stream); }

}  // namespace dgc
