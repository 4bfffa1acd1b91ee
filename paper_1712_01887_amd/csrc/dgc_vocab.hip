// Softmax cross entropy of an output layer without its logits in memory, and its gradients.

#include "dgc_layers.h"

namespace dgc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;   // rows and columns of a workgroup's part of a product
constexpr int kDepth = 16;  // of the sum at a time
constexpr int kPiece = 8192;  // columns of the vocabulary whose P are kept at a time

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// A row's weight, zero where it has no label; `label` is cut to a column that is there.
__device__ __forceinline__ float live_weight(const VocabArgs& v, int row, int& label) {
  label = v.labels[row];
  if (label < 0 || label >= v.vocab) {
    label = -1;
    return 0.0f;
  }
  return v.row_weight ? v.row_weight[row] : 1.0f;
}

// sum[i][j] = sum over k < depth of x(4 ty + i, k) y(4 tx + j, k) for a tile of 64 x 64.
template <typename X, typename Y>
__device__ __forceinline__ void multiply(float (&sum)[4][4], int depth, X x, Y y) {
  __shared__ float xs[kDepth][kTile + 4], ys[kDepth][kTile + 4];
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i / 4][i % 4] = 0.0f;
  for (int k0 = 0; k0 < depth; k0 += kDepth) {
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
      const int r = i / kDepth, k = i % kDepth;
      xs[k][r] = k0 + k < depth ? x(r, k0 + k) : 0.0f;
      ys[k][r] = k0 + k < depth ? y(r, k0 + k) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i / 4][i % 4] = fmaf(xs[k][4 * ty + i / 4], ys[k][4 * tx + i % 4], sum[i / 4][i % 4]);
  }
}

template <typename T>
__device__ __forceinline__ void logits_tile(float (&sum)[4][4], const VocabArgs& v, int row0, int column0) {
  const T* hidden = static_cast<const T*>(v.hidden);
  const T* weight = static_cast<const T*>(v.weight);
  multiply(sum, v.width,
           [&](int r, int k) { return row0 + r < v.rows ? to_float(hidden[(row0 + r) * v.hidden_stride + k]) : 0.0f; },
           [&](int c, int k) { return column0 + c < v.vocab ? to_float(weight[(column0 + c) * v.weight_stride + k]) : 0.0f; });
}

// The largest logit and the sum of exponentials of every row of a tile; a label's logit where it lies in the tile.
template <typename T>
__global__ __launch_bounds__(kThreads) void statistics_kernel(const VocabArgs v, float2* parts, float* at_label) {
  const int row0 = blockIdx.y * kTile, column0 = blockIdx.x * kTile;
  float z[4][4];
  logits_tile<T>(z, v, row0, column0);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 4 * ty + i;
    float top = -INFINITY, sum = 0.0f;
    for (int j = 0; j < 4; ++j) {
      const int column = column0 + 4 * tx + j;
      if (column >= v.vocab) z[i][j] = -INFINITY;
      if (row < v.rows && column == v.labels[row]) at_label[row] = z[i][j];
      top = fmaxf(top, z[i][j]);
    }
    for (int m = 1; m < 16; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    const float shift = top == -INFINITY ? 0.0f : top;
    for (int j = 0; j < 4; ++j) sum += exp2f((z[i][j] - shift) * 1.44269504f);
    for (int m = 1; m < 16; m *= 2) sum += __shfl_xor(sum, m);
    if (tx == 0 && row < v.rows) parts[(int64_t)row * gridDim.x + blockIdx.x] = make_float2(shift, sum);
  }
}

__global__ __launch_bounds__(kThreads) void join_kernel(const VocabArgs v, const float2* parts, const float* at_label, int tiles) {
  const int row = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  __shared__ float2 waves[kThreads / 64];
  float top = -INFINITY, sum = 0.0f;
  for (int i = threadIdx.x; i < tiles; i += kThreads) top = fmaxf(top, parts[(int64_t)row * tiles + i].x);
  for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
  if (lane == 0) waves[wave].x = top;
  __syncthreads();
  for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, waves[i].x);
  for (int i = threadIdx.x; i < tiles; i += kThreads) {
    const float2 p = parts[(int64_t)row * tiles + i];
    sum += p.y * exp2f((p.x - top) * 1.44269504f);
  }
  for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
  if (lane == 0) waves[wave].y = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0f;
    for (int i = 0; i < kThreads / 64; ++i) sum += waves[i].y;
    const float lse = top + logf(sum);
    int label;
    const float w = live_weight(v, row, label);
    if (v.lse) v.lse[row] = lse;
    if (v.loss) v.loss[row] = w != 0.0f ? w * (lse - at_label[row]) : 0.0f;
    if (v.diag_flags && v.labels[row] >= v.vocab) atomicOr(v.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
  }
}

// P of a piece of the vocabulary that begins at `first`.
template <typename T>
__global__ __launch_bounds__(kThreads) void shares_kernel(const VocabArgs v, float* shares, int first) {
  const int row0 = blockIdx.y * kTile, column0 = first + blockIdx.x * kTile;
  float z[4][4];
  logits_tile<T>(z, v, row0, column0);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 4 * ty + i;
    if (row >= v.rows) continue;
    int label;
    const float w = live_weight(v, row, label);
    if (v.diag_flags && v.labels[row] >= v.vocab) atomicOr(v.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
    for (int j = 0; j < 4; ++j) {
      const int column = column0 + 4 * tx + j;
      float p = exp2f((z[i][j] - v.lse[row]) * 1.44269504f) - (column == label ? 1.0f : 0.0f);
      if (column >= v.vocab || w == 0.0f) p = 0.0f;
      shares[(int64_t)row * kPiece + column - first] = p;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dhidden_kernel(const VocabArgs v, const float* shares, float* total, int first, int columns) {
  const int row0 = blockIdx.y * kTile, column0 = blockIdx.x * kTile;
  const T* weight = static_cast<const T*>(v.weight);
  float sum[4][4];
  multiply(sum, columns, [&](int r, int k) { return row0 + r < v.rows ? shares[(int64_t)(row0 + r) * kPiece + k] : 0.0f; },
           [&](int c, int k) { return column0 + c < v.width ? to_float(weight[(int64_t)(first + k) * v.weight_stride + column0 + c]) : 0.0f; });
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 4 * ty + i, column = column0 + 4 * tx + j;
      if (row >= v.rows || column >= v.width) continue;
      float x = sum[i][j];
      float* t = total + (int64_t)row * v.width + column;
      if (first) x += *t;
      *t = x;
      int label;
      if (first + columns == v.vocab) static_cast<T*>(v.dhidden)[row * v.dhidden_stride + column] = from_float<T>(x * live_weight(v, row, label));
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dweight_kernel(const VocabArgs v, const float* shares, int first, int columns) {
  const int row0 = blockIdx.y * kTile, column0 = blockIdx.x * kTile;
  const T* hidden = static_cast<const T*>(v.hidden);
  int label;
  float sum[4][4];
  multiply(sum, v.rows, [&](int r, int k) { return row0 + r < columns ? shares[(int64_t)k * kPiece + row0 + r] : 0.0f; },
           [&](int c, int k) {
             const float w = live_weight(v, k, label);
             return column0 + c < v.width && w != 0.0f ? w * to_float(hidden[k * v.hidden_stride + column0 + c]) : 0.0f;
           });
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 4 * ty + i, column = column0 + 4 * tx + j;
      if (row < columns && column < v.width) static_cast<T*>(v.dweight)[(first + row) * v.dweight_stride + column] = from_float<T>(sum[i][j]);
    }
}

int tiles_of(int64_t n) { return (int)((n + kTile - 1) / kTile); }

template <typename T>
hipError_t forward(const VocabArgs& v, void* workspace, hipStream_t stream) {
  const int tiles = tiles_of(v.vocab);
  float2* parts = static_cast<float2*>(workspace);
  float* at_label = reinterpret_cast<float*>(static_cast<char*>(workspace) + whole((size_t)v.rows * tiles * 8));
  statistics_kernel<T><<<dim3(tiles, tiles_of(v.rows)), kThreads, 0, stream>>>(v, parts, at_label);
  join_kernel<<<v.rows, kThreads, 0, stream>>>(v, parts, at_label, tiles);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const VocabArgs& v, void* workspace, hipStream_t stream) {
  float* shares = static_cast<float*>(workspace);
  float* total = reinterpret_cast<float*>(static_cast<char*>(workspace) + whole((size_t)v.rows * kPiece * 4));
  for (int first = 0; first < v.vocab; first += kPiece) {
    const int columns = v.vocab - first < kPiece ? v.vocab - first : kPiece;
    if (v.rows > 0) shares_kernel<T><<<dim3(tiles_of(columns), tiles_of(v.rows)), kThreads, 0, stream>>>(v, shares, first);
    if (v.rows > 0 && v.dhidden)
      dhidden_kernel<T><<<dim3(tiles_of(v.width), tiles_of(v.rows)), kThreads, 0, stream>>>(v, shares, total, first, columns);
    if (v.dweight)
      dweight_kernel<T><<<dim3(tiles_of(v.width), tiles_of(columns)), kThreads, 0, stream>>>(v, shares, first, columns);
  }
  return hipGetLastError();
}

}  // namespace

size_t vocab_workspace_bytes(int32_t /*dtype*/, int32_t rows, int32_t vocab, int32_t width, bool backward) {
  if (!backward) return whole((size_t)rows * tiles_of(vocab) * 8) + whole((size_t)rows * 4);
  return whole((size_t)rows * kPiece * 4) + whole((size_t)rows * width * 4);
}

hipError_t launch_vocab_forward(const VocabArgs& v, void* workspace, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return forward<float>(v, workspace, stream);
    case DGC_F16: return forward<_Float16>(v, workspace, stream);
    default: return forward<__bf16>(v, workspace, stream);
  }
}

hipError_t launch_vocab_backward(const VocabArgs& v, void* workspace, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return backward<float>(v, workspace, stream);
    case DGC_F16: return backward<_Float16>(v, workspace, stream);
    default: return backward<__bf16>(v, workspace, stream);
  }
}

}  // namespace dgc
