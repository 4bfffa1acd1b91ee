// Linear attention with a decay for each head, and its gradients.

#include "dgc_layers.h"

namespace dgc {
namespace {

constexpr int kColumns = 32;   // columns of the state to a workgroup
constexpr int kParts = 8;      // threads that share a column's rows
constexpr int kThreads = kColumns * kParts;
constexpr int kRows = DGC_HEAD_MAX / kParts;

// One step after the other.  A workgroup has kColumns columns of a state: a thread has every kParts-th element of one of
// them.  out_i = sum over the rows is added up over the kParts threads in LDS, in their order.
template <typename T>
__global__ __launch_bounds__(kThreads) void walk_steps_kernel(const WalkArgs w) {
  __shared__ float vectors[2][DGC_HEAD_MAX];
  __shared__ float sums[kParts][kColumns];
  const int tiles = (w.dc + kColumns - 1) / kColumns;
  const int tile = (int)(blockIdx.x % tiles), head = (int)(blockIdx.x / tiles % w.heads);
  const int64_t sequence = blockIdx.x / tiles / w.heads;
  const int64_t lo = w.row_offsets ? w.row_offsets[sequence] : sequence * w.max_length;
  const int64_t hi = w.row_offsets ? w.row_offsets[sequence + 1] : lo + w.max_length;
  const SequenceRows rows(lo, hi, w.rows, w.max_length);
  const int column = tile * kColumns + (int)threadIdx.x % kColumns, part = (int)threadIdx.x / kColumns;
  const bool mine = column < w.dc;
  const int64_t state = (sequence * w.heads + head) * w.da * w.dc + (int64_t)column * w.state_c;
  float s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = i * kParts + part;
    s[i] = w.first && mine && r < w.da ? w.first[state + (int64_t)r * w.state_a] : 0.0f;
  }
  const float d = exp2f(w.log_decay[head] * 1.44269504f);
  const T* a = static_cast<const T*>(w.a.data) + head * w.a.head_stride;
  const T* b = static_cast<const T*>(w.b.data) + head * w.b.head_stride;
  const T* c = static_cast<const T*>(w.c.data) + head * w.c.head_stride;
  T* out = static_cast<T*>(w.out.data) + head * w.out.head_stride;
  for (int64_t t = 0; t < rows.length; ++t) {
    const int64_t row = rows.begin + (w.reverse ? rows.length - 1 - t : t);
    __syncthreads();
    for (int i = threadIdx.x; i < w.da; i += kThreads) {
      vectors[0][i] = to_float(a[row * w.a.row_stride + i]);
      vectors[1][i] = to_float(b[row * w.b.row_stride + i]);
    }
    const float value = mine ? to_float(c[row * w.c.row_stride + column]) * w.scale : 0.0f;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = i * kParts + part;
      if (r < w.da) {
        s[i] = fmaf(vectors[1][r], value, w.late ? s[i] : d * s[i]);
        sum = fmaf(vectors[0][r], s[i], sum);
        if (w.late) s[i] *= d;
      }
    }
    sums[part][threadIdx.x % kColumns] = sum;
    __syncthreads();
    if (part == 0 && mine) {
      for (int i = 1; i < kParts; ++i) sum += sums[i][threadIdx.x];
      out[row * w.out.row_stride + column] = from_float<T>(sum * w.out_scale);
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = i * kParts + part;
    if (w.last && mine && r < w.da) w.last[state + (int64_t)r * w.state_a] = s[i];
  }
}

}  // namespace

int64_t walk_workgroups(int64_t sequences, int32_t heads, int32_t dc) {
  return sequences * heads * ((dc + kColumns - 1) / kColumns);
}

hipError_t launch_walk(const WalkArgs& w, void* /*workspace*/, int32_t dtype, hipStream_t stream) {
  const uint32_t groups = (uint32_t)walk_workgroups(w.sequences, w.heads, w.dc);
  switch (dtype) {
    case DGC_F32: walk_steps_kernel<float><<<groups, kThreads, 0, stream>>>(w); break;
    case DGC_F16: walk_steps_kernel<_Float16><<<groups, kThreads, 0, stream>>>(w); break;
    default: walk_steps_kernel<__bf16><<<groups, kThreads, 0, stream>>>(w); break;
  }
  return hipGetLastError();
}

}  // namespace dgc
