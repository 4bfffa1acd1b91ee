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
template <typename T>
__device__ __forceinline__ float to_float(T x) {
  return static_cast<float>(x);
}
// To 16 bits: once, to the nearest, ties to even.
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  return static_cast<T>(x);
}

template <int BYTES>
struct WordOf {
  using type = uint32_t;
};
template <>
struct WordOf<2> {
  using type = uint16_t;
};

// N elements that lie behind each other, aligned to the whole of them, as the words they are loaded in: elements of 16
// bits would take a register each.
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  using Word = typename WordOf<sizeof(T) * N>::type;
  static constexpr int kWords = (int)(sizeof(T) * N / sizeof(Word));
  static constexpr int kPerWord = N / kWords;
  Word w[kWords];
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[j]);
    } else {
      const uint32_t word = w[j / kPerWord];
      if constexpr (__is_same(T, __bf16)) return __uint_as_float(j % kPerWord ? word & 0xffff0000u : word << 16);
      return static_cast<float>(__builtin_bit_cast(T, (uint16_t)(j % kPerWord ? word >> 16 : word)));
    }
  }
  __device__ __forceinline__ void set(const float (&v)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = __float_as_uint(v[j]);
    } else if constexpr (N == 1) {
      w[0] = __builtin_bit_cast(uint16_t, from_float<T>(v[0]));
    } else {
#pragma unroll
      for (int j = 0; j < N; j += 2)
        w[j / 2] = (uint32_t)__builtin_bit_cast(uint16_t, from_float<T>(v[j])) | (uint32_t)__builtin_bit_cast(uint16_t, from_float<T>(v[j + 1])) << 16;
    }
  }
  // From here on the compiler takes the words for new ones: it will not keep what it has made of them.
  __device__ __forceinline__ void renew() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
  }
};

}  // namespace dgc
#endif  // DGC_OPERATORS_H_
