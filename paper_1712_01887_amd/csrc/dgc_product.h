// Products of matrices of 16-bit elements on the matrix units, a tile to a workgroup: the common part of the kernels of
// dgc_vocab.hip, which differ in what they do with a tile's sums.
#ifndef DGC_PRODUCT_H_
#define DGC_PRODUCT_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dgc_device.h"

namespace dgc {

typedef float Sums __attribute__((ext_vector_type(16)));
typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
// 16 bytes at any element's address, which loads and stores take.
typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));

template <typename E>
struct Matrix;
template <>
struct Matrix<__bf16> {
  typedef __bf16 Fragment __attribute__((ext_vector_type(8)));
  typedef __bf16 Half __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ Sums multiply(Fragment a, Fragment b, Sums c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Half turned(const __bf16* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) Half*)p);
  }
};
template <>
struct Matrix<_Float16> {
  typedef _Float16 Fragment __attribute__((ext_vector_type(8)));
  typedef _Float16 Half __attribute__((ext_vector_type(4)));
  typedef __fp16 Read __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ Sums multiply(Fragment a, Fragment b, Sums c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Half turned(const _Float16* p) {
    return __builtin_bit_cast(Half, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) Read*)p));
  }
};

// A matrix in memory, `rows` rows `stride` bytes apart, `row_bytes` of each there; `plane` bytes on lies its next part.
// Every row starts at a multiple of 4 bytes and has whole ones.
struct Operand {
  const char* data;
  int64_t stride, plane;
  int32_t rows, row_bytes;
};

constexpr int kDepth = 64;  // of the sum at a time; of operands of three parts, whose tiles have to fit LDS together, half of it
template <int PARTS>
constexpr int kDepthOf = PARTS == 1 ? kDepth : kDepth / 2;

// A tile of rows x columns, by waves_m x waves_n wavefronts.
template <int M, int N, int WAVES_M, int WAVES_N>
struct Tile {
  static constexpr int kM = M, kN = N, kWavesM = WAVES_M, kWavesN = WAVES_N;
  static constexpr int kWaves = WAVES_M * WAVES_N, kThreads = 64 * kWaves;
  static constexpr int kBlocksM = M / WAVES_M / 32, kBlocksN = N / WAVES_N / 32;  // of 32 x 32 to a wavefront
};

// One side of a tile: SIDE rows (or, ACROSS, columns) of an operand, DEPTH of the other kind at a time.
//
// Loads go from memory to LDS without registers in between: 64 lanes leave 64 pieces of 16 bytes behind each other, so that
// what is swizzled is which piece a lane asks for.  Along: 128 (or 64) bytes to a row, whose eight (four) pieces are exchanged
// by half (a quarter of) the row's number, so that the 16 rows that 16 lanes read lie in 16 different places of 256 bytes, all
// the banks there are.
// Across: the sum runs over the rows; blocks of 64 bytes are exchanged by the row's number, so that the four rows from which
// 16 lanes take 4 elements of a column each lie in different banks.
template <typename E, int SIDE, bool ACROSS, int WAVES, int DEPTH>
struct Side {
  static_assert(DEPTH == 32 || DEPTH == 64, "the places of pieces");
  static constexpr int kElements = SIDE * DEPTH;
  static constexpr int kLoads = kElements * 2 / 1024 / WAVES;  // to a wavefront, of 1024 bytes
  static_assert(kLoads * WAVES * 1024 == kElements * 2, "whole loads");
  static constexpr int kPieces = (ACROSS ? SIDE : DEPTH) / 8;  // of 16 bytes to a row in LDS
  const char* base;
  int64_t stride, plane;
  int32_t rows, row_bytes;  // left from `base` on; rows of the array
  uint32_t offset[kLoads];

  static __device__ __forceinline__ int exchange(int row) { return ACROSS ? (SIDE >= 128 ? row & 3 : (row >> 1) & 1) : DEPTH == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }

  // The tile begins at row (or column) `first`.
  __device__ __forceinline__ void start(const Operand& o, int first, int wave, int lane) {
    stride = o.stride;
    plane = o.plane;
    base = ACROSS ? o.data + (int64_t)first * 2 : o.data + first * o.stride;
    rows = ACROSS ? o.rows : o.rows - first;
    row_bytes = ACROSS ? o.row_bytes - first * 2 : o.row_bytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = (wave * kLoads + i) * 64 + lane, row = piece / kPieces, at = piece % kPieces;
      const int wanted = ACROSS ? (((at >> 2) ^ exchange(row)) << 2 | (at & 3)) : at ^ exchange(row);
      offset[i] = (uint32_t)row * (uint32_t)stride + (uint32_t)wanted * 16u;
    }
  }

  // Elements [k, k + DEPTH) of the sum, of part `part`.  Behind the array's last row, zeros: the buffer ends there.
  __device__ __forceinline__ void load(E* lds, int k, int part, int wave) const {
    const char* from = base + part * plane + (ACROSS ? (int64_t)k * stride : (int64_t)k * 2);
    const int have = ACROSS ? rows - k : rows, most = ACROSS ? DEPTH : SIDE;
    const int64_t bytes = have <= 0 ? 0 : (int64_t)((have < most ? have : most) - 1) * stride + row_bytes - (ACROSS ? 0 : k * 2);
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)(uint32_t)bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + i) * 512), 16, (int)offset[i], 0, 0, 0);
  }

  // Elements from `left` on of every row in LDS, which are not the row's.
  static __device__ __forceinline__ void clear(E* lds, int left, int threads) {
    for (int i = threadIdx.x; i < SIDE * kPieces; i += threads) {
      const int row = i / kPieces, piece = i % kPieces;
      if (piece * 8 + 8 <= left) continue;
      E* p = lds + row * DEPTH + ((piece ^ exchange(row)) << 3);
      for (int j = left > piece * 8 ? left - piece * 8 : 0; j < 8; ++j) p[j] = (E)0.0f;
    }
  }

  // What lane `lane` holds of 32 rows (or columns) from `at` on, 16 elements of the sum from `k` on: row lane % 32, eight
  // elements from 8 (lane / 32) on.
  static __device__ __forceinline__ typename Matrix<E>::Fragment fragment(const E* lds, int at, int k, int lane) {
    if constexpr (ACROSS) {
      const int l = lane & 15, row = k + 8 * (lane >> 5) + (l >> 2), column = at + (lane & 16) + 4 * (l & 3);
      const E* p = lds + row * SIDE + (((column >> 5) ^ exchange(row)) << 5) + (column & 31);
      const auto lo = Matrix<E>::turned(p), hi = Matrix<E>::turned(p + 4 * SIDE);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = at + (lane & 31), piece = k / 8 + (lane >> 5);
      return *reinterpret_cast<const typename Matrix<E>::Fragment*>(lds + row * DEPTH + ((piece ^ exchange(row)) << 3));
    }
  }
};

// sums[i][j]: of rows m0 + 32 i + lane % 32 of a wavefront's part of the tile and its columns n0 + 32 j + 8 (e / 4) +
// 4 (lane / 32) + e % 4 in element e, over `depth` elements of the sum from `from` on.  The sum goes by whole steps of kDepthOf.
// Of operands in one part of which neither is ACROSS, what is behind the last one's end in LDS (the next row's elements, or
// whatever lies between rows) is cleared; otherwise a row of zeros has to stand behind it on one side.
//
// Operands in three parts: the six products of parts i and j with i + j < 3, the small ones first.  All the parts of a tile are
// in LDS at a time, so that a fragment that is read is multiplied up to three times: read for each product by itself, as many
// bytes of LDS would be wanted as it can give.
//
// While a tile in LDS is multiplied the next one is on its way to another; a barrier a tile.
template <typename E, typename T, bool ACROSS_A, bool ACROSS_B, int PARTS>
__device__ __forceinline__ void multiply_tile(Sums (&sums)[T::kBlocksM][T::kBlocksN], const Operand& a, const Operand& b, int m0, int n0, int from, int depth) {
  static_assert(PARTS == 1 || PARTS == 3, "parts");
  constexpr int kStep = kDepthOf<PARTS>;
  using A = Side<E, T::kM, ACROSS_A, T::kWaves, kStep>;
  using B = Side<E, T::kN, ACROSS_B, T::kWaves, kStep>;
  __shared__ __align__(16) E a0[PARTS * A::kElements], a1[PARTS * A::kElements], b0[PARTS * B::kElements], b1[PARTS * B::kElements];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wave_m = wave / T::kWavesN * (T::kBlocksM * 32), wave_n = wave % T::kWavesN * (T::kBlocksN * 32);
  A side_a;
  B side_b;
  side_a.start(a, m0, wave, lane);
  side_b.start(b, n0, wave, lane);
#pragma unroll
  for (int i = 0; i < T::kBlocksM; ++i)
#pragma unroll
    for (int j = 0; j < T::kBlocksN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sums[i][j][e] = 0.0f;
  const int tiles = (depth + kStep - 1) / kStep;
  int k = from;  // of the tile that is loaded next
  auto load = [&](E* to_a, E* to_b) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      side_a.load(to_a + p * A::kElements, k, p, wave);
      side_b.load(to_b + p * B::kElements, k, p, wave);
    }
    k += kStep;
  };
  auto trim = [&](E* in_a, E* in_b) {
    if constexpr (!ACROSS_A && !ACROSS_B && PARTS == 1) {
      const int left = depth % kStep;
      if (left == 0) return;
      A::clear(in_a, left, T::kThreads);
      B::clear(in_b, left, T::kThreads);
      __syncthreads();
    }
  };
  // The fragments of a step of 16 are read while the step before it is multiplied, and no sooner: more of them do not fit
  // beside the sums.
  auto compute = [&](const E* from_a, const E* from_b) {
    typename Matrix<E>::Fragment fa[2][PARTS][T::kBlocksM], fb[2][PARTS][T::kBlocksN];
    auto read = [&](int set, int d) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
#pragma unroll
        for (int j = 0; j < T::kBlocksN; ++j) fb[set][p][j] = B::fragment(from_b + p * B::kElements, wave_n + 32 * j, d, lane);
#pragma unroll
        for (int i = 0; i < T::kBlocksM; ++i) fa[set][p][i] = A::fragment(from_a + p * A::kElements, wave_m + 32 * i, d, lane);
      }
    };
    read(0, 0);
#pragma unroll
    for (int step = 0; step < kStep / 16; ++step) {
      if (step + 1 < kStep / 16) read((step + 1) % 2, 16 * step + 16);
#pragma unroll
      for (int both = PARTS - 1; both >= 0; --both)
#pragma unroll
        for (int p = 0; p <= both; ++p)
#pragma unroll
          for (int i = 0; i < T::kBlocksM; ++i)
#pragma unroll
            for (int j = 0; j < T::kBlocksN; ++j) sums[i][j] = Matrix<E>::multiply(fb[step % 2][both - p][j], fa[step % 2][p][i], sums[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (tiles <= 0) return;
  load(a0, b0);
  int t = 0;
  for (; t + 2 < tiles; t += 2) {
    __syncthreads();
    load(a1, b1);
    compute(a0, b0);
    __syncthreads();
    load(a0, b0);
    compute(a1, b1);
  }
  __syncthreads();
  if (t + 1 < tiles) load(a1, b1);
  else trim(a0, b0);
  compute(a0, b0);
  if (t + 1 == tiles) return;
  __syncthreads();
  trim(a1, b1);
  compute(a1, b1);
}

// Stores a wavefront's block of 32 x 32 results in 16 bits, lane's row lane % 32 and columns 8 (e / 4) + 4 (lane / 32) + e % 4,
// by way of LDS, so that a lane has 16 bytes and a store 64 of each row that it meets; as the lanes hold them it is 8 of 32
// rows.  put(row, column, four words) gets eight elements.
constexpr int kBlockPitch = 40;
template <typename E, typename Put>
__device__ __forceinline__ void store_block(E* mine, const float (&x)[16], int lane, Put put) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    typename Matrix<E>::Half four;
#pragma unroll
    for (int j = 0; j < 4; ++j) four[j] = (E)x[4 * q + j];
    *reinterpret_cast<Words2*>(mine + (lane & 31) * kBlockPitch + 8 * q + 4 * (lane >> 5)) = __builtin_bit_cast(Words2, four);
  }
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = i * 16 + lane / 4, column = lane % 4 * 8;
    put(row, column, *reinterpret_cast<const Words4*>(mine + row * kBlockPitch + column));
  }
  wave_lds_fence();
}

// Which tile a workgroup takes.  Workgroups go to the eight dies in turn: a die gets neighbouring tiles, eight rows of tiles
// at a time, so that what they share is in its own cache.
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int& m, int& n) {
  const int total = tiles_m * tiles_n, die = id & 7, q = total >> 3, r = total & 7;
  int t = die * q + (die < r ? die : r) + (id >> 3);
  const int group = 8 * tiles_n, first = t / group * 8;
  const int height = tiles_m - first < 8 ? tiles_m - first : 8;
  t -= first * tiles_n;
  m = first + t % height;
  n = t / height;
}

}  // namespace dgc
#endif  // DGC_PRODUCT_H_
