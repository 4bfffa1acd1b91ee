// Linear attention with a decay for each head, and its gradients.
//
// All of it is one operator (WalkArgs).  Short sequences go step by step; others by chunks of 32 steps, in which
//   out = (a b^T o D) c + d^(i+1) a S,      S <- d^32 S + (d^(31-j) b)^T c
// are products of matrices.  The matrix units take bfloat16: what is in 16 or 32 bits is taken apart into bfloat16 parts (one
// of a bfloat16, two of a binary16, three of a binary32; the shares a b^T and the state two, or three for 32-bit results;
// what goes into the state three), whose products are exact and are summed in binary32.  Parts are cut off, so that none
// passes the type's end, and the last one is rounded: two parts leave 2^-15 of a value out, three 2^-23.  A result in 16 bits,
// which is rounded to 2^-9 or 2^-12 at the end, is formed from two, one in 32 bits and every state from three.

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

// ---- chunks ------------------------------------------------------------------------------------
constexpr int kChunk = 32;

typedef __bf16 Eight __attribute__((ext_vector_type(8)));
typedef __bf16 Four __attribute__((ext_vector_type(4)));
typedef float Block __attribute__((ext_vector_type(16)));  // 32 x 32 of a wavefront: column lane % 32, rows 8 (e / 4) + 4 (lane / 32) + e % 4
typedef uint32_t Words __attribute__((ext_vector_type(4)));

template <typename T>
constexpr int kPartsOf = sizeof(T) == 4 ? 3 : __is_same(T, __bf16) ? 1 : 2;  // of an element
template <typename T>
constexpr int kMiddleParts = sizeof(T) == 4 ? 3 : 2;  // of shares and of a state that is read
constexpr int kIntoState = 3;

__device__ __forceinline__ uint32_t upper_halves(float low, float high) { return __builtin_amdgcn_perm(__float_as_uint(high), __float_as_uint(low), 0x07060302u); }
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// Eight values as PARTS fragments.
template <int PARTS>
__device__ __forceinline__ void take_apart(const float (&x)[8], Eight (&parts)[PARTS]) {
  float left[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) left[i] = x[i];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    Words w;
    if (p + 1 < PARTS) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = upper_halves(left[2 * i], left[2 * i + 1]);
      parts[p] = __builtin_bit_cast(Eight, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) left[i] -= cut(left[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) parts[p][i] = (__bf16)left[i];
    }
  }
}

__device__ __forceinline__ Block multiply(Eight a, Eight b, Block c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// The products of parts i and j with i + j < WEIGHT, the small ones first.
template <int WEIGHT, int A, int B>
__device__ __forceinline__ void multiply_parts(const Eight (&a)[A], const Eight (&b)[B], Block& c) {
#pragma unroll
  for (int sum = A + B - 2; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < A; ++i)
      if (sum < WEIGHT && sum - i >= 0 && sum - i < B) c = multiply(a[i], b[sum - i], c);
}

// d^n of a head.
struct Decay {
  float log2;
  __device__ __forceinline__ float power(int64_t n) const { return n > 0 ? __builtin_amdgcn_exp2f((float)n * log2) : 1.0f; }
};

// Where rows of a and b lie in LDS, and of c.  A row of a or b is read two ways: 16 bytes by each of 16 lanes that have a row
// each, and, for the turned reads, four rows by 16 lanes that ask for 8 bytes each.  Pieces of 16 bytes are exchanged by the
// row's number so that both meet different banks.  Of 16 elements the units of four lie in the order 0, 2, 1, 3: the eight that
// a lane holds of the state, rows 4 h .. and 8 + 4 h .., are then one piece.
template <int DIM>
struct Rows {
  static constexpr int kElements = kChunk * DIM;
  static __device__ __forceinline__ int exchange(int row) {
    return DIM >= 128 ? (row & 3) << 2 | (row >> 2 & 3) : DIM == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : row >> 2 & 3;
  }
  static __device__ __forceinline__ int at(int row, int piece, int half) { return row * DIM + ((piece ^ exchange(row)) << 3) + half * 4; }
  // elements [8 piece, 8 piece + 8) of a row
  static __device__ __forceinline__ void store(__bf16* lds, int row, int piece, Eight x) {
    const int pair = piece & ~1, half = piece & 1;
    *reinterpret_cast<Four*>(lds + at(row, pair, half)) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
    *reinterpret_cast<Four*>(lds + at(row, pair + 1, half)) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
  }
  // of row lane % 32, elements 16 group + 4 h + {0 .. 3, 8 .. 11}, h = lane / 32
  static __device__ __forceinline__ Eight along(const __bf16* lds, int group, int lane) {
    return *reinterpret_cast<const Eight*>(lds + at(lane & 31, 2 * group + (lane >> 5), 0));
  }
  // of element 32 block + lane % 32, rows 16 group + 4 h + {0 .. 3, 8 .. 11}
  static __device__ __forceinline__ Eight across(const __bf16* lds, int block, int group, int lane) {
    const int l = lane & 15, row = 16 * group + 4 * (lane >> 5) + (l >> 2), piece = 4 * block + (lane >> 4 & 1) * 2 + (l & 1);
    return pair(lds + at(row, piece, l >> 1 & 1), lds + at(row + 8, piece, l >> 1 & 1));
  }
  static __device__ __forceinline__ Eight pair(const __bf16* p, const __bf16* q) {
    const Four lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) Four*)p);
    const Four hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) Four*)q);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Pieces of 8 elements of a chunk's rows on their way from memory to LDS, by THREADS threads.
template <typename T, int DIM, int THREADS>
struct Pieces {
  static constexpr int kCount = kChunk * DIM / 8 / THREADS;
  static_assert(kCount * THREADS * 8 == kChunk * DIM, "whole pieces");
  alignas(16) T held[kCount][8];

  // `rows` rows from `base` on, `stride` elements apart, `dim` elements of each; zeros elsewhere.
  __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int dim, bool wide) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int piece = i * THREADS + (int)threadIdx.x, row = piece / (DIM / 8), column = piece % (DIM / 8) * 8;
      const T* from = base + row * stride + column;
      if (wide) {
        uint4* to = reinterpret_cast<uint4*>(held[i]);
        const bool there = row < rows && column < dim;
#pragma unroll
        for (int w = 0; w < (int)sizeof(T) / 2; ++w) to[w] = there ? reinterpret_cast<const uint4*>(from)[w] : make_uint4(0, 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) held[i][j] = row < rows && column + j < dim ? from[j] : (T)0.0f;
      }
    }
  }
  template <typename Store>
  __device__ __forceinline__ void store(Store put) const {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int piece = i * THREADS + (int)threadIdx.x, row = piece / (DIM / 8);
      Eight parts[kPartsOf<T>];
      if constexpr (__is_same(T, __bf16)) {
        parts[0] = *reinterpret_cast<const Eight*>(held[i]);
      } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = to_float(held[i][j]);
        take_apart(x, parts);
      }
#pragma unroll
      for (int p = 0; p < kPartsOf<T>; ++p) put(p, row, piece % (DIM / 8), parts[p]);
    }
  }
};

// c: a wavefront reads its 32 columns turned, and nothing else.
template <int DIM>
struct Columns {
  static constexpr int kElements = kChunk * DIM;
  static __device__ __forceinline__ int at(int row, int piece, int half) {
    const int exchange = DIM >= 128 ? row & 3 : DIM == 64 ? row >> 1 & 1 : 0;
    return row * DIM + (((piece >> 2 ^ exchange) << 2 | (piece & 3)) << 3) + half * 4;
  }
  static __device__ __forceinline__ void store(__bf16* lds, int row, int piece, Eight x) { *reinterpret_cast<Eight*>(lds + at(row, piece, 0)) = x; }
  static __device__ __forceinline__ Eight across(const __bf16* lds, int block, int group, int lane) {
    const int l = lane & 15, row = 16 * group + 4 * (lane >> 5) + (l >> 2), piece = 4 * block + (lane >> 4 & 1) * 2 + (l >> 1 & 1);
    return Rows<DIM>::pair(lds + at(row, piece, l & 1), lds + at(row + 8, piece, l & 1));
  }
};

// A workgroup's part of the work: steps [begin, begin + length) of a sequence, in the order in which they are walked.
struct Segment {
  int64_t sequence, slot, row, length;  // the array row of its first step
  bool first, last;                     // of its sequence

  // Without segments a slot is a sequence.  With them, those of sequence s are at offset(s) / steps + s and behind it: no two
  // of different sequences are the same, since offset(s + 1) / steps + 1 is at least offset(s) / steps + (its segments).
  __device__ __forceinline__ Segment(const WalkArgs& w, int64_t slot_, int64_t steps) : slot(slot_) {
    int64_t index = 0;
    sequence = slot;
    if (steps > 0) {
      int64_t lo = 0, hi = w.sequences;  // the last sequence whose first slot is not behind this one
      while (hi - lo > 1) {
        const int64_t middle = (lo + hi) / 2;
        if (first_slot(w, middle, steps) <= slot) lo = middle;
        else hi = middle;
      }
      sequence = lo;
      index = slot - first_slot(w, lo, steps);
    }
    const SequenceRows rows = rows_of(w, sequence);
    const int64_t begin = index * steps;
    length = rows.length - begin;
    last = steps == 0 || length <= steps;
    if (!last) length = steps;
    first = index == 0;
    if (index < 0 || (index > 0 && length <= 0)) length = -1;  // no such segment
    row = w.reverse ? rows.begin + rows.length - 1 - begin : rows.begin + begin;
  }
  static __device__ __forceinline__ SequenceRows rows_of(const WalkArgs& w, int64_t s) {
    const int64_t lo = w.row_offsets ? w.row_offsets[s] : s * w.max_length;
    return SequenceRows(lo, w.row_offsets ? w.row_offsets[s + 1] : lo + w.max_length, w.rows, w.max_length);
  }
  static __device__ __forceinline__ int64_t first_slot(const WalkArgs& w, int64_t s, int64_t steps) {
    return SequenceRows::inside(w.row_offsets ? w.row_offsets[s] : s * w.max_length, w.rows) / steps + s;
  }
};

struct Slots {
  int64_t count, steps;  // steps of a segment, a multiple of kChunk; 0: sequences are not cut
  float* states;         // [slot][head][...] as w.first; may be null
};

// A workgroup walks a segment of a sequence for one head and WAVES * 32 columns of c, a wavefront with 32 columns of the state
// in its registers.  OUT: out and, behind the sequence's last segment, `last`; otherwise what the segment adds to the state.
//
// Of a chunk every wavefront forms a b^T for itself, as 32 x 32 shares whose layout is that of the operand they are next, and
// so is the state's: neither goes through LDS.  While a chunk is worked on the next one's rows are on their way to registers.
template <typename T, int DA, int WAVES, bool OUT>
__global__ __launch_bounds__(64 * WAVES, DA <= 128 && sizeof(T) == 2 ? 2 : 1) void walk_chunks_kernel(const WalkArgs w, const Slots slots) {
  constexpr int kThreads = 64 * WAVES, kInput = kPartsOf<T>, kMiddle = kMiddleParts<T>, kBlocks = DA / 32, DC = 32 * WAVES;
  constexpr int kWeight = __is_same(T, __bf16) ? 2 : 3, kWeightIn = 3;
  using R = Rows<DA>;
  using Cs = Columns<DC>;
  // two buffers where they leave room for a second workgroup, or fit at all
  constexpr int kBuffers = kInput * (2 * R::kElements + Cs::kElements) * 2 <= 40960 ? 2 : 1;
  __shared__ __align__(16) __bf16 lds_a[kBuffers][OUT ? kInput * R::kElements : 8], lds_b[kBuffers][kInput * R::kElements], lds_c[kBuffers][kInput * Cs::kElements];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane >> 5;
  const int tiles = (w.dc + DC - 1) / DC;
  const int tile = (int)(blockIdx.x % tiles), head = (int)(blockIdx.x / tiles % w.heads);
  const Segment seg(w, blockIdx.x / tiles / w.heads, slots.steps);
  if (seg.length < 0 || (!OUT && seg.last)) return;
  const int column0 = tile * DC, column = column0 + 32 * wave + (lane & 31);
  const Decay d{w.log_decay[head] * 1.44269504f};

  Block state[kBlocks];
  const float* from = OUT && slots.steps > 0 && !seg.first ? slots.states + (seg.slot * w.heads + head) * w.da * w.dc : OUT && w.first ? w.first + (seg.sequence * w.heads + head) * w.da * w.dc : nullptr;
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 32 * i + 8 * (e / 4) + 4 * h + e % 4;
      state[i][e] = from && r < w.da && column < w.dc ? from[(int64_t)r * w.state_a + (int64_t)column * w.state_c] : 0.0f;
    }

  const int64_t sign = w.reverse ? -1 : 1;
  const int64_t step_a = sign * w.a.row_stride, step_b = sign * w.b.row_stride, step_c = sign * w.c.row_stride;
  const T* a = OUT ? static_cast<const T*>(w.a.data) + head * w.a.head_stride + seg.row * w.a.row_stride : nullptr;
  const T* b = static_cast<const T*>(w.b.data) + head * w.b.head_stride + seg.row * w.b.row_stride;
  const T* c = static_cast<const T*>(w.c.data) + head * w.c.head_stride + seg.row * w.c.row_stride + column0;
  auto wide = [](const dgc_heads& x, int dim) {
    return reinterpret_cast<uintptr_t>(x.data) % 16 == 0 && (x.row_stride * sizeof(T)) % 16 == 0 && (x.head_stride * sizeof(T)) % 16 == 0 && dim % 8 == 0;
  };
  const bool wide_a = OUT && wide(w.a, w.da), wide_b = wide(w.b, w.da), wide_c = wide(w.c, w.dc);

  // weights: of a share of step j in step i = lane % 32, of a step that goes into the state
  float share_weight[16], state_weight[2][8];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int j = 8 * (e / 4) + 4 * h + e % 4;
    share_weight[e] = j <= (lane & 31) ? d.power((lane & 31) - j) * w.scale : 0.0f;
    state_weight[e / 8][e % 8] = d.power(kChunk - 1 - j + w.late) * w.scale;
  }
  const float query_weight = d.power((lane & 31) + 1 - w.late);

  Pieces<T, DA, kThreads> next_a, next_b;
  Pieces<T, DC, kThreads> next_c;
  auto load = [&](int64_t at) {
    const int rows = (int)(seg.length - at < kChunk ? seg.length - at : kChunk);
    if constexpr (OUT) next_a.load(a + at * step_a, step_a, rows, w.da, wide_a);
    next_b.load(b + at * step_b, step_b, rows, w.da, wide_b);
    next_c.load(c + at * step_c, step_c, rows, w.dc - column0, wide_c);
  };
  if (seg.length > 0) load(0);
  int buffer = 0;
  for (int64_t at = 0; at < seg.length; at += kChunk, buffer = (buffer + 1) % kBuffers) {
    const int rows = (int)(seg.length - at < kChunk ? seg.length - at : kChunk);
    if (kBuffers == 1 && at > 0) __syncthreads();
    if constexpr (OUT) next_a.store([&](int p, int row, int piece, Eight x) { R::store(lds_a[buffer] + p * R::kElements, row, piece, x); });
    next_b.store([&](int p, int row, int piece, Eight x) { R::store(lds_b[buffer] + p * R::kElements, row, piece, x); });
    next_c.store([&](int p, int row, int piece, Eight x) { Cs::store(lds_c[buffer] + p * Cs::kElements, row, piece, x); });
    __syncthreads();  // of two buffers, the other one was read before the barrier of the chunk before this one
    if (at + kChunk < seg.length) load(at + kChunk);

    Eight turned_c[2][kInput];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int p = 0; p < kInput; ++p) turned_c[k][p] = Cs::across(lds_c[buffer] + p * Cs::kElements, wave, k, lane);

    if constexpr (OUT) {
      Block shares, out;
#pragma unroll
      for (int e = 0; e < 16; ++e) shares[e] = out[e] = 0.0f;
      // the rows' next elements are read while these are multiplied, and no sooner: registers
      Eight row_a[2][kInput], row_b[2][kInput];
      auto read = [&](int k) {
#pragma unroll
        for (int p = 0; p < kInput; ++p) {
          row_a[k % 2][p] = R::along(lds_a[buffer] + p * R::kElements, k, lane);
          row_b[k % 2][p] = R::along(lds_b[buffer] + p * R::kElements, k, lane);
        }
      };
      read(0);
#pragma unroll
      for (int k = 0; k < 2 * kBlocks; ++k) {
        if (k + 1 < 2 * kBlocks) read(k + 1);
        multiply_parts<3>(row_b[k % 2], row_a[k % 2], shares);
        Eight part[kMiddle];
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = state[k / 2][k % 2 * 8 + e];
        take_apart(s, part);
        multiply_parts<kWeight>(part, row_a[k % 2], out);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        out[e] *= query_weight;
        shares[e] *= share_weight[e];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Eight part[kMiddle];
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = shares[k * 8 + e];
        take_apart(s, part);
        multiply_parts<kWeight>(turned_c[k], part, out);
      }
      if ((lane & 31) < rows) {
        T* to = static_cast<T*>(w.out.data) + head * w.out.head_stride + (seg.row + sign * (at + (lane & 31))) * w.out.row_stride + column0 + 32 * wave;
        const bool whole = reinterpret_cast<uintptr_t>(w.out.data) % (4 * sizeof(T)) == 0 && (w.out.row_stride | w.out.head_stride) % 4 == 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = 8 * q + 4 * h, left = w.dc - column0 - 32 * wave - n;
          alignas(16) T four[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) four[j] = from_float<T>(out[4 * q + j] * w.out_scale);
          if (whole && left >= 4) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(to + n) = *reinterpret_cast<const uint4*>(four);
            else *reinterpret_cast<uint2*>(to + n) = *reinterpret_cast<const uint2*>(four);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (j < left) to[n + j] = four[j];
          }
        }
      }
    }

    if (rows < kChunk) {  // the segment's last chunk
#pragma unroll
      for (int e = 0; e < 16; ++e) state_weight[e / 8][e % 8] = d.power(rows - 1 - (8 * (e / 4) + 4 * h + e % 4) + w.late) * w.scale;
    }
    const float kept = d.power(rows);
    Eight into[2][kIntoState];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = 0.0f;
#pragma unroll
        for (int p = kInput - 1; p >= 0; --p) x[e] += (float)turned_c[k][p][e];
        x[e] *= state_weight[k][e];
      }
      take_apart(x, into[k]);
    }
    Eight turned_b[2][kInput];
    auto read = [&](int k) {
#pragma unroll
      for (int p = 0; p < kInput; ++p) turned_b[k % 2][p] = R::across(lds_b[buffer] + p * R::kElements, k / 2, k % 2, lane);
    };
    read(0);
#pragma unroll
    for (int k = 0; k < 2 * kBlocks; ++k) {
      if (k + 1 < 2 * kBlocks) read(k + 1);
      if (k % 2 == 0) state[k / 2] *= kept;
      multiply_parts<kWeightIn>(turned_b[k % 2], into[k % 2], state[k / 2]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  float* to = OUT ? (seg.last && w.last ? w.last + (seg.sequence * w.heads + head) * w.da * w.dc : nullptr)
                  : slots.states + ((seg.slot + 1) * w.heads + head) * w.da * w.dc;
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 32 * i + 8 * (e / 4) + 4 * h + e % 4;
      if (to && r < w.da && column < w.dc) to[(int64_t)r * w.state_a + (int64_t)column * w.state_c] = state[i][e];
    }
}

// What the segments of a sequence add, joined to the state in front of each: slot i + 1 of a sequence holds what its segment i
// adds, and is left with the state in front of segment i + 1.  A thread to an element; a few segments' loads on their way.
__global__ __launch_bounds__(256) void join_kernel(const WalkArgs w, const Slots slots) {
  constexpr int kAhead = 8;
  const int64_t size = (int64_t)w.da * w.dc, groups = (size + 255) / 256;
  const int head = (int)(blockIdx.x / groups % w.heads);
  const int64_t sequence = blockIdx.x / groups / w.heads, element = blockIdx.x % groups * 256 + threadIdx.x;
  const int64_t length = Segment::rows_of(w, sequence).length, segments = (length + slots.steps - 1) / slots.steps;
  if (element >= size) return;
  const float kept = Decay{w.log_decay[head] * 1.44269504f}.power(slots.steps);
  float state = w.first ? w.first[(sequence * w.heads + head) * size + element] : 0.0f;
  float* at = slots.states + ((Segment::first_slot(w, sequence, slots.steps) + 1) * w.heads + head) * size + element;
  for (int64_t i = 0; i + 1 < segments; i += kAhead) {
    float added[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) added[j] = i + j + 1 < segments ? at[(i + j) * w.heads * size] : 0.0f;
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i + j + 1 < segments) {
        state = fmaf(kept, state, added[j]);
        at[(i + j) * w.heads * size] = state;
      }
  }
}

template <typename T, int DA, bool OUT>
hipError_t launch_chunks(const WalkArgs& w, const Slots& slots, hipStream_t stream) {
  const int waves = w.dc <= 32 ? 1 : w.dc <= 64 ? 2 : 4;
  const uint32_t groups = (uint32_t)(slots.count * w.heads * ((w.dc + 32 * waves - 1) / (32 * waves)));
  if (waves == 1) walk_chunks_kernel<T, DA, 1, OUT><<<groups, 64, 0, stream>>>(w, slots);
  else if (waves == 2) walk_chunks_kernel<T, DA, 2, OUT><<<groups, 128, 0, stream>>>(w, slots);
  else walk_chunks_kernel<T, DA, 4, OUT><<<groups, 256, 0, stream>>>(w, slots);
  return hipGetLastError();
}

template <typename T, bool OUT>
hipError_t launch_chunks(const WalkArgs& w, const Slots& slots, hipStream_t stream) {
  return w.da <= 64 ? launch_chunks<T, 64, OUT>(w, slots, stream) : w.da <= 128 ? launch_chunks<T, 128, OUT>(w, slots, stream) : launch_chunks<T, 256, OUT>(w, slots, stream);
}

template <bool OUT>
hipError_t launch_chunks(const WalkArgs& w, const Slots& slots, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return launch_chunks<float, OUT>(w, slots, stream);
    case DGC_F16: return launch_chunks<_Float16, OUT>(w, slots, stream);
    default: return launch_chunks<__bf16, OUT>(w, slots, stream);
  }
}

constexpr int64_t kStepsAtMost = 4;      // of sequences that go step by step
constexpr int64_t kWorkgroups = 512;     // that fill the device
constexpr int64_t kSegmentLeast = 256;

Slots slots_of(int64_t rows, int64_t sequences, int64_t max_length, int32_t heads, int32_t dims, void* workspace) {
  Slots s{sequences, 0, static_cast<float*>(workspace)};
  const int64_t tiles = (dims + 127) / 128, whole = sequences * heads * tiles;
  if (max_length <= 2 * kSegmentLeast || whole >= kWorkgroups / 2) return s;
  // as many segments as fill the device, of kSegmentLeast steps at least
  const int64_t wanted = std::max<int64_t>(1, kWorkgroups / (heads * tiles));
  s.steps = std::max(kSegmentLeast, (rows / wanted + kChunk - 1) / kChunk * kChunk);
  if (s.steps >= max_length) s.steps = 0;
  else s.count = rows / s.steps + sequences;
  return s;
}

}  // namespace

int64_t walk_workgroups(int64_t sequences, int32_t heads, int32_t dc) {
  return sequences * heads * ((dc + kColumns - 1) / kColumns);
}

size_t walk_workspace_bytes(int64_t rows, int64_t sequences, int64_t max_length, int32_t heads, int32_t da, int32_t dc) {
  const Slots s = slots_of(rows, sequences, max_length, heads, std::max(da, dc), nullptr);
  return s.steps == 0 ? 0 : ((size_t)(s.count + 1) * heads * da * dc * 4 + 255) / 256 * 256;
}

hipError_t launch_walk_states(const WalkArgs& w, void* workspace, int32_t dtype, hipStream_t stream) {
  const Slots slots = slots_of(w.rows, w.sequences, w.max_length, w.heads, std::max(w.da, w.dc), workspace);
  if (slots.steps == 0) return hipSuccess;
  const hipError_t err = launch_chunks<false>(w, slots, dtype, stream);
  if (err != hipSuccess) return err;
  const int64_t groups = ((int64_t)w.da * w.dc + 255) / 256;
  join_kernel<<<(uint32_t)(w.sequences * w.heads * groups), 256, 0, stream>>>(w, slots);
  return hipGetLastError();
}

hipError_t launch_walk(const WalkArgs& w, void* workspace, int32_t dtype, hipStream_t stream) {
  if (w.max_length > kStepsAtMost) return launch_chunks<true>(w, slots_of(w.rows, w.sequences, w.max_length, w.heads, std::max(w.da, w.dc), workspace), dtype, stream);
  const uint32_t groups = (uint32_t)walk_workgroups(w.sequences, w.heads, w.dc);
  switch (dtype) {
    case DGC_F32: walk_steps_kernel<float><<<groups, kThreads, 0, stream>>>(w); break;
    case DGC_F16: walk_steps_kernel<_Float16><<<groups, kThreads, 0, stream>>>(w); break;
    default: walk_steps_kernel<__bf16><<<groups, kThreads, 0, stream>>>(w); break;
  }
  return hipGetLastError();
}

}  // namespace dgc
