// Linear attention with a decay for each head, and its gradients.
//
// All of it is one operator (WalkArgs).  Short sequences go step by step; others by chunks of 32 steps, in which
//   out = (a b^T o D) c + d^(i+1) a S,      S <- d^32 S + (d^(31-j) b)^T c
// are products of matrices.  The matrix units take bfloat16: what is in 16 or 32 bits is taken apart into bfloat16 parts (one
// of a bfloat16, two of a binary16, three of a binary32; the shares a b^T and the state two, or three for 32-bit results;
// what goes into the state three), whose products are exact and are summed in binary32.  Parts are cut off, so that none
// passes the type's end, and the last one is rounded: two parts leave 2^-15 of a value out, three 2^-23.  A result in 16 bits,
// which is rounded to 2^-9 or 2^-12 at the end, is formed from two, one in 32 bits and every state from three.

#include <algorithm>
#include <type_traits>

#include "dgc_device.h"
#include "dgc_layers.h"

namespace dgc {
namespace {

struct Walks {  // of one launch
  WalkArgs walk[kWalksMax];
  int32_t count;
  uint32_t first;  // place of the launch's first workgroup
};

// Which walk a workgroup takes part in, and as which of a walk's workgroups.  Those of several walks that read the same rows
// stand side by side, on one die (workgroups go to the eight dies in turn), so that one's rows are in its cache for the others.
__device__ __forceinline__ int64_t place(const Walks& walks, int& walk) {
  const uint32_t at = walks.first + blockIdx.x, round = 8 * (uint32_t)walks.count, in = at % round;
  walk = (int)(in / 8);
  return (int64_t)(at / round) * 8 + in % 8;
}
inline uint32_t places(int64_t groups, int count) { return (uint32_t)((groups + 7) / 8 * 8 * count); }

// A launch has less than 2^32 threads: workgroups beyond them, of very many sequences, are launched behind the others.
template <int THREADS, typename... More>
void launch_places(void (*kernel)(Walks, More...), Walks walks, uint32_t places, hipStream_t stream, More... more) {
  constexpr uint32_t kMost = UINT32_MAX / THREADS;
  for (uint32_t left = places; left > 0;) {
    const uint32_t groups = std::min(left, kMost);
    walks.first = places - left;
    kernel<<<groups, THREADS, 0, stream>>>(walks, more...);
    left -= groups;
  }
}

// ---- steps -------------------------------------------------------------------------------------
constexpr int kColumns = 32;  // columns of the state to a workgroup at least
constexpr int kThreads = 256;

// One step after the other: what bounds it is the state, which is read and written once.  A thread has four of COLUMNS columns
// and up to ROWS of their rows in registers; o is summed over the rows of a wavefront by exchanges, over the wavefronts in LDS,
// in their order.  Everything that a step reads is asked for at once.
template <typename T, int COLUMNS, int ROWS>
__global__ __launch_bounds__(kThreads) void walk_steps_kernel(const Walks walks) {
  constexpr int kRowThreads = kThreads * 4 / COLUMNS, kRows = ROWS;  // a thread's rows are kRowThreads apart
  int which;
  const int64_t group = place(walks, which);
  const WalkArgs& w = walks.walk[which];
  __shared__ float4 sums[2][kThreads / 64][COLUMNS / 4];
  const int tiles = (w.dc + COLUMNS - 1) / COLUMNS;
  const int tile = (int)(group % tiles), head = (int)(group / tiles % w.heads);
  const int64_t sequence = group / tiles / w.heads;
  if (sequence >= w.sequences) return;  // whole rounds of the dies, and the walk with the most tiles
  const int64_t lo = w.row_offsets ? w.row_offsets[sequence] : sequence * w.max_length;
  const int64_t hi = w.row_offsets ? w.row_offsets[sequence + 1] : lo + w.max_length;
  const SequenceRows rows(lo, hi, w.rows, w.max_length);
  const int column = tile * COLUMNS + 4 * ((int)threadIdx.x % (COLUMNS / 4)), row0 = (int)threadIdx.x / (COLUMNS / 4);
  const int columns = w.dc - column;  // that are there, from this thread's first on
  const bool whole = columns >= 4 && w.state_c == 1 && w.state_a % 4 == 0;
  const bool whole_first = whole && reinterpret_cast<uintptr_t>(w.first) % 16 == 0, whole_last = whole && reinterpret_cast<uintptr_t>(w.last) % 16 == 0;
  const int64_t at = (sequence * w.heads + head) * w.da * w.dc + (int64_t)column * w.state_c;
  float s[kRows][4];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = row0 + i * kRowThreads;
    const float* from = w.first + at + (int64_t)r * w.state_a;
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
    if (!w.first || r >= w.da) continue;
    if (whole_first) {
      const float4 x = *reinterpret_cast<const float4*>(from);
      s[i][0] = x.x, s[i][1] = x.y, s[i][2] = x.z, s[i][3] = x.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < columns) s[i][j] = from[(int64_t)j * w.state_c];
    }
  }
  const float d = exp2f(w.log_decay[head] * 1.44269504f), before = w.late ? 1.0f : d, after = w.late ? d : 1.0f;
  const T* a = static_cast<const T*>(w.a.data) + head * w.a.head_stride;
  const T* b = static_cast<const T*>(w.b.data) + head * w.b.head_stride;
  const T* c = static_cast<const T*>(w.c.data) + head * w.c.head_stride + column;
  T* out = static_cast<T*>(w.out.data) + head * w.out.head_stride + column;
  for (int64_t t = 0; t < rows.length; ++t) {
    const int64_t row = rows.begin + (w.reverse ? rows.length - 1 - t : t);
    float x[kRows], y[kRows], z[4], sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = row0 + i * kRowThreads;
      x[i] = r < w.da ? to_float(a[row * w.a.row_stride + r]) : 0.0f;
      y[i] = r < w.da ? to_float(b[row * w.b.row_stride + r]) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = j < columns ? to_float(c[row * w.c.row_stride + j]) * w.scale : 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (row0 + i * kRowThreads < w.da)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = fmaf(y[i], z[j], before * s[i][j]);
          sum[j] = fmaf(x[i], s[i][j], sum[j]);
          s[i][j] *= after;
        }
#pragma unroll
    for (int m = COLUMNS / 4; m < 64; m *= 2)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += __shfl_xor(sum[j], m);
    // of two rows of sums the other one may still be read
    if (threadIdx.x % 64 < COLUMNS / 4) sums[t & 1][threadIdx.x / 64][threadIdx.x % 64] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (threadIdx.x < COLUMNS / 4) {
      for (int i = 1; i < kThreads / 64; ++i) {
        const float4 other = sums[t & 1][i][threadIdx.x];
        sum[0] += other.x, sum[1] += other.y, sum[2] += other.z, sum[3] += other.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < columns) out[row * w.out.row_stride + j] = from_float<T>(sum[j] * w.out_scale);
    }
  }
  if (!w.last) return;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = row0 + i * kRowThreads;
    float* to = w.last + at + (int64_t)r * w.state_a;
    if (r >= w.da) continue;
    if (whole_last) {
      *reinterpret_cast<float4*>(to) = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < columns) to[(int64_t)j * w.state_c] = s[i][j];
    }
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
  __device__ __forceinline__ float power(int n) const { return n > 0 ? __builtin_amdgcn_exp2f((float)n * log2) : 1.0f; }
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

// 16 bytes at any element's address, which loads take.
typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));

// Pieces of 8 elements of a chunk's rows on their way from memory to LDS, by THREADS threads.  NARROW: of rows that may be
// shorter than a piece, element by element; were both ways in one kernel, what they leave in registers would be waited for
// where they meet.
template <typename T, int DIM, int THREADS, bool NARROW>
struct Pieces {
  static constexpr int kCount = kChunk * DIM / 8 / THREADS;
  static_assert(kCount * THREADS * 8 == kChunk * DIM, "whole pieces");
  alignas(16) T held[kCount][8];
  uint32_t offset[kCount];  // bytes from the chunk's row with the lowest address

  static __device__ __forceinline__ int row(int i) { return (i * THREADS + (int)threadIdx.x) / (DIM / 8); }
  static __device__ __forceinline__ int column(int i) { return (i * THREADS + (int)threadIdx.x) % (DIM / 8) * 8; }

  // Elements from `first` on, `dim` of them to the end, of rows that are `stride` elements apart.  Every piece is loaded, one
  // that is not there from a place that is, and what is wrong with it is put right when it is stored: were loads masked, or
  // two ways of loading in one kernel, the registers they leave would be waited for here.  A piece that the row ends in is
  // loaded as the row's last eight elements, which may begin in front of `first`, but not of the row.
  __device__ __forceinline__ void start(int64_t stride, int first, int dim, bool reverse, int skipped) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int there = row(i) < skipped ? skipped : row(i);
      const int at = first + (NARROW ? (column(i) < dim ? column(i) : 0) : column(i) + 8 <= dim ? column(i) : dim - 8);
      offset[i] = ((uint32_t)(reverse ? kChunk - 1 - there : there) * (uint32_t)stride + (uint32_t)at) * (uint32_t)sizeof(T);
    }
  }
  // The chunk whose row with the lowest address is at `lowest`.
  __device__ __forceinline__ void load(const T* lowest, int dim) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const char* from = reinterpret_cast<const char*>(lowest) + offset[i];
      if constexpr (!NARROW) {
#pragma unroll
        for (int w = 0; w < (int)sizeof(T) / 2; ++w) reinterpret_cast<Loose*>(held[i])[w] = reinterpret_cast<const Loose*>(from)[w];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) held[i][j] = column(i) + j < dim ? reinterpret_cast<const T*>(from)[j] : (T)0.0f;
      }
    }
  }
  // Zeros for rows in front of `skipped` and elements behind the row's end.
  template <typename Store>
  __device__ __forceinline__ void store(int dim, int skipped, Store put) {
    const bool right = dim >= DIM && skipped == 0;  // nothing is wrong
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      if (!right) {
        const int left = row(i) < skipped ? 0 : dim - column(i);
        const int down = !NARROW && left > 0 && left < 8 ? 8 - left : 0;
#pragma unroll
        for (int by = 4; by > 0; by /= 2)
#pragma unroll
          for (int j = 0; j < 8; ++j) held[i][j] = down & by ? (j + by < 8 ? held[i][(j + by) & 7] : (T)0.0f) : held[i][j];
#pragma unroll
        for (int j = 0; j < 8; ++j) held[i][j] = left > 0 ? held[i][j] : (T)0.0f;
      }
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
      for (int p = 0; p < kPartsOf<T>; ++p) put(p, row(i), column(i) / 8, parts[p]);
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
  bool last;                            // of its sequence

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
};

// A workgroup walks a segment of a sequence for one head and WAVES * 32 columns of c, a wavefront with 32 columns of the state
// in its registers.  OUT: out and, behind the sequence's last segment, `last`; otherwise what the segment adds to the state.
//
// Of a chunk every wavefront forms a b^T for itself, as 32 x 32 shares whose layout is that of the operand they are next, and
// so is the state's: neither goes through LDS.  While a chunk is worked on the next one's rows are on their way to registers.
//
// Bound by memory and by issue alike: 65536 steps of 16 heads of 128 x 128 in bfloat16, forward and backward, ask for 18 and write
// 4 arrays of 268 MB (4.5 GB come from memory) in 1560 to 1620 us; without loads 1340, without stores 1410, with neither product
// 1170 to 1280.  By the profiler's counters vector instructions take 60 % of the cycles and products 43 %.
template <typename T, int DA, int WAVES, bool OUT, bool NARROW>
__global__ __launch_bounds__(64 * WAVES, DA <= 128 && sizeof(T) == 2 ? 2 : 1) void walk_chunks_kernel(const Walks walks, const Slots slots) {
  int which;
  const int64_t group = place(walks, which);
  const WalkArgs& w = walks.walk[which];
  constexpr int kThreads = 64 * WAVES, kInput = kPartsOf<T>, kMiddle = kMiddleParts<T>, kBlocks = DA / 32, DC = 32 * WAVES;
  constexpr int kWeight = __is_same(T, __bf16) ? 2 : 3, kWeightIn = 3;
  using R = Rows<DA>;
  using Cs = Columns<DC>;
  // two buffers where they leave room for a second workgroup, or fit at all
  constexpr int kBuffers = kInput * (2 * R::kElements + Cs::kElements) * 2 <= 40960 ? 2 : 1;
  __shared__ __align__(16) __bf16 lds_a[kBuffers][OUT ? kInput * R::kElements : 8], lds_b[kBuffers][kInput * R::kElements], lds_c[kBuffers][kInput * Cs::kElements];
  constexpr int kPitch = 40;
  __shared__ __align__(16) T staged[OUT && sizeof(T) == 2 ? WAVES : 1][OUT && sizeof(T) == 2 ? kChunk * kPitch : 8];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane >> 5;
  const int tiles = (w.dc + DC - 1) / DC;
  const int tile = (int)(group % tiles), head = (int)(group / tiles % w.heads);
  if (group / tiles / w.heads >= slots.count) return;  // whole rounds of the dies, and the walk with the most tiles
  const Segment seg(w, group / tiles / w.heads, slots.steps);
  if (seg.length < 0 || (!OUT && seg.last)) return;
  const int column0 = tile * DC, column = column0 + 32 * wave + (lane & 31);
  const Decay d{w.log_decay[head] * 1.44269504f};

  Block state[kBlocks];
  // Where sequences are cut, a first segment has its state from the workspace too: the last one may leave `last` in its place.
  const float* from = !OUT ? nullptr : slots.steps > 0 ? w.states + (seg.slot * w.heads + head) * w.da * w.dc : w.first ? w.first + (seg.sequence * w.heads + head) * w.da * w.dc : nullptr;
  if (from) from += (int64_t)(4 * h) * w.state_a + (int64_t)column * w.state_c;
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool there = from && 32 * i + 8 * q + 4 * h + j < w.da && column < w.dc;
        state[i][4 * q + j] = there ? from[(32 * i + 8 * q + j) * w.state_a] : 0.0f;
      }

  const int64_t sign = w.reverse ? -1 : 1;
  const T* a = OUT ? static_cast<const T*>(w.a.data) + head * w.a.head_stride : nullptr;
  const T* b = static_cast<const T*>(w.b.data) + head * w.b.head_stride;
  const T* c = static_cast<const T*>(w.c.data) + head * w.c.head_stride;

  const int64_t step_out = sign * w.out.row_stride;
  T* out_rows = OUT ? static_cast<T*>(w.out.data) + head * w.out.head_stride + seg.row * w.out.row_stride + column0 + 32 * wave : nullptr;

  // Weights.  Of a share of step j in step i = lane % 32: d^(i - j), from LDS at j - i + 31, zeros behind 31.  Of a step j that
  // goes into the state: d^(31 - j); of the lane's eight, j = 16 k + 4 h + {0 .. 3, 8 .. 11}, a power of its own for either k,
  // times one that all lanes have.  A segment's first chunk is the short one, if one is, and takes the window's end.
  __shared__ float share_weights[2 * kChunk];
  if (threadIdx.x < 2 * kChunk) share_weights[threadIdx.x] = threadIdx.x < kChunk ? d.power(kChunk - 1 - (int)threadIdx.x) * w.scale : 0.0f;
  const int behind = 4 * h - (lane & 31) + kChunk - 1;
  float uniform[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) uniform[e] = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, d.power(e < 4 ? 11 - e : 7 - e) * w.scale)));
  const float into_weight[2] = {d.power(20 - 4 * h + w.late), d.power(4 - 4 * h + w.late)};
  const int short_by = (int)(-seg.length & (kChunk - 1));
  // The state in registers is the state without the decay of the last `since` steps, `factor`: to multiply all of it once a
  // chunk would be a tenth of the arithmetic.  Decays that leave less than 2^-20 are caught up with.
  float query_weight = d.power((lane & 31) - short_by + 1 - w.late), factor = 1.0f;
  int since = 0;

  Pieces<T, DA, kThreads, NARROW> next_a, next_b;
  Pieces<T, DC, kThreads, NARROW> next_c;
  const int64_t stride_a = w.a.row_stride, stride_b = w.b.row_stride, stride_c = w.c.row_stride;
  const bool reverse = w.reverse;
  const int da = w.da, dc = w.dc - column0;
  auto start = [&](int skipped) {
    if constexpr (OUT) next_a.start(stride_a, 0, da, reverse, skipped);
    next_b.start(stride_b, 0, da, reverse, skipped);
    next_c.start(stride_c, column0, dc, reverse, skipped);
  };
  auto load = [&](int64_t at) {
    const int64_t lowest = seg.row + (reverse ? -at - (kChunk - 1) : at);
    if constexpr (OUT) next_a.load(a + lowest * stride_a, da);
    next_b.load(b + lowest * stride_b, da);
    next_c.load(c + lowest * stride_c, dc);
  };
  start(short_by);
  if (seg.length > 0) load(-short_by);
  start(0);
  int buffer = 0;
  for (int64_t at = -short_by; at < seg.length; at += kChunk, buffer = (buffer + 1) % kBuffers) {
    const int skipped = at < 0 ? short_by : 0;
    if (kBuffers == 1) __syncthreads();
    if constexpr (OUT) next_a.store(da, skipped, [&](int p, int row, int piece, Eight x) { R::store(lds_a[buffer] + p * R::kElements, row, piece, x); });
    next_b.store(da, skipped, [&](int p, int row, int piece, Eight x) { R::store(lds_b[buffer] + p * R::kElements, row, piece, x); });
    next_c.store(dc, skipped, [&](int p, int row, int piece, Eight x) { Cs::store(lds_c[buffer] + p * Cs::kElements, row, piece, x); });
    __syncthreads();  // of two buffers, the other one was read before the barrier of the chunk before this one
    if (at + kChunk < seg.length) load(at + kChunk);
    __builtin_amdgcn_sched_barrier(0);

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
      // and the state's next elements are taken apart: a product of matrices occupies its unit for as long as the other one
      // takes for eight instructions, so that a third of them goes behind each of three products
      Eight part[2][kMiddle];
      auto apart = [&](int k) {
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = state[k / 2][k % 2 * 8 + e];
        take_apart(s, part[k % 2]);
      };
      read(0);
      apart(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 2 * kBlocks; ++k) {
        if (k + 1 < 2 * kBlocks) {
          read(k + 1);
          apart(k + 1);
        }
        multiply_parts<3>(row_b[k % 2], row_a[k % 2], shares);
        multiply_parts<kWeight>(part[k % 2], row_a[k % 2], out);
        if constexpr (__is_same(T, __bf16)) {
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      const float query = query_weight * factor;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        out[e] *= query;
        shares[e] *= share_weights[behind + 8 * (e / 4) + e % 4];
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
      float result[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) result[e] = out[e] * w.out_scale;
      if constexpr (sizeof(T) == 2) {
        // Through LDS, so that a lane has 16 bytes of a row and a store 64 bytes of each row that it meets.  As the lanes hold
        // them, 8 bytes of 32 rows each, a chunk is four times as many requests to the cache: 65536 x 16 x 128 forward and
        // backward 1650 us, this way 1575.
        T* mine = staged[wave];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          Pack<T, 4> four;
          const float x[4] = {result[4 * q], result[4 * q + 1], result[4 * q + 2], result[4 * q + 3]};
          four.set(x);
          *reinterpret_cast<Pack<T, 4>*>(mine + (lane & 31) * kPitch + 8 * q + 4 * h) = four;
        }
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = i * 16 + lane / 4, piece = lane % 4 * 8, left = w.dc - column0 - 32 * wave - piece;
          const T* from = mine + row * kPitch + piece;
          T* to = out_rows + (at + row) * step_out + piece;
          if (at + row < 0) continue;
          if (left >= 8) {
            *reinterpret_cast<Loose*>(to) = *reinterpret_cast<const Words*>(from);
          } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
              if (j < left) to[j] = from[j];
          }
        }
        wave_lds_fence();
      } else if (at + (lane & 31) >= 0) {
        // 16 bytes of 32 rows each; through LDS 20 x 350 x 12 x 64 took 196 us instead of 142, in more registers
        T* to = out_rows + (at + (lane & 31)) * step_out;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = 8 * q + 4 * h, left = w.dc - column0 - 32 * wave - n;
          if (left >= 4) {
            const float4 x = make_float4(result[4 * q], result[4 * q + 1], result[4 * q + 2], result[4 * q + 3]);
            *reinterpret_cast<Loose*>(to + n) = __builtin_bit_cast(Loose, x);
          } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
              if (j < left) to[n + j] = result[4 * q + j];
          }
        }
      }
    }

    const float before = factor;
    since += at < 0 ? kChunk - short_by : kChunk;
    factor = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, d.power(since))));
    if (!(factor >= 0x1p-20f && factor <= 0x1p20f)) {
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) state[i] *= d.power(at < 0 ? kChunk - short_by : kChunk) * before;
      since = 0;
      factor = 1.0f;
    }
    const float inverse = __builtin_amdgcn_rcpf(factor), into_scale[2] = {into_weight[0] * inverse, into_weight[1] * inverse};
    Eight into[2][kIntoState];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = (float)turned_c[k][kInput - 1][e];
#pragma unroll
        for (int p = kInput - 2; p >= 0; --p) x[e] += (float)turned_c[k][p][e];
        x[e] *= into_scale[k] * uniform[e];
      }
      take_apart(x, into[k]);
    }
    __builtin_amdgcn_sched_barrier(0);
    Eight turned_b[2][kInput];
    auto read = [&](int k) {
#pragma unroll
      for (int p = 0; p < kInput; ++p) turned_b[k % 2][p] = R::across(lds_b[buffer] + p * R::kElements, k / 2, k % 2, lane);
    };
    read(0);
#pragma unroll
    for (int k = 0; k < 2 * kBlocks; ++k) {
      if (k + 1 < 2 * kBlocks) read(k + 1);
      multiply_parts<kWeightIn>(turned_b[k % 2], into[k % 2], state[k / 2]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (at < 0) query_weight = d.power((lane & 31) + 1 - w.late);
  }

  float* to = OUT ? (seg.last && w.last ? w.last + (seg.sequence * w.heads + head) * w.da * w.dc : nullptr)
                  : w.states + ((seg.slot + 1) * w.heads + head) * w.da * w.dc;
  // the compiler would keep the addresses of the first loads until here
  int again = lane;
  asm volatile("" : "+v"(again));
  const int column_again = column0 + 32 * wave + (again & 31);
  if (!to || column_again >= w.dc) return;
  float* first = to + (int64_t)(4 * (again >> 5)) * w.state_a + (int64_t)column_again * w.state_c;
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q, first += 8 * (int64_t)w.state_a)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (32 * i + 8 * q + 4 * (again >> 5) + j < w.da) first[j * w.state_a] = state[i][4 * q + j] * factor;
}

// What the segments of a sequence add, joined to the state in front of each: slot i + 1 of a sequence holds what its segment i
// adds, and slot i is left with the state in front of segment i.  A thread to an element; a few segments' loads on their way.
__global__ __launch_bounds__(256) void join_kernel(const Walks walks, const Slots slots) {
  const WalkArgs& w = walks.walk[blockIdx.y];
  constexpr int kAhead = 8;
  const int64_t size = (int64_t)w.da * w.dc, groups = (size + 255) / 256;
  const int head = (int)(blockIdx.x / groups % w.heads);
  const int64_t sequence = blockIdx.x / groups / w.heads, element = blockIdx.x % groups * 256 + threadIdx.x;
  const int64_t length = Segment::rows_of(w, sequence).length, segments = (length + slots.steps - 1) / slots.steps;
  if (element >= size) return;
  const float kept = Decay{w.log_decay[head] * 1.44269504f}.power((int)slots.steps);
  float state = w.first ? w.first[(sequence * w.heads + head) * size + element] : 0.0f;
  float* at = w.states + (Segment::first_slot(w, sequence, slots.steps) * w.heads + head) * size + element;
  *at = state;
  at += w.heads * size;
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

// What the kernels of a walk are made for: rows of the state and its columns to a workgroup, OUT: as above.
struct Made {
  int rows, waves;
  bool narrow;
  explicit Made(const WalkArgs& w) : rows(w.da <= 64 ? 64 : w.da <= 128 ? 128 : 256), waves(w.dc <= 32 ? 1 : w.dc <= 64 ? 2 : 4), narrow(w.da < 8 || w.dc < 8) {
    if (narrow) {
      waves = 4;
      if (rows == 128) rows = 256;
    }
  }
  bool operator==(const Made& o) const { return rows == o.rows && waves == o.waves && narrow == o.narrow; }
};

template <typename T, bool OUT>
void launch_chunks(const Walks& walks, int count, const Slots& slots, hipStream_t stream) {
  const Made made(walks.walk[0]);
  int32_t dc = 0;
  for (int i = 0; i < count; ++i) dc = std::max(dc, walks.walk[i].dc);
  const uint32_t grid = places(slots.count * walks.walk[0].heads * ((dc + 32 * made.waves - 1) / (32 * made.waves)), count);
  auto go = [&](auto rows, auto waves, auto narrow) {
    launch_places<64 * decltype(waves)::value>(walk_chunks_kernel<T, decltype(rows)::value, decltype(waves)::value, OUT, decltype(narrow)::value>, walks, grid, stream, slots);
  };
  auto with_waves = [&](auto rows) {
    if (made.waves == 1) go(rows, std::integral_constant<int, 1>(), std::false_type());
    else if (made.waves == 2) go(rows, std::integral_constant<int, 2>(), std::false_type());
    else go(rows, std::integral_constant<int, 4>(), std::false_type());
  };
  if (made.narrow && made.rows == 64) go(std::integral_constant<int, 64>(), std::integral_constant<int, 4>(), std::true_type());
  else if (made.narrow) go(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), std::true_type());
  else if (made.rows == 64) with_waves(std::integral_constant<int, 64>());
  else if (made.rows == 128) with_waves(std::integral_constant<int, 128>());
  else with_waves(std::integral_constant<int, 256>());
}

template <typename T>
void launch_steps(const Walks& walks, int count, hipStream_t stream) {
  // 128 columns to a workgroup where all walks have more than 64 of them, and up to 128 rows: 512 bytes of a row to a wavefront's
  // load, and a thread has 8 or 16 loads on their way (64 x 16 states of 64 x 128: 17.2 us, 3.9 TB/s; by 32 columns 22.8).  Of 64
  // columns half the threads would have none: 64 x 16 states of 64 x 64 by 32 columns 10.4 us, 3.2 TB/s, by 128 13.0; 256 x 16 30.7
  // and 40.6
  int32_t rows = 0, least = DGC_HEAD_MAX, most = 0;
  for (int i = 0; i < count; ++i) {
    rows = std::max(rows, walks.walk[i].da);
    least = std::min(least, walks.walk[i].dc);
    most = std::max(most, walks.walk[i].dc);
  }
  const int64_t heads = walks.walk[0].sequences * walks.walk[0].heads;
  auto go = [&](auto columns, auto held) {
    constexpr int kWide = decltype(columns)::value;
    launch_places<kThreads>(walk_steps_kernel<T, kWide, decltype(held)::value>, walks, places(heads * ((most + kWide - 1) / kWide), count), stream);
  };
  if (least > 64 && rows <= 64) go(std::integral_constant<int, 128>(), std::integral_constant<int, 8>());
  else if (least > 64 && rows <= 128) go(std::integral_constant<int, 128>(), std::integral_constant<int, 16>());
  else if (rows <= 64) go(std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
  else go(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
}

template <typename F>
void with_type(int32_t dtype, F f) {
  if (dtype == DGC_F32) f(0.0f);
  else if (dtype == DGC_F16) f((_Float16)0.0f);
  else f((__bf16)0.0f);
}

// A step that goes by itself costs a reduction and a barrier, a chunk of up to 32 some 5 us whatever it holds.
constexpr int64_t kStepsAtMost = 4;      // of sequences that go step by step
constexpr int64_t kWorkgroups = 512;     // that fill the device
constexpr int64_t kSegmentLeast = 128;   // steps; a state of 128 x 128 is as many bytes as 128 rows of k and v in bfloat16
constexpr int64_t kCutLongerThan = 512;  // steps of the longest sequence
constexpr int64_t kCutBelow = 136, kCutRaggedBelow = 256;  // workgroups without cutting, of sequences of one length and of different ones

// Cutting sequences into segments fills the device and shortens the longest one's chain of chunks, and reads k and v a second time.
// Both sides in us, cut and whole, forward / forward and backward:
//   equal sequences of 4096 x 128 x 128 bfloat16   64 workgroups 132 and 300 / 470 and 599, 128: 243 and 301 / 843 and 751,
//                                                  144: 327 and 302 / 1033 and 786, 192: 402 and 303 / 1283 and 1032
//   different ones, up to 4000 x 64 x 64 binary16  160: 176 and 355 / 556 and 736, 256: 323 and 358 / 974 and 1022,
//                  up to 1500                      384: 216 and 169 / 627 and 492
//   short ones                                     8 x 300 x 12 x 64 x 64 bfloat16 36 and 28 / 81 and 62, 2 x 512 x 16 x 128 x 128 43 and 47 / 99 and 94
//   segments of 128, and of 256 at least           1024 x 16 x 128 x 128 bfloat16 40 and 51 / 90 and 105, 4096 x 4 x 64 x 64 30 and 39 / 65 and 79;
//                  of 64                           35 / 96 and 28 / 64
Slots slots_of(int64_t rows, int64_t sequences, int64_t max_length, int32_t heads, int32_t dims, bool ragged) {
  Slots s{sequences, 0};
  const int64_t tiles = (dims + 127) / 128, whole = sequences * heads * tiles;
  if (max_length <= kCutLongerThan || whole >= (ragged ? kCutRaggedBelow : kCutBelow)) return s;
  // as many segments as fill the device, of kSegmentLeast steps at least
  const int64_t wanted = std::max<int64_t>(1, kWorkgroups / (heads * tiles));
  s.steps = std::max(kSegmentLeast, (rows / wanted + kChunk - 1) / kChunk * kChunk);
  if (s.steps >= max_length) s.steps = 0;
  else s.count = rows / s.steps + sequences;
  return s;
}

Slots slots_of(const WalkArgs& w) { return slots_of(w.rows, w.sequences, w.max_length, w.heads, std::max(w.da, w.dc), w.row_offsets != nullptr); }

// Calls f(walks, count) for the walks that one kernel can take together.
template <typename F>
void together(const WalkArgs* w, int count, F f) {
  bool done[kWalksMax] = {};
  for (int i = 0; i < count; ++i) {
    if (done[i]) continue;
    Walks walks{};
    int n = 0;
    for (int j = i; j < count; ++j)
      if (!done[j] && Made(w[j]) == Made(w[i])) {
        walks.walk[n++] = w[j];
        done[j] = true;
      }
    walks.count = n;
    f(walks, n);
  }
}

}  // namespace

int64_t walk_workgroups(int64_t sequences, int32_t heads, int32_t dc) {
  return sequences * heads * ((dc + kColumns - 1) / kColumns);
}

size_t walk_workspace_bytes(int64_t rows, int64_t sequences, int64_t max_length, int32_t heads, int32_t da, int32_t dc, bool ragged) {
  const Slots s = slots_of(rows, sequences, max_length, heads, std::max(da, dc), ragged);
  return s.steps == 0 ? 0 : ((size_t)(s.count + 1) * heads * da * dc * 4 + 255) / 256 * 256;
}

hipError_t launch_walk_states(const WalkArgs* w, int count, int32_t dtype, hipStream_t stream) {
  const Slots slots = slots_of(w[0]);
  if (slots.steps == 0) return hipSuccess;
  together(w, count, [&](const Walks& walks, int n) {
    with_type(dtype, [&](auto t) { launch_chunks<decltype(t), false>(walks, n, slots, stream); });
    const int64_t groups = ((int64_t)w[0].da * w[0].dc + 255) / 256;
    join_kernel<<<dim3((uint32_t)(w[0].sequences * w[0].heads * groups), (uint32_t)n), 256, 0, stream>>>(walks, slots);
  });
  return hipGetLastError();
}

hipError_t launch_walks(const WalkArgs* w, int count, int32_t dtype, hipStream_t stream) {
  if (w[0].max_length > kStepsAtMost) {
    together(w, count, [&](const Walks& walks, int n) {
      with_type(dtype, [&](auto t) { launch_chunks<decltype(t), true>(walks, n, slots_of(w[0]), stream); });
    });
  } else {
    Walks walks{};
    for (int i = 0; i < count; ++i) walks.walk[i] = w[i];
    walks.count = count;
    with_type(dtype, [&](auto t) { launch_steps<decltype(t)>(walks, count, stream); });
  }
  return hipGetLastError();
}

}  // namespace dgc
