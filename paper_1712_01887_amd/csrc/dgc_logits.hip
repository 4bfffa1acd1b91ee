// Operators on rows of logits: a teacher's largest ones as pairs, and the loss of a student against such pairs
// with its gradient.

#include "dgc_device.h"
#include "dgc_operators.h"

namespace dgc {
namespace {

constexpr float kLog2E = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kInf = __builtin_inff();

// A value that is the same in every lane, in a register of the wavefront's.
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Sum or maximum over the wavefront, the same in every lane.
__device__ __forceinline__ float wave_sum_f(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max_f(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// ---- a row ------------------------------------------------------------------------------------------------
// A workgroup of NT threads takes a row in vectors of 16 bytes, vector v by thread v mod NT: CH of them to a thread, which
// keeps them in registers from the row's only read on, or, with CH = 0 (rows longer than the registers hold), reads them
// again in every pass.  The few elements behind the last whole vector go to one thread each.  Places behind the row's end
// hold -inf.
template <typename T, int NT, int CH>
struct Row {
  static constexpr int E = 16 / (int)sizeof(T);
  using Vector = Pack<T, E>;
  struct __attribute__((packed, aligned(sizeof(T)))) Loose {  // a row starts where any element may
    Vector v;
  };
  Vector held[CH > 0 ? CH : 1];
  float rest;

  static __device__ __forceinline__ Vector nothing() {
    constexpr uint32_t word = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u;
    Vector p;
#pragma unroll
    for (int i = 0; i < Vector::kWords; ++i) p.w[i] = word;
    return p;
  }
  static __device__ __forceinline__ Vector load(const T* z, int v) { return reinterpret_cast<const Loose*>(z + (uint32_t)v * (uint32_t)E)->v; }
  // The whole vectors of a row as a buffer resource (data format 32, offsets in bytes): behind its end nothing is read or
  // stored, and so nowhere in the row of a null pointer.
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const T* z, int vocab) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)z, 0, z ? (int)((uint32_t)(vocab / E) * 16u) : 0, 0x00020000);
  }
  static __device__ __forceinline__ uint32_t offset(uint32_t thread, int i) { return (thread + (uint32_t)(i * NT)) * 16u; }
  // Vector i of this thread.
  __device__ __forceinline__ void read(__amdgpu_buffer_rsrc_t z, uint32_t thread, int i) {
    held[i] = __builtin_bit_cast(Vector, __builtin_amdgcn_raw_buffer_load_b128(z, offset(thread, i), 0, 0));
  }
  static __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t g, uint32_t thread, int i, const Vector& v) {
    typedef uint32_t four __attribute__((ext_vector_type(4)));
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(four, v), g, offset(thread, i), 0, 0);
  }
  __device__ __forceinline__ void read_rest(const T* z, int vocab) {
    const uint32_t at = (uint32_t)(vocab / E * E) + threadIdx.x;  // may pass 2^31
    rest = z && at < (uint32_t)vocab ? to_float(z[at]) : -kInf;
  }
  __device__ __forceinline__ void read(__amdgpu_buffer_rsrc_t from) {
#pragma unroll
    for (int i = 0; i < CH; ++i) read(from, threadIdx.x, i);
  }
  __device__ __forceinline__ void read(const T* z, int vocab) {
    read(buffer(z, vocab));
    read_rest(z, vocab);
  }
  // Piece k of NT x CH vectors of a longer row.
  __device__ __forceinline__ void read_piece(const T* z, int whole, int k) {
    const int first = k * NT * CH, vectors = whole - first < NT * CH ? whole - first : NT * CH;
    read(buffer(z ? z + (int64_t)first * E : nullptr, vectors * E));
  }
  __device__ __forceinline__ void cut_piece(int whole, int k) { cut((whole - k * NT * CH) * E); }
  // Before a row that was read is used: its end.
  __device__ __forceinline__ void cut(int vocab) {
    const int whole = vocab / E;
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if ((i + 1) * NT > whole) {
        const Vector none = nothing();
#pragma unroll
        for (int j = 0; j < Vector::kWords; ++j) held[i].w[j] = i * NT + (int)threadIdx.x < whole ? held[i].w[j] : none.w[j];
      }
  }
  // Between two passes: what the first has made of the elements is not kept, it would take several times the registers.
  __device__ __forceinline__ void renew() {
#pragma unroll
    for (int i = 0; i < CH; ++i) held[i].renew();
  }
  // f(vector, its number) for every vector of this thread
  template <typename F>
  __device__ __forceinline__ void each(const T* z, int vocab, F f) const {
    if constexpr (CH > 0) {
#pragma unroll
      for (int i = 0; i < CH; ++i) f(held[i], i * NT + (int)threadIdx.x);
    } else {
      const int whole = vocab / E;
#pragma unroll 4
      for (int v = threadIdx.x; v < whole; v += NT) f(load(z, v), v);
    }
  }
  __device__ __forceinline__ float largest(const T* z, int vocab) const {
    float m = rest;
    each(z, vocab, [&](const Vector& p, int) {
#pragma unroll
      for (int j = 0; j < E; ++j) m = fmaxf(m, p.get(j));
    });
    return m;
  }
};

// What the wavefronts of a workgroup leave for each other.
template <int NT>
struct Between {
  float largest[NT / 64];
  float2 sums[NT / 64];
  __device__ __forceinline__ float max_of() const {
    float m = largest[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) m = fmaxf(m, largest[i]);
    return uniform(m);
  }
  __device__ __forceinline__ float2 sum_of() const {
    float2 s = sums[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) s.x += sums[i].x, s.y += sums[i].y;
    return float2{uniform(s.x), uniform(s.y)};
  }
};

// ---- top logits ---------------------------------------------------------------------------------------------
// A whole number that orders as the logits do, zero for those that are never chosen (NaN, -inf); both zeros are one.
__device__ __forceinline__ uint32_t order_key(float z) {
  if (!(z > -kInf)) return 0u;
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// LDS of a workgroup.  Two keys to a thread where there are few threads: with no more keys than k, the floor would be the
// least of them.
template <int NT>
struct TopShared {
  static constexpr int kCandidates = NT < 256 ? 512 : 1024, kVectors = NT < 256 ? 128 : 1024, kKeys = NT <= 256 ? 2 * NT : NT;
  float2 sums[NT / 64];                        // largest and sum of the wavefronts
  uint4 vectors[kVectors];                     // those with an element that reaches the floor
  int32_t numbers[kVectors];
  unsigned long long candidates[kCandidates];  // key, then index from the highest
  uint32_t rank[kCandidates];
  uint32_t keys[kKeys];
  uint32_t histogram[256];
  uint32_t totals[NT / 64];
  uint32_t floor, count, hits, prefix, wanted;
};

// A key that at least k of the `n` keys in LDS reach, its low 16 bits zero; 1 if fewer than k are not zero.  One wavefront.
template <int N>
__device__ __forceinline__ uint32_t floor_of(const uint32_t* keys, int k, int lane) {
  constexpr int kEach = (N + 63) / 64;
  uint32_t mine[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine[i] = i * 64 + lane < N ? keys[i * 64 + lane] : 0u;
  uint32_t found = 0;
  for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
    const uint32_t probe = found | bit;
    int passed = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) passed += __popcll(__ballot(mine[i] >= probe));
    if (passed >= k) found = probe;
  }
  return found ? found : 1u;
}

// The value of a lane of the same four: the neighbour's (0xb1) or that of the other two (0x4e).
template <int PERM>
__device__ __forceinline__ float neighbour(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), PERM, 0xf, 0xf, false));
}

// Of the vectors listed, those that still reach the floor.
template <typename T, int NT>
__device__ __forceinline__ void thin_out(TopShared<NT>& s, uint32_t listed, float least) {
  constexpr int kVectors = TopShared<NT>::kVectors, kEach = kVectors / NT > 0 ? kVectors / NT : 1, E = 16 / (int)sizeof(T);
  uint4 mine[kEach];
  int32_t number[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const uint32_t at = (uint32_t)(i * NT) + threadIdx.x;
    if (at < listed) mine[i] = s.vectors[at], number[i] = s.numbers[at];
  }
  if (threadIdx.x == 0) s.hits = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if ((uint32_t)(i * NT) + threadIdx.x < listed) {
      const Pack<T, E> p = __builtin_bit_cast(Pack<T, E>, mine[i]);
      float m = p.get(0);
#pragma unroll
      for (int j = 1; j < E; ++j) m = fmaxf(m, p.get(j));
      if (m >= least) {
        const uint32_t at = atomicAdd(&s.hits, 1u);
        s.vectors[at] = mine[i];
        s.numbers[at] = number[i];
      }
    }
  }
  __syncthreads();
}

// So many threads to a candidate that all have work, each with its share of the others to compare with, four of them at a
// time; a single wavefront with several candidates to a lane looks at what it has read for HELD of them (4096 rows of 500 in
// bfloat16 to their 256 largest: one by one 357 us, others in fours 164, HELD = 4 too 100; 2048 x 131072 to 256: 188 and 160).
template <int NT, uint32_t HELD>
__device__ __forceinline__ void count_better(TopShared<NT>& s, uint32_t n, uint32_t span) {
  const uint32_t parts = span >= NT || span == 0 ? 1u : NT / span;  // a power of two
  for (uint32_t t = threadIdx.x; t < span * parts; t += NT * HELD) {
    const uint32_t part = t / span, c = t - part * span;
    unsigned long long key[HELD];
    uint32_t better[HELD];
#pragma unroll
    for (uint32_t m = 0; m < HELD; ++m) key[m] = s.candidates[c + m * NT < span ? c + m * NT : c], better[m] = 0;
#pragma unroll 1
    for (uint32_t i = part; i < n; i += 4 * parts) {
      const unsigned long long others[4] = {s.candidates[i], s.candidates[i + parts], s.candidates[i + 2 * parts], s.candidates[i + 3 * parts]};
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (uint32_t m = 0; m < HELD; ++m) better[m] += others[j] > key[m];
    }
#pragma unroll
    for (uint32_t m = 0; m < HELD; ++m)
      if (c + m * NT < n && better[m]) atomicAdd(&s.rank[c + m * NT], better[m]);
  }
}

// The exact way, for rows in which too many logits reach the floor (ties above all): the k-th largest key by its bytes from
// the highest, then all logits above it and the first few, by index, of those that equal it.  The row is read again in every
// pass.
template <typename T, int NT>
__device__ __forceinline__ void select_exactly(const T* z, int vocab, int k, TopShared<NT>& s) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t prefix = 0, wanted = (uint32_t)k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += NT) s.histogram[i] = 0;
    __syncthreads();
    for (uint32_t first = 0; first < (uint32_t)vocab; first += NT) {
      const uint32_t j = first + threadIdx.x;
      const uint32_t key = j < (uint32_t)vocab ? order_key(to_float(z[j])) : 0u;
      const bool counts = key != 0 && (shift == 24 || key >> (shift + 8) == prefix);
      const uint32_t bin = (key >> shift) & 255u;
      const unsigned long long all = __ballot(counts);
      if (all) {  // the bin that one of the lanes names, once for all that name it
        const int leader = __ffsll(all) - 1;
        const uint32_t one = __builtin_amdgcn_readlane(bin, leader);
        const unsigned long long same = __ballot(counts && bin == one);
        if (lane == leader) atomicAdd(&s.histogram[one], (uint32_t)__popcll(same));
        if (counts && bin != one) atomicAdd(&s.histogram[bin], 1u);
      }
    }
    __syncthreads();
    if (w == 0) {  // lane l: bins 255 - 4 l and the three below
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = s.histogram[255 - 4 * lane - i], sum += c[i];
      uint32_t above = wave_inclusive_sum(sum) - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < wanted && above + c[i] >= wanted) s.prefix = prefix << 8 | (uint32_t)(255 - 4 * lane - i), s.wanted = wanted - above;
        above += c[i];
      }
    }
    __syncthreads();
    prefix = s.prefix;
    wanted = s.wanted;
  }
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  uint32_t seen = 0;  // equal ones before this turn, in ascending order
  for (uint32_t first = 0; first < (uint32_t)vocab; first += NT) {
    const uint32_t j = first + threadIdx.x;
    const uint32_t key = j < (uint32_t)vocab ? order_key(to_float(z[j])) : 0u;
    const unsigned long long equal = __ballot(key == prefix);
    bool taken = key > prefix;
    if (seen < wanted) {
      if (lane == 0) s.totals[w] = (uint32_t)__popcll(equal);
      __syncthreads();
      uint32_t at = seen + (uint32_t)__popcll(equal & ((1ull << lane) - 1));
      for (int i = 0; i < NT / 64; ++i) {
        if (i < w) at += s.totals[i];
        seen += s.totals[i];
      }
      taken |= key == prefix && at < wanted;
      __syncthreads();
    }
    if (taken) s.candidates[atomicAdd(&s.count, 1u)] = (unsigned long long)key << 32 | ~j;
  }
  __syncthreads();
}

// A floor that at least k logits reach is the k-th largest of the threads' largest; hardly more reach it (of N keys some
// -N ln(1 - k / N) logits), unless ties or neighbours crowd there.  A row goes by in pieces of NT x CH vectors, the next one
// on its way while one is looked at: the vectors that reach the floor of what has gone by are listed in LDS, in the end
// their elements that reach the last floor, and these are ranked by counting.  Each logit is read once, and takes a maximum
// and, for the log-sum-exp, an exponential against the thread's own largest so far.
//   4096 x 131072 in bfloat16, 64 pairs: 218 us, 4.9 TB/s of 6.5 that a bare kernel reaches.  A row held in registers as a
//   whole took 302: nothing was on its way while it was ranked.  8 x 32768 7.1 us, 700 x 10000 in 32 bits 14.3: a row's chain
//   of piece, floor, list and rank, about 5 us behind its loads.  Few rows leave most of the device idle, as a row is one
//   workgroup's: 1 x 131072 takes 18 us, to 256 pairs 32.  With 512 threads 7 to 13 registers are spilled (24 to 48 bytes of scratch).
template <typename T, int NT, int CH>
__global__ __launch_bounds__(NT, NT < 512 || CH > 4 ? 4 : 6) void top_logits_kernel(TopArgs a) {
  using Piece = Row<T, NT, CH>;
  constexpr int E = Piece::E;
  constexpr uint32_t kCandidates = TopShared<NT>::kCandidates, kVectors = TopShared<NT>::kVectors;
  constexpr int kKeys = TopShared<NT>::kKeys;
  __shared__ TopShared<NT> s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = a.inv_temperature * kLog2E;
  const int whole = a.vocab / E, pieces = whole > 0 ? (whole + NT * CH - 1) / (NT * CH) : 1;
  Piece piece;
  int64_t r = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + r * a.row_stride;
  piece.read_piece(z, whole, 0);
  piece.read_rest(z, a.vocab);
  for (;;) {
    if (threadIdx.x == 0) s.count = s.hits = 0;
    const float rest = piece.rest;
    const int64_t next = r + gridDim.x;
    const T* z_next = next < a.rows ? static_cast<const T*>(a.logits) + next * a.row_stride : nullptr;
    float largest[2] = {rest, -kInf};           // of even and odd vectors or halves of them
    float m = -kInf, sum = 0.0f;                // of this thread: sum of exp((z - m) / T)
    float least = 0.0f;
    for (int k = 0; k < pieces; ++k) {
      asm volatile("" : "+s"(a.vocab));
      Piece now = piece;
      now.cut_piece(whole, k);
      const bool more = k + 1 < pieces;
      piece.read_piece(more ? z : z_next, whole, more ? k + 1 : 0);
      float top[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float low = now.held[i].get(0), high = now.held[i].get(E / 2);
#pragma unroll
        for (int j = 1; j < E / 2; ++j) low = fmaxf(low, now.held[i].get(j)), high = fmaxf(high, now.held[i].get(E / 2 + j));
        largest[0] = fmaxf(largest[0], low);
        largest[1] = fmaxf(largest[1], high);
        top[i] = fmaxf(low, high);
      }
      const float seen = fmaxf(largest[0], largest[1]);
      now.renew();
      if (a.out_lse) {
        const float shift = seen == -kInf ? 0.0f : seen;
        sum *= exp2_fast((m - shift) * c);
        m = seen;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) sum += exp2_fast((now.held[i].get(j) - shift) * c);
        if (k == 0) sum += exp2_fast((rest - shift) * c);
        now.renew();
      }
      if ((k & (k - 1)) == 0 || k + 1 == pieces) {  // the floor of what has gone by, when that has doubled
        const int fold = a.k * 8 <= kKeys ? 4 : a.k * 4 <= kKeys ? 2 : 1;  // fewer keys do where k is small
        float keyed[2] = {kKeys == NT ? seen : largest[0], largest[1]};
#pragma unroll
        for (int i = 0; i < kKeys / NT; ++i) {
          if (fold > 1) keyed[i] = fmaxf(keyed[i], neighbour<0xb1>(keyed[i]));
          if (fold > 2) keyed[i] = fmaxf(keyed[i], neighbour<0x4e>(keyed[i]));
          if (lane % fold == 0) s.keys[(i * NT + (int)threadIdx.x) / fold] = order_key(keyed[i]);
        }
        __syncthreads();
        if (w == 0) {
          const uint32_t floor = fold == 4   ? floor_of<kKeys / 4>(s.keys, a.k, lane)
                                 : fold == 2 ? floor_of<kKeys / 2>(s.keys, a.k, lane)
                                             : floor_of<kKeys>(s.keys, a.k, lane);
          if (lane == 0) s.floor = floor;
        }
        const uint32_t listed = __builtin_amdgcn_readfirstlane(s.hits);
        __syncthreads();
        const uint32_t floor = __builtin_amdgcn_readfirstlane(s.floor);
        least = floor > 1u ? key_value(floor) : -3.402823466e38f;  // whatever can be chosen
        if (listed > kVectors / 2 && listed <= kVectors) thin_out<T, NT>(s, listed, least);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (top[i] >= least) {
          const uint32_t at = atomicAdd(&s.hits, 1u);
          if (at < kVectors) s.vectors[at] = __builtin_bit_cast(uint4, now.held[i]), s.numbers[at] = (k * CH + i) * NT + (int)threadIdx.x;
        }
    }
    piece.read_rest(z_next, a.vocab);
    auto list = [&](float value, int j) {
      const uint32_t at = atomicAdd(&s.count, 1u);
      if (at < kCandidates) s.candidates[at] = (unsigned long long)order_key(value) << 32 | (uint32_t)~j;
    };
    if (rest >= least) list(rest, whole * E + (int)threadIdx.x);
    if (a.out_lse) {
      const float all = wave_max_f(m);
      const float total = wave_sum_f(sum * exp2_fast((m - (all == -kInf ? 0.0f : all)) * c));
      if (lane == 0) s.sums[w] = float2{all, total};
    }
    __syncthreads();
    const uint32_t hits = __builtin_amdgcn_readfirstlane(s.hits);
    for (uint32_t i = threadIdx.x; i < hits * E && hits <= kVectors; i += NT) {
      const float value = to_float(reinterpret_cast<const T*>(s.vectors)[i]);
      if (value >= least) list(value, s.numbers[i / E] * E + (int)(i % E));
    }
    if (a.out_lse && threadIdx.x == 0) {
      float all = s.sums[0].x, total = 0.0f;
      for (int i = 1; i < NT / 64; ++i) all = fmaxf(all, s.sums[i].x);
      all = all == -kInf ? 0.0f : all;
      for (int i = 0; i < NT / 64; ++i) total += s.sums[i].y * exp2_fast((s.sums[i].x - all) * c);
      a.out_lse[r] = all * a.inv_temperature + kLn2 * __log2f(total);
    }
    __syncthreads();
    uint32_t n = __builtin_amdgcn_readfirstlane(s.count);
    if (hits > kVectors || n > kCandidates) {
      __syncthreads();
      select_exactly<T, NT>(z, a.vocab, a.k, s);
      n = __builtin_amdgcn_readfirstlane(s.count);
    }
    const uint32_t span = (n + 63u) & ~63u;
    for (uint32_t i = threadIdx.x; i < span; i += NT) {
      s.rank[i] = 0;
      if (i >= n) s.candidates[i] = 0;  // less than any, so that no four need a look at the end
    }
    __syncthreads();
    if (NT == 64 && span > NT) count_better<NT, 4>(s, n, span);
    else count_better<NT, 1>(s, n, span);
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < n; c += NT) {
      const uint32_t rank = s.rank[c];
      if (rank < (uint32_t)a.k) {
        a.out_idx[r * a.k + rank] = (int)~(uint32_t)s.candidates[c];
        a.out_val[r * a.k + rank] = key_value((uint32_t)(s.candidates[c] >> 32));
      }
    }
    for (int c = (int)n + (int)threadIdx.x; c < a.k; c += NT) {
      a.out_idx[r * a.k + c] = -1;
      a.out_val[r * a.k + c] = -kInf;
    }
    if (!z_next) return;
    r = next;
    z = z_next;
    __syncthreads();
  }
}

// ---- distillation ---------------------------------------------------------------------------------------------
constexpr int kPairs = DGC_TOP_MAX / 64;  // of a lane of the first wavefront

template <int NT>
struct DistillShared {
  Between<NT> between;
  float mass, kl;
  int32_t at[DGC_TOP_MAX];  // the pairs' elements, what they hold, and the teacher's share
  float z_at[DGC_TOP_MAX], p[DGC_TOP_MAX];
};

// One workgroup takes a row at a time and, with CH > 0, reads it once: largest logit, sum of exponentials, gradient, all from
// registers, with two exchanges through LDS.  The first wavefront sees to the pairs in between (their logits are gathered while
// the row comes in), and writes the few elements that pairs and the label name once more behind the others.
//   4096 x 131072 in bfloat16, loss and gradient, a temperature of two and hard labels: 500 us, 4.3 TB/s (2.1 GB; with the row
//   read three times and 256 threads 1862).  Such a row takes half the registers of a compute unit, so that only one is there:
//   its loads go out while the row before it is stored, but the exchanges stand alone, and the arithmetic, some 23
//   instructions an element, is 310 us of the whole.  The loss alone 256 us, 4.2 TB/s.  1111 x 32771 in binary16 50 us (146 MB),
//   20 x 10000 in 32 bits 6.5.
// With CH = 0, rows that registers do not hold are read three times (the loss alone: twice), the later times from nearer
// memory in part, and nothing is on its way between two of them: 2048 x 131072 in 32 bits 642 us and the loss alone 307 (2.1 and
// 1.1 GB to move: 3.3 and 3.5 TB/s), 2048 x 140000 in bfloat16 395 and 194 (2.9 TB/s).
// The exponentials of an element at the temperature and without one: not needed or the same, the square of the first (a
// temperature of two: 500 us where one of its own takes 525 for 4096 x 131072, 50.4 and 54.7 for 1111 x 32771), or one of its own.
enum { kOnce, kSquare, kTwice };
template <int MODE>
__device__ __forceinline__ float2 powers(float z, float c) {
  const float e = exp2_fast(z * c);
  return float2{e, MODE == kOnce ? 0.0f : MODE == kSquare ? e * e : exp2_fast(z * kLog2E)};
}
template <typename T, int NT, int CH, int MODE, bool GRAD>
__global__ __launch_bounds__(NT) void distill_kernel(DistillArgs a) {
  constexpr int E = Row<T, NT, CH>::E;
  __shared__ DistillShared<NT> s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float tau = a.temperature, inv_tau = 1.0f / tau, c = inv_tau * kLog2E;
  Row<T, NT, CH> row;
  int64_t r = blockIdx.x;
  float weight = a.row_weight ? uniform(a.row_weight[r]) : 1.0f;
  row.read(weight != 0.0f ? static_cast<const T*>(a.logits) + r * a.row_stride : nullptr, a.vocab);
  for (;;) {
    asm volatile("" : "+s"(a.vocab));  // places of vectors are counted anew for every row, not kept in registers
    const T* z = static_cast<const T*>(a.logits) + r * a.row_stride;
    T* grad = GRAD ? static_cast<T*>(a.grad) + r * a.grad_stride : nullptr;
    const int64_t next = r + gridDim.x;
    const float next_weight = next < a.rows ? (a.row_weight ? uniform(a.row_weight[next]) : 1.0f) : 0.0f;
    int y = a.labels ? __builtin_amdgcn_readfirstlane(a.labels[r]) : -1;
    // the pairs, and the logits they and the label name: the first wavefront's
    int at[kPairs];
    float t[kPairs], z_at[kPairs], z_y = 0.0f;
    bool named = false;  // the label is one of the pairs
    if (w == 0) {
      bool bad = y >= a.vocab;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const int p = i * 64 + lane;
        at[i] = p < a.k ? a.top_idx[r * a.k + p] : -1;
        bad |= at[i] >= a.vocab;
        if (at[i] >= a.vocab || a.hard_weight == 1.0f) at[i] = -1;  // without weight, also an infinite divergence counts nothing
        t[i] = at[i] >= 0 ? a.top_val[r * a.k + p] * inv_tau : -kInf;
        z_at[i] = at[i] >= 0 ? to_float(z[at[i]]) : 0.0f;
        named |= at[i] >= 0 && at[i] == y;
      }
      if (bad && a.diag_flags) atomicOr(a.diag_flags, (uint32_t)DGC_DIAG_BAD_INDEX);
      if (y >= 0 && y < a.vocab) z_y = to_float(z[y]);
      named = __any(named);
    }
    if (y >= a.vocab) y = -1;
    bool live = weight != 0.0f;
    float shift = 0.0f, cs = 0.0f, ch = 0.0f, soft = 0.0f, hard = 0.0f;
    if (live) {
      row.cut(a.vocab);
      const float wave = wave_max_f(row.largest(z, a.vocab));
      row.renew();
      if (lane == 0) s.between.largest[w] = wave;
      __syncthreads();
      const float m = s.between.max_of();
      shift = m == -kInf ? 0.0f : m;
      float2 sums{0.0f, 0.0f};
      auto add = [&](float zj) {
        const float2 e = powers<MODE>(zj - shift, c);
        sums.x += e.x;
        if (MODE != kOnce) sums.y += e.y;
      };
      row.each(z, a.vocab, [&](const Pack<T, E>& v, int) {
#pragma unroll
        for (int j = 0; j < E; ++j) add(v.get(j));
      });
      add(row.rest);
      row.renew();
      sums.x = wave_sum_f(sums.x);
      if (MODE != kOnce) sums.y = wave_sum_f(sums.y);
      if (lane == 0) s.between.sums[w] = sums;
      if (w == 0) {
        float log_p[kPairs], from;
        if (a.top_lse) {
          from = a.top_lse[r];
        } else {  // from their largest on: rounded beside it, the logarithm of their sum would move all shares alike
          float tm = t[0];
#pragma unroll
          for (int i = 1; i < kPairs; ++i) tm = fmaxf(tm, t[i]);
          tm = wave_max_f(tm);
          tm = tm == -kInf ? 0.0f : tm;
          float total = 0.0f;
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            t[i] -= tm;
            total += at[i] >= 0 ? __expf(t[i]) : 0.0f;
          }
          total = wave_sum_f(total);
          from = total > 0.0f ? __logf(total) : 0.0f;
        }
        float mass = 0.0f, kl = 0.0f;  // of the divergence, what does not need the row's sum
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          log_p[i] = t[i] - from;
          const float p = at[i] >= 0 ? __expf(log_p[i]) : 0.0f;
          z_at[i] -= shift;
          mass += p;
          kl += p != 0.0f ? p * (log_p[i] - z_at[i] * inv_tau) : 0.0f;
          s.at[i * 64 + lane] = at[i];
          s.z_at[i * 64 + lane] = z_at[i];
          s.p[i * 64 + lane] = p;
        }
        mass = wave_sum_f(mass);
        kl = wave_sum_f(kl);
        z_y -= shift;
        if (lane == 0) s.mass = mass, s.kl = kl;
      }
      __syncthreads();
      sums = s.between.sum_of();
      const float mass = uniform(s.mass);
      live = sums.x != 0.0f;  // zero: nothing but -inf
      if (MODE == kOnce) sums.y = sums.x;
      if (live) {
        soft = weight * (1.0f - a.hard_weight) * tau;
        hard = y >= 0 ? weight * a.hard_weight : 0.0f;
        cs = soft * mass / sums.x;
        ch = hard / sums.y;
        if (a.loss && threadIdx.x == 0)
          a.loss[r] = weight * ((1.0f - a.hard_weight) * tau * tau * (s.kl + mass * __logf(sums.x)) + (y >= 0 ? a.hard_weight * (__logf(sums.y) - z_y) : 0.0f));
      }
    }
    if (!live && a.loss && threadIdx.x == 0) a.loss[r] = 0.0f;
    if (MODE == kOnce) cs += ch;  // one exponential stands for both
    const T* z_next = next_weight != 0.0f ? static_cast<const T*>(a.logits) + next * a.row_stride : nullptr;
    const __amdgpu_buffer_rsrc_t from = Row<T, NT, CH>::buffer(z_next, a.vocab);
    const uint32_t behind = (uint32_t)(a.vocab / E * E) + threadIdx.x;
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));  // offsets of vectors are counted anew for every row, not kept in registers
    auto value = [&](float zj) {
      const float2 e = powers<MODE>(zj, c);
      return MODE == kOnce ? cs * e.x : fmaf(ch, e.y, cs * e.x);
    };
    if constexpr (GRAD) {
      auto of = [&](const Pack<T, E>& v) {
        float g[E];
#pragma unroll
        for (int j = 0; j < E; ++j) g[j] = value(v.get(j) - shift);
        Pack<T, E> out;
        out.set(g);
        return out;
      };
      if (!live)  // (what the sweep below forms of such a row is not stored)
        for (uint32_t j = threadIdx.x; j < (uint32_t)a.vocab; j += NT) grad[j] = from_float<T>(0.0f);
      if constexpr (CH > 0) {  // the next row comes in where this one goes out
        const __amdgpu_buffer_rsrc_t to = Row<T, NT, CH>::buffer(live ? grad : nullptr, a.vocab);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          Row<T, NT, CH>::store(to, thread, i, of(row.held[i]));
          row.read(from, thread, i);
          __builtin_amdgcn_sched_barrier(1);  // no load before the registers it fills are free
        }
      } else if (live) {
        row.each(z, a.vocab, [&](const Pack<T, E>& v, int number) {
          reinterpret_cast<typename Row<T, NT, CH>::Loose*>(grad + (uint32_t)number * (uint32_t)E)->v = of(v);
        });
      }
      if (live && behind < (uint32_t)a.vocab) grad[behind] = from_float<T>(value(row.rest - shift));
    } else {
#pragma unroll
      for (int i = 0; i < CH; ++i) row.read(from, thread, i);
    }
    row.read_rest(z_next, a.vocab);
    if (GRAD && live) {
      __syncthreads();
      if (w == 0) {  // the few elements that a pair or the label names, once more
        for (int i = lane; i < a.k; i += 64) {
          const int j = s.at[i];
          if (j >= 0) grad[j] = from_float<T>(value(s.z_at[i]) - soft * s.p[i] - (j == y ? hard : 0.0f));
        }
        if (lane == 0 && y >= 0 && !named) grad[y] = from_float<T>(value(z_y) - hard);
      }
    }
    if (next >= a.rows) return;
    r = next;
    weight = next_weight;
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------
// Workgroups that walk all rows, as many as the device holds at a time (asked for once: it takes longer than a launch).
template <typename T, int NT, int CH, typename ARGS, void (*KERNEL)(ARGS)>
hipError_t launch_rows(const ARGS& a, hipStream_t stream) {
  static const int per_unit = [] {
    int n = 0;
    return hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, NT, 0) == hipSuccess && n > 0 ? n : 1;
  }();
  const int64_t most = (int64_t)per_unit * compute_units();
  KERNEL<<<dim3((unsigned)(a.rows < most ? a.rows : most)), NT, 0, stream>>>(a);
  return hipGetLastError();
}

struct PickTop {
  template <typename T, typename ARGS>
  static hipError_t launch(const ARGS& a, hipStream_t stream) {
    const int64_t vectors = ceil_div(a.vocab, 16 / (int64_t)sizeof(T));
#define DGC_ROW(NT, CH) return launch_rows<T, NT, CH, TopArgs, &top_logits_kernel<T, NT, CH>>(a, stream)
    if (vectors <= 64) DGC_ROW(64, 1);
    if (vectors <= 256) DGC_ROW(256, 1);
    if (vectors <= 1024) DGC_ROW(256, 4);
    // Few rows: what one of them takes is what counts, so fewer pieces (333 rows of 10000 in 32 bits, 64 pairs: 11.0 us in
    // pieces of 8 vectors a thread, 12.4 in pieces of 4; 512 of 32000 in bfloat16 14.9 and 16.6).  Many: workgroups to a compute
    // unit (1024 of those 27.4 and 24.7, 4096 77.6 and 74; 2048 of 131072, 256 pairs: 179 and 154).
    if (a.rows <= 2 * compute_units()) DGC_ROW(512, 8);
    DGC_ROW(512, 4);
#undef DGC_ROW
  }
};
template <int MODE, bool GRAD>
struct PickDistill {
  template <typename T, typename ARGS>
  static hipError_t launch(const ARGS& a, hipStream_t stream) {
    const int64_t vectors = ceil_div(a.vocab, 16 / (int64_t)sizeof(T));
#define DGC_ROW(NT, CH) return launch_rows<T, NT, CH, DistillArgs, &distill_kernel<T, NT, CH, MODE, GRAD>>(a, stream)
    // Few enough vectors to a thread that several rows are on a compute unit at a time, few enough threads that they do not wait
    // for each other long.  2048 rows, loss and gradient at a temperature of two with labels / the loss alone, in us:
    //   vocabulary      512 x 6      512 x 10     512 x 14     1024 x 16    not held
    //   16001 bfloat16  40 / 21      59 / 32      75 / 38      161 / 85     63 / 43
    //   20000           40 / 22      59 / 31      75 / 40      161 / 81     63 / 42
    //   32000                        67 / 33      83 / 41      161 / 83     98 / 52
    //   40000                        77 / 37      91 / 41      165 / 85     117 / 53
    //   50000                                     101 / 44     174 / 88     155 / 64
    //   57000                                     112 / 46     181 / 90     175 / 70
    //   64000                                                  186 / 93     194 / 80
    //   100352                                                 225 / 114    284 / 142
    //   131072                                                 266 / 128    357 / 177
    //   10000 binary32  32 / 21      39 / 25      43 / 26      84 / 52      57 / 40
    //   20000                        70 / 34      72 / 33      108 / 57     97 / 45
    //   32768                                                  137 / 64     155 / 59
    // Threads without a vector cost as much as the others: from one size to the next the time steps up, most behind 57344
    // elements of 16 bits and 28672 of 32.  There the loss alone would do better without registers (64000 and 32768 above).
    if (vectors <= 64) DGC_ROW(64, 1);
    if (vectors <= 256) DGC_ROW(256, 1);
    if (vectors <= 1024) DGC_ROW(256, 4);
    if (vectors <= 3072) DGC_ROW(512, 6);
    if (vectors <= 5120) DGC_ROW(512, 10);
    if (vectors <= 7168) DGC_ROW(512, 14);
    if (vectors <= 16384) DGC_ROW(1024, 16);
    DGC_ROW(1024, 0);
#undef DGC_ROW
  }
};

template <typename PICK, typename ARGS>
hipError_t launch_type(const ARGS& a, int32_t dtype, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return PICK::template launch<float>(a, stream);
    case DGC_F16: return PICK::template launch<_Float16>(a, stream);
    default: return PICK::template launch<__bf16>(a, stream);
  }
}

template <int MODE>
hipError_t launch_mode(const DistillArgs& a, int32_t dtype, hipStream_t stream) {
  return a.grad ? launch_type<PickDistill<MODE, true>>(a, dtype, stream) : launch_type<PickDistill<MODE, false>>(a, dtype, stream);
}

}  // namespace

hipError_t launch_top_logits(const TopArgs& a, int32_t dtype, hipStream_t stream) { return launch_type<PickTop>(a, dtype, stream); }
hipError_t launch_distill(const DistillArgs& a, int32_t dtype, hipStream_t stream) {
  if (!a.labels || a.temperature == 1.0f) return launch_mode<kOnce>(a, dtype, stream);
  if (a.temperature == 2.0f) return launch_mode<kSquare>(a, dtype, stream);
  return launch_mode<kTwice>(a, dtype, stream);
}

}  // namespace dgc
