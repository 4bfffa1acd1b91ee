// The gated linear recurrence: h_t = a_t h_{t-1} + b_t x_t with a = sigmoid(gate), forward and backward.

#include "dgc_operators.h"

namespace dgc {

bool scan_chained(const ScanArgs& a);
int64_t scan_word_rows(const ScanArgs& a);

namespace {

struct Gates {
  float a, b;  // sigmoid(f), sigmoid(-f): neither is formed as one minus the other, so both keep their relative accuracy
};

__device__ __forceinline__ Gates gates_of(float f) {
  const float t = __expf(-fabsf(f));
  const float s = __builtin_amdgcn_rcpf(1.0f + t);
  const float ts = t * s;
  return f < 0.0f ? Gates{ts, s} : Gates{s, ts};
}

// Rows [begin, begin + length) of a sequence, cut to the arrays and to max_length whatever the offsets say.
__device__ __forceinline__ void sequence_rows(const ScanArgs& a, int64_t s, int64_t& begin, int64_t& length) {
  if (!a.row_offsets) {
    begin = s * a.max_length;
    length = a.max_length;
    return;
  }
  const int64_t lo = a.row_offsets[s], hi = a.row_offsets[s + 1];
  begin = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
  length = (hi > a.rows ? a.rows : hi) - begin;
  length = length < 0 ? 0 : length > a.max_length ? a.max_length : length;
}

// Where the state in front of step c * kStateRows of a sequence is kept: no two of them at one place, all below
// rows / kStateRows + sequences.
constexpr int kStateRows = DGC_SCAN_STATE_ROWS;
__device__ __forceinline__ int64_t state_row(int64_t s, int64_t begin, int64_t c) { return begin / kStateRows + s + c; }

// ---- tiles -------------------------------------------------------------------------------------
// A wavefront takes kWaveRows steps of kBlock channels: VEC channels to a lane, 64 / VEC lanes to a row and so VEC groups
// of lanes that take kWaveRows / VEC steps each, one after the other in registers.  A group's steps together are
// h_out = A h_in + H; groups are joined by shuffles, the W wavefronts of a tile through LDS.
constexpr int kWaveRows = 32;
constexpr int kBlock = 64;
static_assert(kStateRows % kWaveRows == 0, "a kept state lies in front of a wavefront's first step");

// Tiles of one sequence and one block of channels follow each other.  What a tile does to a state is left in a word of its
// own (A with its sign bit set, H), which is read by the tiles behind it in its group of kGroup tiles; the last tile of a
// group leaves the state behind it instead (1.0 with the sign bit set, state).  A tile joins, in order, the state in front
// of its group and the words of the group's tiles before its own: always the same sums, whoever comes first.
// A word is stored and loaded whole, so that it needs no fence; zero says that it is not there yet.
constexpr int kGroup = 32;

struct Chain {
  unsigned long long* words;  // [tile rows][channels]; null: a workgroup walks all tiles of a sequence and block
  uint32_t* ticket;
  uint32_t tickets;           // (tile row, block) in all
  int64_t tile_rows;          // without row_offsets: tiles of a sequence
};

__device__ __forceinline__ unsigned long long chain_word(float a, float h) {
  // a NaN leaves no finite state, whatever comes in
  if (!(a <= 1.0f)) h = __builtin_nanf(""), a = 1.0f;
  return (unsigned long long)(__float_as_uint(a) | 0x80000000u) << 32 | __float_as_uint(h);
}

__device__ __forceinline__ unsigned long long wait_for(const unsigned long long* p) {
  unsigned long long w;
  while (!((w = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) >> 63)) __builtin_amdgcn_s_sleep(1);
  return w;
}

// The state in front of the tile at `position` of its chain (in the direction of travel), whose words lie `step` behind
// those of the one before it (`first`: in front of the first group).  The rows of words waited for belong to lower tickets, and every ticket's workgroup leaves
// its row, whatever the offsets hold: they run, or have run, and none of them waits for this one, so every wait ends.
__device__ __forceinline__ float chain_state(const unsigned long long* word, int64_t step, int64_t position, float first) {
  const int before = (int)(position % kGroup);
  const unsigned long long* p = word - before * step;
  float state = first;
  if (position > before) state = __uint_as_float((uint32_t)wait_for(p - step));
  for (int i = 0; i < before; ++i, p += step) {
    const unsigned long long w = wait_for(p);
    state = fmaf(__uint_as_float((uint32_t)(w >> 32) & 0x7fffffffu), state, __uint_as_float((uint32_t)w));
  }
  return state;
}

struct Tile {
  int64_t sequence, begin, length;
  int64_t index, count;  // in its sequence
  int64_t word_row;      // of its words
  int32_t block;
  bool there;
};

// Tile `ticket`.  Equal sequences: all first tiles, then all second ones.  With offsets: tile row
// begin / rows + sequence + index, as for the kept states; rows of that numbering between two sequences stay empty.
template <int ROWS, bool REVERSE>
__device__ __forceinline__ Tile tile_of(const ScanArgs& a, const Chain& chain, uint32_t ticket) {
  const uint32_t blocks = (uint32_t)((a.channels + kBlock - 1) / kBlock);
  Tile t;
  uint32_t row = ticket / blocks;
  t.block = (int32_t)(ticket - row * blocks);
  if (!a.row_offsets) {
    const uint32_t sequences = (uint32_t)a.sequences;
    const uint32_t c = row / sequences;
    t.sequence = row - c * sequences;
    sequence_rows(a, t.sequence, t.begin, t.length);
    t.count = chain.tile_rows;
    t.index = REVERSE ? t.count - 1 - c : c;
    t.word_row = t.sequence * t.count + t.index;
    t.there = true;
    return t;
  }
  if (REVERSE) row = chain.tickets / blocks - 1 - row;
  // the last sequence whose first tile row is not behind this one
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, hi = a.sequences;
  while (hi - lo > 1) {
    const int64_t stride = (hi - lo + 63) / 64;
    const int64_t at = lo + lane * stride;
    int64_t begin = 0, length = 0;
    if (at < hi) sequence_rows(a, at, begin, length);
    const bool before = at < hi && begin / ROWS + at <= row;
    const int passed = __popcll(__ballot(before));
    const int64_t next = lo + passed * stride;
    lo = passed ? next - stride : lo;
    hi = next < hi && passed ? next : passed ? hi : lo + 1;
  }
  t.sequence = __builtin_amdgcn_readfirstlane((int)lo);
  sequence_rows(a, t.sequence, t.begin, t.length);
  t.count = (t.length + ROWS - 1) / ROWS;
  t.count = t.count < 1 ? 1 : t.count;
  t.index = (int64_t)row - (t.begin / ROWS + t.sequence);
  t.word_row = row;
  t.there = t.index >= 0 && t.index < t.count;
  return t;
}

// A tile row that belongs to no sequence leaves a word all the same: with offsets that do not ascend, some tile may look
// for it.
__device__ __forceinline__ void skip_tile(const ScanArgs& a, const Chain& chain, const Tile& t, int64_t channel) {
  if (threadIdx.x < 64 && channel < a.channels)
    __hip_atomic_store(chain.words + t.word_row * a.channels + channel, chain_word(1.0f, 0.0f), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// VEC elements of every step of a lane; steps behind the last one are not read.
template <typename T, int VEC, int S>
__device__ __forceinline__ void load_steps(const T* p, int64_t stride, uint32_t lane_offset, int steps, bool full, Pack<T, VEC> (&out)[S]) {
  if (full) {
#pragma unroll
    for (int i = 0; i < S; ++i) out[i] = *reinterpret_cast<const Pack<T, VEC>*>(p + i * stride + lane_offset);
  } else {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      out[i] = Pack<T, VEC>{};
      if (i < steps) out[i] = *reinterpret_cast<const Pack<T, VEC>*>(p + i * stride + lane_offset);
    }
  }
}

template <typename T, int VEC, int S>
__device__ __forceinline__ void store_steps(T* p, int64_t stride, uint32_t lane_offset, int steps, int i, const Pack<T, VEC>& v) {
  if (i < steps) *reinterpret_cast<Pack<T, VEC>*>(p + i * stride + lane_offset) = v;
}

// (A, H) of the lane groups in front of this one; A, H become those up to and with this one.
template <int VEC, bool DOWN>
__device__ __forceinline__ void join_groups(float (&A)[VEC], float (&H)[VEC], float (&A0)[VEC], float (&H0)[VEC], int group) {
  constexpr int kLanes = 64 / VEC;
#pragma unroll
  for (int o = kLanes; o < 64; o *= 2) {
    const bool has = DOWN ? group < VEC - o / kLanes : group >= o / kLanes;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float pa = DOWN ? __shfl_down(A[j], o) : __shfl_up(A[j], o), ph = DOWN ? __shfl_down(H[j], o) : __shfl_up(H[j], o);
      if (has) {
        H[j] = fmaf(A[j], ph, H[j]);
        A[j] *= pa;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    A0[j] = 1.0f;
    H0[j] = 0.0f;
    if (VEC > 1) {
      const float pa = DOWN ? __shfl_down(A[j], kLanes) : __shfl_up(A[j], kLanes), ph = DOWN ? __shfl_down(H[j], kLanes) : __shfl_up(H[j], kLanes);
      if (DOWN ? group < VEC - 1 : group > 0) {
        A0[j] = pa;
        H0[j] = ph;
      }
    }
  }
}

template <typename T, int VEC, int W, bool FREE, bool CHAIN>
__global__ __launch_bounds__(W * 64) void scan_forward_kernel(ScanArgs a, Chain chain) {
  constexpr int S = kWaveRows / VEC, kLanes = 64 / VEC, kRows = W * kWaveRows;
  __shared__ float2 part[W][kBlock];
  __shared__ float start[W][kBlock];
  __shared__ uint32_t next;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = lane / kLanes, col = (lane % kLanes) * VEC;
  uint32_t ticket = blockIdx.x;
  if (CHAIN) {
    if (threadIdx.x == 0) next = atomicAdd(chain.ticket, 1u);
    __syncthreads();
    ticket = next;
    if (ticket >= chain.tickets) return;
  }
  Tile t{};
  if (!CHAIN) {
    const uint32_t blocks = (uint32_t)((a.channels + kBlock - 1) / kBlock);
    t.sequence = ticket / blocks;
    t.block = (int32_t)(ticket - (uint32_t)t.sequence * blocks);
    sequence_rows(a, t.sequence, t.begin, t.length);
    t.count = (t.length + kRows - 1) / kRows;
    t.count = t.count < 1 ? 1 : t.count;
    t.there = true;
  }
  float carried = 0.0f;  // wavefront 0, lane by channel: the state in front of the tile
  for (;;) {
    uint32_t taken = 0;
    if (CHAIN) {
      if (threadIdx.x == 0) taken = atomicAdd(chain.ticket, 1u);
      t = tile_of<kRows, false>(a, chain, ticket);
    }
    const int64_t channel = (int64_t)t.block * kBlock + lane;
    const int64_t d = (int64_t)t.block * kBlock + col;
    if (t.there) {
      const int64_t row = t.index * kRows + w * kWaveRows;  // of the sequence, the wavefront's first
      const int64_t left = t.length - row - group * S;
      const int steps = d < a.channels ? (int)(left < 0 ? 0 : left > S ? S : left) : 0;
      const bool full = __all(steps == S);
      const int64_t at = t.begin + row;
      Pack<T, VEC> rf[S], rx[S];
      load_steps<T, VEC, S>(static_cast<const T*>(a.gate) + at * a.gate_stride, a.gate_stride, (uint32_t)(group * S * a.gate_stride + d), steps, full, rf);
      load_steps<T, VEC, S>(static_cast<const T*>(a.x) + at * a.x_stride, a.x_stride, (uint32_t)(group * S * a.x_stride + d), steps, full, rx);
      float ca[S][VEC], cu[S][VEC];
      float A[VEC], H[VEC], A0[VEC], H0[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) A[j] = 1.0f, H[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < S; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const Gates g = gates_of(to_float(rf[i].e[j]));
          const float xt = to_float(rx[i].e[j]);
          ca[i][j] = g.a;
          cu[i][j] = FREE ? xt : g.b * xt;
        }
        if (!full && i >= steps) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) ca[i][j] = 1.0f, cu[i][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          H[j] = fmaf(ca[i][j], H[j], cu[i][j]);
          A[j] *= ca[i][j];
        }
      }
      join_groups<VEC, false>(A, H, A0, H0, group);
      if (group == VEC - 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) part[w][col + j] = float2{A[j], H[j]};
      }
      __syncthreads();
      if (w == 0) {
        if (channel < a.channels) {
          const int64_t carry_at = t.sequence * a.channels + channel;
          float state = carried;
          if (CHAIN ? t.index < kGroup : t.index == 0) state = a.first ? a.first[carry_at] : 0.0f;
          if (CHAIN) {
            unsigned long long* word = chain.words + t.word_row * a.channels + channel;
            const bool closes = t.index % kGroup == kGroup - 1;
            if (!closes) {
              float ta = 1.0f, th = 0.0f;
#pragma unroll
              for (int v = 0; v < W; ++v) {
                th = fmaf(part[v][lane].x, th, part[v][lane].y);
                ta *= part[v][lane].x;
              }
              __hip_atomic_store(word, chain_word(ta, th), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            state = chain_state(word, a.channels, t.index, state);
          }
#pragma unroll
          for (int v = 0; v < W; ++v) {
            start[v][lane] = state;
            state = fmaf(part[v][lane].x, state, part[v][lane].y);
          }
          carried = state;
          if (CHAIN && t.index % kGroup == kGroup - 1)
            __hip_atomic_store(chain.words + t.word_row * a.channels + channel, chain_word(1.0f, state), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (t.index + 1 == t.count && a.last) a.last[carry_at] = state;
        }
        if (CHAIN && threadIdx.x == 0) next = taken;
      }
      __syncthreads();
      float state[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = start[w][col + j];
      if (a.states && group == 0 && steps > 0 && w % (kStateRows / kWaveRows) == 0) {
        float* kept = a.states + state_row(t.sequence, t.begin, row / kStateRows) * a.channels + d;
#pragma unroll
        for (int j = 0; j < VEC; ++j) kept[j] = state[j];
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = fmaf(A0[j], state[j], H0[j]);
      T* h = static_cast<T*>(a.h) + at * a.h_stride;
      const uint32_t lane_offset = (uint32_t)(group * S * a.h_stride + d);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        Pack<T, VEC> out;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          state[j] = fmaf(ca[i][j], state[j], cu[i][j]);
          out.e[j] = from_float<T>(state[j]);
        }
        store_steps<T, VEC, S>(h, a.h_stride, lane_offset, steps, i, out);
      }
    } else if (CHAIN) {
      skip_tile(a, chain, t, channel);
      __syncthreads();
      if (threadIdx.x == 0) next = taken;
      __syncthreads();
    }
    if (CHAIN) {
      ticket = next;
      if (ticket >= chain.tickets) return;
    } else if (++t.index == t.count) {
      return;
    }
  }
}

// The smaller of sigmoid(f) and sigmoid(-f), its sign bit set where it is the first: one register that gives both back,
// the larger as one minus the smaller, which keeps the relative accuracy of each.
__device__ __forceinline__ float fold_gates(float f) {
  const float t = __expf(-fabsf(f));
  const float m = t * __builtin_amdgcn_rcpf(1.0f + t);
  return f < 0.0f ? -m : m;
}
__device__ __forceinline__ Gates unfold_gates(float v) {
  const float m = fabsf(v), o = 1.0f - m;
  return (__float_as_uint(v) >> 31) ? Gates{m, o} : Gates{o, m};
}

// The same tiles from the last to the first.  A wavefront forms its states again from the kept one in front of it (an odd
// one by way of its neighbour's steps), and the gradient runs through the tiles as the state does in the forward pass.
template <typename T, int VEC, int W, bool FREE, bool CHAIN>
__global__ __launch_bounds__(W * 64, 3) void scan_backward_kernel(ScanArgs a, Chain chain) {
  constexpr int S = kWaveRows / VEC, kLanes = 64 / VEC, kRows = W * kWaveRows;
  static_assert(kStateRows == 2 * kWaveRows && W % 2 == 0, "two wavefronts to a kept state");
  __shared__ float2 part[W][kBlock];
  __shared__ float back[W][kBlock];
  __shared__ float start[W][kBlock];
  __shared__ uint32_t next;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = lane / kLanes, col = (lane % kLanes) * VEC;
  uint32_t ticket = blockIdx.x;
  if (CHAIN) {
    if (threadIdx.x == 0) next = atomicAdd(chain.ticket, 1u);
    __syncthreads();
    ticket = next;
    if (ticket >= chain.tickets) return;
  }
  Tile t{};
  if (!CHAIN) {
    const uint32_t blocks = (uint32_t)((a.channels + kBlock - 1) / kBlock);
    t.sequence = ticket / blocks;
    t.block = (int32_t)(ticket - (uint32_t)t.sequence * blocks);
    sequence_rows(a, t.sequence, t.begin, t.length);
    t.count = (t.length + kRows - 1) / kRows;
    t.count = t.count < 1 ? 1 : t.count;
    t.index = t.count - 1;
    t.there = true;
  }
  float carried = 0.0f;
  for (;;) {
    uint32_t taken = 0;
    if (CHAIN) {
      if (threadIdx.x == 0) taken = atomicAdd(chain.ticket, 1u);
      t = tile_of<kRows, true>(a, chain, ticket);
    }
    const int64_t channel = (int64_t)t.block * kBlock + lane;
    const int64_t d = (int64_t)t.block * kBlock + col;
    if (t.there) {
      const int64_t row = t.index * kRows + w * kWaveRows;
      const int64_t left = t.length - row - group * S;
      const int steps = d < a.channels ? (int)(left < 0 ? 0 : left > S ? S : left) : 0;
      const bool full = __all(steps == S);
      const int64_t at = t.begin + row;
      Pack<T, VEC> rf[S], rx[S], rd[S];
      load_steps<T, VEC, S>(static_cast<const T*>(a.gate) + at * a.gate_stride, a.gate_stride, (uint32_t)(group * S * a.gate_stride + d), steps, full, rf);
      load_steps<T, VEC, S>(static_cast<const T*>(a.x) + at * a.x_stride, a.x_stride, (uint32_t)(group * S * a.x_stride + d), steps, full, rx);
      load_steps<T, VEC, S>(static_cast<const T*>(a.dh) + at * a.dh_stride, a.dh_stride, (uint32_t)(group * S * a.dh_stride + d), steps, full, rd);
      float state[VEC];  // the kept state in front of the pair of wavefronts
      {
        const int64_t pair_row = row - (w & 1) * kWaveRows;
#pragma unroll
        for (int j = 0; j < VEC; ++j) state[j] = 0.0f;
        if (d < a.channels && pair_row < t.length) {
          const float* kept = a.states + state_row(t.sequence, t.begin, pair_row / kStateRows) * a.channels + d;
#pragma unroll
          for (int j = 0; j < VEC; ++j) state[j] = kept[j];
        }
      }
      float cm[S][VEC];
      float A[VEC], H[VEC], A0[VEC], H0[VEC], B[VEC], G[VEC], B0[VEC], G0[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) A[j] = 1.0f, H[j] = 0.0f, G[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        if (!full && i >= steps) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) rx[i].e[j] = rd[i].e[j] = from_float<T>(0.0f), cm[i][j] = 0.0f;  // a = 1, b = 0
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) cm[i][j] = fold_gates(to_float(rf[i].e[j]));
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const Gates g = unfold_gates(cm[i][j]);
          const float xt = to_float(rx[i].e[j]);
          H[j] = fmaf(g.a, H[j], FREE ? xt : g.b * xt);
          A[j] *= g.a;
        }
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) B[j] = A[j];
#pragma unroll
      for (int i = S - 1; i >= 0; --i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) G[j] = unfold_gates(cm[i][j]).a * (to_float(rd[i].e[j]) + G[j]);
      join_groups<VEC, false>(A, H, A0, H0, group);
      join_groups<VEC, true>(B, G, B0, G0, group);
      if (group == VEC - 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) part[w][col + j] = float2{A[j], H[j]};
      }
      if (group == 0) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) back[w][col + j] = G[j];
      }
      __syncthreads();
      if (w == 0) {
        if (channel < a.channels) {
          const int64_t carry_at = t.sequence * a.channels + channel;
          const int64_t position = t.count - 1 - t.index;
          float flow = carried;
          if (CHAIN ? position < kGroup : position == 0) flow = a.first ? a.first[carry_at] : 0.0f;
          if (CHAIN) {
            unsigned long long* word = chain.words + t.word_row * a.channels + channel;
            const bool closes = position % kGroup == kGroup - 1;
            if (!closes) {
              float ta = 1.0f, th = 0.0f;
#pragma unroll
              for (int v = W - 1; v >= 0; --v) {
                th = fmaf(part[v][lane].x, th, back[v][lane]);
                ta *= part[v][lane].x;
              }
              __hip_atomic_store(word, chain_word(ta, th), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            flow = chain_state(word, -a.channels, position, flow);
          }
#pragma unroll
          for (int v = W - 1; v >= 0; --v) {
            start[v][lane] = flow;
            flow = fmaf(part[v][lane].x, flow, back[v][lane]);
          }
          carried = flow;
          if (CHAIN && position % kGroup == kGroup - 1)
            __hip_atomic_store(chain.words + t.word_row * a.channels + channel, chain_word(1.0f, flow), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (t.index == 0 && a.last) a.last[carry_at] = flow;
        }
        if (CHAIN && threadIdx.x == 0) next = taken;
      }
      if (w & 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) state[j] = fmaf(part[w - 1][col + j].x, state[j], part[w - 1][col + j].y);
      }
      float before[S][VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = fmaf(A0[j], state[j], H0[j]);
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const Gates g = unfold_gates(cm[i][j]);
          const float xt = to_float(rx[i].e[j]);
          before[i][j] = FREE ? state[j] : state[j] - xt;
          state[j] = fmaf(g.a, state[j], FREE ? xt : g.b * xt);
        }
      __syncthreads();
      float flow[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) flow[j] = fmaf(B0[j], start[w][col + j], G0[j]);
      T* dgate = static_cast<T*>(a.dgate) + at * a.dgate_stride;
      T* dx = static_cast<T*>(a.dx) + at * a.dx_stride;
      const uint32_t gate_offset = (uint32_t)(group * S * a.dgate_stride + d), x_offset = (uint32_t)(group * S * a.dx_stride + d);
#pragma unroll
      for (int i = S - 1; i >= 0; --i) {
        Pack<T, VEC> og, ox;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const Gates g = unfold_gates(cm[i][j]);
          const float gt = to_float(rd[i].e[j]) + flow[j];
          ox.e[j] = from_float<T>(FREE ? gt : g.b * gt);
          og.e[j] = from_float<T>(gt * before[i][j] * (g.a * g.b));
          flow[j] = g.a * gt;
        }
        store_steps<T, VEC, S>(dx, a.dx_stride, x_offset, steps, i, ox);
        store_steps<T, VEC, S>(dgate, a.dgate_stride, gate_offset, steps, i, og);
      }
    } else if (CHAIN) {
      skip_tile(a, chain, t, channel);
      __syncthreads();
      if (threadIdx.x == 0) next = taken;
      __syncthreads();
    }
    if (CHAIN) {
      ticket = next;
      if (ticket >= chain.tickets) return;
    } else if (--t.index < 0) {
      return;
    }
  }
}

template <typename T, int VEC, int W, bool CHAIN>
hipError_t launch_tiles(const ScanArgs& a, const Chain& chain, uint32_t groups, bool free_input, bool backward, hipStream_t stream) {
  auto kernel = backward ? (free_input ? scan_backward_kernel<T, VEC, W, true, CHAIN> : scan_backward_kernel<T, VEC, W, false, CHAIN>)
                         : (free_input ? scan_forward_kernel<T, VEC, W, true, CHAIN> : scan_forward_kernel<T, VEC, W, false, CHAIN>);
  kernel<<<dim3(groups), W * 64, 0, stream>>>(a, chain);
  return hipGetLastError();
}

// Sequences of up to so many steps are walked by one workgroup each (and block of channels).
constexpr int kTileWaves = 4;
constexpr int kTileRows = kTileWaves * kWaveRows;
constexpr int kChainGroups = 4 * 256;

template <typename T, int VEC>
hipError_t launch_vec(const ScanArgs& a, void* workspace, bool free_input, bool backward, hipStream_t stream) {
  const int64_t blocks = ceil_div(a.channels, kBlock);
  Chain chain{};
  if (!scan_chained(a)) {
    const uint32_t groups = (uint32_t)(a.sequences * blocks);
    if (a.max_length <= 2 * kWaveRows) return launch_tiles<T, VEC, 2, false>(a, chain, groups, free_input, backward, stream);
    return launch_tiles<T, VEC, kTileWaves, false>(a, chain, groups, free_input, backward, stream);
  }
  chain.ticket = static_cast<uint32_t*>(workspace);
  chain.words = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + 256);
  chain.tile_rows = ceil_div(a.max_length, kTileRows);
  chain.tickets = (uint32_t)(scan_word_rows(a) * blocks);
  const hipError_t e = launch_clear_words(static_cast<uint32_t*>(workspace), scan_workspace_bytes(a) / 4, stream);
  if (e != hipSuccess) return e;
  const uint32_t groups = chain.tickets < (uint32_t)kChainGroups ? chain.tickets : (uint32_t)kChainGroups;
  return launch_tiles<T, VEC, kTileWaves, true>(a, chain, groups, free_input, backward, stream);
}

// Channels to a lane: as many as all rows are aligned for, eight bytes of them at most.
template <typename T>
hipError_t launch(const ScanArgs& a, void* workspace, bool free_input, bool backward, hipStream_t stream) {
  uint64_t bits = (uint64_t)a.channels * sizeof(T);
  for (const void* p : {a.gate, a.x, static_cast<const void*>(a.h), a.dh, static_cast<const void*>(a.dgate), static_cast<const void*>(a.dx)})
    bits |= reinterpret_cast<uintptr_t>(p);
  for (int64_t stride : {a.gate_stride, a.x_stride, a.h_stride, a.dh_stride, a.dgate_stride, a.dx_stride})
    bits |= (uint64_t)stride * sizeof(T);
  if (sizeof(T) == 2 && bits % 8 == 0) return launch_vec<T, sizeof(T) == 2 ? 4 : 2>(a, workspace, free_input, backward, stream);
  if (bits % (2 * sizeof(T)) == 0) return launch_vec<T, 2>(a, workspace, free_input, backward, stream);
  return launch_vec<T, 1>(a, workspace, free_input, backward, stream);
}

}  // namespace

int64_t scan_word_rows(const ScanArgs& a) {
  return a.row_offsets ? a.rows / kTileRows + a.sequences : a.sequences * ceil_div(a.max_length, kTileRows);
}

bool scan_chained(const ScanArgs& a) { return a.max_length > kTileRows; }

int64_t scan_workgroups(const ScanArgs& a) {
  return (scan_chained(a) ? scan_word_rows(a) : a.sequences) * ceil_div(a.channels, kBlock);
}

size_t scan_workspace_bytes(const ScanArgs& a) {
  if (!scan_chained(a)) return 0;
  return 256 + ((size_t)scan_word_rows(a) * (size_t)a.channels * sizeof(unsigned long long) + 255) / 256 * 256;
}

hipError_t launch_scan(const ScanArgs& a, void* workspace, int32_t dtype, bool free_input, bool backward, hipStream_t stream) {
  switch (dtype) {
    case DGC_F32: return launch<float>(a, workspace, free_input, backward, stream);
    case DGC_F16: return launch<_Float16>(a, workspace, free_input, backward, stream);
    default: return launch<__bf16>(a, workspace, free_input, backward, stream);
  }
}

}  // namespace dgc
