// The gated linear recurrence: h_t = a_t h_{t-1} + b_t x_t with a = sigmoid(gate), forward and backward.

#include "dgc_operators.h"
#include "dgc_steps.h"

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
  const SequenceRows cut(a.row_offsets[s], a.row_offsets[s + 1], a.rows, a.max_length);
  begin = cut.begin;
  length = cut.length;
}

// Where the state in front of step c * kStateRows of a sequence is kept: no two of them at one place, all below
// rows / kStateRows + sequences.
constexpr int kStateRows = DGC_SCAN_STATE_ROWS;
__device__ __forceinline__ int64_t state_row(int64_t s, int64_t begin, int64_t c) { return begin / kStateRows + s + c; }

// ---- tiles -------------------------------------------------------------------------------------
// How a wavefront takes its share of a tile: VEC channels to a lane, GROUPS groups of lanes that take S steps each, one
// after the other in registers.  A row's piece is 64 / GROUPS lanes wide (256 bytes where the rows' alignment allows it).
// A group's steps together are h_out = A h_in + H; groups are joined by shuffles, wavefronts through LDS.
template <typename T_, int VEC, int GROUPS, int S>
struct Shape {
  using T = T_;
  static constexpr int kVec = VEC, kGroups = GROUPS, kSteps = S;
  static constexpr int kLanes = 64 / GROUPS;
  static constexpr int kBlock = kLanes * VEC;                   // channels
  static constexpr int kRows = GROUPS * S;                      // of a wavefront
  static constexpr int kStateWaves = kStateRows / kRows;        // wavefronts to a kept state
  static_assert(kStateRows % kRows == 0, "a kept state lies in front of a wavefront's first step");
  static_assert(kRows <= kWaveRows && sizeof(T) <= 4, "offsets of a wavefront's rows take 32 bits");
};

// Where a tile lies, for the wavefronts that work on it.
struct Place {
  int64_t row;    // of the arrays, its first
  int64_t left;   // steps of the sequence from there on
  int64_t state;  // row of the kept state in front of it
  int64_t sequence;
  int64_t word_row;  // of its words
  int64_t position;  // in its sequence, in the direction of travel
  int32_t block;     // of channels
  int32_t last;      // no tile follows
  int32_t there;
};

__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ Place uniform(const Place& p) {
  return Place{uniform(p.row), uniform(p.left), uniform(p.state), uniform(p.sequence), uniform(p.word_row), uniform(p.position),
               __builtin_amdgcn_readfirstlane(p.block), __builtin_amdgcn_readfirstlane(p.last), __builtin_amdgcn_readfirstlane(p.there)};
}

// What of a place one lane works on.
struct Share {
  int64_t at;  // row of the arrays, the wavefront's first
  int64_t d;   // channel, the lane's first
  int group;   // of lanes
  int steps;   // of the lane
  int rows;    // of the wavefront
  bool full;   // no lane of the wavefront has fewer steps than all
};

template <typename SHAPE>
__device__ __forceinline__ Share share_of(const ScanArgs& a, const Place& p, int w, int lane) {
  constexpr int S = SHAPE::kSteps, kRows = SHAPE::kRows;
  Share h;
  h.group = lane / SHAPE::kLanes;
  h.d = (int64_t)p.block * SHAPE::kBlock + (lane % SHAPE::kLanes) * SHAPE::kVec;
  h.at = p.row + w * kRows;
  const int64_t left = p.left - w * kRows;
  h.rows = (int)(left < 0 ? 0 : left > kRows ? kRows : left);
  const int mine = h.rows - h.group * S;
  h.steps = h.d < a.channels ? (mine < 0 ? 0 : mine > S ? S : mine) : 0;
  h.full = __all(h.steps == S);
  return h;
}

// The wavefront's rows of an array as a buffer resource: an offset behind the last of them reads zeros and stores nothing,
// and one register to a lane is all that addresses take.  (Data format 32 in word 3, no swizzle, offsets in bytes.)
constexpr int kBufferFormat = 0x00020000;

template <typename T, int VEC, int S>
struct Steps {
  __amdgpu_buffer_rsrc_t rsrc;
  StepOffsets offsets;
  __device__ __forceinline__ Steps(const void* array, int64_t stride, const Share& h)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc((void*)(static_cast<const T*>(array) + h.at * stride), 0,
                                               (int)StepOffsets::buffer_bytes(h.rows, (uint32_t)stride * (uint32_t)sizeof(T)), kBufferFormat)),
        offsets(h.steps, h.group * S, (uint32_t)h.d * (uint32_t)sizeof(T), (uint32_t)stride * (uint32_t)sizeof(T)) {}
  __device__ __forceinline__ Pack<T, VEC> load(int i) const {
    const uint32_t at = offsets.at(i);
    if constexpr (sizeof(T) * VEC == 8) return __builtin_bit_cast(Pack<T, VEC>, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0));
    else if constexpr (sizeof(T) * VEC == 4) return __builtin_bit_cast(Pack<T, VEC>, __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0));
    else return __builtin_bit_cast(Pack<T, VEC>, __builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0));
  }
  __device__ __forceinline__ void store(int i, const Pack<T, VEC>& v) const {
    const uint32_t at = offsets.at(i);
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(T) * VEC == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(two, v), rsrc, at, 0, 0);
    else if constexpr (sizeof(T) * VEC == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rsrc, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), rsrc, at, 0, 0);
  }
};

// VEC elements of every step of a lane, zeros behind the last one.
template <typename T, int VEC, int S>
__device__ __forceinline__ void load_steps(const void* array, int64_t stride, const Share& h, Pack<T, VEC> (&out)[S]) {
  const Steps<T, VEC, S> steps(array, stride, h);
#pragma unroll
  for (int i = 0; i < S; ++i) out[i] = steps.load(i);
}

// (A0, H0) of the lane groups in front of this one (DOWN: behind it); A, H become those up to and with this one.
template <int GROUPS, bool DOWN, int VEC>
__device__ __forceinline__ void join_groups(float (&A)[VEC], float (&H)[VEC], float (&A0)[VEC], float (&H0)[VEC], int group) {
  constexpr int kLanes = 64 / GROUPS;
  auto other = [](float x, int lanes) { return DOWN ? __shfl_down(x, lanes) : __shfl_up(x, lanes); };
#pragma unroll
  for (int o = 1; o < GROUPS; o *= 2) {
    const bool has = DOWN ? group < GROUPS - o : group >= o;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float pa = other(A[j], o * kLanes), ph = other(H[j], o * kLanes);
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
    if (GROUPS > 1) {
      const float pa = other(A[j], kLanes), ph = other(H[j], kLanes);
      if (DOWN ? group < GROUPS - 1 : group > 0) {
        A0[j] = pa;
        H0[j] = ph;
      }
    }
  }
}

// ---- one wavefront's share of a tile, forward ------------------------------------------------------
template <typename SHAPE>
struct ForwardInput {
  using T = typename SHAPE::T;
  static constexpr int VEC = SHAPE::kVec, S = SHAPE::kSteps;
  Pack<T, VEC> gate[S], x[S];
  __device__ __forceinline__ void load(const ScanArgs& a, const Place&, int, const Share& h) {
    load_steps<T, VEC, S>(a.gate, a.gate_stride, h, gate);
    load_steps<T, VEC, S>(a.x, a.x_stride, h, x);
  }
};

template <typename SHAPE_, int W, bool FREE>
struct ForwardTile {
  using SHAPE = SHAPE_;
  using T = typename SHAPE::T;
  static constexpr int VEC = SHAPE::kVec, S = SHAPE::kSteps, kBlock = SHAPE::kBlock, kStateWaves = SHAPE::kStateWaves;
  static constexpr bool kReverse = false;
  using Input = ForwardInput<SHAPE>;
  struct Parts {  // what a tile's wavefronts leave in LDS
    float2 of[W][kBlock];
  };
  float ca[S][VEC], cu[S][VEC], A0[VEC], H0[VEC];

  // Gates and inputs of every step, and what the wavefront does to a state.
  __device__ __forceinline__ void fold(const Input& in, const Share& h, int w, int col, Parts& parts) {
    float A[VEC], H[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.0f, H[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const Gates g = gates_of(in.gate[i].get(j));
        const float xt = in.x[i].get(j);
        ca[i][j] = g.a;
        cu[i][j] = FREE ? xt : g.b * xt;
      }
    }
    if (!h.full) {  // steps behind the last one leave the state alone
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) ca[i][j] = i < h.steps ? ca[i][j] : 1.0f, cu[i][j] = i < h.steps ? cu[i][j] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        H[j] = fmaf(ca[i][j], H[j], cu[i][j]);
        A[j] *= ca[i][j];
      }
    }
    join_groups<SHAPE::kGroups, false>(A, H, A0, H0, h.group);
    if (h.group == SHAPE::kGroups - 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) parts.of[w][col + j] = float2{A[j], H[j]};
    }
  }

  __device__ __forceinline__ void between(const Parts&, int, int) {}

  // One lane by channel: (A, H) of the tile's wavefronts in the direction of travel, the i-th.
  static __device__ __forceinline__ float2 part(const Parts& parts, int i, int channel) { return parts.of[i][channel]; }

  // The states, from the one in front of the tile.
  __device__ __forceinline__ void apply(const ScanArgs& a, const Place& p, const Share& h, int w, int col, const Parts& parts,
                                        float (&state)[VEC]) {
    for (int v = 0; v < w; ++v) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = fmaf(parts.of[v][col + j].x, state[j], parts.of[v][col + j].y);
    }
    if (a.states && h.group == 0 && h.steps > 0 && w % kStateWaves == 0) {
      float* kept = a.states + (p.state + w / kStateWaves) * a.channels + h.d;
#pragma unroll
      for (int j = 0; j < VEC; ++j) kept[j] = state[j];
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) state[j] = fmaf(A0[j], state[j], H0[j]);
    const Steps<T, VEC, S> out(a.h, a.h_stride, h);
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = fmaf(ca[i][j], state[j], cu[i][j]);
      Pack<T, VEC> v;
      v.set(state);
      out.store(i, v);
    }
  }
};

// ---- the same backward ---------------------------------------------------------------------------------
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

template <typename SHAPE>
struct BackwardInput {
  using T = typename SHAPE::T;
  static constexpr int VEC = SHAPE::kVec, S = SHAPE::kSteps;
  Pack<T, VEC> gate[S], x[S], dh[S];
  float state[VEC];  // the kept one in front of the wavefront, or of one of the few before it
  __device__ __forceinline__ void load(const ScanArgs& a, const Place& p, int w, const Share& h) {
    load_steps<T, VEC, S>(a.gate, a.gate_stride, h, gate);
    load_steps<T, VEC, S>(a.x, a.x_stride, h, x);
    load_steps<T, VEC, S>(a.dh, a.dh_stride, h, dh);
#pragma unroll
    for (int j = 0; j < VEC; ++j) state[j] = 0.0f;
    if (h.d < a.channels && w / SHAPE::kStateWaves * kStateRows < p.left) {
      const float* kept = a.states + (p.state + w / SHAPE::kStateWaves) * a.channels + h.d;
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = kept[j];
    }
  }
};

// A wavefront forms its states again from the kept one in front of it (an odd one by way of its neighbour's steps); the
// gradient runs through the tiles, from the last to the first, as the state does in the forward pass.
template <typename SHAPE_, int W, bool FREE>
struct BackwardTile {
  using SHAPE = SHAPE_;
  using T = typename SHAPE::T;
  static constexpr int VEC = SHAPE::kVec, S = SHAPE::kSteps, kBlock = SHAPE::kBlock, kStateWaves = SHAPE::kStateWaves;
  static constexpr bool kReverse = true;
  static_assert(W % kStateWaves == 0, "tiles start at kept states");
  using Input = BackwardInput<SHAPE>;
  struct Parts {
    float2 of[W][kBlock];  // forward
    float back[W][kBlock];
  };
  float cm[S][VEC], before[S][VEC], A0[VEC], H0[VEC], B0[VEC], G0[VEC], state[VEC];
  Pack<T, VEC> x[S], dh[S];

  __device__ __forceinline__ void fold(const Input& in, const Share& h, int w, int col, Parts& parts) {
    float A[VEC], H[VEC], B[VEC], G[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.0f, H[j] = 0.0f, G[j] = 0.0f, state[j] = in.state[j];
#pragma unroll
    for (int i = 0; i < S; ++i) {
      x[i] = in.x[i];
      dh[i] = in.dh[i];  // zero behind the last step
#pragma unroll
      for (int j = 0; j < VEC; ++j) cm[i][j] = fold_gates(in.gate[i].get(j));
    }
    if (!h.full) {  // a = 1, b = 0 there
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) cm[i][j] = i < h.steps ? cm[i][j] : 0.0f;
    }
    keep_folded();
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const Gates g = unfold_gates(cm[i][j]);
        const float xt = x[i].get(j);
        H[j] = fmaf(g.a, H[j], FREE ? xt : g.b * xt);
        A[j] *= g.a;
        G[j] = fmaf(A[j], dh[i].get(j), G[j]);  // what dh of this step leaves in front of the first one
      }
    }
    keep_folded();
#pragma unroll
    for (int j = 0; j < VEC; ++j) B[j] = A[j];
    join_groups<SHAPE::kGroups, false>(A, H, A0, H0, h.group);
    join_groups<SHAPE::kGroups, true>(B, G, B0, G0, h.group);
    if (h.group == SHAPE::kGroups - 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) parts.of[w][col + j] = float2{A[j], H[j]};
    }
    if (h.group == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) parts.back[w][col + j] = G[j];
    }
  }

  // The compiler would rather keep both factors of all steps, in twice the registers, than form them again.
  __device__ __forceinline__ void keep_folded() {
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) asm volatile("" : "+v"(cm[i][j]));
      x[i].renew();
      dh[i].renew();
    }
  }

  static __device__ __forceinline__ float2 part(const Parts& parts, int i, int channel) {
    return float2{parts.of[W - 1 - i][channel].x, parts.back[W - 1 - i][channel]};
  }

  // While the gradient is on its way: the states once more, h_{t-1} - x_t of every step.
  __device__ __forceinline__ void between(const Parts& parts, int w, int col) {
    for (int v = w / kStateWaves * kStateWaves; v < w; ++v) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) state[j] = fmaf(parts.of[v][col + j].x, state[j], parts.of[v][col + j].y);
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) state[j] = fmaf(A0[j], state[j], H0[j]);
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const Gates g = unfold_gates(cm[i][j]);
        const float xt = x[i].get(j);
        before[i][j] = FREE ? state[j] : state[j] - xt;
        state[j] = fmaf(g.a, state[j], FREE ? xt : g.b * xt);
      }
    keep_folded();
  }

  __device__ __forceinline__ void apply(const ScanArgs& a, const Place&, const Share& h, int w, int col, const Parts& parts,
                                        float (&flow)[VEC]) {
    for (int v = W - 1; v > w; --v) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) flow[j] = fmaf(parts.of[v][col + j].x, flow[j], parts.back[v][col + j]);
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) flow[j] = fmaf(B0[j], flow[j], G0[j]);
    const Steps<T, VEC, S> out_gate(a.dgate, a.dgate_stride, h), out_x(a.dx, a.dx_stride, h);
#pragma unroll
    for (int i = S - 1; i >= 0; --i) {
      float vg[VEC], vx[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const Gates g = unfold_gates(cm[i][j]);
        const float gt = dh[i].get(j) + flow[j];
        vx[j] = FREE ? gt : g.b * gt;
        vg[j] = gt * before[i][j] * (g.a * g.b);
        flow[j] = g.a * gt;
      }
      Pack<T, VEC> og, ox;
      og.set(vg);
      ox.set(vx);
      out_x.store(i, ox);
      out_gate.store(i, og);
    }
  }
};

// ---- a few steps: a thread walks VEC channels of one sequence --------------------------------------------------
// What bounds this is the launch: 256 streams of 1500 channels in 32 bits, one step, 3.0 us forward and 3.2 backward; by tiles,
// of which a wavefront uses one row then, 19 and 37.  Four steps 4.8 and 6.2 us, by tiles 20 and 39.  Tiles do not win beyond
// four either (five steps 21 and 40 us by them, 5.5 and 8.4 with room for 16 here, and 16 steps 22 and 40 against 14 and 21): the
// limit keeps the registers of a single step few, which takes 3.4 and 4.2 us with room for 16 and 3.1 and 3.5 with room for 8.
constexpr int kShort = 4;
constexpr int kShortThreads = 256;

template <typename T, int VEC, bool FREE, bool REVERSE>
__global__ __launch_bounds__(kShortThreads) void scan_short_kernel(ScanArgs a, uint32_t first) {
  const uint32_t groups = (uint32_t)((a.channels / VEC + kShortThreads - 1) / kShortThreads);  // of a sequence
  const uint32_t number = first + blockIdx.x;
  const int64_t s = number / groups;
  const int64_t d = ((int64_t)(number - (uint32_t)s * groups) * kShortThreads + threadIdx.x) * VEC;
  if (d >= a.channels) return;
  int64_t begin, length;
  sequence_rows(a, s, begin, length);
  auto at = [&](const void* array, int64_t stride, int t) {
    return reinterpret_cast<const Pack<T, VEC>*>(static_cast<const T*>(array) + (begin + t) * stride + d);
  };
  auto to = [&](void* array, int64_t stride, int t) {
    return reinterpret_cast<Pack<T, VEC>*>(static_cast<T*>(array) + (begin + t) * stride + d);
  };
  Pack<T, VEC> gate[kShort]{}, x[kShort]{}, dh[kShort]{};
#pragma unroll
  for (int t = 0; t < kShort; ++t)
    if (t < length) {
      gate[t] = *at(a.gate, a.gate_stride, t);
      x[t] = *at(a.x, a.x_stride, t);
      if (REVERSE) dh[t] = *at(a.dh, a.dh_stride, t);
    }
  float carry[VEC], state[VEC], before[kShort][VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) carry[j] = a.first ? a.first[s * a.channels + d + j] : 0.0f;
  float* kept = a.states ? a.states + state_row(s, begin, 0) * a.channels + d : nullptr;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    state[j] = carry[j];
    if (REVERSE) state[j] = length > 0 ? kept[j] : 0.0f;
    if (!REVERSE && kept && length > 0) kept[j] = state[j];
  }
#pragma unroll
  for (int t = 0; t < kShort; ++t)
    if (t < length) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const Gates g = gates_of(gate[t].get(j));
        const float xt = x[t].get(j);
        before[t][j] = state[j];
        state[j] = fmaf(g.a, state[j], FREE ? xt : g.b * xt);
      }
      if (!REVERSE) {
        Pack<T, VEC> h;
        h.set(state);
        *to(a.h, a.h_stride, t) = h;
      }
    }
  if (REVERSE) {
#pragma unroll
    for (int t = kShort - 1; t >= 0; --t)
      if (t < length) {
        float vg[VEC], vx[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const Gates g = gates_of(gate[t].get(j));
          const float gt = dh[t].get(j) + carry[j], inner = FREE ? before[t][j] : before[t][j] - x[t].get(j);
          vx[j] = FREE ? gt : g.b * gt;
          vg[j] = gt * inner * (g.a * g.b);
          carry[j] = g.a * gt;
        }
        Pack<T, VEC> og, ox;
        og.set(vg);
        ox.set(vx);
        *to(a.dx, a.dx_stride, t) = ox;
        *to(a.dgate, a.dgate_stride, t) = og;
      }
  }
  if (a.last) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.last[s * a.channels + d + j] = REVERSE ? carry[j] : state[j];
  }
}

// ---- short sequences: a workgroup walks the tiles of one sequence and block ---------------------------------
// One pass over the data: 512 sequences of 128 x 2048 in bfloat16 forward 153 us (5.3 TB/s), backward 258 (5.2); 20 x 35 x 1500 in
// 32 bits 4.5 and 7.2, a launch and a chain of loads, steps, exchange and stores.  A tile has the rows of one kept state: with
// twice as many 183 and 416 us, 6.0 and 12.5 (in 32 bits 512 x 128 x 1024 139 and 272, 149 and 249 as it is).  Backward, 170 to
// 243 registers in 16 bits leave two wavefronts to a SIMD.  Of sequences shorter than 64 steps only a part of the rows is
// there: 2048 x 32 x 2048 takes 204 and 484 us.
template <typename TILE, int W>
__global__ __launch_bounds__(W * 64) void scan_walk_kernel(ScanArgs a, uint32_t first) {
  using SHAPE = typename TILE::SHAPE;
  constexpr int VEC = SHAPE::kVec, kBlock = SHAPE::kBlock, kRows = W * SHAPE::kRows;
  __shared__ typename TILE::Parts parts[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane % SHAPE::kLanes * VEC;
  const uint32_t blocks = (uint32_t)((a.channels + kBlock - 1) / kBlock);
  const uint32_t s = (first + blockIdx.x) / blocks, block = first + blockIdx.x - s * blocks;
  int64_t begin, length;
  sequence_rows(a, s, begin, length);
  const int64_t count = length > 0 ? (length + kRows - 1) / kRows : 1;
  const int64_t d = (int64_t)block * kBlock + col;
  float carry[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) carry[j] = a.first && d + j < a.channels ? a.first[s * a.channels + d + j] : 0.0f;
  for (int64_t i = 0; i < count; ++i) {
    const int64_t index = TILE::kReverse ? count - 1 - i : i;
    const Place p{begin + index * kRows, length - index * kRows, state_row(s, begin, index * (kRows / kStateRows)), s, 0, i,
                  (int32_t)block, 0, 1};
    const Share h = share_of<SHAPE>(a, p, w, lane);
    typename TILE::Input in;
    TILE tile;
    in.load(a, p, w, h);
    tile.fold(in, h, w, col, parts[i & 1]);
    __syncthreads();
    tile.between(parts[i & 1], w, col);
    float state[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) state[j] = carry[j];
#pragma unroll
    for (int v = 0; v < W; ++v)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float2 part = TILE::part(parts[i & 1], v, col + j);
        carry[j] = fmaf(part.x, carry[j], part.y);
      }
    tile.apply(a, p, h, w, col, parts[i & 1], state);
  }
  if (a.last && w == 0 && lane < SHAPE::kLanes && d < a.channels) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.last[s * a.channels + d + j] = carry[j];
  }
}

// ---- long sequences: tiles side by side ---------------------------------------------------------------------
// Tiles of one sequence and block of channels follow each other.  What a tile does to a state is left in a word of its own
// (A with its sign bit set, H), which is read by the tiles behind it in its group of kGroup tiles; the last tile of a group,
// and the first of a sequence, leave the state behind them instead (0 with the sign bit set, state).  A tile joins, in order,
// the state in front of its group and the words of the group's tiles before its own: always the same sums, whoever comes
// first.  A word is stored and loaded whole, so that it needs no fence; zero says that it is not there yet.
constexpr int kGroup = 16;

struct Chain {
  unsigned long long* words;  // [tile rows][channels]
  uint32_t* ticket;
  uint32_t tickets;   // (tile row, block) in all
  int64_t tile_rows;  // without row_offsets: tiles of a sequence
};

__device__ __forceinline__ unsigned long long chain_word(float a, float h) {
  // a NaN leaves no finite state, whatever comes in
  if (!(a <= 1.0f)) h = __builtin_nanf(""), a = 1.0f;
  return (unsigned long long)(__float_as_uint(a) | 0x80000000u) << 32 | __float_as_uint(h);
}

// The state in front of the tile at `position` > 0 of its chain (in the direction of travel), whose words lie `step` behind
// those of the one before it.  The rows of words waited for belong to lower tickets, and every ticket's workgroup leaves
// its row, whatever the offsets hold: they run, or have run, and none of them waits for this one, so every wait ends.  All
// words are asked for at once.
__device__ __forceinline__ float chain_state(const unsigned long long* word, int64_t step, int64_t position) {
  const int before = (int)(position % kGroup);
  const int n = before + (position > before ? 1 : 0);
  unsigned long long v[kGroup];
  for (;;) {
    unsigned long long all = ~0ull;
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      v[i] = __hip_atomic_load(word - (n - (i < n ? i : n - 1)) * step, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int i = 0; i < kGroup; ++i) all &= v[i];
    if (all >> 63) break;
    __builtin_amdgcn_s_sleep(1);
  }
  float state = 0.0f;  // the first word is a state
#pragma unroll
  for (int i = 0; i < kGroup; ++i)
    if (i < n) state = fmaf(__uint_as_float((uint32_t)(v[i] >> 32) & 0x7fffffffu), state, __uint_as_float((uint32_t)v[i]));
  return state;
}

// Tile `ticket`.  Equal sequences: all first tiles, then all second ones.  With offsets: tile row
// begin / ROWS + sequence + index, as for the kept states; rows of that numbering between two sequences stay empty.
template <int ROWS, int BLOCK, bool REVERSE>
__device__ __forceinline__ Place tile_of(const ScanArgs& a, const Chain& chain, uint32_t ticket) {
  const uint32_t blocks = (uint32_t)((a.channels + BLOCK - 1) / BLOCK);
  uint32_t row = ticket / blocks;
  Place p;
  p.block = (int32_t)(ticket - row * blocks);
  int64_t begin, length, index, count;
  if (!a.row_offsets) {
    const uint32_t sequences = (uint32_t)a.sequences;
    p.position = row / sequences;
    p.sequence = row - (uint32_t)p.position * sequences;
    sequence_rows(a, p.sequence, begin, length);
    count = chain.tile_rows;
    index = REVERSE ? count - 1 - p.position : p.position;
    p.word_row = p.sequence * count + index;
    p.there = 1;
  } else {
    if (REVERSE) row = chain.tickets / blocks - 1 - row;
    // the last sequence whose first tile row is not behind this one
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = a.sequences;
    while (hi - lo > 1) {
      const int64_t stride = (hi - lo + 63) / 64;
      const int64_t at = lo + lane * stride;
      if (at < hi) sequence_rows(a, at, begin, length);
      const bool before = at < hi && begin / ROWS + at <= row;
      const int passed = __popcll(__ballot(before));
      const int64_t next = lo + passed * stride;
      if (passed) {
        lo = next - stride;
        hi = next < hi ? next : hi;
      } else {
        hi = lo + 1;
      }
    }
    p.sequence = __builtin_amdgcn_readfirstlane((int)lo);
    sequence_rows(a, p.sequence, begin, length);
    count = length > 0 ? (length + ROWS - 1) / ROWS : 1;
    index = (int64_t)row - (begin / ROWS + p.sequence);
    p.position = REVERSE ? count - 1 - index : index;
    p.word_row = row;
    p.there = index >= 0 && index < count;
  }
  p.row = begin + index * ROWS;
  p.left = length - index * ROWS;
  p.state = state_row(p.sequence, begin, index * (ROWS / kStateRows));
  p.last = p.position + 1 == count;
  return p;
}

// The next tile that is there; `there` is zero behind the last one.  A tile row that belongs to no sequence leaves words
// all the same: with offsets that do not ascend, some tile may look for them.
template <int ROWS, int BLOCK, bool REVERSE>
__device__ __forceinline__ Place next_tile(const ScanArgs& a, const Chain& chain, int lane) {
  for (;;) {
    uint32_t ticket = 0;
    if (lane == 0) ticket = atomicAdd(chain.ticket, 1u);
    ticket = __builtin_amdgcn_readfirstlane(ticket);
    if (ticket >= chain.tickets) return Place{};
    const Place p = tile_of<ROWS, BLOCK, REVERSE>(a, chain, ticket);
    if (p.there) return p;
    for (int64_t channel = (int64_t)p.block * BLOCK + lane; channel < (int64_t)(p.block + 1) * BLOCK && channel < a.channels; channel += 64)
      __hip_atomic_store(chain.words + p.word_row * a.channels + channel, chain_word(1.0f, 0.0f), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// A barrier for what lies in LDS: loads that are on their way stay on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Every element is read once: gates and inputs stay in registers (backward: the folded gates, and the states formed again)
// while the chain brings the state.  65536 x 2048 in bfloat16, one sequence, with the clear of the words (5.7 us): forward 197 us
// (4.1 TB/s), backward 362 (3.7); 65536 x 1024 in 32 bits 179 and 306, 65536 x 2047 in bfloat16, two bytes a lane, 281 and 414.
// What bounds it in 16 bits is that nothing covers a workgroup's wait for the chain: ten wavefronts of 97 or 98 registers
// forward and of 168 backward (5 to 8 more of those are spilled, 24 to 36 bytes of scratch) leave room for one workgroup to a
// compute unit, where 96 would for two, and all of them load, wait and store side by side.  Two passes over the data would
// move 1.34 and 2.15 GB, 206 and 330 us at the 6.5 TB/s of a bare kernel.
// Tried: the tile's own wavefronts seeing to the chain (224 to 247 and 332 to 357 us), tiles of 64 steps (288 and 397 at best), groups of
// 8 and of 32 tiles (more hops, more words to read), tickets from several counters (240 to 292 and 348 to 390: rows of memory
// are then read piece by piece), gates formed twice to have more workgroups (260 to 315 forward).
// W wavefronts work on tiles; those behind them, one to 64 channels, see to the chain: the first of them takes tickets, all
// leave words, and wait for those of other tiles.
template <typename TILE, int W, int RESIDENT>
__global__ __launch_bounds__(W * 64 + TILE::kBlock, RESIDENT) void scan_chain_kernel(ScanArgs a, Chain chain) {
  using SHAPE = typename TILE::SHAPE;
  constexpr int VEC = SHAPE::kVec, kBlock = SHAPE::kBlock, kRows = W * SHAPE::kRows;
  __shared__ typename TILE::Parts parts[2];
  __shared__ Place places[2];
  __shared__ float carry[kBlock];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= W) {
    if (w == W) {
      const Place p = next_tile<kRows, kBlock, TILE::kReverse>(a, chain, lane);
      if (lane == 0) places[0] = p;
    }
    lds_barrier();
    for (int turn = 0;; turn ^= 1) {
      const Place p = uniform(places[turn]);
      if (!p.there) return;
      if (w == W) {
        const Place next = next_tile<kRows, kBlock, TILE::kReverse>(a, chain, lane);
        if (lane == 0) places[turn ^ 1] = next;
      }
      lds_barrier();
      const int mine = (w - W) * 64 + lane;
      const int64_t channel = (int64_t)p.block * kBlock + mine;
      if (channel < a.channels) {
        const bool closes = p.position == 0 || p.position % kGroup == kGroup - 1;
        unsigned long long* word = chain.words + p.word_row * a.channels + channel;
        float A = 1.0f, H = 0.0f;
#pragma unroll
        for (int v = 0; v < W; ++v) {
          const float2 part = TILE::part(parts[turn], v, mine);
          H = fmaf(part.x, H, part.y);
          A *= part.x;
        }
        if (!closes) __hip_atomic_store(word, chain_word(A, H), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int64_t carried = p.sequence * a.channels + channel;
        float state;
        if (p.position == 0)
          state = a.first ? a.first[carried] : 0.0f;
        else
          state = chain_state(word, TILE::kReverse ? -a.channels : a.channels, p.position);
        carry[mine] = state;
        state = fmaf(A, state, H);
        if (closes) __hip_atomic_store(word, chain_word(0.0f, state), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (p.last && a.last) a.last[carried] = state;
      }
      lds_barrier();
    }
  }
  const int col = lane % SHAPE::kLanes * VEC;
  lds_barrier();
  for (int turn = 0;; turn ^= 1) {
    const Place p = uniform(places[turn]);
    if (!p.there) return;
    const Share h = share_of<SHAPE>(a, p, w, lane);
    typename TILE::Input in;
    in.load(a, p, w, h);
    TILE tile;
    tile.fold(in, h, w, col, parts[turn]);
    lds_barrier();
    tile.between(parts[turn], w, col);
    lds_barrier();
    float state[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) state[j] = carry[col + j];
    tile.apply(a, p, h, w, col, parts[turn], state);
  }
}

// Sequences of more steps than a tile holds are cut into tiles.
constexpr int kTileRows = 128;
constexpr int kChainGroups = 4 * 256;  // more than are resident at a time: those that find no ticket left end at once

// A launch has less than 2^32 threads: workgroups beyond them, of many short sequences, are launched behind the others.
template <int THREADS>
hipError_t launch_all(void (*kernel)(ScanArgs, uint32_t), const ScanArgs& a, int64_t groups, hipStream_t stream) {
  constexpr int64_t kMost = (int64_t)UINT32_MAX / THREADS;
  for (int64_t first = 0; first < groups; first += kMost) {
    kernel<<<dim3((uint32_t)(groups - first < kMost ? groups - first : kMost)), THREADS, 0, stream>>>(a, (uint32_t)first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <template <typename, int, bool> class TILE, typename SHAPE, bool FREE>
hipError_t launch_tiles(const ScanArgs& a, void* workspace, hipStream_t stream) {
  const int64_t blocks = ceil_div(a.channels, SHAPE::kBlock);
  constexpr int kWaves = kTileRows / SHAPE::kRows;
  if (a.max_length <= kShort) {
    using T = typename SHAPE::T;
    const int64_t groups = ceil_div(a.channels / SHAPE::kVec, kShortThreads) * a.sequences;
    return launch_all<kShortThreads>(scan_short_kernel<T, SHAPE::kVec, FREE, TILE<SHAPE, kWaves, FREE>::kReverse>, a, groups, stream);
  }
  if (!scan_chained(a)) {
    constexpr int W = SHAPE::kStateWaves;
    return launch_all<W * 64>(scan_walk_kernel<TILE<SHAPE, W, FREE>, W>, a, a.sequences * blocks, stream);
  }
  Chain chain{};
  chain.ticket = static_cast<uint32_t*>(workspace);
  chain.words = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + 256);
  chain.tile_rows = ceil_div(a.max_length, kTileRows);
  chain.tickets = (uint32_t)(scan_word_rows(a) * blocks);
  const hipError_t e = launch_clear_words(static_cast<uint32_t*>(workspace), scan_workspace_bytes(a) / 4, stream);
  if (e != hipSuccess) return e;
  const uint32_t groups = chain.tickets < (uint32_t)kChainGroups ? chain.tickets : (uint32_t)kChainGroups;
  using Kernel = TILE<SHAPE, kWaves, FREE>;
  constexpr int kResident = Kernel::kReverse ? 3 : 4;
  scan_chain_kernel<Kernel, kWaves, kResident><<<groups, kWaves * 64 + SHAPE::kBlock, 0, stream>>>(a, chain);
  return hipGetLastError();
}

template <typename SHAPE>
hipError_t launch_shape(const ScanArgs& a, void* workspace, bool free_input, bool backward, hipStream_t stream) {
  if (backward)
    return free_input ? launch_tiles<BackwardTile, SHAPE, true>(a, workspace, stream) : launch_tiles<BackwardTile, SHAPE, false>(a, workspace, stream);
  return free_input ? launch_tiles<ForwardTile, SHAPE, true>(a, workspace, stream) : launch_tiles<ForwardTile, SHAPE, false>(a, workspace, stream);
}

// Channels to a lane: as many as all rows are aligned for, eight bytes of them at most.
template <typename T>
hipError_t launch(const ScanArgs& a, void* workspace, bool free_input, bool backward, hipStream_t stream) {
  uint64_t bits = (uint64_t)a.channels * sizeof(T);
  for (const void* p : {a.gate, a.x, static_cast<const void*>(a.h), a.dh, static_cast<const void*>(a.dgate), static_cast<const void*>(a.dx)})
    bits |= reinterpret_cast<uintptr_t>(p);
  for (int64_t stride : {a.gate_stride, a.x_stride, a.h_stride, a.dh_stride, a.dgate_stride, a.dx_stride})
    bits |= (uint64_t)stride * sizeof(T);
  if constexpr (sizeof(T) == 2) {
    if (bits % 8 == 0) return launch_shape<Shape<T, 4, 2, 8>>(a, workspace, free_input, backward, stream);
    if (bits % 4 == 0) return launch_shape<Shape<T, 2, 1, 16>>(a, workspace, free_input, backward, stream);
  } else {
    if (bits % 8 == 0) return launch_shape<Shape<T, 2, 2, 8>>(a, workspace, free_input, backward, stream);
  }
  return launch_shape<Shape<T, 1, 1, 16>>(a, workspace, free_input, backward, stream);
}

}  // namespace

int64_t scan_word_rows(const ScanArgs& a) {
  return a.row_offsets ? a.rows / kTileRows + a.sequences : a.sequences * ceil_div(a.max_length, kTileRows);
}

// Long sequences are cut into tiles that wait for each other, unless there are so many of them (times blocks of 64
// channels, of which a workgroup has two in 16 bits at 8 or 4 bytes a lane) that walking them fills the device well enough, and
// none is much longer than the mean.  In us, tiles side by side and one behind the other, forward / backward in bfloat16, by
// that number: 228 (12 x 1500 x 1200) 45/71 and 59/127; 456 (24 of them) 78/151 and 68/163; 512 (16 x 1024 x 2048) 56/104 and
// 45/108; 768 (24) 82/144 and 79/135; 912 (48 x 1500 x 1200) 155/276 and 141/251, of 187 to 1500 steps 111/183 and 95/169; 2048
// (64 x 1024 x 2048) 191/350 and 172/277.  In 32 bits 480 (20 x 200 x 1500) 31/38 and 19/30.  Around the limit the two directions
// do not agree, and sequences of two tiles would rather be walked below it as well: 192 (8 x 200 x 1500) 17/20 and 11/19.
constexpr int64_t kWalkBlocks = 384;
bool scan_chained(const ScanArgs& a) {
  if (a.max_length <= kTileRows) return false;
  return a.sequences * ceil_div(a.channels, 64) < kWalkBlocks || a.max_length > 4 * (a.rows / a.sequences);
}

int64_t scan_workgroups(const ScanArgs& a) {
  return (scan_chained(a) ? scan_word_rows(a) : a.sequences) * ceil_div(a.channels, 64);
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
