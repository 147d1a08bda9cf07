// Rotary positions on several axes behind the norm of the heads, forward and backward.
//
// Every element is read once and written once, so HBM bounds the time of many tokens (16 + 16 heads of 64 in bf16 are 8 KB a token).  A
// thread block works on one tensor.  Its warps take tokens: the lanes compute a token's cosines and sines once, a pair each, for all
// heads; then the heads pass through, each on as many lanes as hold it in runs of `PU` pairs.  A lane holds both elements of its pairs, so
// that turning them needs no exchange, and the norm of a head is a sum over its lanes.  Weights and biases of the lane's elements stay in
// registers, which is what a block for each tensor is for: read from shared memory for every head they kept its data path busy to 83%
// (30 frames: 79 us, with registers 68).  Runs of later heads arrive by asynchronous copies, each thread's for itself, so that no
// load is waited for.  100 frames (137,400 tokens): 207 us, in a loop of calls 213, 5.3 TB/s; two copies of the same size side by side reach
// 5.8.  Five blocks on the SM instead of four: the same on their own, 228 us in a loop (fewer registers, so that values are computed again).
//
// Angles: a frequency is kept as the 64-bit fraction of a turn that one position advances by.  position * fraction modulo 2^64 is the exact
// product modulo one turn, whatever the position; its upper 32 bits go to sincospi.
#include <cmath>
#include <type_traits>

#include "elements.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace avggt {

namespace {

constexpr int kWarps = 4;
constexpr int kBlocksPerSm = 4, kBackBlocksPerSm = 3;      // as the launch bounds have it
constexpr int kMaxPairs = 128;      // head_dim <= 256
constexpr int kMaxTable = 256;      // pairs of the tokens that a warp works on together: 32 lanes of at most eight
constexpr int kMaxTokens = 8;       // of them, so that their positions on three axes are a warp's
constexpr int kMaxSegs = 4;         // blocks of pairs: up to three axes, and the elements that are not turned

// Stages of the pipeline of copies, of which all but one are in flight.
__host__ __device__ constexpr int stages_of(int stage_bytes) { return stage_bytes == 0 ? 0 : 4; }

struct RotaryTensor {
  const char* in;                   // forward: the heads; backward: the gradient of the turned heads
  char* out;
  const char* x;                    // backward with a norm: the heads
  int64_t in_ts, in_hs, out_ts, out_hs, x_ts, x_hs;   // strides in bytes
  const float* weight;
  const float* bias;
  int heads;
  int heads_at_once;                // of a token that a warp works on together: a chunk
  int tokens_at_once;               // more than one where a token's heads leave lanes over
  int chunks;                       // of a token's heads
  int first_block, n_blocks;        // the thread blocks that work on this tensor
};

struct RotaryArgs {
  RotaryTensor t[3];                // Q, K, V (V is copied)
  const int32_t* positions;
  float* partials;                  // backward: [n_blocks of Q, then of K][2][d]
  int n_tokens, n_axes, d, n_pairs;
  int units;                        // runs of PU pairs in a head
  int lanes;                        // lanes of a head, a power of two
  int n_segs;
  int seg_start[kMaxSegs + 1];      // in pairs
  int norm;
  float eps, inv_d, sign;           // sign: 1, or -1 to turn back
  int split;                        // a warp takes one chunk instead of every so-many-th token
  uint64_t turn[kMaxPairs];
  int8_t axis[kMaxPairs];           // -1: not turned
};

// Behind the pipeline in shared memory: each warp's table of its token's cosines and sines, and in the end (backward) its rows of sums.
struct RotarySmem {
  float *cosine, *sine, *sums;
};

// Pairs of a warp's table.  What shared memory a block does not take is left to the cache that the copies pass through.
__host__ __device__ constexpr int table_pairs(bool groups) { return groups ? kMaxTable : kMaxPairs; }

template <bool GROUPS> __device__ __forceinline__ RotarySmem rotary_smem(unsigned char* base) {
  constexpr int kTable = table_pairs(GROUPS);
  float* p = reinterpret_cast<float*>(base);
  return {p + (threadIdx.x >> 5) * 2 * kTable, p + (threadIdx.x >> 5) * 2 * kTable + kTable, p + kWarps * 2 * kTable};
}

// Elements of the first halves of a unit's pairs, and of the second.
template <int PU, bool ADJ>
__device__ __forceinline__ void unit_offsets(const RotaryArgs& a, int unit, int& lo, int& hi) {
  const int p = unit * PU;
  if (ADJ) {
    lo = 2 * p;
    hi = lo + PU;
    return;
  }
  lo = hi = 0;
#pragma unroll
  for (int s = 0; s < kMaxSegs; ++s)
    if (s < a.n_segs && p >= a.seg_start[s] && p < a.seg_start[s + 1]) {
      lo = a.seg_start[s] + p;                       // 2 * start + (p - start)
      hi = lo + (a.seg_start[s + 1] - a.seg_start[s]);
    }
}

// A sum over a head's lanes.  LANES: their number, or 0 where it is not known to the compiler.
template <int LANES> __device__ __forceinline__ float head_sum(float v, int lanes) {
  if constexpr (LANES > 0) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  } else {
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  return v;
}

// Element index, within the 2 * PU values of a unit, of the first and the second of pair i.
template <int PU, bool ADJ> __device__ __forceinline__ constexpr int first_of(int i) { return ADJ ? 2 * i : i; }
template <int PU, bool ADJ> __device__ __forceinline__ constexpr int second_of(int i) { return ADJ ? 2 * i + 1 : PU + i; }

// Where a lane's units are in a head: in bytes, of the halves of the first unit's pairs from the head's start, and of the others from the
// first half of the first.
template <typename T, int PU, int NU, bool ADJ>
struct LaneUnits {
  uint32_t head, token;              // the lane's head of a chunk and its token of those at once
  int first;                         // bytes of the first half of its first unit
  int lo[NU], hi[NU];                // from there on
  int pair[NU];                      // the first pair in the warp's table
  bool have[NU];
  __device__ __forceinline__ LaneUnits(const RotaryArgs& a, const RotaryTensor& t, int lane, int lanes, bool groups) {
    const uint32_t place = lane / lanes;
    token = groups ? place / t.heads_at_once : 0;
    head = place - token * t.heads_at_once;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int unit = lane % lanes + i * 32;
      have[i] = unit < a.units;
      unit_offsets<PU, ADJ>(a, have[i] ? unit : 0, lo[i], hi[i]);
      pair[i] = static_cast<int>(token) * a.n_pairs + (have[i] ? unit * PU : 0);
      lo[i] *= static_cast<int>(sizeof(T));
      hi[i] *= static_cast<int>(sizeof(T));
    }
    first = lo[0];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      lo[i] -= first;
      hi[i] -= first;
    }
  }
  // The weights' elements
  __device__ __forceinline__ int lo_element(int i) const { return (first + lo[i]) / static_cast<int>(sizeof(T)); }
  __device__ __forceinline__ int hi_element(int i) const { return (first + hi[i]) / static_cast<int>(sizeof(T)); }
};

// A lane's units of a head.  From a pipeline stage in shared memory where runs have at least four bytes (each thread fetches and reads
// its own 16, 8 or 4 bytes, so that nothing but the thread's own wait stands between; what is never fetched is zeroed once), else
// straight from memory.
template <typename T, int PU, int NU, bool ADJ>
struct HeadRuns {
  using R = Run<T, PU>;
  using Units = LaneUnits<T, PU, NU, ADJ>;
  static constexpr bool kAsync = R::kBytes >= 4;
  static constexpr int kApart = 32 * kWarps * R::kBytes;                   // bytes between a thread's runs
  static constexpr int kStageBytes = kAsync ? 2 * NU * kApart : 0;
  R lo[NU], hi[NU];

  static __device__ __forceinline__ void fetch(uint32_t own, const char* p, const Units& u) {   // own: the thread's first run in the stage
#pragma unroll
    for (int i = 0; i < NU; ++i)
      if (u.have[i]) {
        R::load_async(own + 2 * i * kApart, p + u.lo[i]);
        R::load_async(own + (2 * i + 1) * kApart, p + u.hi[i]);
      }
  }
  static __device__ __forceinline__ void clear(unsigned char* own, int bytes) {
    if constexpr (kAsync)
      for (int at = 0; at < bytes; at += kApart)
#pragma unroll
        for (int w = 0; w < R::kBytes; w += 4) *reinterpret_cast<uint32_t*>(own + at + w) = 0u;
  }
  __device__ __forceinline__ void take(const unsigned char* own) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      lo[i].load(own + 2 * i * kApart);
      hi[i].load(own + (2 * i + 1) * kApart);
    }
  }
  __device__ __forceinline__ void load(const char* p, const Units& u, bool on) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (u.have[i] && on) {
        lo[i].load(p + u.lo[i]);
        hi[i].load(p + u.hi[i]);
      } else {
        lo[i].zero();
        hi[i].zero();
      }
    }
  }
  __device__ __forceinline__ void store(char* p, const Units& u, bool on) const {
#pragma unroll
    for (int i = 0; i < NU; ++i)
      if (u.have[i] && on) {
        lo[i].store(p + u.lo[i]);
        hi[i].store(p + u.hi[i]);
      }
  }
  __device__ __forceinline__ void values(float (&v)[NU][2 * PU]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < PU; ++e) {
        v[i][e] = lo[i].value(e);
        v[i][PU + e] = hi[i].value(e);
      }
  }
  __device__ __forceinline__ void set(const float (&v)[NU][2 * PU]) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      lo[i].set(v[i]);
      hi[i].set(v[i] + PU);
    }
  }
};

// x <- x - mean of the head (lanes' units that it does not have stay zero).
template <int PU, int NU, int LANES>
__device__ __forceinline__ void centre(float (&x)[NU][2 * PU], const bool (&have)[NU], const RotaryArgs& a) {
  if (a.norm != AVGGT_NORM_LAYER) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i) sum += sum_of<2 * PU>(x[i]);
  const float mean = head_sum<LANES>(sum, a.lanes) * a.inv_d;
#pragma unroll
  for (int i = 0; i < NU; ++i) add_each<2 * PU>(x[i], have[i] ? -mean : 0.f);
}

// The unit's pairs turned by the angles of c and s.
template <int PU, bool ADJ>
__device__ __forceinline__ void turn_pairs(float (&x)[2 * PU], const float (&c)[PU], const float (&s)[PU]) {
  if constexpr (!ADJ && PU % 2 == 0) {
#pragma unroll
    for (int e = 0; e < PU; e += 2) {
      const uint64_t lo = two(x + e), hi = two(x + PU + e), cc = two(c + e), ss = two(s + e);
      put_two(sub_f32x2(mul_f32x2(lo, cc), mul_f32x2(hi, ss)), x + e);
      put_two(fma_f32x2(lo, ss, mul_f32x2(hi, cc)), x + PU + e);
    }
  } else {
#pragma unroll
    for (int e = 0; e < PU; ++e) {
      float& p0 = x[first_of<PU, ADJ>(e)];
      float& p1 = x[second_of<PU, ADJ>(e)];
      const float turned = p0 * c[e] - p1 * s[e];
      p1 = p0 * s[e] + p1 * c[e];
      p0 = turned;
    }
  }
}

template <int N>
__device__ __forceinline__ void read_floats(const float* p, float* v) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 q = *reinterpret_cast<const float4*>(p + i);
      v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = p[i];
  }
}

// The table of a warp's token: its cosines and sines, a lane's N pairs of them, 32 apart.  Pairs that are not turned (and those that the
// head does not have) turn by nothing.  The positions of the next token are read while the warp works on the one before.
template <int N>
struct TokenAngles {
  uint64_t turn[N];
  const int32_t* at[N];
  int pos[N];
  __device__ __forceinline__ TokenAngles(const RotaryArgs& a, uint32_t token, int, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = lane + 32 * i;
      const int axis = p < a.n_pairs ? a.axis[p] : -1;
      turn[i] = axis >= 0 ? a.turn[p] : 0;
      at[i] = a.positions + static_cast<uint64_t>(token) * a.n_axes + (axis >= 0 ? axis : 0);
    }
  }
  __device__ __forceinline__ void read() {
#pragma unroll
    for (int i = 0; i < N; ++i) pos[i] = *at[i];
  }
  __device__ __forceinline__ void step(int64_t elements) {
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] += elements;
  }
  __device__ __forceinline__ void fill(const RotaryArgs& a, const RotarySmem& s, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(pos[i])) * turn[i];     // of 2^64 a turn
      float c, sn;
      // upper half as a signed fraction of a turn; sincospi takes half turns
      sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &sn, &c);
      s.cosine[lane + 32 * i] = c;
      s.sine[lane + 32 * i] = sn * a.sign;
    }
  }
};

// The same for several tokens at once, whose tables follow one another.  Their positions are read by as many lanes as there are.
template <int N>
struct GroupAngles {
  uint64_t turn[N];
  int axis[N];
  const int32_t* at;                 // the lane's position of the tokens
  int64_t left;                      // positions from there on
  int tokens, pos = 0;
  __device__ __forceinline__ GroupAngles(const RotaryArgs& a, uint32_t token, int tokens_at_once, int lane) : tokens(tokens_at_once) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = lane + 32 * i;
      axis[i] = p < a.n_pairs ? a.axis[p] : -1;
      turn[i] = axis[i] >= 0 ? a.turn[p] : 0;
      if (axis[i] < 0) axis[i] = 0;
    }
    const int64_t first = static_cast<int64_t>(token) * a.n_axes + lane;
    at = a.positions + first;
    left = lane < tokens * a.n_axes ? static_cast<int64_t>(a.n_tokens) * a.n_axes - first : 0;
  }
  __device__ __forceinline__ void read() {
    if (left > 0) pos = *at;
  }
  __device__ __forceinline__ void step(int64_t elements) {
    at += elements;
    left -= elements;
  }
  __device__ __forceinline__ void fill(const RotaryArgs& a, const RotarySmem& s, int lane) const {
    for (int t = 0; t < tokens; ++t)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t p = __shfl_sync(0xffffffffu, pos, t * a.n_axes + axis[i]);
        const uint64_t phase = static_cast<uint64_t>(p) * turn[i];           // of 2^64 a turn
        float c, sn;
        sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f, &sn, &c);
        if (lane + 32 * i < a.n_pairs) {
          s.cosine[t * a.n_pairs + lane + 32 * i] = c;
          s.sine[t * a.n_pairs + lane + 32 * i] = sn * a.sign;
        }
      }
  }
};
// A lane's pairs of a table: heads of at most 32 * that many pairs.
template <int PU, int LANES> constexpr int kPairsOfLane = LANES == 0 ? kMaxPairs / 32 : LANES * PU > 32 ? LANES * PU / 32 : 1;

// What a thread block works on: one tensor, of which its warps take every so-many-th token each (or group of tokens at once), in chunks of
// its heads; with few tokens a warp takes one chunk.
struct Share {
  int which;
  uint32_t token, token_step, chunk, chunks, todo;     // the warp's first token, from there to its next; its first chunk; how many it has
  __device__ __forceinline__ Share(const RotaryArgs& a, bool several) {
    which = static_cast<int>(blockIdx.x) >= a.t[2].first_block ? 2 : static_cast<int>(blockIdx.x) >= a.t[1].first_block ? 1 : 0;
    const RotaryTensor& t = a.t[which];
    const uint32_t at_once = several ? t.tokens_at_once : 1, groups = (static_cast<uint32_t>(a.n_tokens) + at_once - 1) / at_once;
    const uint32_t mine = (blockIdx.x - t.first_block) * kWarps + (threadIdx.x >> 5), step = t.n_blocks * kWarps;
    chunks = t.chunks;
    token_step = step * at_once;
    if (a.split) {
      const uint32_t group = mine / chunks;
      token = group * at_once;
      chunk = mine - group * chunks;
      todo = group < groups ? 1 : 0;
    } else {
      token = mine * at_once;
      chunk = 0;
      todo = mine < groups ? (groups - mine + step - 1) / step * chunks : 0;
    }
  }
};

// A lane's address in a tensor: head by head, `step` bytes each, and from a token's last chunk to the next token's first, `turn` bytes.
struct Steps {
  int64_t step, turn;
  __device__ __forceinline__ Steps(int64_t token_stride, int64_t chunk_stride, const Share& s)
      : step(chunk_stride), turn(static_cast<int64_t>(s.token_step) * token_stride - static_cast<int64_t>(s.chunks - 1) * chunk_stride) {}
};
__device__ __forceinline__ int64_t start_of(int64_t token_stride, int64_t head_stride, uint32_t token, uint32_t head, int first) {
  return static_cast<int64_t>(token) * token_stride + static_cast<int64_t>(head) * head_stride + first;
}

// PU: pairs of a unit; NU: units of a lane.  (PU, NU) is (8, 1) or (4, 1) where runs of that many elements are aligned and no block
// of pairs ends inside one, else (2, 2) or (1, 4).  LANES: lanes of a head, or 0 where the compiler does not know them.
// GROUPS: some tensor's heads leave room for several tokens at once (a variant of its own: 100 frames of 16 heads, which need none of it, took 237 us
// with it and 209 without).
template <typename T, int PU, int NU, bool ADJ, int LANES, bool GROUPS>
__global__ void __launch_bounds__(32 * kWarps, kBlocksPerSm) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  using Runs = HeadRuns<T, PU, NU, ADJ>;
  constexpr int kStageBytes = Runs::kStageBytes, kStages = stages_of(kStageBytes);
  const int lane = threadIdx.x & 31, lanes = LANES > 0 ? LANES : a.lanes;
  const RotarySmem s = rotary_smem<GROUPS>(smem + kStages * kStageBytes);
  const uint32_t own = threadIdx.x * Runs::R::kBytes;
  Runs::clear(smem + own, kStages * kStageBytes);
  const Share share(a, GROUPS);
  const RotaryTensor& t = a.t[share.which];
  const LaneUnits<T, PU, NU, ADJ> u(a, t, lane, lanes, GROUPS);
  const bool turned = share.which < 2, normed = turned && a.norm != AVGGT_NORM_NONE;
  typename std::conditional<GROUPS, GroupAngles<kPairsOfLane<PU, LANES>>, TokenAngles<kPairsOfLane<PU, LANES>>>::type angles(
      a, share.token, t.tokens_at_once, lane);
  const uint32_t at_once = GROUPS ? t.heads_at_once : 32 / lanes, heads = t.heads, n = a.n_tokens;
  const Steps in_steps(t.in_ts, at_once * t.in_hs, share), out_steps(t.out_ts, at_once * t.out_hs, share);
  const char* from = t.in + start_of(t.in_ts, t.in_hs, share.token + u.token, share.chunk * at_once + u.head, u.first);
  char* to = t.out + start_of(t.out_ts, t.out_hs, share.token + u.token, share.chunk * at_once + u.head, u.first);

  // a lane has no head in some chunks (a token's last one), and no token in the last group
  uint32_t to_fetch = share.todo, fetch_head = share.chunk * at_once + u.head, fetch_token = share.token + u.token;
  const auto fetch = [&](uint32_t stage) {
    if (to_fetch > 0) {
      if (fetch_head < heads && (!GROUPS || fetch_token < n)) Runs::fetch(stage, from, u);
      if (--to_fetch > 0) {
        fetch_head += at_once;
        const bool last = fetch_head >= share.chunks * at_once;
        from += last ? in_steps.turn : in_steps.step;
        if (last) {
          fetch_head = u.head;
          fetch_token += share.token_step;
        }
      }
    }
    copy_async_commit();
  };

  grid_dependency_wait();
  grid_launch_dependents();
  if constexpr (Runs::kAsync)
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(smem_u32(smem) + own + i * kStageBytes);
  if (turned && share.todo > 0) angles.read();
  // the tensor's weights and biases of the lane's elements
  float w[NU][2 * PU], b[NU][2 * PU];
  if (normed)
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 2 * PU; ++e) {
        const int at = e < PU ? u.lo_element(i) + e : u.hi_element(i) + e - PU;
        w[i][e] = t.weight ? t.weight[at] : 1.f;
        b[i][e] = t.bias ? t.bias[at] : 0.f;
      }

  float c[NU][PU], sn[NU][PU];
  uint32_t head = share.chunk * at_once + u.head, token = share.token + u.token;
  bool begins = true;                                    // a token
  uint32_t stage = own, last = own + (kStages - 1) * kStageBytes;   // this chunk's, and the one before, which is used up
  for (uint32_t todo = share.todo; todo > 0; --todo) {
    if (begins && turned) {
      __syncwarp();                  // the last token's table has been read
      angles.fill(a, s, lane);
      if (todo > share.chunks) {
        angles.step(static_cast<int64_t>(share.token_step) * a.n_axes);
        angles.read();
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        read_floats<PU>(s.cosine + u.pair[i], c[i]);
        read_floats<PU>(s.sine + u.pair[i], sn[i]);
      }
    }
    const bool on = head < heads && (!GROUPS || token < n);
    Runs runs;
    if constexpr (Runs::kAsync) {
      copy_async_wait<kStages - 2>();
      runs.take(smem + stage);
      fetch(smem_u32(smem) + last);
      last = stage;
      stage = stage >= (kStages - 1) * kStageBytes ? stage - (kStages - 1) * kStageBytes : stage + kStageBytes;
    } else {
      runs.load(from, u, on);
    }
    if (turned) {
      float x[NU][2 * PU];
      runs.values(x);
      if (normed) {
        centre<PU, NU, LANES>(x, u.have, a);
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) sq += dot_of<2 * PU>(x[i], x[i]);
        const float rstd = rsqrtf(head_sum<LANES>(sq, a.lanes) * a.inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          scale_each<2 * PU>(x[i], rstd);
          affine_each<2 * PU>(x[i], w[i], b[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < NU; ++i) turn_pairs<PU, ADJ>(x[i], c[i], sn[i]);
      runs.set(x);
    }
    runs.store(to, u, on);
    head += at_once;
    begins = head >= share.chunks * at_once;
    to += begins ? out_steps.turn : out_steps.step;
    if constexpr (!Runs::kAsync) from += begins ? in_steps.turn : in_steps.step;
    if (begins) {
      head = u.head;
      token += share.token_step;
    }
  }
}

// Backward behind a norm.  With e = the gradient turned back, xhat the standardised head and g = e * weight:
//   dx = rstd * (g - mean(g) - xhat * mean(g * xhat))      (mean(g) with a mean in the norm only; xhat is formed
//                                                           first: rstd^3 leaves the range of 32 bits long before rstd does)
//   dweight = sum of e * xhat, dbias = sum of e            over tokens and heads
// The sums are kept by the lane that holds the elements, over all the tokens of its warp; a thread block works on one tensor, so that a
// lane has one tensor's sums to keep.  The blocks' sums go to the workspace and are added up by rotary_sums_kernel.  With 48 registers of
// sums and weights, 16 of cosines and sines and twelve warps on the SM the issue of instructions (50% of the slots) and their latency
// bound it: 30 frames 102 us, 5 TB/s; with four blocks on the SM the registers spill (151 us).  As it is, of the 72 variants seven spill 4 to
// 20 bytes a thread, six of them runs of eight where the number of lanes is not known to the compiler.
template <typename T, int PU, int NU, bool ADJ, int LANES, bool GROUPS>
__global__ void __launch_bounds__(32 * kWarps, kBackBlocksPerSm) rotary_backward_kernel(const __grid_constant__ RotaryArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  using Runs = HeadRuns<T, PU, NU, ADJ>;
  constexpr int kStageBytes = 2 * Runs::kStageBytes, kStages = stages_of(kStageBytes);     // a head's gradient and its input
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, lanes = LANES > 0 ? LANES : a.lanes;
  const RotarySmem s = rotary_smem<GROUPS>(smem + kStages * kStageBytes);
  const uint32_t own = threadIdx.x * Runs::R::kBytes;
  Runs::clear(smem + own, kStages * kStageBytes);
  const Share share(a, GROUPS);
  const RotaryTensor& t = a.t[share.which];
  const LaneUnits<T, PU, NU, ADJ> u(a, t, lane, lanes, GROUPS);
  const bool turned = share.which < 2;
  typename std::conditional<GROUPS, GroupAngles<kPairsOfLane<PU, LANES>>, TokenAngles<kPairsOfLane<PU, LANES>>>::type angles(
      a, share.token, t.tokens_at_once, lane);
  const uint32_t at_once = GROUPS ? t.heads_at_once : 32 / lanes, heads = t.heads, n = a.n_tokens;
  const Steps grad_steps(t.in_ts, at_once * t.in_hs, share), x_steps(t.x_ts, at_once * t.x_hs, share), out_steps(t.out_ts, at_once * t.out_hs, share);
  const char* grad_from = t.in + start_of(t.in_ts, t.in_hs, share.token + u.token, u.head, u.first);
  const char* x_from = t.x + start_of(t.x_ts, t.x_hs, share.token + u.token, u.head, u.first);
  char* to = t.out + start_of(t.out_ts, t.out_hs, share.token + u.token, u.head, u.first);
  uint32_t to_fetch = share.todo, fetch_head = u.head, fetch_token = share.token + u.token;
  const auto go_on = [&]() {
    fetch_head += at_once;
    const bool last = fetch_head >= share.chunks * at_once;
    grad_from += last ? grad_steps.turn : grad_steps.step;
    x_from += last ? x_steps.turn : x_steps.step;
    if (last) {
      fetch_head = u.head;
      fetch_token += share.token_step;
    }
  };
  const auto fetch = [&](uint32_t stage) {
    if (to_fetch > 0) {
      if (fetch_head < heads && (!GROUPS || fetch_token < n)) {
        Runs::fetch(stage, grad_from, u);
        if (turned) Runs::fetch(stage + Runs::kStageBytes, x_from, u);
      }
      if (--to_fetch > 0) go_on();
    }
    copy_async_commit();
  };
  grid_dependency_wait();
  grid_launch_dependents();
  if constexpr (Runs::kAsync)
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(smem_u32(smem) + own + i * kStageBytes);
  if (turned && share.todo > 0) angles.read();
  float w[NU][2 * PU];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 2 * PU; ++e) w[i][e] = turned && t.weight ? t.weight[e < PU ? u.lo_element(i) + e : u.hi_element(i) + e - PU] : 1.f;

  float dw[NU][2 * PU], db[NU][2 * PU];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 2 * PU; ++e) dw[i][e] = db[i][e] = 0.f;
  const bool short_chunk = heads % at_once != 0 || (GROUPS && n % t.tokens_at_once != 0);      // some lanes have no head, or no token, at times
  uint32_t head = u.head, token = share.token + u.token;
  bool begins = true;                                    // a token
  uint32_t stage = own, last = own + (kStages - 1) * kStageBytes;   // this head's, and the one before, which is used up
  float c[NU][PU], sn[NU][PU];
  for (uint32_t todo = share.todo; todo > 0; --todo) {
    if (begins && turned) {
      __syncwarp();                  // the last token's table has been read
      angles.fill(a, s, lane);
      if (todo > share.chunks) {
        angles.step(static_cast<int64_t>(share.token_step) * a.n_axes);
        angles.read();
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        read_floats<PU>(s.cosine + u.pair[i], c[i]);
        read_floats<PU>(s.sine + u.pair[i], sn[i]);
      }
    }
    const bool on = !short_chunk || (head < heads && (!GROUPS || token < n));
    Runs grad, in;
    if constexpr (Runs::kAsync) {
      copy_async_wait<kStages - 2>();
      grad.take(smem + stage);
      if (turned) in.take(smem + stage + Runs::kStageBytes);
      fetch(smem_u32(smem) + last);
      last = stage;
      stage = stage >= (kStages - 1) * kStageBytes ? stage - (kStages - 1) * kStageBytes : stage + kStageBytes;
    } else {
      grad.load(grad_from, u, on);
      if (turned) in.load(x_from, u, on);
      if (todo > 1) go_on();
    }
    if (turned) {
      float x[NU][2 * PU], g[NU][2 * PU];
      if constexpr (Runs::kAsync) {                      // stages keep what an earlier chunk left where the token has no head
        if (short_chunk && !on)
#pragma unroll
          for (int i = 0; i < NU; ++i) {
            grad.lo[i].zero();
            grad.hi[i].zero();
            in.lo[i].zero();
            in.hi[i].zero();
          }
      }
      in.values(x);
      grad.values(g);
      centre<PU, NU, LANES>(x, u.have, a);
      // sum of squares, sum of g, sum of g x: one round of exchanges
      float sq = 0.f, sum = 0.f, dot = 0.f, gw[NU][2 * PU];
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        turn_pairs<PU, ADJ>(g[i], c[i], sn[i]);
        accumulate<2 * PU>(db[i], g[i]);
        multiply<2 * PU>(gw[i], g[i], w[i]);
        sq += dot_of<2 * PU>(x[i], x[i]);
        sum += sum_of<2 * PU>(gw[i]);
        dot += dot_of<2 * PU>(gw[i], x[i]);
      }
      sq = head_sum<LANES>(sq, a.lanes);
      sum = head_sum<LANES>(sum, a.lanes);
      dot = head_sum<LANES>(dot, a.lanes);
      const float rstd = rsqrtf(sq * a.inv_d + a.eps);
      // -rstd * mean(g) and, of xhat, -rstd * mean(g xhat)
      const float shift = a.norm == AVGGT_NORM_LAYER ? -rstd * (sum * a.inv_d) : 0.f, pull = -rstd * (rstd * (dot * a.inv_d));
      const uint64_t rr = pack_f32x2(rstd, rstd), pp = pack_f32x2(pull, pull), sh = pack_f32x2(shift, shift);
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int e = 0; e < 2 * PU; e += 2) {
          const uint64_t xhat = mul_f32x2(two(x[i] + e), rr);
          put_two(fma_f32x2(two(g[i] + e), xhat, two(dw[i] + e)), dw[i] + e);
          put_two(fma_f32x2(two(gw[i] + e), rr, fma_f32x2(xhat, pp, sh)), gw[i] + e);
        }
      grad.set(gw);
    }
    grad.store(to, u, on);
    head += at_once;
    begins = head >= share.chunks * at_once;
    to += begins ? out_steps.turn : out_steps.step;
    if (begins) {
      head = u.head;
      token += share.token_step;
    }
  }
  if (!turned) return;

  // lanes that hold the same elements of other heads, then the warps of the block
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 2 * PU; ++e)
      for (int o = lanes; o < 32; o <<= 1) {
        dw[i][e] += __shfl_xor_sync(0xffffffffu, dw[i][e], o);
        db[i][e] += __shfl_xor_sync(0xffffffffu, db[i][e], o);
      }
  float* rows = s.sums + warp * 2 * a.d;
  if (lane < lanes) {
#pragma unroll
    for (int i = 0; i < NU; ++i)
      if (u.have[i]) {
#pragma unroll
        for (int e = 0; e < 2 * PU; ++e) {
          const int at = e < PU ? u.lo_element(i) + e : u.hi_element(i) + e - PU;
          rows[at] = dw[i][e];
          rows[a.d + at] = db[i][e];
        }
      }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * a.d; e += blockDim.x) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += s.sums[w * 2 * a.d + e];
    a.partials[static_cast<int64_t>(blockIdx.x) * 2 * a.d + e] = v;
  }
}

struct RotarySums {
  const float* partials;
  int first[2], n[2];               // rows of Q and of K
  float* out[2][2];                 // weight, bias
  int d;
};

// Adds up the blocks' sums: 32 columns of one output per thread block, its 32 warps on rows of their own.
__global__ void __launch_bounds__(1024) rotary_sums_kernel(const __grid_constant__ RotarySums a) {
  __shared__ float part[32][33];
  grid_dependency_wait();
  grid_launch_dependents();
  const int which = blockIdx.y >> 1, kind = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float* out = a.out[which][kind];
  if (out == nullptr) return;
  float v = 0.f;
  if (col < a.d)
#pragma unroll 8
    for (int r = warp; r < a.n[which]; r += 32) v += a.partials[(static_cast<int64_t>(a.first[which] + r) * 2 + kind) * a.d + col];
  part[warp][lane] = v;
  __syncthreads();
  v = part[lane][warp];             // column `warp`, row group `lane`
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && blockIdx.x * 32 + warp < a.d) out[blockIdx.x * 32 + warp] = v;
}

bool multiple(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(bytes - 1)) == 0; }

int type_size(int type) { return type == AVGGT_TYPE_FP32 ? 4 : 2; }

// Runs of that many bytes at any of a tensor's heads are aligned.
bool runs_aligned(const void* p, int64_t ts, int64_t hs, int run) {
  const int64_t bytes = run > 16 ? 16 : run;
  return multiple(p, bytes) && ts % bytes == 0 && hs % bytes == 0;
}

using RotaryKernel = void (*)(RotaryArgs);
struct RotaryVariant {
  RotaryKernel kernel;
  int smem;                         // bytes of the pipeline and the tables
};

template <typename T, int PU, int NU, bool ADJ, int LANES, bool BACK>
RotaryVariant rotary_variant(bool groups) {
  constexpr int stage = (BACK ? 2 : 1) * HeadRuns<T, PU, NU, ADJ>::kStageBytes, smem = stages_of(stage) * stage;
  // with the sums of the gradient, what a thread block has without asking
  static_assert(smem + kWarps * 2 * kMaxTable * 4 + (BACK ? 2 * kWarps * 2 * kMaxPairs * 4 : 0) <= 48 * 1024, "shared memory");
  const int bytes = smem + kWarps * 2 * table_pairs(groups) * 4;
  if constexpr (BACK)
    return {groups ? rotary_backward_kernel<T, PU, NU, ADJ, LANES, true> : rotary_backward_kernel<T, PU, NU, ADJ, LANES, false>, bytes};
  else
    return {groups ? rotary_kernel<T, PU, NU, ADJ, LANES, true> : rotary_kernel<T, PU, NU, ADJ, LANES, false>, bytes};
}

template <typename T, bool ADJ, bool BACK>
RotaryVariant rotary_instance(int pu, int lanes, bool groups) {
  switch (pu) {
    case 8:                          // 16-bit heads; of 64 and of 128 elements, their sums are a fixed number of exchanges
      if constexpr (sizeof(T) == 2)
        return lanes == 4   ? rotary_variant<T, 8, 1, ADJ, 4, BACK>(groups)
               : lanes == 8 ? rotary_variant<T, 8, 1, ADJ, 8, BACK>(groups)
                            : rotary_variant<T, 8, 1, ADJ, 0, BACK>(groups);
    case 4: return lanes == 8 ? rotary_variant<T, 4, 1, ADJ, 8, BACK>(groups) : rotary_variant<T, 4, 1, ADJ, 0, BACK>(groups);
    case 2: return rotary_variant<T, 2, 2, ADJ, 0, BACK>(groups);
    default: return rotary_variant<T, 1, 4, ADJ, 0, BACK>(groups);
  }
}

template <bool BACK>
RotaryVariant rotary_instance_of(int type, bool adjacent, int pu, int lanes, bool groups) {
  switch (type) {
    case AVGGT_TYPE_BF16:
      return adjacent ? rotary_instance<__nv_bfloat16, true, BACK>(pu, lanes, groups) : rotary_instance<__nv_bfloat16, false, BACK>(pu, lanes, groups);
    case AVGGT_TYPE_FP16: return adjacent ? rotary_instance<__half, true, BACK>(pu, lanes, groups) : rotary_instance<__half, false, BACK>(pu, lanes, groups);
    default: return adjacent ? rotary_instance<float, true, BACK>(pu, lanes, groups) : rotary_instance<float, false, BACK>(pu, lanes, groups);
  }
}

// Pairs, blocks of pairs, axes and frequencies.
void describe_pairs(const avggt_rotary_params& p, RotaryArgs* a) {
  constexpr long double to_turns = 18446744073709551616.0L / 6.283185307179586476925286766559L;   // 2^64 / (2 pi)
  const bool shared = (p.flags & AVGGT_ROTARY_SHARED_LADDER) != 0;
  int turned = 0;
  for (int i = 0; i < p.n_axes; ++i) turned += p.pairs[i];
  a->n_pairs = p.head_dim / 2;
  a->n_segs = 0;
  int at = 0;
  // Rungs one behind the other by products in more than 64 bits of floating point: 128 of them are still exact to 2^-56, and take a
  // twentieth of what as many powers take.
  long double frequency = 1.0L, ratio = 1.0L;
  for (int i = 0; i < p.n_axes; ++i) {
    const int n = shared ? turned : p.pairs[i];
    if (!shared && n > 0) a->seg_start[a->n_segs++] = at;
    if (n > 0 && (!shared || at == 0)) {
      frequency = 1.0L;
      ratio = std::pow(static_cast<long double>(p.theta), -1.0L / n);
    }
    for (int j = 0; j < p.pairs[i]; ++j, ++at, frequency *= ratio) {
      a->axis[at] = static_cast<int8_t>(i);
      a->turn[at] = static_cast<uint64_t>(frequency * to_turns);
    }
  }
  if (shared && turned > 0) a->seg_start[a->n_segs++] = 0;
  if (at < a->n_pairs) a->seg_start[a->n_segs++] = at;
  for (; at < a->n_pairs; ++at) {
    a->axis[at] = -1;
    a->turn[at] = 0;
  }
  for (int s = a->n_segs; s <= kMaxSegs; ++s) a->seg_start[s] = a->n_pairs;
}

// The longest run of pairs, up to 16 bytes, that ends where a block of pairs ends and is aligned in every array of the call.
int choose_unit(const RotaryArgs& a, int size, bool adjacent) {
  for (int pu = size == 4 ? 4 : 8; pu > 1; pu >>= 1) {
    bool fits = a.n_pairs <= 32 * pu * (pu == 2 ? 2 : 1);
    for (int s = 0; fits && !adjacent && s <= a.n_segs; ++s) fits = a.seg_start[s] % pu == 0;
    fits = fits && a.n_pairs % pu == 0;
    for (int i = 0; fits && i < 3; ++i) {
      const RotaryTensor& t = a.t[i];
      if (t.in == nullptr) continue;
      fits = runs_aligned(t.in, t.in_ts, t.in_hs, pu * size) && runs_aligned(t.out, t.out_ts, t.out_hs, pu * size) &&
             (t.x == nullptr || runs_aligned(t.x, t.x_ts, t.x_hs, pu * size));
    }
    if (fits) return pu;
  }
  return 1;
}

// Units and lanes of a head; of each tensor, the heads and the tokens that a warp works on together.  Heads that leave lanes over make
// room for more tokens (147 frames with one head of Q and of K: 172 -> 57 us).  Returns whether they do.
bool set_units(RotaryArgs* a, int pu) {
  a->units = a->n_pairs / pu;
  a->lanes = 1;
  while (a->lanes < 32 && a->lanes < a->units) a->lanes <<= 1;
  const int places = 32 / a->lanes;
  bool groups = false;
  for (RotaryTensor& t : a->t) {
    t.heads_at_once = places;
    while (t.heads_at_once / 2 >= t.heads && places / t.heads_at_once < kMaxTokens) t.heads_at_once /= 2;
    t.tokens_at_once = places / t.heads_at_once;
    t.chunks = t.in == nullptr ? 0 : (t.heads + t.heads_at_once - 1) / t.heads_at_once;
    groups = groups || (t.in != nullptr && t.tokens_at_once > 1);
  }
  return groups;
}

// Thread blocks of each tensor: in proportion to what a token of it costs (a chunk that is turned, the table of angles, a chunk that is
// copied), at most one for each four of its tokens (of its chunks, if they are shared out one by one).  Returns their number.
unsigned share_blocks(RotaryArgs* a, int64_t most, int chunk_cost, int table_cost, int copy_cost) {
  int64_t cost[3], all = 0;
  for (int i = 0; i < 3; ++i) {
    const int chunks = a->t[i].chunks;
    const int tokens = a->t[i].tokens_at_once;
    cost[i] = chunks == 0 ? 0 : i < 2 ? 8 * chunk_cost * chunks / tokens + 8 * table_cost : 8 * copy_cost * chunks / tokens;   // 8: kMaxTokens
    all += cost[i];
  }
  int64_t at = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t groups = (static_cast<int64_t>(a->n_tokens) + a->t[i].tokens_at_once - 1) / a->t[i].tokens_at_once;
    const int64_t items = groups * (a->split ? a->t[i].chunks : 1), needed = (items + kWarps - 1) / kWarps;
    int64_t n = cost[i] * most / all;
    if (a->split || n > needed) n = needed;
    else if (n < 1) n = 1;
    if (cost[i] == 0) n = 0;
    a->t[i].first_block = static_cast<int>(at);
    a->t[i].n_blocks = static_cast<int>(n);
    at += n;
  }
  return static_cast<unsigned>(at);
}

}  // namespace

size_t rotary_ws_bytes(const avggt_rotary_params& p, int sm_count) {
  return p.norm == AVGGT_NORM_NONE ? 0 : static_cast<size_t>(sm_count) * kBackBlocksPerSm * 2 * p.head_dim * sizeof(float);
}

static void set_tensor(RotaryTensor* t, const avggt_heads* in, const avggt_heads* out, const avggt_heads* x, int heads, int size) {
  *t = RotaryTensor{};
  t->heads = heads;
  if (in == nullptr) return;
  t->in = static_cast<const char*>(in->data);
  t->in_ts = in->token_stride * size;
  t->in_hs = in->head_stride * size;
  t->out = static_cast<char*>(out->data);
  t->out_ts = out->token_stride * size;
  t->out_hs = out->head_stride * size;
  if (x) {
    t->x = static_cast<const char*>(x->data);
    t->x_ts = x->token_stride * size;
    t->x_hs = x->head_stride * size;
  }
}

cudaError_t launch_rotary(const avggt_rotary_params& p, int sm_count, const int32_t* positions, const avggt_heads* const in[3],
                          const avggt_heads* const out[3], const float* const weight[2], const float* const bias[2], bool turn_back,
                          cudaStream_t st) {
  RotaryArgs a = {};
  for (int i = 0; i < 3; ++i) set_tensor(&a.t[i], in[i], out[i], nullptr, i == 0 ? p.heads_q : p.heads_k, type_size(p.type));
  for (int i = 0; i < 2; ++i) {
    a.t[i].weight = weight[i];
    a.t[i].bias = bias[i];
  }
  a.positions = positions;
  a.n_tokens = static_cast<int>(p.n_tokens);
  a.n_axes = p.n_axes;
  a.d = p.head_dim;
  a.norm = p.norm;
  a.eps = p.eps;
  a.inv_d = 1.f / static_cast<float>(p.head_dim);
  a.sign = turn_back ? -1.f : 1.f;
  describe_pairs(p, &a);
  const bool adjacent = (p.flags & AVGGT_ROTARY_ADJACENT) != 0;
  const int pu = choose_unit(a, type_size(p.type), adjacent);
  const bool groups = set_units(&a, pu);
  // Few tokens leave SMs without a warp: a warp then takes one chunk, as long as all of them are on the GPU at once.
  const int64_t chunks = a.t[0].chunks + a.t[1].chunks + a.t[2].chunks;
  a.split = a.n_tokens * chunks <= static_cast<int64_t>(sm_count) * kBlocksPerSm * kWarps ? 1 : 0;
  const unsigned blocks = share_blocks(&a, sm_count * kBlocksPerSm, 4, 3, 3);
  const RotaryVariant v = rotary_instance_of<false>(p.type, adjacent, pu, a.lanes, groups);
  return launch_dependent(v.kernel, blocks, 32 * kWarps, v.smem, st, a);
}

cudaError_t launch_rotary_backward(const avggt_rotary_params& p, int sm_count, const int32_t* positions, const avggt_heads* const in[3],
                                   const avggt_heads* const out[3], const avggt_heads* const x[2], const float* const weight[2],
                                   float* const dweight[2], float* const dbias[2], void* ws, cudaStream_t st) {
  RotaryArgs a = {};
  for (int i = 0; i < 3; ++i) set_tensor(&a.t[i], in[i], out[i], i < 2 ? x[i] : nullptr, i == 0 ? p.heads_q : p.heads_k, type_size(p.type));
  for (int i = 0; i < 2; ++i) a.t[i].weight = weight[i];
  a.positions = positions;
  a.partials = static_cast<float*>(ws);
  a.n_tokens = static_cast<int>(p.n_tokens);
  a.n_axes = p.n_axes;
  a.d = p.head_dim;
  a.norm = p.norm;
  a.eps = p.eps;
  a.inv_d = 1.f / static_cast<float>(p.head_dim);
  a.sign = -1.f;
  describe_pairs(p, &a);
  const bool adjacent = (p.flags & AVGGT_ROTARY_ADJACENT) != 0;
  const int pu = choose_unit(a, type_size(p.type), adjacent);
  const bool groups = set_units(&a, pu);
  const unsigned blocks = share_blocks(&a, sm_count * kBackBlocksPerSm, 7, 3, 5);
  const RotaryVariant v = rotary_instance_of<true>(p.type, adjacent, pu, a.lanes, groups);
  const cudaError_t e = launch_dependent(v.kernel, blocks, 32 * kWarps, v.smem + 2 * kWarps * a.d * 4, st, a);
  if (e != cudaSuccess) return e;
  RotarySums r = {};
  r.partials = a.partials;
  r.d = a.d;
  bool any = false;
  for (int i = 0; i < 2; ++i) {
    r.first[i] = a.t[i].first_block;
    r.n[i] = a.t[i].n_blocks;
    r.out[i][0] = dweight[i];
    r.out[i][1] = dbias[i];
    any = any || dweight[i] || dbias[i];
  }
  if (!any) return cudaSuccess;
  // a grid of 4 rows: the outputs that are not asked for end at once
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.d + 31) / 32), 4);
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rotary_sums_kernel, r);
}

}  // namespace avggt
