// What the kernels of the residual stream have in common (residual_forward.cuh, residual_backward.cuh).  What a call launches: residual_norm.cu.
//
// The stream between two branches of a block:
//   p = post(y),  r = alpha x + gate p,  h = norm(r) * weight + bias
// One pass: a row is read once, stays on the SM for its norms' sums, and is written once.  The time is bound by HBM (four arrays forward, six
// backward).
#pragma once

#include <initializer_list>
#include <mutex>

#include "elements.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace avggt {

constexpr int kRun = 8;              // channels of a run
constexpr int kSpan = 32 * kRun;     // channels of a warp's run: run i of a warp is that far behind run 0
constexpr int kWarpRows = 4;         // warps of a block in which each warp has rows of its own
constexpr int kWarpThreads = 32 * kWarpRows;

// ---- a row's threads: a warp, or a block's.  A thread has RUNS times eight channels.  How they lie goes by the rows' types and alignment:
//   16  runs of eight channels (16-bit types: 16 bytes)
//    8  two groups of four channels, 128 apart (16 bytes of 32-bit types, 8 of 16-bit ones): neighbouring lanes read what is one piece
//       in memory, where runs of eight would have them read half a sector at a time
//    4  pairs of channels, 64 apart: neighbouring lanes read neighbouring words
//    2  channels 32 apart, read one at a time
template <int LAY, bool BLOCK, int RUNS>
struct Channels {
  int first, end;                    // the thread's first channel; the row's number of channels
  __device__ __forceinline__ explicit Channels(int channels) : end(channels) {
    const int lane = threadIdx.x & 31, warp = BLOCK ? threadIdx.x >> 5 : 0;
    first = warp * RUNS * kSpan + lane * (LAY / 2);
  }
  // Channel e of run i exists.
  __device__ __forceinline__ bool has(int i, int e) const {
    return first + i * kSpan + (LAY == 16 ? 0 : LAY == 8 ? e / 4 * 128 : LAY == 4 ? e / 2 * 64 + e % 2 : 32 * e) < end;
  }
  // Run i of a row; `p` is the address of the row's channel `first`.
  template <typename T> __device__ __forceinline__ void read(Run<T, kRun>& q, const char* p, int i) const {
    p += i * (kSpan * sizeof(T));
    const int left = end - first - i * kSpan;
    if constexpr (LAY == 16) {
      if (left > 0) q.load(p);
      else q.zero();
    } else if constexpr (LAY == 8) {
      q.load_quads(p, left);
    } else if constexpr (LAY == 4) {
      q.load_pairs(p, left);
    } else {
      q.load_spread(p, left);
    }
  }
  template <typename T> __device__ __forceinline__ void write(const float (&v)[kRun], char* p, int i) const {
    Run<T, kRun> q;
    q.set(v);
    p += i * (kSpan * sizeof(T));
    const int left = end - first - i * kSpan;
    if constexpr (LAY == 16) {
      if (left > 0) q.store(p);
    } else if constexpr (LAY == 8) {
      q.store_quads(p, left);
    } else if constexpr (LAY == 4) {
      q.store_pairs(p, left);
    } else {
      q.store_spread(p, left);
    }
  }
  // A parameter's, or `fallback` where there is none; zero in channels that the row does not have.
  __device__ __forceinline__ void read_param(float (&v)[kRun], const float* row, int i, float fallback) const {
    if (row != nullptr) {
      Run<float, kRun> q;
      read(q, reinterpret_cast<const char*>(row + first), i);
      q.values(v);
    } else {
#pragma unroll
      for (int e = 0; e < kRun; ++e) v[e] = has(i, e) ? fallback : 0.f;
    }
  }
  // v <- v - mean in the channels that the row has (the others stay zero)
  __device__ __forceinline__ void centre(float (&v)[RUNS][kRun], float mean) const {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      if constexpr (LAY == 16) {
        add_each<kRun>(v[i], has(i, 0) ? -mean : 0.f);
      } else if constexpr (LAY == 8) {
        add_each<4>(v[i], has(i, 0) ? -mean : 0.f);
        add_each<4>(v[i] + 4, has(i, 4) ? -mean : 0.f);
      } else {
#pragma unroll
        for (int e = 0; e < kRun; ++e)
          if (has(i, e)) v[i][e] -= mean;
      }
    }
  }
};

template <int RUNS> __device__ __forceinline__ float sum_all(const float (&v)[RUNS][kRun]) {
  float s = sum_of<kRun>(v[0]);
#pragma unroll
  for (int i = 1; i < RUNS; ++i) s += sum_of<kRun>(v[i]);
  return s;
}
template <int RUNS> __device__ __forceinline__ float dot_all(const float (&v)[RUNS][kRun], const float (&w)[RUNS][kRun]) {
  float s = dot_of<kRun>(v[0], w[0]);
#pragma unroll
  for (int i = 1; i < RUNS; ++i) s += dot_of<kRun>(v[i], w[i]);
  return s;
}

// Each of N values (a power of two) summed over the row's threads, the sums to all of them.  Lanes first exchange halves of the values,
// so that N sums cost N - 1 exchanges and a chain of five instead of 5 N.  The warps of a row (up to WARPS; 1: nothing to do) meet in
// `scratch` [2][MOST][32], whose halves take turns, so that one barrier does; `turn` is the offset of the next one.  MOST: the largest N
// that it is used with.
template <int WARPS, int MOST, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* scratch, int& turn) {
  constexpr int kLanes = 32 / N;     // that end with the same value's sum
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = N, o = 16; n > 1; n >>= 1, o >>= 1)
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const bool upper = lane & o;
      const float give = upper ? v[i] : v[i + n / 2], keep = upper ? v[i + n / 2] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  float s = v[0];
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if constexpr (WARPS > 1) {
    float* buf = scratch + turn + lane / kLanes * 32;
    turn ^= MOST * 32;
    const int warps = blockDim.x >> 5, sub = lane % kLanes;
    if (sub == 0) buf[threadIdx.x >> 5] = s;
    __syncthreads();
    s = sub < warps ? buf[sub] : 0.f;
#pragma unroll
    for (int w = kLanes; w < WARPS; w += kLanes)
      if (sub + w < warps) s += buf[sub + w];
#pragma unroll
    for (int o = (kLanes < WARPS ? kLanes : WARPS) / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  if constexpr (N > 1 || WARPS > 1) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __shfl_sync(0xffffffffu, s, n * kLanes);
  } else {
    v[0] = s;
  }
}

// The pipeline of copies: a thread brings its own channels of later rows to shared memory and reads them back itself, so that only its
// own wait stands between.  A stage holds a batch of rows of each array, in pieces of 16, 8 or 4 bytes, THREADS of them between a
// thread's.  What is never copied (channels that the row does not have, arrays that the call does not have) is zeroed once.
template <typename T, int LAY, int THREADS, int RUNS>
struct Staged {
  static constexpr uint32_t kPiece = LAY == 16 ? 16 : LAY == 8 ? 4 * sizeof(T) : 4, kApart = THREADS * kPiece, kPieces = kRun * sizeof(T) / kPiece,
                            kRunBytes = kPieces * kApart, kBytes = RUNS * kRunBytes;
  static constexpr int kChannels = kPiece >= sizeof(T) ? kPiece / sizeof(T) : 1;       // of a piece
  static __device__ __forceinline__ uint32_t own() { return threadIdx.x * kPiece; }
  template <typename C> static __device__ __forceinline__ void fetch(uint32_t at, const char* p, const C& ch) {
    at += own();
#pragma unroll
    for (int i = 0; i < RUNS; ++i, at += kRunBytes, p += kSpan * sizeof(T))
#pragma unroll
      for (uint32_t k = 0; k < kPieces; ++k)
        if (ch.has(i, k * kChannels))
          copy_async<kPiece, false>(at + k * kApart, p + (LAY == 8 ? k * 128 * sizeof(T) : LAY == 4 ? Run<T, kRun>::pair_word(k) * 4 : k * 16));
  }
  static __device__ __forceinline__ void take(Run<T, kRun>& q, const unsigned char* at, int i) {
    at += own() + i * kRunBytes;
#pragma unroll
    for (uint32_t k = 0; k < kPieces; ++k) {
      if constexpr (kPiece == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(at + k * kApart);
        q.w[4 * k] = v.x; q.w[4 * k + 1] = v.y; q.w[4 * k + 2] = v.z; q.w[4 * k + 3] = v.w;
      } else if constexpr (kPiece == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(at + k * kApart);
        q.w[2 * k] = v.x; q.w[2 * k + 1] = v.y;
      } else {
        q.w[k] = *reinterpret_cast<const uint32_t*>(at + k * kApart);
      }
    }
  }
  // The thread's own pieces of `rows` rows that lie `row_bytes` apart.
  static __device__ __forceinline__ void clear(unsigned char* at, int rows, uint32_t row_bytes) {
    at += own();
    for (int r = 0; r < rows; ++r, at += row_bytes)
#pragma unroll
      for (uint32_t k = 0; k < RUNS * kPieces; ++k)
#pragma unroll
        for (uint32_t b = 0; b < kPiece; b += 4) *reinterpret_cast<uint32_t*>(at + k * kApart + b) = 0u;
  }
};
__device__ __forceinline__ void wait_stages(int stages) {      // two or three
  if (stages == 2) copy_async_wait<0>();
  else copy_async_wait<1>();
}

// ---- launches
// How the channels of a call's rows may lie (Channels), by the addresses and strides of its rows and parameters.
struct RowAlignment {
  uint64_t narrow = 0, wide = 0;     // of 16-bit arrays and of 32-bit ones
  void rows(const avggt_rows* t, int size) {
    if (t == nullptr) return;
    (size == 2 ? narrow : wide) |= reinterpret_cast<uintptr_t>(t->data) | static_cast<uint64_t>(t->stride * size);
  }
  void params(std::initializer_list<const void*> list) {
    for (const void* p : list) wide |= reinterpret_cast<uintptr_t>(p);
  }
  int layout(int channels, int residual_size, int branch_size) const {
    const bool runs = residual_size == 2 && branch_size == 2;
    if (runs && narrow % 16 == 0 && wide % 16 == 0 && channels % kRun == 0) return 16;
    if (!runs && narrow % 8 == 0 && wide % 16 == 0 && channels % 4 == 0) return 8;
    return narrow % 4 == 0 && (channels % 2 == 0 || branch_size == 4) ? 4 : 2;
  }
};
inline int size_of(int type) { return type == AVGGT_TYPE_FP32 ? 4 : 2; }

// An array as the kernels take it: its address, or null, and its stride in bytes.
template <typename P> void set_rows(const avggt_rows* t, int size, P* data, int64_t* stride) {
  *data = t ? static_cast<P>(t->data) : nullptr;
  *stride = t ? t->stride * size : 0;
}

constexpr int kSmemPerSm = 224 * 1024, kSmemPerBlock = 2048;       // what blocks can have; a block's own, beside the pipeline
constexpr int kMostSmem = kSmemPerSm - kSmemPerBlock;              // of a block's pipeline and sums

// Allows an instance the most that any call asks of it, once for each device.  (The limit belongs to the function: set to each call's own
// size, it could be lowered by another host thread between a call's setting and its launch.)
template <auto KERNEL> cudaError_t allow_smem() {
  static std::mutex mu;
  static bool ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (ready[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
  ready[dev] = e == cudaSuccess;
  return e;
}

template <auto KERNEL, typename A>
cudaError_t launch_with_smem(int64_t blocks, unsigned threads, int smem, cudaStream_t st, const A& args) {
  if (smem > 40 * 1024) {            // with the kernels' own, below what needs no asking
    const cudaError_t e = allow_smem<KERNEL>();
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(KERNEL, static_cast<unsigned>(blocks), threads, smem, st, args);
}

// Threads of a row: eight channels each, sixteen where that would be more than 512.
inline int runs_of(int channels) { return channels > 512 * kRun ? 2 : 1; }
inline unsigned threads_of(int channels) {
  const int span = runs_of(channels) * kSpan;
  return static_cast<unsigned>((channels + span - 1) / span * 32);
}

}  // namespace avggt
