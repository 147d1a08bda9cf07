// Element types of the entry points that take more than one: runs of elements moved between memory and registers, and their values
// in 32 bits.  The loads are plain ones (not the read-only path): a kernel may be resident while the kernel before it still writes.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"

namespace avggt {

__device__ __forceinline__ float value_of_bits(uint16_t bits, const __nv_bfloat16*) { return __uint_as_float(static_cast<uint32_t>(bits) << 16); }
__device__ __forceinline__ float value_of_bits(uint16_t bits, const __half*) { return __half2float(__ushort_as_half(bits)); }
__device__ __forceinline__ uint32_t bits_of_two(float a, float b, const __nv_bfloat16*) {   // a in the lower half
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return static_cast<uint32_t>(__bfloat16_as_ushort(t.x)) | static_cast<uint32_t>(__bfloat16_as_ushort(t.y)) << 16;
}
__device__ __forceinline__ uint32_t bits_of_two(float a, float b, const __half*) {
  const __half2 t = __floats2half2_rn(a, b);
  return static_cast<uint32_t>(__half_as_ushort(t.x)) | static_cast<uint32_t>(__half_as_ushort(t.y)) << 16;
}

// N elements of T as they lie in memory; N is a power of two.
template <typename T, int N>
struct Run {
  static constexpr int kBytes = N * static_cast<int>(sizeof(T));
  uint32_t w[kBytes >= 4 ? kBytes / 4 : 1];

  __device__ __forceinline__ void load(const void* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 q = static_cast<const uint4*>(p)[i];
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 q = *static_cast<const uint2*>(p);
      w[0] = q.x; w[1] = q.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *static_cast<const uint32_t*>(p);
    } else {
      w[0] = *static_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(void* p) const {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) static_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else if constexpr (kBytes == 8) {
      *static_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (kBytes == 4) {
      *static_cast<uint32_t*>(p) = w[0];
    } else {
      *static_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    }
  }
  // The same by an asynchronous copy to shared memory (runs of 4, 8 or 16 bytes), from where load reads it.  By way of the first-level
  // cache: lanes' runs may share its sectors.
  static __device__ __forceinline__ void load_async(uint32_t dst, const void* p) { copy_async<kBytes, true>(dst, p); }
  // Two groups of four neighbouring elements, 128 elements apart: neighbouring lanes' groups are neighbours.  Groups from element `end`
  // on are zero.
  __device__ __forceinline__ void load_quads(const void* p, int end) {
    constexpr int kWords = kBytes / 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      Run<T, 4> q;
      if (128 * k < end) q.load(static_cast<const char*>(p) + 128 * k * sizeof(T));
      else q.zero();
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[k * kWords + i] = q.w[i];
    }
  }
  __device__ __forceinline__ void store_quads(void* p, int end) const {
    constexpr int kWords = kBytes / 8;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (128 * k < end) {
        Run<T, 4> q;
#pragma unroll
        for (int i = 0; i < kWords; ++i) q.w[i] = w[k * kWords + i];
        q.store(static_cast<char*>(p) + 128 * k * sizeof(T));
      }
  }
  // Neighbouring pairs of elements, 64 elements apart, at any address that is a multiple of four bytes: neighbouring lanes read neighbouring
  // words.  Zero from element `end` on (16-bit types: an even number).
  __device__ __forceinline__ void load_pairs(const void* p, int end) {
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) {
      const int at = pair_word(i);
      w[i] = at * 4 / static_cast<int>(sizeof(T)) < end ? static_cast<const uint32_t*>(p)[at] : 0u;
    }
  }
  __device__ __forceinline__ void store_pairs(void* p, int end) const {
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) {
      const int at = pair_word(i);
      if (at * 4 / static_cast<int>(sizeof(T)) < end) static_cast<uint32_t*>(p)[at] = w[i];
    }
  }
  // The word of memory that word i of the run is.
  static __device__ __forceinline__ constexpr int pair_word(int i) { return sizeof(T) == 4 ? i / 2 * 64 + i % 2 : i * 32; }
  // Elements 0, 32, 64 ... of p, one at a time, at any address that is a multiple of the element's size: neighbouring lanes read
  // neighbouring elements.  Zero from `end` on.
  __device__ __forceinline__ void load_spread(const void* p, int end) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = 32 * i < end ? static_cast<const uint32_t*>(p)[32 * i] : 0u;
    } else {
      uint32_t half[N];
#pragma unroll
      for (int i = 0; i < N; ++i) half[i] = 32 * i < end ? static_cast<const uint16_t*>(p)[32 * i] : 0u;
      if constexpr (N == 1) {
        w[0] = half[0];
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) w[i / 2] = half[i] | half[i + 1] << 16;
      }
    }
  }
  __device__ __forceinline__ void store_spread(void* p, int end) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (32 * i < end) {
        if constexpr (sizeof(T) == 4) static_cast<uint32_t*>(p)[32 * i] = w[i];
        else static_cast<uint16_t*>(p)[32 * i] = static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& x : w) x = 0u;
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return value_of_bits(static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2]), static_cast<const T*>(nullptr));
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = value(i);
  }
  // v rounded to T once, to nearest even.
  __device__ __forceinline__ void set(const float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(v[i]);
    } else if constexpr (N == 1) {
      w[0] = bits_of_two(v[0], 0.f, static_cast<const T*>(nullptr)) & 0xffffu;
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) w[i / 2] = bits_of_two(v[i], v[i + 1], static_cast<const T*>(nullptr));
    }
  }
};

// ---- pairs of floats in neighbouring array elements: one instruction for two where the array is in registers
__device__ __forceinline__ uint64_t two(const float* v) { return pack_f32x2(v[0], v[1]); }
__device__ __forceinline__ void put_two(uint64_t q, float* v) { unpack_f32x2(q, v[0], v[1]); }

// v <- v + s
template <int N> __device__ __forceinline__ void add_each(float* v, float s) {
  const uint64_t ss = pack_f32x2(s, s);
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(add_f32x2(two(v + i), ss), v + i);
}
// v <- v * s
template <int N> __device__ __forceinline__ void scale_each(float* v, float s) {
  const uint64_t ss = pack_f32x2(s, s);
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(mul_f32x2(two(v + i), ss), v + i);
}
// out <- v * w
template <int N> __device__ __forceinline__ void multiply(float* out, const float* v, const float* w) {
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(mul_f32x2(two(v + i), two(w + i)), out + i);
}
// v <- v * w + b
template <int N> __device__ __forceinline__ void affine_each(float* v, const float* w, const float* b) {
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(fma_f32x2(two(v + i), two(w + i), two(b + i)), v + i);
}
// acc <- acc + v
template <int N> __device__ __forceinline__ void accumulate(float* acc, const float* v) {
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(add_f32x2(two(acc + i), two(v + i)), acc + i);
}
// acc <- acc + v * w
template <int N> __device__ __forceinline__ void accumulate_products(float* acc, const float* v, const float* w) {
#pragma unroll
  for (int i = 0; i < N; i += 2) put_two(fma_f32x2(two(v + i), two(w + i), two(acc + i)), acc + i);
}
template <int N> __device__ __forceinline__ float sum_of(const float* v) {
  uint64_t s = two(v);
#pragma unroll
  for (int i = 2; i < N; i += 2) s = add_f32x2(s, two(v + i));
  float a, b;
  unpack_f32x2(s, a, b);
  return a + b;
}
template <int N> __device__ __forceinline__ float dot_of(const float* v, const float* w) {
  uint64_t s = mul_f32x2(two(v), two(w));
#pragma unroll
  for (int i = 2; i < N; i += 2) s = fma_f32x2(two(v + i), two(w + i), s);
  float a, b;
  unpack_f32x2(s, a, b);
  return a + b;
}

}  // namespace avggt
