// What the kernels around the vocabulary matrices share: bfloat16 <-> float32, groups of consecutive elements as one load or
// store, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "simple_vocab.h"

namespace simple {
namespace vocab {

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
// Round to nearest even; a NaN stays one (its upper half could be all zeros behind the sign and exponent).
__device__ __forceinline__ uint16_t to_bf16(float f) {
  const uint32_t b = __float_as_uint(f);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((b >> 16) | 0x40u);
  return (uint16_t)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) { return (uint32_t)to_bf16(a) | (uint32_t)to_bf16(b) << 16; }
template <typename T> __device__ __forceinline__ T down(float f);
template <> __device__ __forceinline__ float down<float>(float f) { return f; }
template <> __device__ __forceinline__ uint16_t down<uint16_t>(float f) { return to_bf16(f); }

// VEC consecutive elements of T, aligned to their own size together, or to 16 bytes where that is less.
template <typename T, int VEC> struct __align__(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16) Group { T v[VEC]; };
template <typename T, int VEC> __device__ __forceinline__ void load(const T* p, float (&out)[VEC]) {
  const Group<T, VEC> g = *reinterpret_cast<const Group<T, VEC>*>(p);
#pragma unroll
  for (int i = 0; i < VEC; ++i) out[i] = up(g.v[i]);
}
template <typename T, int VEC> __device__ __forceinline__ void store(T* p, const float (&in)[VEC]) {
  Group<T, VEC> g;
#pragma unroll
  for (int i = 0; i < VEC; ++i) g.v[i] = down<T>(in[i]);
  *reinterpret_cast<Group<T, VEC>*>(p) = g;
}

// VEC elements of a row of `len` from its element c < len on, zeros behind its end.  WHOLE: rows are aligned and c + VEC is in the row; else any
// alignment (an access of 16 bytes may start anywhere): a row's last elements come from the VEC that end with it, without a branch ahead of the load.
template <typename T, int VEC, bool WHOLE> __device__ __forceinline__ void load_some(const T* row, int64_t c, int64_t len, float (&out)[VEC]) {
  if constexpr (WHOLE) load<T, VEC>(row + c, out);
  else {
    static_assert(sizeof(T) * VEC == 16 || sizeof(T) * VEC == 8, "one access");
    using Bits = std::conditional_t<sizeof(T) * VEC == 16, unsigned __int128, uint64_t>;
    Bits v = 0;
    if (len >= VEC) {
      __builtin_memcpy(&v, row + min(c, len - VEC), sizeof(v));
      if (c + VEC > len) v >>= 8 * (int)sizeof(T) * (int)(c + VEC - len);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if (i < len) {
          T x;
          x = row[i];
          uint32_t bits = 0;
          __builtin_memcpy(&bits, &x, sizeof(T));
          v |= (Bits)bits << (8 * (int)sizeof(T) * i);
        }
      }
    }
    T e[VEC];
    __builtin_memcpy(e, &v, sizeof(v));
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] = up(e[i]);
  }
}
template <typename T, int VEC, bool WHOLE> __device__ __forceinline__ void put_some(T* p, int64_t n, const T (&v)[VEC]) {
  if constexpr (WHOLE) {
    Group<T, VEC> g;
#pragma unroll
    for (int i = 0; i < VEC; ++i) g.v[i] = v[i];
    *reinterpret_cast<Group<T, VEC>*>(p) = g;
  } else if (n >= VEC) __builtin_memcpy(p, v, sizeof(v));
  else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < n) p[i] = v[i];
  }
}
template <typename T, int VEC, bool WHOLE> __device__ __forceinline__ void store_some(T* p, int64_t n, const float (&in)[VEC]) {
  T v[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = down<T>(in[i]);
  put_some<T, VEC, WHOLE>(p, n, v);
}

// A lane of a product's tile holds four consecutive 16-bit values (two words) of a row, its row's other 16-lane groups the next ones, and the values
// 16 further on are in the next fragment.  `a` and `b` are two such fragments: afterwards the lane holds eight consecutive values, `a` then `b`, at
// 16 * (group / 2) + 8 * (group % 2) from the first fragment's start, so that a store writes 64 bytes of each of 16 rows instead of 32.
__device__ __forceinline__ void eight_of(uint2& a, uint2& b) {
  auto swap = [](uint32_t& x, uint32_t& y) {
    const auto h = __builtin_amdgcn_permlane32_swap(x, y, false, false);  // x's upper half against y's lower
    const auto q = __builtin_amdgcn_permlane16_swap(h[0], h[1], false, false);  // x's odd sixteens against y's even
    x = q[0];
    y = q[1];
  };
  swap(a.x, b.x);
  swap(a.y, b.y);
}

// The first n of eight 16-bit values, to any address of an element (a store of 16 bytes may start anywhere; by single elements dW of 21 tokens with rows of 868
// took three times as long).  PAST: the caches are not to keep them.
template <bool PAST = false> __device__ __forceinline__ void put8(uint16_t* to, int64_t n, uint4 v) {
  if (n >= 8) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    if constexpr (PAST) __builtin_nontemporal_store(words{v.x, v.y, v.z, v.w}, reinterpret_cast<words*>(to));
    else __builtin_memcpy(to, &v, 16);
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) to[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
  }
}

// ---- host side ----
inline bool good_type(int dtype) { return dtype == SIMPLE_F32 || dtype == SIMPLE_BF16; }
inline int64_t type_bytes(int dtype) { return dtype == SIMPLE_F32 ? 4 : 2; }
// Whether rows of `stride` elements of `esz` bytes that start at `p` all start at a multiple of `to` bytes.
inline bool rows_aligned(const void* p, int64_t stride, int64_t esz, int64_t to) {
  return p == nullptr || (((uintptr_t)p & (uintptr_t)(to - 1)) == 0 && ((stride * esz) & (to - 1)) == 0);
}
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Workgroups of a launch at most, of up to 1024 threads: of a grid of 2^32 threads or more the runtime starts what is left modulo 2^32, without an error.
constexpr int64_t LAUNCH_WGS = (int64_t)1 << 21;
inline int launched() { return hipGetLastError() == hipSuccess ? SIMPLE_OK : SIMPLE_EDEVICE; }

}  // namespace vocab
}  // namespace simple
