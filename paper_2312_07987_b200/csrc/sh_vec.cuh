// Vectors of V stored values: held as loaded (what is on its way costs few registers), turned into fp32, stored.
#pragma once
#include "sh_internal.cuh"

template <typename T, int V>
struct ShRaw {
  static constexpr int BYTES = V * (int)sizeof(T);
  uint32_t w[BYTES < 4 ? 1 : BYTES / 4];

  // (aligned to V values; evict-first: nobody reads it again)
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    } else if constexpr (BYTES == 8) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
      w[0] = v.x; w[1] = v.y;
    } else if constexpr (BYTES == 4) {
      w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
    } else {
      w[0] = __ldcs(reinterpret_cast<const unsigned short*>(p));
    }
  }
  __device__ __forceinline__ void take(const unsigned char* s) {             // from shared memory (one value, or 16 bytes and more)
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(s)[i];
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    } else if constexpr (BYTES == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(s);
    } else {
      w[0] = *reinterpret_cast<const unsigned short*>(s);
    }
  }
  __device__ __forceinline__ void put(T* p) const {                          // one value, as it is
    static_assert(V == 1, "");
    if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
  }
  __device__ __forceinline__ void fill(uint32_t word) {
#pragma unroll
    for (int i = 0; i < (BYTES < 4 ? 1 : BYTES / 4); ++i) w[i] = word;
  }
  __device__ __forceinline__ void get(float (&f)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(w[i]);
      else f[i] = sh_to_float<T>(reinterpret_cast<const T*>(w)[i]);
    }
  }
};

template <typename T, int V>
__device__ __forceinline__ void sh_store(T* p, const float (&f)[V]) {
  constexpr int BYTES = V * (int)sizeof(T);
  if constexpr (BYTES >= 4) {
    uint32_t w[BYTES / 4];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
      else reinterpret_cast<T*>(w)[i] = sh_from_float<T>(f[i]);
    }
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else if constexpr (BYTES == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    }
  } else {
    p[0] = sh_from_float<T>(f[0]);
  }
}

// Sum over groups of LANES neighbouring lanes (a power of two), in every lane of a group.
template <int LANES>
__device__ __forceinline__ float sh_group_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Two of them at once: after one exchange each half of a group adds one.
template <int LANES>
__device__ __forceinline__ void sh_group_sums(float& a, float& b) {
  const bool up = threadIdx.x & (LANES / 2);
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, LANES / 2);
#pragma unroll
  for (int o = LANES / 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const float w = __shfl_xor_sync(0xffffffffu, v, LANES / 2);
  a = up ? w : v;
  b = up ? v : w;
}
