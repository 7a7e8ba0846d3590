// Dropout with the residual sum.  The mask is never stored: value (r, c) is kept where its 16 bits, from a counter-based
// generator at counter (c / 8, r, offset), are not below the limit, so the gradient's way back is the same call.
//
// Generator: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011).
#pragma once
#include "sh_vec.cuh"

constexpr int DO_THREADS = 256;

struct DoArgs {
  const void *x, *residual; void* y;
  const unsigned long long* rng;           // device: {seed, offset}
  long long xs, rs, ys;                    // row strides
  unsigned row0, units;                    // first row of this launch; pieces of 8 columns in it
  unsigned upr;                            // pieces in a row
  int cols, limit;
  float scale;
};

__device__ __forceinline__ uint4 sh_philox(uint4 c, uint2 k) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
    c = make_uint4((unsigned)(b >> 32) ^ c.y ^ k.x, (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ k.y, (unsigned)a);
    k.x += 0x9E3779B9u; k.y += 0xBB67AE85u;
  }
  return c;
}

// A thread takes 8 neighbouring columns, one counter.  VEC: rows of x, residual and y keep 16-byte alignment.
template <typename T, bool VEC, bool RES>
static __global__ void __launch_bounds__(DO_THREADS) sh_dropout_kernel(const DoArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const unsigned long long seed = __ldg(a.rng), offset = __ldg(a.rng + 1);
  const unsigned step = gridDim.x * DO_THREADS;
  for (unsigned u = blockIdx.x * DO_THREADS + threadIdx.x; u < a.units; u += step) {
    const unsigned r = u / a.upr, blk = u - r * a.upr;
    const long long row = (long long)a.row0 + r;
    const int c0 = (int)blk * 8, n = min(8, a.cols - c0);
    const T* x = (const T*)a.x + row * a.xs + c0;
    T* y = (T*)a.y + row * a.ys + c0;
    float f[8], res[8];
    if (VEC && n == 8) {
      sh_load<T, 8>(x, f);
      if constexpr (RES) sh_load<T, 8>((const T*)a.residual + row * a.rs + c0, res);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = i < n ? sh_to_float<T>(x[i]) : 0.f;
        if constexpr (RES) res[i] = i < n ? sh_to_float<T>(((const T*)a.residual)[row * a.rs + c0 + i]) : 0.f;
      }
    }
    const uint4 w = sh_philox(make_uint4(blk, (unsigned)row, (unsigned)offset, (unsigned)(offset >> 32)), make_uint2((unsigned)seed, (unsigned)(seed >> 32)));
    const unsigned bits[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int v = (int)(i & 1 ? bits[i / 2] >> 16 : bits[i / 2] & 0xFFFFu);
      const float d = v >= a.limit ? f[i] * a.scale : 0.f;       // (a dropped value does not count, whatever it is)
      f[i] = RES ? d + res[i] : d;
    }
    if (VEC && n == 8) sh_store<T, 8>(y, f);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) if (i < n) y[i] = sh_from_float<T>(f[i]);
    }
  }
}
