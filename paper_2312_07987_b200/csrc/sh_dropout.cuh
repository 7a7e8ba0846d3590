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
  int cols, none;                          // none: nothing is kept
  unsigned limit;                          // what 16 bits in the upper half of a word are compared with
  float scale;
};
// DENSE: whole pieces one behind the other; VECTORS: rows keep 16-byte alignment, a row may end inside a piece; VALUES: anything.
enum { DO_DENSE = 0, DO_VECTORS = 1, DO_VALUES = 2 };

struct ShPhiloxKey { unsigned k[20]; };     // the keys of the ten rounds
__device__ __forceinline__ ShPhiloxKey sh_philox_key(unsigned long long seed) {
  ShPhiloxKey r;
#pragma unroll
  for (int i = 0; i < 10; ++i) { r.k[2 * i] = (unsigned)seed + i * 0x9E3779B9u; r.k[2 * i + 1] = (unsigned)(seed >> 32) + i * 0xBB67AE85u; }
  return r;
}
__device__ __forceinline__ uint4 sh_philox(uint4 c, const ShPhiloxKey& key) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
    c = make_uint4((unsigned)(b >> 32) ^ c.y ^ key.k[2 * i], (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ key.k[2 * i + 1], (unsigned)a);
  }
  return c;
}

// A thread takes pieces of 8 neighbouring columns, one counter each; the next two are on their way while one is worked on.
// The generator is what costs: 20 wide multiplications and as many three-way ors a piece, so its 128 bits serve 8 values, and what
// is left of the work - two operations, a comparison and a selection a value - is kept off addresses.
template <typename T, int MODE, bool RES>
static __global__ void __launch_bounds__(DO_THREADS) sh_dropout_kernel(const DoArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const unsigned long long seed = __ldg(a.rng), offset = __ldg(a.rng + 1);
  const unsigned step = gridDim.x * DO_THREADS, step_r = step / a.upr, step_b = step - step_r * a.upr;
  unsigned u = blockIdx.x * DO_THREADS + threadIdx.x, r = u / a.upr, blk = u - r * a.upr;     // of the piece that is worked on
  constexpr int AHEAD = 2;
  unsigned fu = u, fr = r, fb = blk;                     // of the piece that is fetched
  ShRaw<T, 8> x[AHEAD], res[AHEAD];
  auto next = [&](unsigned& pu, unsigned& pr, unsigned& pb) {
    pu += step;
    pr += step_r; pb += step_b;
    if (pb >= a.upr) { pb -= a.upr; ++pr; }
  };
  auto fetch = [&](int q) {
    if (fu < a.units) {
      const long long at = MODE == DO_DENSE ? (long long)fu * 8 : (long long)fr * a.xs + (long long)fb * 8;
      const T* px = (const T*)a.x + at;
      const T* pr = RES ? (const T*)a.residual + (MODE == DO_DENSE ? at : (long long)fr * a.rs + (long long)fb * 8) : nullptr;
      const int n = a.cols - (int)fb * 8;
      if (MODE == DO_DENSE || (MODE == DO_VECTORS && n >= 8)) {
        x[q].load(px);
        if constexpr (RES) res[q].load(pr);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          reinterpret_cast<T*>(x[q].w)[i] = i < n ? px[i] : T(0.f);
          if constexpr (RES) reinterpret_cast<T*>(res[q].w)[i] = i < n ? pr[i] : T(0.f);
        }
      }
    }
    if constexpr (MODE == DO_DENSE) fu += step;
    else next(fu, fr, fb);
  };
#pragma unroll
  for (int q = 0; q < AHEAD; ++q) fetch(q);
  const ShPhiloxKey key = sh_philox_key(seed);
  while (u < a.units) {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (u >= a.units) break;
      const uint4 w = sh_philox(make_uint4(blk, a.row0 + r, (unsigned)offset, (unsigned)(offset >> 32)), key);
      const unsigned bits[4] = {w.x, w.y, w.z, w.w};
      float f[8], add[8];
      x[q].get(f);
      if constexpr (RES) res[q].get(add);
      fetch(q);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (the value's 16 bits in the upper half of a word; a dropped value does not count, whatever it is)
        const unsigned v = i & 1 ? bits[i / 2] : bits[i / 2] << 16;
        const float d = v >= a.limit && !a.none ? f[i] * a.scale : 0.f;
        f[i] = RES ? d + add[i] : d;
      }
      T* y = (T*)a.y + (MODE == DO_DENSE ? (long long)u * 8 : (long long)r * a.ys + (long long)blk * 8);
      const int n = a.cols - (int)blk * 8;
      if (MODE == DO_DENSE || (MODE == DO_VECTORS && n >= 8)) sh_store<T, 8>(y, f);
      else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) y[i] = sh_from_float<T>(f[i]);
      }
      next(u, r, blk);
    }
  }
}
