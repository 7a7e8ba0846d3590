// Dropout with the residual sum.  The mask is never stored: value (r, c) is kept where its 16 bits, from a counter-based
// generator at counter (c / 8, r, offset), are not below the limit, so the gradient's way back is the same call.
//
// What bounds it: HBM where rows are whole pieces (65536 x 2048 in bf16 with the residual: 129 us, 6.2 TB/s of 6.56 measured; 8192 x 1024 in fp32
// 14.4), the generator's integer multiplications beside it where only 4 bytes a value move (16384 x 2048 in bf16 without: 23.8 us, 5.6 TB/s).
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
  int group_log;                           // rows at any address: lanes to a segment of a row, as a power of two
  unsigned segs, groups;                   // ... segments of a row, and of the launch
  long long values;                        // dense rows of any length: of the launch (units: pieces of 16)
  unsigned limit;                          // what 16 bits in the upper half of a word are compared with
  float scale;
};
// DENSE: whole pieces one behind the other; VECTORS: rows keep 16-byte alignment, a row may end inside a piece.  (Other
// rows: sh_dropout_flat_kernel, sh_dropout_rows_kernel.)
enum { DO_DENSE = 0, DO_VECTORS = 1 };

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

// N values behind their mask, in place: value i's 16 bits are half i of the words.
template <bool RES, int N>
__device__ __forceinline__ void sh_dropout_values(const DoArgs& a, const unsigned (&bits)[N / 2], float (&f)[N], const float (&add)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // (the 16 bits in the upper half of a word; a dropped value does not count, whatever it is)
    const unsigned v = i & 1 ? bits[i / 2] : bits[i / 2] << 16;
    const float d = v >= a.limit && !a.none ? f[i] * a.scale : 0.f;
    f[i] = RES ? d + add[i] : d;
  }
}
// The 8 halves of piece blk of row r.
__device__ __forceinline__ void sh_dropout_bits(const ShPhiloxKey& key, unsigned long long offset, unsigned row, unsigned blk, unsigned* bits) {
  const uint4 w = sh_philox(make_uint4(blk, row, (unsigned)offset, (unsigned)(offset >> 32)), key);
  bits[0] = w.x; bits[1] = w.y; bits[2] = w.z; bits[3] = w.w;
}
// Piece blk of row r behind its mask, in place.
template <bool RES>
__device__ __forceinline__ void sh_dropout_piece(const DoArgs& a, const ShPhiloxKey& key, unsigned long long offset, unsigned r, unsigned blk, float (&f)[8], const float (&add)[8]) {
  unsigned bits[4];
  sh_dropout_bits(key, offset, a.row0 + r, blk, bits);
  sh_dropout_values<RES, 8>(a, bits, f, add);
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
      float f[8], add[8];
      x[q].get(f);
      if constexpr (RES) res[q].get(add);
      fetch(q);
      sh_dropout_piece<RES>(a, key, offset, r, blk, f, add);
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

// Dense rows of any length from 16 columns on: a thread takes 16 values one behind the other, which begin anywhere in a piece and
// may end in the next row.  Their bits are those of three pieces, shifted to the first value by its place in its piece (and, where the
// row ends, those of two of the next row, shifted the other way).  16384 x 2001 in bf16: 36.5 us (3.6 TB/s: four
// generator calls where rows of whole pieces take two); with 8 columns a thread, whose values lie at no vector's address, 91.
template <typename T, bool RES>
static __global__ void __launch_bounds__(DO_THREADS) sh_dropout_flat_kernel(const DoArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const unsigned long long seed = __ldg(a.rng), offset = __ldg(a.rng + 1);
  const unsigned step = gridDim.x * DO_THREADS, cols = (unsigned)a.cols;
  unsigned u = blockIdx.x * DO_THREADS + threadIdx.x;
  const unsigned long long at0 = (unsigned long long)u * 16, by = (unsigned long long)step * 16;
  unsigned r = (unsigned)(at0 / cols), c = (unsigned)(at0 - (unsigned long long)r * cols);
  const unsigned by_r = (unsigned)(by / cols), by_c = (unsigned)(by - (unsigned long long)by_r * cols);
  const ShPhiloxKey key = sh_philox_key(seed);
  ShRaw<T, 16> x, res;
  auto fetch = [&](unsigned p) {
    if (p >= a.units) return;
    const T* px = (const T*)a.x + (long long)p * 16;
    const T* pr = RES ? (const T*)a.residual + (long long)p * 16 : nullptr;
    if ((long long)p * 16 + 16 <= a.values) {
      x.load(px);
      if constexpr (RES) res.load(pr);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool there = (long long)p * 16 + i < a.values;
        reinterpret_cast<T*>(x.w)[i] = there ? px[i] : T(0.f);
        if constexpr (RES) reinterpret_cast<T*>(res.w)[i] = there ? pr[i] : T(0.f);
      }
    }
  };
  fetch(u);
  while (u < a.units) {
    float f[16], add[16];
    x.get(f);
    if constexpr (RES) res.get(add);
    fetch(u + step);
    unsigned w[12], bits[8];
    const unsigned blk = c / 8, s = c % 8;
#pragma unroll
    for (int i = 0; i < 3; ++i) sh_dropout_bits(key, offset, r, blk + i, w + 4 * i);
#pragma unroll
    for (int i = 0; i < 10; ++i) w[i] = s & 4 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 9; ++i) w[i] = s & 2 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) bits[i] = __funnelshift_r(w[i], w[i + 1], s & 1 ? 16 : 0);
    const unsigned left = cols - c;                      // of the row
    if (left < 16) {
      unsigned v[8];
      sh_dropout_bits(key, offset, r + 1, 0, v);
      sh_dropout_bits(key, offset, r + 1, 1, v + 4);
#pragma unroll
      for (int k = 8; k >= 2; k >>= 1)                   // up by `left` halves
#pragma unroll
        for (int i = 7; i >= 0; --i) v[i] = left & k ? (i >= k / 2 ? v[i - k / 2] : 0u) : v[i];
#pragma unroll
      for (int i = 7; i >= 0; --i) v[i] = __funnelshift_l(i ? v[i - 1] : 0u, v[i], left & 1 ? 16 : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned m = (2u * i < left ? 0xFFFFu : 0u) | (2u * i + 1 < left ? 0xFFFF0000u : 0u);
        bits[i] = (bits[i] & m) | (v[i] & ~m);
      }
    }
    sh_dropout_values<RES, 16>(a, bits, f, add);
    T* y = (T*)a.y + (long long)u * 16;
    if ((long long)u * 16 + 16 <= a.values) sh_store<T, 16>(y, f);
    else {
#pragma unroll
      for (int i = 0; i < 16; ++i) if ((long long)u * 16 + i < a.values) y[i] = sh_from_float<T>(f[i]);
    }
    u += step; r += by_r; c += by_c;
    if (c >= cols) { c -= cols; ++r; }
  }
}

// What is left (rows apart and at no vector's address, or very short): lanes that took 8 neighbouring values each would touch every 32-byte sector eight
// times over, so a group of lanes (4 to 32, 8 columns each) reads and writes its segment of a row one value a lane, one behind
// the other, and its pieces go through shared memory.  16384 x 2001 in bf16: 73 us; with each lane's values straight from memory 91.
template <typename T, bool RES>
static __global__ void __launch_bounds__(DO_THREADS) sh_dropout_rows_kernel(const DoArgs a) {
  constexpr int N = 8;
  __shared__ __align__(16) T s_x[DO_THREADS / 32][256], s_r[RES ? DO_THREADS / 32 : 1][256];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const unsigned long long seed = __ldg(a.rng), offset = __ldg(a.rng + 1);
  const ShPhiloxKey key = sh_philox_key(seed);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, G = 1 << a.group_log, g = lane >> a.group_log, j = lane & (G - 1);
  const unsigned step = gridDim.x * (DO_THREADS >> a.group_log);
  T* sx = s_x[warp] + g * 8 * G;                         // the group's segment
  T* sr = RES ? s_r[warp] + g * 8 * G : nullptr;
  // (a warp's groups go round together)
  const unsigned first = (blockIdx.x * (DO_THREADS / 32) + warp) << (5 - a.group_log);
  ShRaw<T, 1> x[N], res[N];
  auto fetch = [&](unsigned u) {
    const unsigned r = u / a.segs, c0 = (u - r * a.segs) * 8 * G;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned c = c0 + i * G + j;
      if (u < a.groups && c < (unsigned)a.cols) {
        x[i].load((const T*)a.x + (long long)r * a.xs + c);
        if constexpr (RES) res[i].load((const T*)a.residual + (long long)r * a.rs + c);
      } else {
        x[i].fill(0);
        if constexpr (RES) res[i].fill(0);
      }
    }
  };
  fetch(first + g);
  for (unsigned w = first; w < a.groups; w += step) {
    const unsigned u = w + g, r = u / a.segs, seg = u - r * a.segs, blk = seg * G + j;
    float f[8], add[8];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i].put(sx + i * G + j);
      if constexpr (RES) res[i].put(sr + i * G + j);
    }
    __syncwarp();
    ShRaw<T, 8> piece;
    piece.take((const unsigned char*)(sx + j * 8));
    piece.get(f);
    if constexpr (RES) { piece.take((const unsigned char*)(sr + j * 8)); piece.get(add); }
    fetch(u + step);
    sh_dropout_piece<RES>(a, key, offset, r, blk, f, add);
    sh_store<T, 8>(sx + j * 8, f);                       // (its own piece, which nobody else reads)
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned c = seg * 8 * G + i * G + j;
      ShRaw<T, 1> out;
      out.take((const unsigned char*)(sx + i * G + j));
      if (u < a.groups && c < (unsigned)a.cols) out.put((T*)a.y + (long long)r * a.ys + c);
    }
    __syncwarp();
  }
}
