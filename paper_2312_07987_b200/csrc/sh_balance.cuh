// The balance loss of the gates, the per-expert counts, and the loss's gradient with respect to the gate logits.
//
//   p = softmax over a gate's E logits,  P_e = mean of p_e over the tokens,  f_e = share of the selections
//   counts:  L = coef sum_gates E sum_e f_e P_e      entropy:  L = coef sum_gates sum_e P_e ln P_e
//   dL/dz_e = p_e (c_e - sum_j p_j c_j),  c_e = dL/dP_e / n:  any constant may be taken off c, so it is kept centred
//
// A row (a token's E logits of one gate) belongs to L neighbouring lanes with W values each.  Between its rounds a thread
// stays with the same gate, so its share of P is W sums in registers.
//
// What bounds it: latency at 24 warps an SM (131072 tokens, 8 gates of 32 experts in bf16: sums 24 us - 84 MB, 3.5 TB/s, issue slots two thirds full,
// HBM 43 %, no warp ready in a third of the cycles -, gradient 25 us - 134 MB, 5.4 TB/s); small calls: the latency of their one or two launches.
// Rows that are no whole aligned vectors are loaded and stored a value at a time: 31 experts in bf16 46 and 193 us, in fp32 37 and 87, 15 in bf16 32 and 88.
#pragma once
#include <cooperative_groups.h>

#include "sh_vec.cuh"

constexpr int BL_THREADS = 256, BL_BLOCKS = 3;     // (two rows a thread on their way, 24 warps an SM: 16 warps 5 % slower, more rows the same)
// Rows of a thread whose p it adds in fp32 (a longer chain, of values of one sign, loses a bit with every doubling): more tokens are taken by
// further launches, which add to the blocks' sums.  (Joined in shared memory inside the loop instead: 0.1 us more at 22 us.)
constexpr int BL_CHAIN = 256;
constexpr int BL_LOSS_THREADS = 512;
constexpr int BL_MAX_BLOCKS = 512;         // blocks of the first kernel at most (rows of partial results)

struct BlArgs {
  const void* z; void* dz;
  const int* idx;                          // [sides, N, H, k]
  const unsigned char* mask;               // [N] or nullptr: tokens that count
  const float* slope; const float* gloss;  // gradient: c [gates, E]; a factor, or nullptr
  long long tokens, zt, dzt;               // zt, dzt: strides of a token in z and dz
  int gates, H, E, k;
  int per, tpb;                            // gates of a block, tokens of a block's round: per * tpb rows
  float* part_p; int* part_n;              // [blocks][gates * E] sums of p; [blocks][gates * E] counts, then [blocks] tokens
  unsigned* ticket;                        // gates whose sums are done (set to zero by the first kernel)
};

// A launch of the sums of several: tokens of all of them (idx), and whether there is something to add to.
struct BlPart { long long all; int add; };

// Rows of a thread that are on their way together: 64 bytes of them.
template <typename T, int W> struct BlAhead { static constexpr int N = W * (int)sizeof(T) >= 32 ? 2 : 4; };

// The lane's W logits of a row, -inf where there are none.  VEC: E = L W, aligned.
template <typename T, int W, bool VEC>
struct BlRow {
  ShRaw<T, VEC ? W : 1> raw[VEC ? 1 : W];
  __device__ __forceinline__ void load(const T* p, int n, bool live) {       // n: logits from p on
    constexpr uint32_t none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;      // -inf (two of them)
    if constexpr (VEC) {
      if (live) raw[0].load(p);
      else raw[0].fill(none);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if (live && i < n) raw[i].load(p + i);
        else raw[i].fill(none);
      }
    }
  }
  __device__ __forceinline__ void get(float2 (&f)[W / 2]) const {
    float g[W];
    if constexpr (VEC) {
      raw[0].get(g);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) { float one[1]; raw[i].get(one); g[i] = one[0]; }
    }
#pragma unroll
    for (int i = 0; i < W / 2; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
  }
};

// (2^-22 relative, and a result below 2^-126 is zero: p is added up over tokens or multiplied by its gradient's factor, both off by as much)
__device__ __forceinline__ float bl_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// exp(z - max) of a row in place of its logits; returns 1 / their sum (__fdividef: 2 units in the last place; the sum is between 1 and 32).  The
// difference first: logits may be as large as their type allows.  The exponent is one fp32 product, so with the difference's rounding a p is off by
// 2 |z - max| roundings of 2^-24: 40 of them at 2e-9.  A row of -inf only has no probabilities: zeros.
template <int W, int L>
__device__ __forceinline__ float bl_softmax(float2 (&f)[W / 2]) {
  float m = fmaxf(f[0].x, f[0].y);
#pragma unroll
  for (int i = 1; i < W / 2; ++i) m = fmaxf(m, fmaxf(f[i].x, f[i].y));
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float log2e = 1.4426950408889634f, b = m == -INFINITY ? 0.f : -m;
  const float2 s2 = make_float2(log2e, log2e), b2 = make_float2(b, b);
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    const float2 x = __fmul2_rn(__fadd2_rn(f[i], b2), s2);
    f[i] = make_float2(bl_exp2(x.x), bl_exp2(x.y));
    sum = __fadd2_rn(sum, f[i]);
  }
  float s = sum.x + sum.y;
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s == 0.f ? 0.f : __fdividef(1.f, s);
}

// A block's share of the sums, tokens tpb at a time from its place among `blocks` blocks on (all: tokens of the call), gates g0 .. g0 + ng - 1: into s_p a row of
// the block's sums of p, into s_n the counts (both cleared or overwritten here), into *s_tokens the tokens that count.
template <typename T, int W, int L, bool VEC, int THREADS>
__device__ __forceinline__ void bl_sums(const BlArgs& a, long long all, int block, int blocks, int g0, int ng, float (*s_p)[W * L + 1], int* s_n, int* s_tokens) {
  constexpr int EP = W * L, AHEAD = BlAhead<T, W>::N, PICKS = 4 / L < 1 ? 1 : 4 / L;
  const int row = threadIdx.x / L, sub = threadIdx.x % L, at = sub * W;
  const int gl = row % a.per, tl = row / a.per, gate = g0 + gl;
  const bool mine = tl < a.tpb && gl < ng;
  for (int i = threadIdx.x; i < ng * EP; i += THREADS) s_n[i] = 0;
  if (threadIdx.x == 0) *s_tokens = 0;
  __syncthreads();
  float2 acc[W / 2];
#pragma unroll
  for (int i = 0; i < W / 2; ++i) acc[i] = make_float2(0.f, 0.f);
  int seen = 0;
  auto count = [&](int e) { if ((unsigned)e < (unsigned)a.E) atomicAdd(&s_n[gl * EP + e], 1); };   // (a slot without an expert is not counted)
  const long long step = (long long)blocks * a.tpb;
  long long t = (long long)block * a.tpb + tl;           // (what is past the last token is not read)
  const T* z = (const T*)a.z + (long long)gate * a.E + at + t * a.zt;
  const int* idx = a.idx + ((long long)(gate / a.H) * all * a.H + gate % a.H + t * a.H) * a.k;
  const long long zstep = step * a.zt, istep = step * a.H * a.k, rounds = (a.tokens - (long long)block * a.tpb + step - 1) / step;
  // (the next AHEAD rows are on their way while one is worked on)
  BlRow<T, W, VEC> rows[AHEAD];
  int picks[AHEAD][PICKS];
  auto fetch = [&](int u) {
    const bool live = mine && t < a.tokens && (!a.mask || a.mask[t]);
    rows[u].load(z, a.E - at, live);
#pragma unroll
    for (int j = 0; j < PICKS; ++j) picks[u][j] = live && sub * PICKS + j < a.k ? __ldcs(idx + sub * PICKS + j) : -1;
    if (live)
      for (int j = L * PICKS + sub; j < a.k; j += L) count(__ldcs(idx + j));
    seen += live;
    t += step; z += zstep; idx += istep;
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) fetch(u);
  for (long long r = 0; r < rounds; r += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      float2 f[W / 2];
      rows[u].get(f);
#pragma unroll
      for (int j = 0; j < PICKS; ++j) count(picks[u][j]);
      fetch(u);
      const float inv = bl_softmax<W, L>(f);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) acc[i] = __ffma2_rn(f[i], make_float2(inv, inv), acc[i]);
    }
  }
  if (mine && gl == 0 && sub == 0 && seen) atomicAdd(s_tokens, seen);
#pragma unroll
  for (int i = 0; i < W / 2; ++i) { s_p[row][at + 2 * i] = acc[i].x; s_p[row][at + 2 * i + 1] = acc[i].y; }
  __syncthreads();
}

// The block's sum of p of every (gate, expert) from its rows' sums, in 64 bits: a gate that is nearly balanced has a gradient of
// what is left of ln P behind its mean, and 256 sums of a size added in 32 bits cost it 5 of its 24 bits.  All threads, then those of the
// columns, in a fixed order.
template <int THREADS, int LD, typename F>
__device__ __forceinline__ void bl_columns(const BlArgs& a, int ng, const float (*s_p)[LD], double* s_part, F store) {
  const int cols = ng * a.E, parts = cols < THREADS ? THREADS / cols : 1;
  for (int c0 = 0; c0 < cols; c0 += THREADS) {             // (one round where parts > 1)
    const int i = threadIdx.x % (parts > 1 ? cols : THREADS), part = parts > 1 ? threadIdx.x / cols : 0, c = c0 + i;
    double sum = 0.0;
    if (part < parts && c < cols) {
      const int q = c / a.E, e = c % a.E;
      for (int k = part; k < a.tpb; k += parts) sum += (double)s_p[k * a.per + q][e];
      s_part[threadIdx.x] = sum;
    }
    __syncthreads();
    if (part == 0 && c < cols) {
      for (int k = 1; k < parts; ++k) sum += s_part[k * cols + i];
      store(c, sum);
    }
    __syncthreads();
  }
}

template <typename T, int W, int L, bool VEC>
static __global__ void __launch_bounds__(BL_THREADS, BL_BLOCKS) sh_balance_sums_kernel(const BlArgs a, const BlPart part) {
  constexpr int EP = W * L, ROWS = BL_THREADS / L;
  __shared__ float s_p[ROWS][EP + 1];
  __shared__ int s_n[ROWS * EP];                         // [gate of the block][expert]
  __shared__ double s_part[BL_THREADS];
  __shared__ int s_tokens;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.ticket = 0;
  const int g0 = blockIdx.y * a.per, ng = min(a.per, a.gates - g0);
  bl_sums<T, W, L, VEC, BL_THREADS>(a, part.all, blockIdx.x, gridDim.x, g0, ng, s_p, s_n, &s_tokens);
  const long long base = (long long)blockIdx.x * a.gates * a.E + (long long)g0 * a.E;
  bl_columns<BL_THREADS, EP + 1>(a, ng, s_p, s_part, [&](int c, double sum) {
    const int n = s_n[c / a.E * EP + c % a.E];
    a.part_p[base + c] = (float)(part.add ? sum + a.part_p[base + c] : sum);      // (hundreds of them, each rounded by itself)
    a.part_n[base + c] = part.add ? n + a.part_n[base + c] : n;
  });
  if (blockIdx.y == 0 && threadIdx.x == 0) {
    int* tokens = a.part_n + (long long)gridDim.x * a.gates * a.E + blockIdx.x;
    *tokens = part.add ? s_tokens + *tokens : s_tokens;
  }
}

struct BlOut {
  const float* part_p; const int* part_n; unsigned* ticket; double* gate_loss;
  int blocks, gates, E, kind;
  double coef;
  float *loss, *prob, *slope; int* counts;
};

// A gate's results from its sums: lane e of a warp has expert e's sum of p and count; in 64 bits.  Returns its share of the loss.
__device__ __forceinline__ double bl_finish(const BlOut& a, int gate, int e, double p, int n, int tokens) {
  const double P = tokens ? p / tokens : 0.0;
  int all = n;
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  const double f = all ? (double)n / all : 0.0;
  // (an expert without any probability has no slope: p is zero wherever it would be used)
  const bool used = e < a.E && (a.kind == 0 || P != 0.0);
  double c = 0.0, l = 0.0;
  if (used) {
    if (a.kind == 0) { l = a.E * f * P; c = a.E * f; }
    else { c = log(P); l = P * c; }
  }
  double sum = c;
  int many = used;
  for (int o = 16; o > 0; o >>= 1) {
    l += __shfl_xor_sync(0xffffffffu, l, o);
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    many += __shfl_xor_sync(0xffffffffu, many, o);
  }
  if (e < a.E) {
    const int o = gate * a.E + e;
    a.counts[o] = n;
    a.prob[o] = (float)P;
    a.slope[o] = used && tokens ? (float)(a.coef * (c - sum / many) / tokens) : 0.f;
  }
  return tokens ? a.coef * l : 0.0;
}

// A gate per block: its experts' sums over the first kernel's blocks in a fixed order; the block that comes last adds the gates'
// losses in order.
static __global__ void __launch_bounds__(BL_LOSS_THREADS) sh_balance_loss_kernel(const BlOut a) {
  constexpr int ROWS = BL_LOSS_THREADS / 32;
  __shared__ double s_p[ROWS][32];
  __shared__ int s_n[ROWS][32], s_t[ROWS], s_last;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int gate = blockIdx.x, e = threadIdx.x & 31, r = threadIdx.x >> 5, cols = a.gates * a.E;
  double p = 0.0;
  int n = 0, tokens = 0;
  for (int b = r; b < a.blocks; b += 16 * ROWS) {
    float vp[16];                                        // (loads of a round in flight together)
    int vn[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const bool there = e < a.E && b + k * ROWS < a.blocks;
      const long long at = (long long)(b + k * ROWS) * cols + gate * a.E + e;
      vp[k] = there ? __ldcg(a.part_p + at) : 0.f;
      vn[k] = there ? __ldcg(a.part_n + at) : 0;
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) { p += (double)vp[k]; n += vn[k]; }
  }
  for (int b = threadIdx.x; b < a.blocks; b += BL_LOSS_THREADS) tokens += __ldcg(a.part_n + (long long)a.blocks * cols + b);
  s_p[r][e] = p; s_n[r][e] = n;
  for (int o = 16; o > 0; o >>= 1) tokens += __shfl_xor_sync(0xffffffffu, tokens, o);
  if (e == 0) s_t[r] = tokens;
  __syncthreads();
  if (r == 0) {
    tokens = s_t[0];
    for (int i = 1; i < ROWS; ++i) { tokens += s_t[i]; p += s_p[i][e]; n += s_n[i][e]; }
    const double l = bl_finish(a, gate, e, p, n, tokens);
    if (e == 0) {
      a.gate_loss[gate] = l;
      __threadfence();
      s_last = atomicAdd(a.ticket, 1u) == (unsigned)a.gates - 1;
    }
  }
  __syncthreads();
  if (s_last && threadIdx.x == 0) {
    __threadfence();
    double sum = 0.0;
    for (int i = 0; i < a.gates; ++i) sum += __ldcg(a.gate_loss + i);
    *a.loss = (float)sum;
  }
}

// Both in one launch, for few rows: a cluster of 8 blocks, whose sums are read over distributed shared memory, a warp to a gate.
// (Such calls are bound by their launches: 2048 tokens, 8 gates of 4 experts, 14.2 us a call, 17.6 with the two kernels.)
constexpr int BL_SMALL_THREADS = 512, BL_CLUSTER = 8;
constexpr int BL_SMALL_COLS = 512, BL_SMALL_GATES = 64;   // gates * experts, gates at most
template <typename T, int W, int L, bool VEC>
static __global__ void __launch_bounds__(BL_SMALL_THREADS, 1) sh_balance_small_kernel(const BlArgs a, const BlOut o) {
  namespace cg = cooperative_groups;
  constexpr int EP = W * L, ROWS = BL_SMALL_THREADS / L;
  __shared__ float s_p[ROWS][EP + 1];
  __shared__ int s_n[BL_SMALL_GATES * EP < 2 * BL_SMALL_COLS ? BL_SMALL_GATES * EP : 2 * BL_SMALL_COLS];
  __shared__ double s_sum[BL_SMALL_COLS], s_part[BL_SMALL_THREADS];
  __shared__ double s_loss[BL_SMALL_GATES];
  __shared__ int s_tokens;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank();
  bl_sums<T, W, L, VEC, BL_SMALL_THREADS>(a, a.tokens, rank, BL_CLUSTER, 0, a.gates, s_p, s_n, &s_tokens);
  bl_columns<BL_SMALL_THREADS, EP + 1>(a, a.gates, s_p, s_part, [&](int c, double sum) { s_sum[c] = sum; });
  cluster.sync();
  const int e = threadIdx.x & 31;
  for (int gate = rank + BL_CLUSTER * (threadIdx.x >> 5); gate < a.gates; gate += BL_CLUSTER * (BL_SMALL_THREADS / 32)) {
    double p = 0.0;
    int n = 0, tokens = 0;
#pragma unroll
    for (int b = 0; b < BL_CLUSTER; ++b) {
      if (e < a.E) {
        p += cluster.map_shared_rank(s_sum, b)[gate * a.E + e];
        n += cluster.map_shared_rank(s_n, b)[gate * EP + e];
      }
      tokens += *cluster.map_shared_rank(&s_tokens, b);
    }
    const double l = bl_finish(o, gate, e, p, n, tokens);
    if (e == 0) cluster.map_shared_rank(s_loss, 0)[gate] = l;
  }
  cluster.sync();                                        // (nobody's shared memory is read behind it)
  if (rank == 0 && threadIdx.x == 0) {
    double sum = 0.0;
    for (int i = 0; i < a.gates; ++i) sum += s_loss[i];
    *o.loss = (float)sum;
  }
}

// dz, or dz += (ADD: fp32, the gates' gradients of a backward pass).
template <typename T, int W, int L, bool VEC, bool ADD>
static __global__ void __launch_bounds__(BL_THREADS, BL_BLOCKS) sh_balance_backward_kernel(const BlArgs a) {
  constexpr int AHEAD = BlAhead<T, W>::N;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int row = threadIdx.x / L, at = (threadIdx.x % L) * W;
  const int g0 = blockIdx.y * a.per, gl = row % a.per, tl = row / a.per, gate = g0 + gl;
  const bool mine = tl < a.tpb && gate < a.gates;
  const float gloss = a.gloss ? __ldg(a.gloss) : 1.f;
  float2 c[W / 2];
#pragma unroll
  for (int i = 0; i < W; ++i) (i & 1 ? c[i / 2].y : c[i / 2].x) = mine && at + i < a.E ? __ldg(a.slope + gate * a.E + at + i) : 0.f;
  const long long step = (long long)gridDim.x * a.tpb;
  long long t = (long long)blockIdx.x * a.tpb + tl;
  const T* z = (const T*)a.z + (long long)gate * a.E + at + t * a.zt;
  T* o = (T*)a.dz + (long long)gate * a.E + at + t * a.dzt;
  const long long zstep = step * a.zt, ostep = step * a.dzt, rounds = (a.tokens - (long long)blockIdx.x * a.tpb + step - 1) / step;
  BlRow<T, W, VEC> rows[AHEAD];
  bool there[AHEAD], live[AHEAD];
  auto fetch = [&](int u) {
    there[u] = mine && t < a.tokens;
    live[u] = there[u] && (!a.mask || a.mask[t]);
    rows[u].load(z, a.E - at, live[u]);
    t += step; z += zstep;
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) fetch(u);
  for (long long r = 0; r < rounds; r += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      float2 f[W / 2];
      rows[u].get(f);
      const bool row = there[u], counts = live[u];
      fetch(u);
      const float inv = bl_softmax<W, L>(f);
      float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) d2 = __ffma2_rn(f[i], c[i], d2);
      float dot = d2.x + d2.y;
#pragma unroll
      for (int q = L / 2; q > 0; q >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, q);
      dot *= -inv;
      const float by = gloss * inv;
      float g[W];
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        const float2 v = __fmul2_rn(__fmul2_rn(f[i], make_float2(by, by)), __fadd2_rn(c[i], make_float2(dot, dot)));
        g[2 * i] = counts ? v.x : 0.f; g[2 * i + 1] = counts ? v.y : 0.f;
      }
      if (row) {
        if constexpr (ADD) {
#pragma unroll
          for (int i = 0; i < W; ++i) if (counts && at + i < a.E) o[i] += g[i];
        } else if constexpr (VEC) {
          sh_store<T, W>(o, g);
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i) if (at + i < a.E) o[i] = sh_from_float<T>(g[i]);
        }
      }
      o += ostep;
    }
  }
}
