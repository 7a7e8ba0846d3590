// The balance loss of the gates, the per-expert counts, and the loss's gradient with respect to the gate logits.
//
//   p = softmax over a gate's E logits,  P_e = mean of p_e over the tokens,  f_e = share of the selections
//   counts:  L = coef sum_gates E sum_e f_e P_e      entropy:  L = coef sum_gates sum_e P_e ln P_e
//   dL/dz_e = p_e (c_e - sum_j p_j c_j),  c_e = dL/dP_e / n:  any constant may be taken off c, so it is kept centred
//
// A row (a token's E logits of one gate) belongs to L neighbouring lanes with W values each.  Between its rounds a thread
// stays with the same gate, so its share of P is W sums in registers.
#pragma once
#include "sh_vec.cuh"

constexpr int BL_THREADS = 256;
constexpr int BL_MAX_BLOCKS = 592;         // blocks of the first kernel at most (rows of partial results)

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

// The lane's W logits of a row.  VEC: E = L W, aligned.
template <typename T, int W, bool VEC>
__device__ __forceinline__ void bl_load(const T* p, int at, int E, float (&f)[W], float none) {
  if constexpr (VEC) {
    sh_load<T, W>(p + at, f);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = at + i < E ? sh_to_float<T>(p[at + i]) : none;
  }
}

template <int L> __device__ __forceinline__ float bl_max(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int L> __device__ __forceinline__ float bl_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// p from a row's logits, in place.  A row of -inf only has no probabilities: zeros.
template <int W, int L>
__device__ __forceinline__ void bl_softmax(float (&f)[W]) {
  float m = f[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, f[i]);
  m = bl_max<L>(m);
  const bool none = m == -INFINITY;                      // (a NaN is no maximum: it comes out of the exponential)
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) { f[i] = __isnanf(f[i]) || !none ? expf(f[i] - m) : 0.f; s += f[i]; }
  s = bl_sum<L>(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < W; ++i) f[i] *= inv;
}

// A block's share of the sums: tokens tpb at a time, blockIdx.y's gates.
template <typename T, int W, int L, bool VEC>
static __global__ void __launch_bounds__(BL_THREADS) sh_balance_sums_kernel(const BlArgs a) {
  constexpr int EP = W * L, ROWS = BL_THREADS / L;
  __shared__ float s_p[ROWS][EP + 1];
  __shared__ int s_n[ROWS * EP];                         // [gate of the block][expert]
  __shared__ int s_tokens;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int row = threadIdx.x / L, at = (threadIdx.x % L) * W;
  const int g0 = blockIdx.y * a.per, ng = min(a.per, a.gates - g0);
  const int gl = row % a.per, tl = row / a.per, gate = g0 + gl;
  const bool mine = tl < a.tpb && gl < ng;
  for (int i = threadIdx.x; i < ng * EP; i += BL_THREADS) s_n[i] = 0;
  if (threadIdx.x == 0) s_tokens = 0;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.ticket = 0;
  __syncthreads();
  float acc[W];
  int seen = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = 0.f;
  const T* z = (const T*)a.z + (long long)gate * a.E;
  const int* idx = a.idx + ((long long)(gate / a.H) * a.tokens * a.H + gate % a.H) * a.k;
  for (long long t0 = (long long)blockIdx.x * a.tpb; t0 < a.tokens; t0 += (long long)gridDim.x * a.tpb) {
    const long long t = t0 + tl;
    const bool live = mine && t < a.tokens && (!a.mask || a.mask[t]);
    float f[W];
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = -INFINITY;
    if (live) bl_load<T, W, VEC>(z + t * a.zt, at, a.E, f, -INFINITY);
    if (live) {
      for (int j = threadIdx.x % L; j < a.k; j += L) {
        const unsigned e = (unsigned)idx[t * a.H * a.k + j];
        if (e < (unsigned)a.E) atomicAdd(&s_n[gl * EP + e], 1);     // (a slot without an expert is not counted)
      }
    }
    bl_softmax<W, L>(f);
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] += f[i];
    seen += live;
  }
  if (mine && gl == 0 && threadIdx.x % L == 0 && seen) atomicAdd(&s_tokens, seen);
#pragma unroll
  for (int i = 0; i < W; ++i) s_p[row][at + i] = acc[i];
  __syncthreads();
  const long long base = (long long)blockIdx.x * a.gates * a.E;
  for (int i = threadIdx.x; i < ng * a.E; i += BL_THREADS) {
    const int q = i / a.E, e = i % a.E;
    float sum = 0.f;
    for (int r = 0; r < a.tpb; ++r) sum += s_p[r * a.per + q][e];
    a.part_p[base + (long long)(g0 + q) * a.E + e] = sum;
    a.part_n[base + (long long)(g0 + q) * a.E + e] = s_n[q * EP + e];
  }
  if (blockIdx.y == 0 && threadIdx.x == 0) a.part_n[(long long)gridDim.x * a.gates * a.E + blockIdx.x] = s_tokens;
}

struct BlOut {
  const float* part_p; const int* part_n; unsigned* ticket; double* gate_loss;
  int blocks, gates, E, kind;
  double coef;
  float *loss, *prob, *slope; int* counts;
};

// A gate per block: its experts' sums over the first kernel's blocks in a fixed order, in 64 bits, its share of the loss
// and the centred slope; the block that comes last adds the gates' losses in order.
static __global__ void __launch_bounds__(BL_THREADS) sh_balance_loss_kernel(const BlOut a) {
  __shared__ double s_p[BL_THREADS];
  __shared__ int s_n[BL_THREADS], s_last;
  __shared__ int s_t[BL_THREADS / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int gate = blockIdx.x, e = threadIdx.x & 31, r = threadIdx.x >> 5, cols = a.gates * a.E;
  double p = 0.0;
  int n = 0, tokens = 0;
  if (e < a.E)
    for (int b = r; b < a.blocks; b += BL_THREADS / 32) {
      p += (double)__ldcg(a.part_p + (long long)b * cols + gate * a.E + e);
      n += __ldcg(a.part_n + (long long)b * cols + gate * a.E + e);
    }
  for (int b = threadIdx.x; b < a.blocks; b += BL_THREADS) tokens += __ldcg(a.part_n + (long long)a.blocks * cols + b);
  s_p[threadIdx.x] = p; s_n[threadIdx.x] = n;
  for (int o = 16; o > 0; o >>= 1) tokens += __shfl_xor_sync(0xffffffffu, tokens, o);
  if (e == 0) s_t[r] = tokens;
  __syncthreads();
  if (r == 0) {
    tokens = 0;
    for (int i = 0; i < BL_THREADS / 32; ++i) { tokens += s_t[i]; if (i) { p += s_p[i * 32 + e]; n += s_n[i * 32 + e]; } }
    const double P = tokens ? p / tokens : 0.0;
    int all = n;
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    const double f = all ? (double)n / all : 0.0;
    // (an expert without any probability has no slope: p is zero wherever it would be used)
    double c = 0.0, l = 0.0, mean = 0.0;
    if (e < a.E) {
      if (a.kind == 0) { l = a.E * f * P; c = a.E * f; }
      else if (P != 0.0) { c = log(P); l = P * c; }
    }
    const int used = a.kind == 0 || P != 0.0;
    double cs = e < a.E && used ? c : 0.0;
    int cn = e < a.E && used;
    for (int o = 16; o > 0; o >>= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, o);
      cs += __shfl_xor_sync(0xffffffffu, cs, o);
      cn += __shfl_xor_sync(0xffffffffu, cn, o);
    }
    mean = cn ? cs / cn : 0.0;
    if (e < a.E) {
      const int o = gate * a.E + e;
      a.counts[o] = n;
      a.prob[o] = (float)P;
      a.slope[o] = used && tokens ? (float)(a.coef * (c - mean) / tokens) : 0.f;
    }
    if (e == 0) {
      a.gate_loss[gate] = tokens ? a.coef * l : 0.0;
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

// dz, or dz += (ADD: fp32, the gates' gradients of a backward pass).
template <typename T, int W, int L, bool VEC, bool ADD>
static __global__ void __launch_bounds__(BL_THREADS) sh_balance_backward_kernel(const BlArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int row = threadIdx.x / L, at = (threadIdx.x % L) * W;
  const int g0 = blockIdx.y * a.per, gl = row % a.per, tl = row / a.per, gate = g0 + gl;
  const bool mine = tl < a.tpb && gate < a.gates;
  const float gloss = a.gloss ? __ldg(a.gloss) : 1.f;
  float c[W];
#pragma unroll
  for (int i = 0; i < W; ++i) c[i] = mine && at + i < a.E ? __ldg(a.slope + gate * a.E + at + i) : 0.f;
  const T* z = (const T*)a.z + (long long)gate * a.E;
  T* dz = (T*)a.dz + (long long)gate * a.E;
  for (long long t0 = (long long)blockIdx.x * a.tpb; t0 < a.tokens; t0 += (long long)gridDim.x * a.tpb) {
    const long long t = t0 + tl;
    const bool there = mine && t < a.tokens, live = there && (!a.mask || a.mask[t]);
    float f[W];
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = -INFINITY;
    if (live) bl_load<T, W, VEC>(z + t * a.zt, at, a.E, f, -INFINITY);
    bl_softmax<W, L>(f);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) dot = fmaf(f[i], c[i], dot);
    dot = bl_sum<L>(dot);
    if (!there) continue;                                // (no shuffle below)
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = live ? gloss * (f[i] * (c[i] - dot)) : 0.f;
    T* o = dz + t * a.dzt;
    if constexpr (ADD) {
#pragma unroll
      for (int i = 0; i < W; ++i) if (live && at + i < a.E) o[at + i] += f[i];
    } else if constexpr (VEC) {
      sh_store<T, W>(o + at, f);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) if (at + i < a.E) o[at + i] = sh_from_float<T>(f[i]);
    }
  }
}
