// Norms of queries and keys per head with the position rotation in the same pass, and the backward pass of both.
//
//   r = (mean(x^2) + eps)^-1/2,  y = s Rot(pos) (g x r);   u = s Rot(-pos) dy,  dg = sum u x r,  dx = r (g u - x r mean(g u x r))
//
// A row (one token's head) belongs to `lanes` neighbouring lanes with NV vectors of V values each, in registers from the
// load to the store: x is read once and y written once, the mean is a butterfly over the group.  A pair of rotated columns
// never leaves its lane: neighbouring columns lie in one vector, columns half the rotated width apart in two vectors of the
// same lane.  A group takes several heads of one token, which share the angles.
//
// Angles are turns in 64-bit fixed point: the frequency (divided by 2 pi) times the position, modulo 2^64, is the fraction
// of a turn without any rounding that grows with the position; sincospif of its upper 32 bits is off by 2^-25 turns at most.
#pragma once
#include "sh_vec.cuh"

constexpr int QN_THREADS = 256;
constexpr int QN_MAX_D = 256;
constexpr int QN_MAX_BLOCKS = 1024;       // blocks of the backward kernel at most (rows of its partial gain gradients)

struct QnSide {
  const void* x; const void* dy; void* out;              // out: y, or dx
  const float* gain;
  float* dgain;                                          // nullptr: not wanted
  long long xb, xt, xh, yb, yt, yh, ob, ot, oh;          // strides of batch, token, head (elements): of x, dy, out
  int heads, chunks;                                     // chunks of up to `per` heads
  float scale;
};
struct QnArgs {
  QnSide s[2];
  const void* pos;                                       // [batch, seq] or nullptr: the token's place in its sequence
  int pos64, next;                                       // next: rotated pairs are neighbouring columns
  int seq, D, R;                                         // R: rotated columns
  int lanes, per;                                        // lanes to a row; heads to a group
  long long tokens;                                      // batch * seq
  int blocks0;                                           // backward: blocks of the queries (the rest: keys)
  float eps;
  float* part;                                           // backward: [blocks][D]
  unsigned long long freq[QN_MAX_D / 2];                 // turns per position of each pair, times 2^64
};

// The columns of a lane's vectors (-1: none): vector i at (lane + i lanes) V, with neighbouring pairs inside a vector; or,
// PAIRED, vectors 2 j and 2 j + 1 in the two halves of the rotated columns, or of the columns behind them.  (Vectors of one
// value, where the addresses allow no more, are paired in either order.)
template <int V, int NV, bool PAIRED>
__device__ __forceinline__ void qn_columns(const QnArgs& a, int l, int (&col)[NV]) {
  if constexpr (!PAIRED) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (l + i * a.lanes) * V;
      col[i] = c < a.D ? c : -1;
    }
  } else {
    const int h = a.R / 2, t = (a.D - a.R) / 2;
#pragma unroll
    for (int j = 0; j < NV / 2; ++j) {
      const int p = (l + j * a.lanes) * V;
      if (V == 1 && a.next) {
        col[2 * j] = 2 * p < a.D ? 2 * p : -1;
        col[2 * j + 1] = 2 * p < a.D ? 2 * p + 1 : -1;
        continue;
      }
      const bool rot = p < h, tail = !rot && p - h < t;
      col[2 * j] = rot ? p : tail ? a.R + p - h : -1;
      col[2 * j + 1] = rot ? h + p : tail ? a.R + t + p - h : -1;
    }
  }
}

// cos and sin of a lane's pairs at a position: pair p of a vector (neighbouring) or of two vectors (halves).
template <int V, int NV, bool PAIRED>
__device__ __forceinline__ void qn_angles(const QnArgs& a, const unsigned long long* freq, long long pos, const int (&col)[NV], float (&cs)[NV * V / 2], float (&sn)[NV * V / 2]) {
#pragma unroll
  for (int i = 0; i < NV * V / 2; ++i) {
    int pair, at;                                        // the pair's number and its first column
    bool rot;
    if constexpr (PAIRED) {
      const bool next = V == 1 && a.next;
      at = col[2 * (i / V)] + i % V; pair = next ? at / 2 : at;
      rot = col[2 * (i / V)] >= 0 && pair < a.R / 2;
    } else {
      at = col[i / (V / 2)] + 2 * (i % (V / 2)); pair = at / 2;
      rot = col[i / (V / 2)] >= 0 && at < a.R;
    }
    cs[i] = 1.f; sn[i] = 0.f;
    if (rot) {
      const unsigned long long turns = (unsigned long long)pos * freq[pair];
      sincospif((float)(int)(turns >> 32) * 4.656612873077393e-10f, &sn[i], &cs[i]);   // (2^-31: half turns)
    }
  }
}

template <int V, int NV, bool PAIRED, bool BACK>
__device__ __forceinline__ void qn_rotate(float (&f)[NV][V], const float (&cs)[NV * V / 2], const float (&sn)[NV * V / 2]) {
#pragma unroll
  for (int i = 0; i < NV * V / 2; ++i) {
    float& p = PAIRED ? f[2 * (i / V)][i % V] : f[i / (V / 2)][2 * (i % (V / 2))];
    float& q = PAIRED ? f[2 * (i / V) + 1][i % V] : f[i / (V / 2)][2 * (i % (V / 2)) + 1];
    const float s = BACK ? -sn[i] : sn[i], x = p, y = q;
    p = x * cs[i] - y * s;
    q = x * s + y * cs[i];
  }
}

__device__ __forceinline__ long long qn_position(const QnArgs& a, long long token, int t) {
  if (!a.pos) return t;
  return a.pos64 ? __ldg((const long long*)a.pos + token) : (long long)__ldg((const int*)a.pos + token);
}

__device__ __forceinline__ long long qn_div(long long n, int d) { return n >> 32 ? n / d : (long long)((unsigned)n / (unsigned)d); }

// V = 1 without pairs: nothing is rotated (d_head may be odd).
template <typename T, int V, int NV, bool PAIRED>
static __global__ void __launch_bounds__(QN_THREADS) sh_qk_norm_kernel(const __grid_constant__ QnArgs a) {
  __shared__ unsigned long long s_freq[QN_MAX_D / 2];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int P = V > 1 || PAIRED ? NV * V / 2 : 1;
  for (int i = threadIdx.x; i < a.R / 2; i += QN_THREADS) s_freq[i] = a.freq[i];
  if (a.R) __syncthreads();
  const int l = threadIdx.x & (a.lanes - 1);
  const long long item = (long long)blockIdx.x * (QN_THREADS / a.lanes) + threadIdx.x / a.lanes;
  const int chunks = a.s[0].chunks + a.s[1].chunks;
  const long long token = qn_div(item, chunks);
  const bool live = token < a.tokens;                    // (a warp's groups shuffle together: none leaves early)
  int chunk = (int)(item - token * chunks);
  const int side = chunk >= a.s[0].chunks;
  const QnSide& s = a.s[side];
  if (side) chunk -= a.s[0].chunks;
  const long long b = qn_div(token, a.seq);
  const int t = (int)(token - b * a.seq);
  int col[NV];
  qn_columns<V, NV, PAIRED>(a, l, col);
  float cs[P], sn[P];
  if constexpr (V > 1 || PAIRED)
    if (a.R && live) qn_angles<V, NV, PAIRED>(a, s_freq, qn_position(a, token, t), col, cs, sn);
  float g[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) g[i][j] = s.scale * (s.gain && col[i] >= 0 ? __ldg(s.gain + col[i] + j) : 1.f);
  const T* x = (const T*)s.x + b * s.xb + t * s.xt;
  T* y = (T*)s.out + b * s.ob + t * s.ot;
  const int h0 = chunk * a.per;
  const float inv = 1.f / (float)a.D;
  // the same number of rounds for every group of a warp; two heads' loads in flight
  for (int j = 0; j < a.per; j += 2) {
    float f[2][NV][V];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (live && h0 + j + u < s.heads && j + u < a.per && col[i] >= 0) {
          sh_load<T, V>(x + (h0 + j + u) * s.xh + col[i], f[u][i]);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) f[u][i][v] = 0.f;
        }
      }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) ss = fmaf(f[u][i][v], f[u][i][v], ss);
      const float r = rsqrtf(fmaf(sh_group_sum(ss, a.lanes), inv, a.eps));
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) f[u][i][v] *= r * g[i][v];
      if constexpr (V > 1 || PAIRED)
        if (a.R) qn_rotate<V, NV, PAIRED, false>(f[u], cs, sn);
      if (live && h0 + j + u < s.heads && j + u < a.per) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (col[i] >= 0) sh_store<T, V>(y + (h0 + j + u) * s.oh + col[i], f[u][i]);
      }
    }
  }
}

// The first `blocks0` blocks take the queries, the others the keys, each in rounds over its side's (token, chunk of heads).
// A thread adds its columns' share of the gain gradients over its rows; the block's groups are added in order in shared
// memory, the blocks by sh_qk_norm_gain_kernel: the same bits on every run.
template <typename T, int V, int NV, bool PAIRED>
static __global__ void __launch_bounds__(QN_THREADS) sh_qk_norm_backward_kernel(const __grid_constant__ QnArgs a) {
  __shared__ unsigned long long s_freq[QN_MAX_D / 2];
  extern __shared__ float s_sum[];                       // [groups][D]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int P = V > 1 || PAIRED ? NV * V / 2 : 1;
  for (int i = threadIdx.x; i < a.R / 2; i += QN_THREADS) s_freq[i] = a.freq[i];
  if (a.R) __syncthreads();
  const int l = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = QN_THREADS / a.lanes;
  const int side = (int)blockIdx.x >= a.blocks0;
  const QnSide& s = a.s[side];
  const int block = side ? blockIdx.x - a.blocks0 : blockIdx.x, blocks = side ? gridDim.x - a.blocks0 : a.blocks0;
  int col[NV];
  qn_columns<V, NV, PAIRED>(a, l, col);
  float g[NV][V], dg[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      g[i][j] = s.gain && col[i] >= 0 ? __ldg(s.gain + col[i] + j) : 1.f;
      dg[i][j] = 0.f;
    }
  const float inv = 1.f / (float)a.D;
  const long long items = a.tokens * s.chunks, step = (long long)blocks * groups;
  // (rounds: the same for every group of the block)
  for (long long first = (long long)block * groups; first < items; first += step) {
    const long long item = first + group;
    const bool live = item < items;
    const long long token = live ? qn_div(item, s.chunks) : 0;
    const int h0 = live ? (int)(item - token * s.chunks) * a.per : 0;
    const long long b = qn_div(token, a.seq);
    const int t = (int)(token - b * a.seq);
    float cs[P], sn[P];
    if constexpr (V > 1 || PAIRED)
      if (a.R && live) qn_angles<V, NV, PAIRED>(a, s_freq, qn_position(a, token, t), col, cs, sn);
    const T* x = (const T*)s.x + b * s.xb + t * s.xt;
    const T* dy = (const T*)s.dy + b * s.yb + t * s.yt;
    T* dx = (T*)s.out + b * s.ob + t * s.ot;
    for (int j = 0; j < a.per; ++j) {
      const int h = h0 + j;
      const bool row = live && h < s.heads;
      float f[NV][V], u[NV][V];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (row && col[i] >= 0) {
          sh_load<T, V>(x + h * s.xh + col[i], f[i]);
          sh_load<T, V>(dy + h * s.yh + col[i], u[i]);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) f[i][v] = u[i][v] = 0.f;
        }
      }
      if constexpr (V > 1 || PAIRED)
        if (a.R) qn_rotate<V, NV, PAIRED, true>(u, cs, sn);
      float ss = 0.f, wx = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          u[i][v] *= s.scale;
          ss = fmaf(f[i][v], f[i][v], ss);
          wx = fmaf(u[i][v] * g[i][v], f[i][v], wx);
        }
      ss = sh_group_sum(ss, a.lanes);
      wx = sh_group_sum(wx, a.lanes);
      const float r = rsqrtf(fmaf(ss, inv, a.eps)), m = wx * inv * r * r;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (row) dg[i][v] = fmaf(u[i][v], f[i][v] * r, dg[i][v]);
          u[i][v] = r * fmaf(-f[i][v], m, u[i][v] * g[i][v]);
        }
      if (row) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (col[i] >= 0) sh_store<T, V>(dx + h * s.oh + col[i], u[i]);
      }
    }
  }
  if (!s.dgain) return;                                  // (the whole block)
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (col[i] >= 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) s_sum[group * a.D + col[i] + v] = dg[i][v];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < a.D; c += QN_THREADS) {
    float sum = 0.f;
    for (int q = 0; q < groups; ++q) sum += s_sum[q * a.D + c];
    a.part[(long long)blockIdx.x * a.D + c] = sum;
  }
}

// dgain[c] = sum over a side's blocks, in 64 bits, in a fixed order.  Blocks of 32 columns x 32 rows of partial sums.
struct QnGain { const float* part; float* dgain[2]; int first[3]; int D; };     // side i: rows first[i] .. first[i + 1] - 1
static __global__ void __launch_bounds__(1024) sh_qk_norm_gain_kernel(QnGain a) {
  __shared__ double s_sum[32][33];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int side = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
  float* out = a.dgain[side];
  if (!out) return;                                      // (the whole block)
  double sum = 0.0;
  if (c < a.D)
    for (int i = a.first[side] + threadIdx.y; i < a.first[side + 1]; i += 32) sum += (double)__ldcg(a.part + (long long)i * a.D + c);
  s_sum[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.y == 0 && c < a.D) {
    sum = 0.0;
    for (int i = 0; i < 32; ++i) sum += s_sum[i][threadIdx.x];
    out[c] = (float)sum;
  }
}
