// Norms of queries and keys per head with the position rotation in the same pass, and the backward pass of both.
//
//   r = (mean(x^2) + eps)^-1/2,  y = s Rot(pos) (g x r);   u = s Rot(-pos) dy,  dg = sum u x r,  dx = r (g u - x r mean(g u x r))
//
// A row (one token's head) belongs to LANES neighbouring lanes with NV vectors of V values each, in registers from the
// load to the store: x is read once and y written once, the mean is a butterfly over the group.  A pair of rotated columns
// never leaves its lane: neighbouring columns lie in one vector, columns half the rotated width apart in two vectors of the
// same lane.  A group takes several heads of one token, which share the angles.
//
// Angles are turns in 64-bit fixed point: the frequency (divided by 2 pi) times the position, modulo 2^64, is the fraction
// of a turn without any rounding that grows with the position; its upper 32 bits as a float are off by 2^-26 turns at most.
//
// What bounds it: HBM forward (16384 tokens, 40 heads of 128 in bf16: 59 us, 5.7 TB/s of 6.56 measured; 16 heads in fp32: 45 us, 6.0), where a
// group's heads are many; else what a group does once (angles, factors, addresses: as much as for three rows).  Backward, 16 heads: in
// fp32 68 us, 5.9 TB/s; in bf16 42 us, 4.8 TB/s: latency at 24 warps an SM - issue slots 62 % full, HBM 43 %, no warp ready in 37 % of the cycles; a
// warp waits as long for the exchanges across lanes as for memory, and longest for the instruction before.
// Rows in flight through shared memory (cp.async) instead of registers: 92 and 72 us.
#pragma once
#include "sh_vec.cuh"

constexpr int QN_THREADS = 256;
constexpr int QN_MAX_D = 256;
constexpr int QN_PAIRS = QN_MAX_D / 2;    // (as many as the widest row's lanes hold)
// The backward kernel's vectors are of 4 values at most (8 of a 16-bit type: 128 registers and spills; 33.5 M values of 16384 tokens, 16 heads
// of 128: 56 us, with 4 42), and its blocks 3 to an SM, which leaves the paired variants of 16-bit types 16 to 60 bytes of spills (fp32, whose rows on their way are twice as large, vectors of one value, and six of two: 2; 8 x 256
// tokens in fp32: 13.5 us with 3, 9.0 with 2).
constexpr int QN_BACKWARD_V = 4;
template <typename T, int V, int NV> __host__ __device__ constexpr int qn_backward_blocks() { return sizeof(T) == 4 || V == 1 || NV == 6 ? 2 : 3; }
constexpr int QN_CHAIN = 512;
constexpr int QN_MAX_BLOCKS = 1024;       // blocks of the backward kernel at most (rows of its partial gain gradients)

// Division of 0 <= n < 2^31 by d >= 1 (0: nothing is divided): (n + upper half of n m) >> s.
struct QnDiv { unsigned d, m, s; };
inline QnDiv qn_divisor(unsigned d) {
  QnDiv r{d, 0, 0};
  if (d == 0) return r;
  while ((1ull << r.s) < d) ++r.s;
  r.m = (unsigned)(((1ull << 32) * ((1ull << r.s) - d)) / d + 1);
  return r;
}

struct QnSide {
  const void* x; const void* dy; void* out;              // out: y, or dx
  const float* gain;
  float* dgain;                                          // nullptr: not wanted
  long long xb, xt, xh, yb, yt, yh, ob, ot, oh;          // strides of batch, token, head (elements): of x, dy, out
  long long from, to;                                    // backward: (token, chunk) numbers of this launch
  int heads;
  QnDiv chunks;                                          // chunks of up to `per` heads
  float scale;
};
struct QnArgs {
  QnSide s[2];
  const void* pos;                                       // [batch, seq] or nullptr: the token's place in its sequence
  int pos64, next;                                       // next: rotated pairs are neighbouring columns
  QnDiv seq, chunks;                                     // chunks: of both sides
  int large;                                             // (token, chunk) numbers of 2^31 and more
  int D, R;                                              // R: rotated columns
  int per;                                               // heads to a group
  long long tokens;                                      // batch * seq
  int blocks0;                                           // backward: blocks of the queries (the rest: keys)
  float eps;
  float* part;                                           // backward: [blocks][D]
  unsigned long long freq[QN_MAX_D / 2];                 // turns per position of each pair, times 2^64
};

// The columns of a lane's vectors (-1: none): vector i at (lane + i LANES) V, with neighbouring pairs inside a vector; or,
// PAIRED, vectors 2 j and 2 j + 1 in the two halves of the rotated columns, or of the columns behind them.  (Vectors of one
// value, where the addresses allow no more, are paired in either order.)
template <int V, int NV, int LANES, bool PAIRED>
__device__ __forceinline__ void qn_columns(const QnArgs& a, int l, int (&col)[NV]) {
  if constexpr (!PAIRED) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (l + i * LANES) * V;
      col[i] = c < a.D ? c : -1;
    }
  } else {
    const int h = a.R / 2, t = (a.D - a.R) / 2;
#pragma unroll
    for (int j = 0; j < NV / 2; ++j) {
      const int p = (l + j * LANES) * V;
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

// Vector i of a row whose lane's first vector is at p.  (Without pairs the distance is known to the compiler.)
template <int V, int NV, int LANES, bool PAIRED, typename T>
__device__ __forceinline__ T* qn_vector(T* p, const int (&col)[NV], int i) {
  return p + (PAIRED ? col[i] - col[0] : i * LANES * V);
}

// The lane's values as pairs (A, B) that a rotation mixes, two pairs to a register pair (packed fp32 arithmetic: two
// operations an instruction).  Pair n is made of two neighbouring values, or of value n % V of vectors 2 (n / V) and + 1.
template <int V, bool PAIRED> __device__ __forceinline__ constexpr int qn_vec_a(int n) { return PAIRED ? 2 * (n / V) : 2 * n / V; }
template <int V, bool PAIRED> __device__ __forceinline__ constexpr int qn_vec_b(int n) { return PAIRED ? 2 * (n / V) + 1 : (2 * n + 1) / V; }
template <int V, bool PAIRED> __device__ __forceinline__ constexpr int qn_at_a(int n) { return PAIRED ? n % V : 2 * n % V; }
template <int V, bool PAIRED> __device__ __forceinline__ constexpr int qn_at_b(int n) { return PAIRED ? n % V : (2 * n + 1) % V; }

template <int P> struct QnPairs { float2 a[P / 2], b[P / 2]; };

__device__ __forceinline__ float& qn_half(float2& v, int h) { return h ? v.y : v.x; }

template <typename T, int V, int NV, bool PAIRED>
__device__ __forceinline__ void qn_get(const ShRaw<T, V> (&raw)[NV], QnPairs<NV * V / 2>& x) {
  float f[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) raw[i].get(f[i]);
#pragma unroll
  for (int n = 0; n < NV * V / 2; ++n) {
    qn_half(x.a[n / 2], n & 1) = f[qn_vec_a<V, PAIRED>(n)][qn_at_a<V, PAIRED>(n)];
    qn_half(x.b[n / 2], n & 1) = f[qn_vec_b<V, PAIRED>(n)][qn_at_b<V, PAIRED>(n)];
  }
}
template <typename T, int V, int NV, int LANES, bool PAIRED>
__device__ __forceinline__ void qn_put(T* p, const int (&col)[NV], QnPairs<NV * V / 2>& x) {
  float f[NV][V];
#pragma unroll
  for (int n = 0; n < NV * V / 2; ++n) {
    f[qn_vec_a<V, PAIRED>(n)][qn_at_a<V, PAIRED>(n)] = qn_half(x.a[n / 2], n & 1);
    f[qn_vec_b<V, PAIRED>(n)][qn_at_b<V, PAIRED>(n)] = qn_half(x.b[n / 2], n & 1);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (col[i] >= 0) sh_store<T, V>(qn_vector<V, NV, LANES, PAIRED>(p, col, i), f[i]);
}

// The lane's gains: ones where there are none.
template <int V, int NV, bool PAIRED>
__device__ __forceinline__ void qn_gains(const float* gain, const int (&col)[NV], QnPairs<NV * V / 2>& g) {
  ShRaw<float, V> raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    raw[i].fill(0x3F800000u);
    if (gain && col[i] >= 0) raw[i].load(gain + col[i]);
  }
  qn_get<float, V, NV, PAIRED>(raw, g);
}

// The frequencies into shared memory; zeros behind the rotated columns, whose cos and sin are then 1 and 0 without a branch.
__device__ __forceinline__ void qn_frequencies(const QnArgs& a, unsigned long long* freq) {
  for (int i = threadIdx.x; i < QN_PAIRS; i += QN_THREADS) freq[i] = i < a.R / 2 ? a.freq[i] : 0ull;
}

// cos and sin of the lane's pair n at a position.  16-bit results: the special function unit's (off by 2^-21, where a result's half
// step is 2^-12 at least); fp32: sincospif.
template <typename T, int V, int NV, int LANES, bool PAIRED>
__device__ __forceinline__ void qn_angle(const unsigned long long* freq, int l, long long pos, int n, float* cs, float* sn) {
  // (pairs in the order of the lanes' columns: neighbours by their first column, halves by the first one's)
  const int pair = PAIRED ? (l + n / V * LANES) * V + n % V : ((l + 2 * n / V * LANES) * V + 2 * n % V) / 2;
  const unsigned long long f = freq[pair];
  // (the upper half of the product's lower 64 bits: half turns times 2^31)
  const float x = (float)(int)(__umulhi((unsigned)pos, (unsigned)f) + (unsigned)pos * (unsigned)(f >> 32) + (unsigned)(pos >> 32) * (unsigned)f);
  if constexpr (sizeof(T) == 2) __sincosf(x * (3.14159265f * 4.656612873077393e-10f), sn, cs);
  else sincospif(x * 4.656612873077393e-10f, sn, cs);
}

__device__ __forceinline__ long long qn_position(const QnArgs& a, long long token, int t) {
  if (!a.pos) return t;
  return a.pos64 ? __ldg((const long long*)a.pos + token) : (long long)__ldg((const int*)a.pos + token);
}
__device__ __forceinline__ long long qn_div(const QnArgs& a, long long n, const QnDiv& d) {
  return a.large ? n / d.d : (long long)((__umulhi((unsigned)n, d.m) + (unsigned)n) >> d.s);
}

// V = 1 without pairs: nothing is rotated (d_head may be odd).
template <typename T, int V, int NV, int LANES, bool PAIRED>
static __global__ void __launch_bounds__(QN_THREADS, 3) sh_qk_norm_kernel(const __grid_constant__ QnArgs a) {
  __shared__ __align__(16) unsigned long long s_freq[QN_PAIRS];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int P = NV * V / 2;
  if (a.R) qn_frequencies(a, s_freq);
  const int l = threadIdx.x % LANES;
  const long long item = (long long)blockIdx.x * (QN_THREADS / LANES) + threadIdx.x / LANES;
  const long long token = qn_div(a, item, a.chunks);
  const bool live = token < a.tokens;                    // (a warp's groups shuffle together: none leaves early)
  int chunk = (int)(item - token * a.chunks.d);
  const int side = chunk >= (int)a.s[0].chunks.d;
  const QnSide& s = a.s[side];
  if (side) chunk -= a.s[0].chunks.d;
  const long long b = qn_div(a, token, a.seq);
  const int t = (int)(token - b * a.seq.d);
  const int h0 = chunk * a.per, n = live ? min(a.per, s.heads - h0) : 0;
  int col[NV];
  qn_columns<V, NV, LANES, PAIRED>(a, l, col);
  const T* px = (const T*)s.x + b * s.xb + t * s.xt + h0 * s.xh + col[0];
  T* py = (T*)s.out + b * s.ob + t * s.ot + h0 * s.oh + col[0];
  // The next two heads' values are on their way while one is worked on; the same number of rounds for every group of a warp.
  // (A lane without columns keeps its zeros, a group without a next head what it has: it is not stored.)
  ShRaw<T, V> raw[2][NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) { raw[0][i].fill(0); raw[1][i].fill(0); }
  auto fetch = [&](int j, ShRaw<T, V> (&to)[NV]) {
    if (j < n) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (col[i] >= 0) to[i].load(qn_vector<V, NV, LANES, PAIRED>(px, col, i));
    }
    px += s.xh;
  };
  fetch(0, raw[0]); fetch(1, raw[1]);
  const long long pos = live && a.R ? qn_position(a, token, t) : 0;
  QnPairs<P> g;
  qn_gains<V, NV, PAIRED>(s.gain, col, g);
  if (a.R) __syncthreads();                              // the frequencies
  // y = r (A ga cs - B gb sn, A ga sn + B gb cs): gains, scale and angles in four factors a pair, for all of the heads
  QnPairs<P> fa, fb;
#pragma unroll
  for (int m = 0; m < P; ++m) {
    float cs = 1.f, sn = 0.f;
    if constexpr (V > 1 || PAIRED)
      if (a.R) qn_angle<T, V, NV, LANES, PAIRED>(s_freq, l, pos, m, &cs, &sn);
    const float ga = s.scale * qn_half(g.a[m / 2], m & 1), gb = s.scale * qn_half(g.b[m / 2], m & 1);
    qn_half(fa.a[m / 2], m & 1) = ga * cs; qn_half(fa.b[m / 2], m & 1) = -gb * sn;
    qn_half(fb.a[m / 2], m & 1) = ga * sn; qn_half(fb.b[m / 2], m & 1) = gb * cs;
  }
  const float inv = 1.f / (float)a.D;
  for (int j0 = 0; j0 < a.per; j0 += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      QnPairs<P> x, y;
      qn_get<T, V, NV, PAIRED>(raw[u], x);
      fetch(j0 + u + 2, raw[u]);
      float2 ss = make_float2(0.f, 0.f);
#pragma unroll
      for (int m = 0; m < P / 2; ++m) {
        ss = __ffma2_rn(x.a[m], x.a[m], ss);
        ss = __ffma2_rn(x.b[m], x.b[m], ss);
        y.a[m] = __ffma2_rn(x.a[m], fa.a[m], __fmul2_rn(x.b[m], fa.b[m]));
        y.b[m] = __ffma2_rn(x.a[m], fb.a[m], __fmul2_rn(x.b[m], fb.b[m]));
      }
      const float r = rsqrtf(fmaf(sh_group_sum<LANES>(ss.x + ss.y), inv, a.eps));
      const float2 rr = make_float2(r, r);
#pragma unroll
      for (int m = 0; m < P / 2; ++m) { y.a[m] = __fmul2_rn(y.a[m], rr); y.b[m] = __fmul2_rn(y.b[m], rr); }
      if (j0 + u < n) qn_put<T, V, NV, LANES, PAIRED>(py, col, y);
      py += s.oh;
    }
  }
}

// The first `blocks0` blocks take the queries, the others the keys, each in rounds over its side's (token, chunk of heads).
// A thread adds its columns' share of the gain gradients over its rows; the block's groups are added in order in shared
// memory, the blocks by sh_qk_norm_gain_kernel: the same bits on every run.  A thread's fp32 sum is of QN_CHAIN rows at most (a longer one, of values
// of one sign, loses a bit with every doubling): more rows are taken by further launches, which add to the blocks' sums.  (Sums kept
// in 64 bits in shared memory beside the thread's, joined in the loop: 16384 tokens, 16 heads of 128 in bf16 48.8 us, as it is 42.2.)
template <typename T, int V, int NV, int LANES, bool PAIRED>
static __global__ void __launch_bounds__(QN_THREADS, qn_backward_blocks<T, V, NV>()) sh_qk_norm_backward_kernel(const __grid_constant__ QnArgs a) {
  __shared__ __align__(16) unsigned long long s_freq[QN_PAIRS];
  extern __shared__ float s_sum[];                       // [groups][D]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int P = NV * V / 2, GROUPS = QN_THREADS / LANES;
  if (a.R) qn_frequencies(a, s_freq);
  if (a.R) __syncthreads();
  const int l = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int side = (int)blockIdx.x >= a.blocks0;
  const QnSide& s = a.s[side];
  const int block = side ? blockIdx.x - a.blocks0 : blockIdx.x, blocks = side ? gridDim.x - a.blocks0 : a.blocks0;
  int col[NV];
  qn_columns<V, NV, LANES, PAIRED>(a, l, col);
  QnPairs<P> g, dg;
  qn_gains<V, NV, PAIRED>(s.gain, col, g);
#pragma unroll
  for (int m = 0; m < P / 2; ++m) dg.a[m] = dg.b[m] = make_float2(0.f, 0.f);
  const float inv = 1.f / (float)a.D;
  const long long items = s.to, step = (long long)blocks * GROUPS;
  // (rounds: the same for every group of the block)
  for (long long first = s.from + (long long)block * GROUPS; first < items; first += step) {
    const long long item = first + group;
    const bool live = item < items;
    const long long token = live ? qn_div(a, item, s.chunks) : 0;
    const int h0 = live ? (int)(item - token * s.chunks.d) * a.per : 0, n = live ? min(a.per, s.heads - h0) : 0;
    const long long b = qn_div(a, token, a.seq);
    const int t = (int)(token - b * a.seq.d);
    const T* px = (const T*)s.x + b * s.xb + t * s.xt + h0 * s.xh + col[0];
    const T* pd = (const T*)s.dy + b * s.yb + t * s.yt + h0 * s.yh + col[0];
    T* po = (T*)s.out + b * s.ob + t * s.ot + h0 * s.oh + col[0];
    // (as in the forward pass: the next two heads' values on their way)
    ShRaw<T, V> rx[2][NV], ry[2][NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) { rx[0][i].fill(0); rx[1][i].fill(0); ry[0][i].fill(0); ry[1][i].fill(0); }
    auto fetch = [&](int j, ShRaw<T, V> (&x)[NV], ShRaw<T, V> (&y)[NV]) {
      if (j < n) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (col[i] >= 0) {
            x[i].load(qn_vector<V, NV, LANES, PAIRED>(px, col, i));
            y[i].load(qn_vector<V, NV, LANES, PAIRED>(pd, col, i));
          }
      }
      px += s.xh; pd += s.yh;
    };
    fetch(0, rx[0], ry[0]); fetch(1, rx[1], ry[1]);
    const long long pos = live && a.R ? qn_position(a, token, t) : 0;
    float2 cs[P / 2], sn[P / 2];                         // times the scale
#pragma unroll
    for (int m = 0; m < P; ++m) {
      float c = 1.f, d = 0.f;
      if constexpr (V > 1 || PAIRED)
        if (a.R) qn_angle<T, V, NV, LANES, PAIRED>(s_freq, l, pos, m, &c, &d);
      qn_half(cs[m / 2], m & 1) = s.scale * c; qn_half(sn[m / 2], m & 1) = s.scale * d;
    }
    for (int j0 = 0; j0 < a.per; j0 += 2) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        QnPairs<P> x, y, u;
        qn_get<T, V, NV, PAIRED>(rx[q], x);
        qn_get<T, V, NV, PAIRED>(ry[q], y);
        fetch(j0 + q + 2, rx[q], ry[q]);
        // u = s Rot(-pos) dy;  t = u x;  sums of x^2 and of g t;  dx = r (g u) - r m x
        float2 ss = make_float2(0.f, 0.f), wx = ss;
#pragma unroll
        for (int m = 0; m < P / 2; ++m) {
          u.a[m] = __ffma2_rn(y.a[m], cs[m], __fmul2_rn(y.b[m], sn[m]));
          u.b[m] = __ffma2_rn(y.b[m], cs[m], __fmul2_rn(y.a[m], make_float2(-sn[m].x, -sn[m].y)));
          ss = __ffma2_rn(x.a[m], x.a[m], ss);
          ss = __ffma2_rn(x.b[m], x.b[m], ss);
          y.a[m] = __fmul2_rn(u.a[m], x.a[m]);
          y.b[m] = __fmul2_rn(u.b[m], x.b[m]);
          wx = __ffma2_rn(y.a[m], g.a[m], wx);
          wx = __ffma2_rn(y.b[m], g.b[m], wx);
          u.a[m] = __fmul2_rn(u.a[m], g.a[m]);
          u.b[m] = __fmul2_rn(u.b[m], g.b[m]);
        }
        float sum = ss.x + ss.y, dot = wx.x + wx.y;
        sh_group_sums<LANES>(sum, dot);
        float r = rsqrtf(fmaf(sum, inv, a.eps));
        if (j0 + q >= n) r = 0.f;                        // (no row: what is left of the last one does not count)
        const float rm = -(dot * inv * r * r) * r;
        const float2 r2 = make_float2(r, r), rm2 = make_float2(rm, rm);
#pragma unroll
        for (int m = 0; m < P / 2; ++m) {
          dg.a[m] = __ffma2_rn(y.a[m], r2, dg.a[m]);
          dg.b[m] = __ffma2_rn(y.b[m], r2, dg.b[m]);
          u.a[m] = __ffma2_rn(x.a[m], rm2, __fmul2_rn(u.a[m], r2));
          u.b[m] = __ffma2_rn(x.b[m], rm2, __fmul2_rn(u.b[m], r2));
        }
        if (j0 + q < n) qn_put<T, V, NV, LANES, PAIRED>(po, col, u);
        po += s.oh;
      }
    }
  }
  if (!s.dgain) return;                                  // (the whole block)
#pragma unroll
  for (int m = 0; m < P; ++m) {
    const int ca = col[qn_vec_a<V, PAIRED>(m)], cb = col[qn_vec_b<V, PAIRED>(m)];
    if (ca >= 0) s_sum[group * a.D + ca + qn_at_a<V, PAIRED>(m)] = qn_half(dg.a[m / 2], m & 1);
    if (cb >= 0) s_sum[group * a.D + cb + qn_at_b<V, PAIRED>(m)] = qn_half(dg.b[m / 2], m & 1);
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.D; c += QN_THREADS) {
    float* part = a.part + (long long)blockIdx.x * a.D + c;
    float sum = 0.f;
    for (int q = 0; q < GROUPS; ++q) sum += s_sum[q * a.D + c];
    *part = s.from ? *part + sum : sum;
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
  for (int i = a.first[side] + threadIdx.y; i < a.first[side + 1]; i += 8 * 32) {
    float v[8];                                          // (loads of a round in flight together)
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c < a.D && i + 32 * k < a.first[side + 1] ? __ldcg(a.part + (long long)(i + 32 * k) * a.D + c) : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)v[k];
  }
  s_sum[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.y == 0 && c < a.D) {
    sum = 0.0;
    for (int i = 0; i < 32; ++i) sum += s_sum[i][threadIdx.x];
    out[c] = (float)sum;
  }
}
