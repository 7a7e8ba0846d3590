// Operators of a training step around the layer's projections and its selection: norms of queries and keys with the
// position rotation (sh_qknorm.cuh), the balance loss of the gates (sh_balance.cuh), dropout (sh_dropout.cuh).
// Argument checks and launches; every entry point is documented in include/switchhead.h.
#include <cmath>
#include <initializer_list>
#include <utility>

#include "sh_launch.cuh"
#include "sh_qknorm.cuh"
#include "sh_balance.cuh"
#include "sh_dropout.cuh"

namespace {

size_t elem_bytes(int dtype) { return dtype == SH_F32 ? 4 : 2; }

bool dtype_ok(int dtype, bool f16) {
  if (dtype == SH_F32 || dtype == SH_BF16 || (f16 && dtype == SH_F16)) return true;
  sh_set_error(f16 ? "dtype must be SH_F32, SH_BF16 or SH_F16 (got %d)" : "dtype must be SH_F32 or SH_BF16 (got %d)", dtype);
  return false;
}

// Pointers that a kernel reads or writes as elements of `size` bytes (NULL: not used).
bool aligned_to(size_t size, const char* what, std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if ((uintptr_t)p % size) { sh_set_error("%s must be aligned to %zu bytes", what, size); return false; }
  return true;
}

// SMs of the current device.
int device_sms(int* n) {
  static int sms[64];                                      // (an SM count is written once or several times with the same value)
  int dev = 0;
  SH_CUDA_CHECK(cudaGetDevice(&dev));
  int v = dev < 64 ? __atomic_load_n(&sms[dev], __ATOMIC_RELAXED) : 0;
  if (v == 0) {
    SH_CUDA_CHECK(cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev));
    if (dev < 64) __atomic_store_n(&sms[dev], v, __ATOMIC_RELAXED);
  }
  *n = v;
  return SH_OK;
}

int pow2_at_least(int n) { int p = 1; while (p < n) p *= 2; return p; }

// ---- norms of queries and keys ----

// Two elements of an output at one address: its rows of `width` values are not as far apart in a dimension of more than one.
bool apart(const char* what, long long width, std::initializer_list<std::pair<long long, long long>> dims) {
  for (auto& d : dims)
    if (d.first > 1 && d.second < width && d.second > -width) {
      sh_set_error("%s: elements of an output must not share an address (rows of %lld values, a stride of %lld)", what, width, d.second);
      return false;
    }
  return true;
}

// Values a vector may have: every address and every run of columns is a multiple of it.
int vector_width(const sh_qk_norm_args& a, const sh_qk_norm_backward_args* back) {
  const int size = (int)elem_bytes(a.dtype);
  long long all = a.d_head;                                // (what has to be a multiple: a power of two of it is its lowest bit)
  if (a.rotated && a.halves) all |= a.rotated / 2 | (a.d_head - a.rotated) / 2;
  auto add = [&](const sh_heads& h, int heads) {
    if (heads == 0) return;
    all |= (long long)((uintptr_t)h.data / size);
    if (a.batch > 1) all |= h.batch_stride;
    if (a.seq > 1) all |= h.token_stride;
    if (heads > 1) all |= h.head_stride;
  };
  add(a.q, a.q_heads); add(a.q_out, a.q_heads); add(a.k, a.k_heads); add(a.k_out, a.k_heads);
  for (const float* g : {a.gq, a.gk}) all |= ((uintptr_t)g / 4) & 3;      // (loaded four at a time)
  if (back) { add(back->dq, a.q_heads); add(back->dk, a.k_heads); }
  int v = back && QN_BACKWARD_V < 16 / size ? QN_BACKWARD_V : 16 / size;
  while (all & (v - 1)) v /= 2;
  return v;
}

int qn_check(const sh_qk_norm_args& a, const sh_qk_norm_backward_args* back) {
  if (!dtype_ok(a.dtype, true)) return SH_ERR_INVALID_ARG;
  if (a.batch < 0 || a.seq < 0) { sh_set_error("batch and seq must not be negative (got %d, %d)", a.batch, a.seq); return SH_ERR_INVALID_ARG; }
  if (a.q_heads < 0 || a.k_heads < 0) { sh_set_error("q_heads and k_heads must not be negative (got %d, %d)", a.q_heads, a.k_heads); return SH_ERR_INVALID_ARG; }
  if (a.d_head < 1 || a.d_head > QN_MAX_D) { sh_set_error("d_head must be in 1..%d (got %d)", QN_MAX_D, a.d_head); return SH_ERR_INVALID_ARG; }
  if (a.rotated < 0 || a.rotated > a.d_head || a.rotated % 2) { sh_set_error("rotated must be even and in 0..d_head (got %d, d_head %d)", a.rotated, a.d_head); return SH_ERR_INVALID_ARG; }
  if (a.rotated && a.d_head % 2) { sh_set_error("a rotation needs an even d_head (got %d)", a.d_head); return SH_ERR_UNSUPPORTED; }
  if (a.rotated && !(a.base > 0.0 && std::isfinite(a.base))) { sh_set_error("rotary base must be positive and finite (got %g)", a.base); return SH_ERR_INVALID_ARG; }
  if (!(a.eps > 0.f && std::isfinite(a.eps))) { sh_set_error("eps must be positive and finite (got %g)", (double)a.eps); return SH_ERR_INVALID_ARG; }
  if (!std::isfinite(a.q_scale)) { sh_set_error("q_scale must be finite (got %g)", (double)a.q_scale); return SH_ERR_INVALID_ARG; }
  if (!aligned_to(4, "gains and their gradients", {a.gq, a.gk, back ? back->dgq : nullptr, back ? back->dgk : nullptr})) return SH_ERR_INVALID_ARG;
  if (a.batch == 0 || a.seq == 0) return SH_OK;
  if (!aligned_to(a.positions_64 ? 8 : 4, "positions", {a.positions})) return SH_ERR_INVALID_ARG;
  struct Side { const char *in, *out; const sh_heads &x, &y; const sh_heads* dy; int heads; };
  const Side sides[2] = {{"q", "q_out", a.q, a.q_out, back ? &back->dq : nullptr, a.q_heads}, {"k", "k_out", a.k, a.k_out, back ? &back->dk : nullptr, a.k_heads}};
  for (const Side& s : sides) {
    if (s.heads == 0) continue;
    if (!s.x.data || !s.y.data) { sh_set_error("%s and %s must not be NULL", s.in, s.out); return SH_ERR_INVALID_ARG; }
    if (s.dy && !s.dy->data) { sh_set_error("d%s must not be NULL", s.in); return SH_ERR_INVALID_ARG; }
    if (!aligned_to(elem_bytes(a.dtype), "q, k, their outputs and gradients", {s.x.data, s.y.data, s.dy ? s.dy->data : nullptr})) return SH_ERR_INVALID_ARG;
    if (!apart(s.out, a.d_head, {{a.batch, s.y.batch_stride}, {a.seq, s.y.token_stride}, {s.heads, s.y.head_stride}})) return SH_ERR_INVALID_ARG;
  }
  return SH_OK;
}

// The kernel's arguments.
void qn_fill(const sh_qk_norm_args& p, const sh_qk_norm_backward_args* back, QnArgs& a) {
  const sh_heads none{};
  auto side = [&](QnSide& s, const sh_heads& x, const sh_heads& out, const sh_heads& dy, const float* gain, float* dgain, int heads, float scale) {
    s.x = x.data; s.xb = x.batch_stride; s.xt = x.token_stride; s.xh = x.head_stride;
    s.out = out.data; s.ob = out.batch_stride; s.ot = out.token_stride; s.oh = out.head_stride;
    s.dy = dy.data; s.yb = dy.batch_stride; s.yt = dy.token_stride; s.yh = dy.head_stride;
    s.gain = gain; s.dgain = dgain; s.heads = heads; s.scale = scale;
  };
  side(a.s[0], p.q, p.q_out, back ? back->dq : none, p.gq, back ? back->dgq : nullptr, p.q_heads, p.q_scale);
  side(a.s[1], p.k, p.k_out, back ? back->dk : none, p.gk, back ? back->dgk : nullptr, p.k_heads, 1.f);
  a.pos = p.positions; a.pos64 = p.positions_64 != 0;
  a.next = p.rotated && !p.halves;
  a.seq = qn_divisor((unsigned)p.seq); a.D = p.d_head; a.R = p.rotated;
  a.tokens = (long long)p.batch * p.seq;
  a.eps = p.eps;
  a.blocks0 = 0; a.part = nullptr;
  // (frequencies by one multiplication each, 64 bits of mantissa: the roundings and the ratio's own add up, base >= 1, to less than 4 units of 2^-64
  //  turns at any pair - 62 relative at the last of 128 -, with the cut to 64 bits 2^-30 turns at position 2^31)
  if (p.rotated) {
    const long double two_pi = 6.283185307179586476925286766559005768L, ratio = powl((long double)p.base, -2.0L / p.rotated);
    long double f = 1.0L / two_pi;
    for (int i = 0; i < p.rotated / 2; ++i, f *= ratio) a.freq[i] = (unsigned long long)((f < 1.0L ? f : f - floorl(f)) * 18446744073709551616.0L);
  }
}

constexpr int qn_vectors(int v) { return v >= 4 ? 2 : v == 2 ? 4 : 8; }
// Vectors of two values and d_head 129 to 192: six to a lane, 16 lanes, where 32 with four each leave a third or more of them idle.  (20398 tokens, 10
// heads each of queries and keys, six / four, us: 132 in halves, bf16, 80 / 117, backward 137 / 215; 190 next to one another 78 / 95, 114 / 162; fp32, 132 127 / 132, 190 140 / 136.
// Not fp32 backward, whose rows on their way do not fit 128 registers then - 200 to 480 bytes of spills: 132 273 / 188, 190 230 / 191; 2048 tokens,
// 4 heads each of 132, 11.2 / 10.8.)
constexpr int QN_SIX = 6;
bool qn_six(int v, int d_head, bool f32, bool backward) { return v == 2 && d_head > 128 && d_head <= 192 && !(f32 && backward); }
// Lanes to a row: 4 to 32 (vectors of two values, where a quarter of the rotated width is odd, or less: 16 or 32).
int qn_lanes(int v, int d_head, bool f32, bool backward) {
  if (qn_six(v, d_head, f32, backward)) return 16;
  const int n = pow2_at_least((d_head + v * qn_vectors(v) - 1) / (v * qn_vectors(v))), least = v == 8 ? 4 : v == 4 ? 8 : 16;
  return n > least ? n : least;
}

template <typename T, int V, int LANES, bool PAIRED, int NV = qn_vectors(V)>
int qn_launch(const QnArgs& a, bool backward, bool pdl, int blocks, cudaStream_t st) {
  if constexpr (V <= QN_BACKWARD_V && !(NV == QN_SIX && sizeof(T) == 4))     // (vector_width gives the backward kernel no wider ones)
    if (backward)
      return launch_k(pdl, sh_qk_norm_backward_kernel<T, V, NV, LANES, PAIRED>, dim3((unsigned)blocks), dim3(QN_THREADS), (size_t)(QN_THREADS / LANES) * a.D * 4, st, a);
  return launch_k(pdl, sh_qk_norm_kernel<T, V, NV, LANES, PAIRED>, dim3((unsigned)blocks), dim3(QN_THREADS), 0, st, a);
}

template <typename T, int V, bool PAIRED>
int qn_lanes_of(const QnArgs& a, int lanes, bool backward, bool pdl, int blocks, cudaStream_t st) {
  constexpr int LEAST = V == 8 ? 4 : V == 4 ? 8 : 16;
  if constexpr (V == 2)
    if (qn_six(V, a.D, sizeof(T) == 4, backward)) return qn_launch<T, V, 16, PAIRED, QN_SIX>(a, backward, pdl, blocks, st);
  if (lanes == LEAST) return qn_launch<T, V, LEAST, PAIRED>(a, backward, pdl, blocks, st);
  if constexpr (LEAST < 16)
    if (lanes == 2 * LEAST) return qn_launch<T, V, 2 * LEAST, PAIRED>(a, backward, pdl, blocks, st);
  return qn_launch<T, V, LEAST < 16 ? 4 * LEAST : 32, PAIRED>(a, backward, pdl, blocks, st);
}

template <typename T>
int qn_dispatch(const QnArgs& a, int v, int lanes, bool halves, bool backward, bool pdl, int blocks, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (v == 8) return halves ? qn_lanes_of<T, 8, true>(a, lanes, backward, pdl, blocks, st) : qn_lanes_of<T, 8, false>(a, lanes, backward, pdl, blocks, st);
  if (v >= 4) return halves ? qn_lanes_of<T, 4, true>(a, lanes, backward, pdl, blocks, st) : qn_lanes_of<T, 4, false>(a, lanes, backward, pdl, blocks, st);
  if (v == 2) return halves ? qn_lanes_of<T, 2, true>(a, lanes, backward, pdl, blocks, st) : qn_lanes_of<T, 2, false>(a, lanes, backward, pdl, blocks, st);
  // (nothing rotated: d_head may be odd)
  return a.R ? qn_lanes_of<T, 1, true>(a, lanes, backward, pdl, blocks, st) : qn_lanes_of<T, 1, false>(a, lanes, backward, pdl, blocks, st);
}

int qn_run(const sh_qk_norm_args& p, const sh_qk_norm_backward_args* back, bool pdl, cudaStream_t st, int* launches = nullptr) {
  const bool backward = back != nullptr;
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  const bool halves = p.rotated && p.halves;
  const int v = vector_width(p, back);
  QnArgs a;
  qn_fill(p, back, a);
  const int lanes = qn_lanes(v, p.d_head, p.dtype == SH_F32, backward), groups = QN_THREADS / lanes, most = p.q_heads > p.k_heads ? p.q_heads : p.k_heads;
  // Heads to a group: all of them share a token's angles (16384 tokens, 40 heads of 128: 4 heads 64 us, 8 59, 16 64), but not so many that
  // SMs are left without a block (16 tokens, 8 heads: 4 heads 3.5 us, 1 2.7; 2048 tokens, 4 heads of 76, backward: 2 heads 6.3 us, 1 7.7).
  a.per = most < 8 ? (most < 1 ? 1 : most) : 8;
  auto chunks = [&](int i) { return (a.s[i].heads + a.per - 1) / a.per; };
  while (a.per > 1 && a.tokens * (chunks(0) + chunks(1)) < (long long)sms * groups) a.per = a.per > 2 ? (a.per + 1) / 2 : 1;
  const int c[2] = {chunks(0), chunks(1)};
  const long long items[2] = {a.tokens * c[0], a.tokens * c[1]};
  for (int i = 0; i < 2; ++i) a.s[i].chunks = qn_divisor((unsigned)c[i]);
  a.chunks = qn_divisor((unsigned)(c[0] + c[1]));
  a.large = items[0] + items[1] > (1ll << 31) - (1 << 24);   // (a grid's last round goes past the end)
  long long blocks = (items[0] + items[1] + groups - 1) / groups, step[2] = {0, 0}, many = 1;
  if (backward) {
    long long n[2];
    for (int i = 0; i < 2; ++i) n[i] = (items[i] + groups - 1) / groups;
    const long long fit = (long long)sms * (p.dtype == SH_F32 ? qn_backward_blocks<float, 4, 2>() : v == 1 ? qn_backward_blocks<__half, 1, 8>() : qn_six(v, p.d_head, false, true) ? qn_backward_blocks<__half, 2, QN_SIX>() : qn_backward_blocks<__half, 4, 2>()), cap = fit < QN_MAX_BLOCKS ? fit : QN_MAX_BLOCKS;
    if (n[0] + n[1] > cap) {                               // shares by the sides' rows
      const long long all = n[0] + n[1];
      const long long b0 = n[0] ? (n[0] * cap + all / 2) / all : 0;
      n[0] = n[0] && b0 < 1 ? 1 : n[1] && b0 > cap - 1 ? cap - 1 : b0;
      n[1] = n[1] ? cap - n[0] : 0;
    }
    a.blocks0 = (int)n[0];
    blocks = n[0] + n[1];
    a.part = (float*)back->workspace;
    for (int i = 0; i < 2; ++i) step[i] = n[i] * groups;
    many = back->dgq || back->dgk ? QN_CHAIN / a.per : items[0] + items[1];
  }
  if (blocks > 0x7fffffffll) { sh_set_error("too many rows: batch * seq * heads / %d must be below 2^31", groups); return SH_ERR_UNSUPPORTED; }
  // (backward, with gains: `many` rounds of the grid to a launch, QN_CHAIN rows of a thread)
  bool more = blocks > 0;
  for (long long r = 0; more; r += many) {
    more = false;
    for (int i = 0; i < 2; ++i) {
      a.s[i].from = r * step[i]; a.s[i].to = items[i];
      if (backward && (items[i] - a.s[i].from + step[i] - 1) / (step[i] ? step[i] : 1) > many) { a.s[i].to = a.s[i].from + many * step[i]; more = true; }
    }
    const bool chain = pdl || r > 0;
    int rc = p.dtype == SH_F32 ? qn_dispatch<float>(a, v, lanes, halves, backward, chain, (int)blocks, st)
           : p.dtype == SH_BF16 ? qn_dispatch<__nv_bfloat16>(a, v, lanes, halves, backward, chain, (int)blocks, st)
                                : qn_dispatch<__half>(a, v, lanes, halves, backward, chain, (int)blocks, st);
    if (rc) return rc;
    if (launches) ++*launches;
  }
  if (backward && (back->dgq || back->dgk)) {
    if (launches) ++*launches;
    QnGain g{a.part, {back->dgq, back->dgk}, {0, a.blocks0, (int)blocks}, p.d_head};
    return launch_k(blocks > 0, sh_qk_norm_gain_kernel, dim3((unsigned)((p.d_head + 31) / 32), 2), dim3(32, 32), 0, st, g);
  }
  return SH_OK;
}


// ---- balance loss ----

struct BlPlan { int w, l, per, ny, tpb, nx; bool vec; };

constexpr size_t kBlHead = 256;
size_t bl_losses(long long gates) { return ((size_t)gates * 8 + 255) / 256 * 256; }

// Logits of a lane: 32 bytes of them, fewer where there are no more.
int bl_width(int dtype, int E) { return E <= 4 ? 4 : E <= 8 || dtype == SH_F32 ? 8 : 16; }

// Few rows: one launch (sh_balance_small_kernel), which needs no workspace.  Up to 2^18 logits: 2048 tokens, 8 gates of 4 experts
// 7.5 us on the device against 9.2, 14.2 against 17.6 with the host's part; 8192 tokens (2^18) 12.0 and 9.9, 14.3 and 17.6, of 16 experts (1024
// tokens) 9.5 and 9.9; 2^19: 18 and 11, 19 and 18.  (By the time of a call; the layer's passes, whose launches are chained, take the same rule, and from
// 2^18 logits of few experts on they would do with the other kernel.)
bool bl_small(long long tokens, long long gates, int E) {
  return gates <= BL_SMALL_GATES && gates * E <= BL_SMALL_COLS && tokens * gates * (E < 4 ? 4 : E) <= 1 << 18;
}

// The thread layout for E logits of a gate; `vec`: rows are whole, aligned vectors; `small`: the kernel of one launch.
BlPlan bl_plan(int dtype, long long tokens, int gates, int E, bool aligned, bool small, int sms) {
  BlPlan p;
  p.w = bl_width(dtype, E);
  p.l = pow2_at_least((E + p.w - 1) / p.w);
  p.vec = aligned && E == p.w * p.l;
  const int rows = (small ? BL_SMALL_THREADS : BL_THREADS) / p.l;
  p.ny = (gates + rows - 1) / rows;
  p.per = (gates + p.ny - 1) / p.ny;
  p.tpb = rows / p.per;
  const long long rounds = (tokens + p.tpb - 1) / p.tpb;
  long long cap = (long long)BL_BLOCKS * sms < BL_MAX_BLOCKS ? (long long)BL_BLOCKS * sms : BL_MAX_BLOCKS;
  cap = cap / p.ny < 1 ? 1 : cap / p.ny;
  const long long turns = (rounds + 1) / 2;                // (two rows of a thread at least are on their way together)
  p.nx = (int)(turns < 1 ? 1 : turns < cap ? turns : cap);
  return p;
}

bool bl_aligned(const void* z, long long stride, int gates, int E, int w, int size, long long tokens) {
  const size_t bytes = (size_t)w * size < 16 ? (size_t)w * size : 16;
  return (uintptr_t)z % bytes == 0 && (tokens < 2 || (size_t)stride * size % bytes == 0) && (gates < 2 || (size_t)E * size % bytes == 0);
}

int bl_check(const sh_balance_args& a, bool backward) {
  if (!dtype_ok(a.dtype, false)) return SH_ERR_INVALID_ARG;
  if (a.n_tokens < 0) { sh_set_error("n_tokens must not be negative (got %lld)", (long long)a.n_tokens); return SH_ERR_INVALID_ARG; }
  if (a.sides < 1 || a.n_heads < 1 || a.n_experts < 1 || a.n_experts > 32) {
    sh_set_error("sides and n_heads must be >= 1, n_experts in 1..32 (got %d, %d, %d)", a.sides, a.n_heads, a.n_experts);
    return SH_ERR_INVALID_ARG;
  }
  const long long gates = (long long)a.sides * a.n_heads;
  if (gates > 65535) { sh_set_error("sides * n_heads must be at most 65535 (got %lld)", gates); return SH_ERR_UNSUPPORTED; }
  if (a.n_tokens && !a.logits) { sh_set_error("logits must not be NULL"); return SH_ERR_INVALID_ARG; }
  if (!aligned_to(elem_bytes(a.dtype), "logits and dlogits", {a.logits, backward ? a.dlogits : nullptr})) return SH_ERR_INVALID_ARG;
  if (!aligned_to(4, "idx, loss, prob, slope, counts and gloss", {a.idx, a.loss, a.prob, a.slope, a.counts, a.gloss})) return SH_ERR_INVALID_ARG;
  if (backward) {
    if (!a.slope || (a.n_tokens && !a.dlogits)) { sh_set_error("slope and dlogits must not be NULL"); return SH_ERR_INVALID_ARG; }
    return apart("dlogits", gates * a.n_experts, {{a.n_tokens, a.dtoken_stride}}) ? SH_OK : SH_ERR_INVALID_ARG;
  }
  if (a.k < 1 || a.k > a.n_experts) { sh_set_error("k must be in 1..n_experts (got k=%d, n_experts=%d)", a.k, a.n_experts); return SH_ERR_INVALID_ARG; }
  if (a.n_tokens >= (1ll << 31) / a.k) { sh_set_error("n_tokens * k must be below 2^31 (got %lld, %d)", (long long)a.n_tokens, a.k); return SH_ERR_UNSUPPORTED; }
  if (a.kind != SH_BALANCE_COUNTS && a.kind != SH_BALANCE_ENTROPY) { sh_set_error("unknown kind of balance loss: %d", a.kind); return SH_ERR_INVALID_ARG; }
  if (!std::isfinite(a.coef)) { sh_set_error("coef must be finite (got %g)", (double)a.coef); return SH_ERR_INVALID_ARG; }
  if ((a.n_tokens && !a.idx) || !a.loss || !a.counts || !a.prob || !a.slope) { sh_set_error("idx, loss, counts, prob and slope must not be NULL"); return SH_ERR_INVALID_ARG; }
  const size_t need = sh_balance_workspace_bytes(a.n_tokens, a.sides, a.n_heads, a.n_experts);
  if (need == 0) return SH_OK;
  if (!a.workspace || (uintptr_t)a.workspace % 256) { sh_set_error("workspace must be a device pointer aligned to 256 bytes"); return SH_ERR_WORKSPACE; }
  if (a.workspace_bytes < need) { sh_set_error("workspace too small: %zu bytes given, %zu needed", a.workspace_bytes, need); return SH_ERR_WORKSPACE; }
  return SH_OK;
}

void bl_fill(const sh_balance_args& p, const BlPlan& pl, BlArgs& a) {
  a.z = p.logits; a.dz = p.dlogits; a.idx = p.idx; a.mask = (const unsigned char*)p.mask;
  a.slope = p.slope; a.gloss = p.gloss;
  a.tokens = p.n_tokens; a.zt = p.token_stride; a.dzt = p.dtoken_stride;
  a.gates = p.sides * p.n_heads; a.H = p.n_heads; a.E = p.n_experts; a.k = p.k;
  a.per = pl.per; a.tpb = pl.tpb;
  a.part_p = nullptr; a.part_n = nullptr; a.ticket = nullptr;
}

template <typename T, int W, int L, bool VEC>
int bl_launch(const BlArgs& a, const BlPlan& p, int what, const BlOut* o, const BlPart& part, bool pdl, cudaStream_t st) {
  const dim3 grid((unsigned)p.nx, (unsigned)p.ny);
  if (what == 0 && o) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(BL_CLUSTER); cfg.blockDim = dim3(BL_SMALL_THREADS); cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = BL_CLUSTER; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 2 : 1;
    SH_CUDA_CHECK(cudaLaunchKernelEx(&cfg, sh_balance_small_kernel<T, W, L, VEC>, a, *o));
    return SH_OK;
  }
  if (what == 0) return launch_k(pdl, sh_balance_sums_kernel<T, W, L, VEC>, grid, dim3(BL_THREADS), 0, st, a, part);
  if constexpr (sizeof(T) == 4)
    if (what == 2) return launch_k(pdl, sh_balance_backward_kernel<T, W, L, VEC, true>, grid, dim3(BL_THREADS), 0, st, a);
  return launch_k(pdl, sh_balance_backward_kernel<T, W, L, VEC, false>, grid, dim3(BL_THREADS), 0, st, a);
}

// what: 0 the sums (with `o`: and the loss), 1 dz, 2 dz added (fp32)
int bl_dispatch(int dtype, const BlArgs& a, const BlPlan& p, int what, const BlOut* o, const BlPart& part, bool pdl, cudaStream_t st) {
#define SH_BL(T, W, L) return p.vec ? bl_launch<T, W, L, true>(a, p, what, o, part, pdl, st) : bl_launch<T, W, L, false>(a, p, what, o, part, pdl, st)
  if (dtype == SH_F32) {
    if (p.w == 4) SH_BL(float, 4, 1);
    if (p.l == 1) SH_BL(float, 8, 1);
    if (p.l == 2) SH_BL(float, 8, 2);
    SH_BL(float, 8, 4);
  }
  if (p.w == 4) SH_BL(__nv_bfloat16, 4, 1);
  if (p.w == 8) SH_BL(__nv_bfloat16, 8, 1);
  if (p.l == 1) SH_BL(__nv_bfloat16, 16, 1);
  SH_BL(__nv_bfloat16, 16, 2);
#undef SH_BL
}

BlPlan bl_plan_for(const sh_balance_args& p, bool backward, bool small, int sms) {
  const int gates = p.sides * p.n_heads, size = (int)elem_bytes(p.dtype), w = bl_width(p.dtype, p.n_experts);
  bool aligned = bl_aligned(p.logits, p.token_stride, gates, p.n_experts, w, size, p.n_tokens);
  if (backward) aligned = aligned && bl_aligned(p.dlogits, p.dtoken_stride, gates, p.n_experts, w, size, p.n_tokens);
  return bl_plan(p.dtype, p.n_tokens, gates, p.n_experts, aligned, small, sms);
}

}  // namespace

int sh_run_qk_norm(const sh_qk_norm_args& p, bool pdl, cudaStream_t st) {
  if (int rc = qn_check(p, nullptr)) return rc;
  if (p.batch == 0 || p.seq == 0) return SH_OK;
  return qn_run(p, nullptr, pdl, st);
}

int sh_run_qk_norm_backward(const sh_qk_norm_backward_args& p, bool pdl, cudaStream_t st, int* launches) {
  if (int rc = qn_check(p.norm, &p)) return rc;
  if (p.dgq || p.dgk) {
    const size_t need = sh_qk_norm_workspace_bytes(p.norm.d_head);
    if (!p.workspace || (uintptr_t)p.workspace % 256) { sh_set_error("workspace must be a device pointer aligned to 256 bytes"); return SH_ERR_WORKSPACE; }
    if (p.workspace_bytes < need) { sh_set_error("workspace too small: %zu bytes given, %zu needed", p.workspace_bytes, need); return SH_ERR_WORKSPACE; }
  }
  return qn_run(p.norm, &p, pdl, st, launches);
}

int sh_run_balance_loss(const sh_balance_args& p, bool pdl, cudaStream_t st, int* launches) {
  if (int rc = bl_check(p, false)) return rc;
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  const bool small = bl_small(p.n_tokens, (long long)p.sides * p.n_heads, p.n_experts);
  const BlPlan pl = bl_plan_for(p, false, small, sms);
  BlArgs a;
  bl_fill(p, pl, a);
  BlOut o{};
  o.gates = a.gates; o.E = a.E; o.kind = p.kind; o.coef = p.coef;
  o.loss = p.loss; o.prob = p.prob; o.slope = p.slope; o.counts = p.counts;
  if (launches) ++*launches;                               // (the last one)
  if (small) return bl_dispatch(p.dtype, a, pl, 0, &o, BlPart{}, pdl, st);
  char* ws = (char*)p.workspace;
  a.ticket = (unsigned*)ws;
  a.part_p = (float*)(ws + kBlHead + bl_losses(a.gates));
  a.part_n = (int*)(a.part_p + (size_t)pl.nx * a.gates * a.E);
  const long long most = (long long)BL_CHAIN * pl.nx * pl.tpb;                // tokens of a launch
  for (long long t = 0; t == 0 || t < p.n_tokens; t += most) {
    a.z = (const char*)p.logits + t * p.token_stride * (long long)elem_bytes(p.dtype);
    a.idx = p.idx + t * p.n_heads * p.k;
    a.mask = p.mask ? (const unsigned char*)p.mask + t : nullptr;
    a.tokens = p.n_tokens - t < most ? p.n_tokens - t : most;
    if (int rc = bl_dispatch(p.dtype, a, pl, 0, nullptr, BlPart{p.n_tokens, t > 0}, pdl || t > 0, st)) return rc;
    if (launches) ++*launches;
  }
  o.part_p = a.part_p; o.part_n = a.part_n; o.ticket = a.ticket; o.gate_loss = (double*)(ws + kBlHead);
  o.blocks = pl.nx;
  return launch_k(true, sh_balance_loss_kernel, dim3((unsigned)a.gates), dim3(BL_LOSS_THREADS), 0, st, o);
}

int sh_run_balance_backward(const sh_balance_args& p, bool add, bool pdl, cudaStream_t st) {
  if (int rc = bl_check(p, true)) return rc;
  if (p.n_tokens == 0) return SH_OK;
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  const BlPlan pl = bl_plan_for(p, true, false, sms);
  BlArgs a;
  bl_fill(p, pl, a);
  return bl_dispatch(p.dtype, a, pl, add ? 2 : 1, nullptr, BlPart{}, pdl, st);
}

int sh_run_dropout(const sh_dropout_args& p, bool pdl, cudaStream_t st) {
  if (!dtype_ok(p.dtype, true)) return SH_ERR_INVALID_ARG;
  if (p.rows < 0 || p.cols < 0) { sh_set_error("rows and cols must not be negative (got %lld, %lld)", (long long)p.rows, (long long)p.cols); return SH_ERR_INVALID_ARG; }
  if (p.rows > (1ll << 32) || p.cols > (1ll << 31) - 8) {
    sh_set_error("at most 2^32 rows and 2^31-8 cols (got %lld, %lld)", (long long)p.rows, (long long)p.cols);
    return SH_ERR_UNSUPPORTED;
  }
  if (!(p.p >= 0.0 && p.p <= 1.0)) { sh_set_error("p must be in 0..1 (got %g)", p.p); return SH_ERR_INVALID_ARG; }
  if (p.rows == 0 || p.cols == 0) return SH_OK;
  if (!apart("y", p.cols, {{p.rows, p.y_stride}})) return SH_ERR_INVALID_ARG;
  if (!p.x || !p.y || !p.rng) { sh_set_error("x, y and rng must not be NULL"); return SH_ERR_INVALID_ARG; }
  if (!aligned_to(8, "rng", {p.rng}) || !aligned_to(elem_bytes(p.dtype), "x, residual and y", {p.x, p.residual, p.y})) return SH_ERR_INVALID_ARG;
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  const size_t size = elem_bytes(p.dtype);
  auto aligned = [&](const void* q, long long stride) { return (uintptr_t)q % 16 == 0 && (p.rows == 1 || (size_t)stride * size % 16 == 0); };
  const bool vec = aligned(p.x, p.x_stride) && aligned(p.y, p.y_stride) && (!p.residual || aligned(p.residual, p.residual_stride));
  const bool whole = p.rows == 1 || (p.x_stride == p.cols && p.y_stride == p.cols && (!p.residual || p.residual_stride == p.cols));   // one run of values
  const bool dense = vec && whole && p.cols % 8 == 0;
  const bool base = (((uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)p.residual) & 15) == 0;
  const bool flat = !vec && whole && base && p.cols >= 16 && p.rows < (1ll << 34) / p.cols;
  DoArgs a;
  a.rng = (const unsigned long long*)p.rng;
  a.xs = p.x_stride; a.rs = p.residual_stride; a.ys = p.y_stride;
  a.cols = (int)p.cols;
  a.upr = (unsigned)((p.cols + 7) / 8);
  a.group_log = 2;
  while (a.group_log < 5 && (1u << a.group_log) < a.upr) ++a.group_log;
  a.segs = (unsigned)((a.upr + (1u << a.group_log) - 1) >> a.group_log);
  const int limit = (int)lrint(p.p * 65536.0);
  a.none = limit > 65535; a.limit = a.none ? 0u : (unsigned)limit << 16;
  a.scale = a.none ? 0.f : (float)(65536.0 / (65536 - limit));
  const long long most = flat ? p.rows : (1ll << 31) / a.upr < 1 ? 1 : (1ll << 31) / a.upr;           // rows of a launch
  for (long long r = 0; r < p.rows; r += most) {
    const long long n = p.rows - r < most ? p.rows - r : most;
    a.x = (const char*)p.x + r * p.x_stride * (long long)size; a.y = (char*)p.y + r * p.y_stride * (long long)size;
    a.residual = p.residual ? (const char*)p.residual + r * p.residual_stride * (long long)size : nullptr;
    a.row0 = (unsigned)r; a.units = (unsigned)(n * a.upr);
    a.groups = (unsigned)(n * a.segs);
    a.values = n * p.cols;
    if (flat) a.units = (unsigned)((a.values + 15) / 16);
    const long long threads = vec || flat ? a.units : (long long)a.groups << a.group_log;
    const long long blocks = (threads + DO_THREADS - 1) / DO_THREADS, cap = 8ll * sms;
    const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
    auto go = [&](auto kern) { return launch_k(pdl, kern, grid, dim3(DO_THREADS), 0, st, a); };
    auto typed = [&](auto zero) {
      using T = decltype(zero);
      if (p.residual) return dense ? go(sh_dropout_kernel<T, DO_DENSE, true>) : vec ? go(sh_dropout_kernel<T, DO_VECTORS, true>)
                           : flat ? go(sh_dropout_flat_kernel<T, true>) : go(sh_dropout_rows_kernel<T, true>);
      return dense ? go(sh_dropout_kernel<T, DO_DENSE, false>) : vec ? go(sh_dropout_kernel<T, DO_VECTORS, false>)
           : flat ? go(sh_dropout_flat_kernel<T, false>) : go(sh_dropout_rows_kernel<T, false>);
    };
    const int rc = p.dtype == SH_F32 ? typed(0.f) : p.dtype == SH_BF16 ? typed(__nv_bfloat16()) : typed(__half());
    if (rc) return rc;
  }
  return SH_OK;
}

extern "C" size_t sh_qk_norm_workspace_bytes(int d_head) {
  return d_head < 1 || d_head > QN_MAX_D ? 0 : (size_t)QN_MAX_BLOCKS * d_head * 4;
}

extern "C" size_t sh_balance_workspace_bytes(int64_t n_tokens, int sides, int n_heads, int n_experts) {
  const long long gates = (long long)sides * n_heads;
  if (sides < 1 || n_heads < 1 || gates > 65535 || n_experts < 1 || n_experts > 32 || bl_small(n_tokens, gates, n_experts)) return 0;
  return kBlHead + bl_losses(gates) + (size_t)BL_MAX_BLOCKS * (gates * n_experts * 8 + 4);
}

// An entry point: the reason of the last failure cleared, the struct of arguments given.
template <typename A, typename F>
static int entry(const A* args, F run) {
  sh_set_error("%s", "");
  if (!args) { sh_set_error("args is NULL"); return SH_ERR_INVALID_ARG; }
  return run(*args);
}

extern "C" int sh_qk_norm(const sh_qk_norm_args* args, void* stream) {
  return entry(args, [&](const sh_qk_norm_args& a) { return sh_run_qk_norm(a, false, (cudaStream_t)stream); });
}
extern "C" int sh_qk_norm_backward(const sh_qk_norm_backward_args* args, void* stream) {
  return entry(args, [&](const sh_qk_norm_backward_args& a) { return sh_run_qk_norm_backward(a, false, (cudaStream_t)stream); });
}
extern "C" int sh_balance_loss(const sh_balance_args* args, void* stream) {
  return entry(args, [&](const sh_balance_args& a) { return sh_run_balance_loss(a, false, (cudaStream_t)stream); });
}
extern "C" int sh_balance_backward(const sh_balance_args* args, void* stream) {
  return entry(args, [&](const sh_balance_args& a) { return sh_run_balance_backward(a, false, false, (cudaStream_t)stream); });
}
extern "C" int sh_dropout(const sh_dropout_args* args, void* stream) {
  return entry(args, [&](const sh_dropout_args& a) { return sh_run_dropout(a, false, (cudaStream_t)stream); });
}
