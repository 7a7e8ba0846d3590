"""The operators of a training step (sh_qk_norm, sh_balance_loss, sh_dropout and their gradients) on the GPU against the fp64
oracle: types, head layouts, odd sizes, strides, padded batches, extreme values, in-place calls, captured calls.

Tolerances.  A stored result is the fp32 result rounded once: off by half a step of its type, eps / 2 of its magnitude.
The fp32 result is off by a number of fp32 roundings (U = 2^-24) of the magnitudes it is put together from, which each
check counts."""
import numpy as np
import pytest
import torch

from oracle import training_operators as op
from paper_2312_07987_b200 import binding as b

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2      # half a step below the normal numbers


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, bound, t):
    """|got - want| within half a step of the type plus bound (an array)."""
    got, want = host(got), np.asarray(want)
    off = np.abs(got - want) - (half(t) * (np.abs(want) + bound) + bound + tiny(t))
    assert not np.isnan(off).any() and (off <= 0).all(), float(off.max())


def draw(shape, t, seed, layout="bthd", extra=0):
    """Values [B, T, H, D] in a layout: dense, the layer's [B, H, T, D], the first columns of a fused projection of `extra` more heads, or
    `odd`: rows an odd number of values (D is even) apart, so that no vector of two is aligned."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, T, H, D = shape
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)
    if layout == "bhtd":
        return r(B, H, T, D).transpose(1, 2)
    if layout == "fused":
        return r(B, T, H + extra, D)[:, :, :H]
    if layout == "odd":
        return r(B, T, H, D + 1)[..., 1:]
    return r(B, T, H, D)


def norm_bounds(x, gain, eps, scale):
    """Per row: the largest normalised value times sqrt(2) (the length of a pair, which a rotation mixes)."""
    n = op.qk_norm(x, gain, None, eps, scale=scale)
    return np.sqrt(2) * np.abs(n).max(-1, keepdims=True)


# the sum of squares: at most 16 additions in a lane, 5 across lanes, so 21 U, of which the root keeps half; rsqrtf 4 U; gain, scale, r: 4 U
NORM_U = 20
# sine and cosine: the angle is off by 2^-26 turns (its upper 32 bits as a float: half a step of 2^-24 of a half turn) = 2 pi 2^-26 = 1.6 U; fp32:
# sincospif by 2 U; 16-bit types: sin.approx and cos.approx by 2^-20.9 (the instruction's documented bound) = 8.6 U and their argument, the
# rounded product of pi, by 1.6 U more; two products and a sum: 3 U
TURN_U = 15

CASES = [  # B, T, Hq, Hk, D, rotated, halves, layout, dtype, q_scale
    (2, 5, 4, 4, 128, 128, False, "fused", "bf16", 1.0),
    (2, 3, 8, 2, 128, 64, True, "fused", "bf16", 0.5),
    (1, 9, 4, 4, 100, 100, False, "bhtd", "f16", 0.1),
    (3, 7, 2, 2, 76, 76, False, "bhtd", "f32", 1.0),
    (3, 7, 2, 3, 76, 76, True, "bthd", "f32", 1.0),
    (1, 1, 1, 1, 64, 64, True, "bthd", "bf16", 1.0),
    (2, 33, 3, 1, 132, 100, False, "bthd", "bf16", 1.0),
    (2, 6, 2, 2, 168, 168, True, "bhtd", "f16", 1.0),
    (1, 17, 2, 2, 256, 256, True, "bthd", "f32", 1.0),
    (1, 4, 5, 2, 255, 0, False, "bthd", "bf16", 1.0),
    (1, 4, 2, 2, 33, 0, False, "bthd", "f32", 1.0),
    (1, 5, 2, 1, 1, 0, False, "bthd", "f32", 1.0),
    (1, 5, 2, 1, 2, 2, False, "bthd", "f16", 1.0),
    (1, 5, 2, 1, 2, 2, True, "bthd", "f32", 1.0),
    (2, 5, 2, 2, 64, 64, False, "odd", "bf16", 1.0),
    (2, 5, 2, 2, 64, 34, True, "odd", "f16", 1.0),
    (2, 5, 2, 2, 250, 250, False, "odd", "f32", 1.0),
    (2, 5, 3, 2, 22, 6, True, "bthd", "bf16", 1.0),
    (1, 3, 17, 9, 32, 32, False, "bthd", "f32", 1.0),
    (5, 97, 4, 4, 32, 32, False, "bthd", "bf16", 1.0),
]


def positions_for(kind, B, T):
    if kind == "none":
        return None, np.broadcast_to(np.arange(T), (B, T))
    g = np.random.default_rng(B * 100 + T)
    p = {"packed": np.arange(T) - np.minimum(np.arange(T), T // 2), "far": np.arange(T) + g.integers(0, 1 << 31, (B, 1)) - T,
         "negative": np.arange(T) - 1000}[kind] + np.zeros((B, T), dtype=np.int64)
    return torch.from_numpy(p.astype(np.int32 if kind != "far" else np.int64)).cuda(), p


@pytest.mark.parametrize("case,pos", [(c, pos) for c in CASES for pos in (("none", "packed", "far", "negative") if c[5] else ("none",))])
def test_norm_and_its_gradients(case, pos):
    B, T, Hq, Hk, D, R, halves, layout, ty, qs = case
    t = TYPES[ty]
    q, k = draw((B, T, Hq, D), t, 1, layout, Hk), draw((B, T, Hk, D), t, 2, layout, Hq)
    dq, dk = draw((B, T, Hq, D), t, 3), draw((B, T, Hk, D), t, 4, "bhtd")
    g = torch.Generator(device="cuda").manual_seed(5)
    gq, gk = (1 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    dev_pos, p = positions_for(pos, B, T)
    eps = 1e-3
    kw = dict(eps=eps, base=500.0, rotated=R, halves=halves)
    yq, yk = b.sh_qk_norm(q, k, gq, gk, positions=dev_pos, q_scale=qs, **kw)
    back = b.sh_qk_norm_backward(q, k, dq, dk, gq, gk, positions=dev_pos, q_scale=qs, **kw)
    # (the oracle's own angle: a product rounded to 2^-53 and a frequency as far off, at every position)
    far = np.abs(p).max() * 2.0 ** -51
    for x, gain, y, scale, dy, dx, dg in ((q, gq, yq, qs, dq, back["dq"], back["dgq"]), (k, gk, yk, 1.0, dk, back["dk"], back["dgk"])):
        assert y.shape == x.shape and y.dtype == t and dx.shape == x.shape
        x, gain, dy = host(x), host(gain), host(dy)
        mag = norm_bounds(x, gain, eps, scale)
        close(y, op.qk_norm(x, gain, p, scale=scale, **kw), mag * ((NORM_U + TURN_U) * U + far), t)
        want, wg = op.qk_norm_backward(x, dy, gain, p, scale=scale, **kw)
        size = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        n, u = x / size, np.sqrt(2) * np.abs(scale * dy).max(-1, keepdims=True)
        w = u * np.abs(gain).max()
        # dx = r (w - n mean(w n)): the turned gradient, the mean (21 additions and products), r twice more than in the forward pass
        close(dx, want, (w + np.abs(n) * w * np.abs(n).mean(-1, keepdims=True)) / size * ((TURN_U + 2 * NORM_U + 21) * U + far), t)
        # a gain's gradient: a row's share as above; additions in fp32 over a thread's rows (at most 64 here) and 256 groups of lanes at most
        share = (u * np.abs(n)).reshape(-1, D).sum(0)
        close(dg, wg, share * ((TURN_U + NORM_U + 4 + 64 + 256) * U + far), torch.float32)


@pytest.mark.parametrize("halves", [False, True])
def test_norm_gradients_against_differences(halves):
    # along random directions of x and of the gain: differences of the fp64 definition, 1e-5 to either side (their own error: 1e-10 times third
    # derivatives of size 10, and 1e-16 / 1e-5 of sums of 1e3), against the kernels' gradients
    B, T, H, D = 2, 7, 3, 32
    q, dq = draw((B, T, H, D), torch.float32, 1), draw((B, T, H, D), torch.float32, 2)
    gain = 1 + 0.3 * torch.randn(D, device="cuda")
    kw = dict(eps=1e-2, base=100.0, rotated=24, halves=halves)
    back = b.sh_qk_norm_backward(q, None, dq, None, gain, None, q_scale=0.7, **kw)
    p = np.broadcast_to(np.arange(T), (B, T))
    f = lambda x, g: (op.qk_norm(x, g, p, scale=0.7, **kw) * host(dq)).sum()
    rg = np.random.default_rng(3)
    for _ in range(3):
        vx, vg = rg.standard_normal((B, T, H, D)), rg.standard_normal(D)
        x, g, h = host(q), host(gain), 1e-5
        size = np.abs(host(dq)).max() * 2.0 / np.sqrt((x * x).mean(-1)).min()
        slope = (f(x + h * vx, g) - f(x - h * vx, g)) / (2 * h)
        assert abs((host(back["dq"]) * vx).sum() - slope) < 80 * U * size * np.abs(vx).sum() + 1e-6
        slope = (f(x, g + h * vg) - f(x, g - h * vg)) / (2 * h)
        assert abs((host(back["dgq"]) * vg).sum() - slope) < 400 * U * np.abs(host(dq)).max() * 4 * B * T * H * np.abs(vg).max() + 1e-6


@pytest.mark.parametrize("kind", ["counts", "entropy"])
def test_balance_gradient_against_differences(kind):
    z, idx, mask = balance_inputs(40, 2, 2, 6, 2, torch.float32, True)
    got = b.sh_balance_loss(z, idx, kind=kind, coef=1.0, mask=mask)
    dz = host(b.sh_balance_backward(z, got["slope"], mask=mask))
    f = lambda v: op.balance(v, idx.cpu().numpy(), kind, 1.0, mask.cpu().numpy())[0]
    rg = np.random.default_rng(4)
    for _ in range(3):
        v, h = rg.standard_normal(z.shape), 1e-5
        slope = (f(host(z) + h * v) - f(host(z) - h * v)) / (2 * h)
        # (each value: 60 U of p c / n with p <= 1 and c <= 6; the differences: 1e-10 and 1e-16 / 1e-5 of a loss of 24)
        assert abs((dz * v).sum() - slope) < 60 * U * 6 / int(mask.sum()) * np.abs(v).sum() + 1e-8


def test_norm_without_gains_or_keys():
    q, dq = draw((2, 6, 3, 40), torch.float32, 1), draw((2, 6, 3, 40), torch.float32, 2)
    y, none = b.sh_qk_norm(q, None, rotated=40)
    assert none is None
    p = np.broadcast_to(np.arange(6), (2, 6))
    close(y, op.qk_norm(host(q), None, p, 1e-6, rotated=40), norm_bounds(host(q), None, 1e-6, 1.0) * (NORM_U + TURN_U) * U, torch.float32)
    back = b.sh_qk_norm_backward(q, None, dq, None, rotated=40)
    assert back["dk"] is None and back["dgq"] is None
    want, _ = op.qk_norm_backward(host(q), host(dq), None, p, 1e-6, rotated=40)
    assert np.abs(host(back["dq"]) - want).max() < 200 * U * np.abs(host(dq)).max() / np.sqrt((host(q) ** 2).mean(-1)).min()
    only = b.sh_qk_norm_backward(q, q, dq, dq, None, torch.ones(40, device="cuda"), rotated=40)        # one side's gain alone
    assert only["dgq"] is None and torch.isfinite(only["dgk"]).all()


def test_norm_of_nothing():
    for shape in ((0, 4, 2, 32), (3, 0, 2, 32), (2, 4, 0, 32)):
        q = torch.zeros(shape, device="cuda")
        k = torch.zeros(shape[:2] + (2, 32), device="cuda") if shape[2] == 0 else q.clone()
        y, _ = b.sh_qk_norm(q, k, rotated=32)
        assert y.shape == shape
        back = b.sh_qk_norm_backward(q, k, q, k, torch.ones(32, device="cuda"), torch.ones(32, device="cuda"), rotated=32)
        assert not back["dgq"].any() and not back["dgk"].any()          # a sum over no rows (or over zeros) is zero


@pytest.mark.parametrize("layout", ["bthd", "bhtd", "fused"])
@pytest.mark.parametrize("halves", [False, True])
def test_norm_in_place_gives_the_same_bits(layout, halves):
    q, k = draw((3, 50, 4, 100), torch.bfloat16, 1, layout, 4), draw((3, 50, 2, 100), torch.bfloat16, 2, layout, 6)
    kw = dict(rotated=48, halves=halves, q_scale=0.3)
    want = b.sh_qk_norm(q, k, **kw)
    got = b.sh_qk_norm(q, k, q_out=q, k_out=k, **kw)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_norm_leaves_what_is_not_its_own():
    whole = torch.full((2, 9, 7, 64), 7.0, device="cuda")
    q, k = torch.randn(2, 5, 3, 32, device="cuda"), torch.randn(2, 5, 2, 32, device="cuda")
    b.sh_qk_norm(q, k, rotated=32, q_out=whole[:, 1:6, 1:4, 16:48], k_out=whole[:, 1:6, 4:6, 16:48])
    own = torch.zeros_like(whole, dtype=torch.bool)
    own[:, 1:6, 1:6, 16:48] = True
    assert (whole[~own] == 7.0).all() and (whole[own] != 7.0).all()


def test_norm_rows_stand_alone():
    q = torch.randn(2, 6, 2, 64, device="cuda")
    q[0, 1] = 0.0
    q[0, 2, 1, 5] = float("nan")
    q[1, 3, 0, 7] = float("inf")
    y, _ = b.sh_qk_norm(q, None, rotated=64)
    bad = torch.zeros(2, 6, 2, dtype=torch.bool, device="cuda")
    bad[0, 2, 1] = bad[1, 3, 0] = True
    assert torch.isfinite(y[~bad]).all() and not y[0, 1].any()
    assert torch.isnan(y[0, 2, 1]).all() and torch.isnan(y[1, 3, 0]).any()
    clean = torch.where(bad[..., None], torch.ones((), device="cuda"), q)
    assert torch.equal(b.sh_qk_norm(clean, None, rotated=64)[0][~bad], y[~bad])
    back = b.sh_qk_norm_backward(q, None, torch.ones_like(q), None, rotated=64)
    assert torch.isfinite(back["dq"][~bad]).all()


def test_norm_offsets_past_32_bits():
    # two sequences 2^32 elements apart, their rows at the two ends of one allocation
    n = (1 << 32) + 4096
    store = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    q = store.as_strided((2, 2, 2, 64), (1 << 32, 128, 64, 1))
    src = torch.randn(2, 2, 2, 64, device="cuda").bfloat16()
    q.copy_(src)
    want, _ = b.sh_qk_norm(src, None, rotated=64)
    b.sh_qk_norm(q, None, rotated=64, q_out=q)
    assert torch.equal(q, want)
    del store, q
    torch.cuda.empty_cache()


def test_norm_of_more_rows_than_31_bits():
    # inputs of one row that every token shares (strides of zero), outputs of their own
    B, T = (1 << 11) + 8, 1 << 20
    row, drow = torch.randn(1, 1, 1, 2, device="cuda").bfloat16(), torch.randn(1, 1, 1, 2, device="cuda").bfloat16()
    q = row.expand(B, T, 1, 2)
    y = torch.empty(B, T, 1, 2, dtype=torch.bfloat16, device="cuda")
    b.sh_qk_norm(q, None, rotated=2, q_out=y)
    few = torch.tensor([0, 1, 777, T - 2, T - 1], device="cuda")
    want, _ = b.sh_qk_norm(row.expand(1, 5, 1, 2), None, rotated=2, positions=few.view(1, 5).int())
    for n in (0, 1, 1023, 2047, 2048, B - 1):
        assert torch.equal(y[n, few], want[0]), n
    del y
    back = b.sh_qk_norm_backward(q, None, drow.expand(B, T, 1, 2), None, rotated=2)["dq"]
    want = b.sh_qk_norm_backward(row.expand(1, 5, 1, 2), None, drow.expand(1, 5, 1, 2), None, rotated=2, positions=few.view(1, 5).int())["dq"]
    for n in (0, 1, 1023, 2047, 2048, B - 1):
        assert torch.equal(back[n, few], want[0]), n
    del back
    torch.cuda.empty_cache()


def test_norm_many_rows_take_every_block():
    # more rows than the backward kernel's blocks take in one round, unequal sides
    q, k = draw((4, 2000, 12, 64), torch.bfloat16, 1), draw((4, 2000, 1, 64), torch.bfloat16, 2)
    dq, dk = draw((4, 2000, 12, 64), torch.bfloat16, 3), draw((4, 2000, 1, 64), torch.bfloat16, 4)
    g = torch.ones(64, device="cuda")
    first, again = (b.sh_qk_norm_backward(q, k, dq, dk, g, g, rotated=64) for _ in range(2))
    p = np.broadcast_to(np.arange(2000), (4, 2000))
    for x, dy, dx, dg, n in ((q, dq, "dq", "dgq", 12), (k, dk, "dk", "dgk", 1)):
        assert torch.equal(first[dx], again[dx]) and torch.equal(first[dg], again[dg])
        want, wg = op.qk_norm_backward(host(x), host(dy), np.ones(64), p, 1e-6, rotated=64)
        assert np.abs(host(first[dx]) - want).max() < 2.0 ** -8 * np.abs(want).max() + 1e-5
        # (random signs: the sum's error is its rows' and additions' errors, far below sqrt(rows) of them each)
        assert np.abs(host(first[dg]) - wg).max() < 64 * U * np.abs(host(x)).max() * np.abs(host(dy)).max() * np.sqrt(8000 * n)


BALANCE = [  # N, sides, H, E, k, dtype, padded
    (64, 2, 2, 4, 2, "f32", False), (1, 1, 1, 2, 1, "f32", False), (1, 2, 3, 32, 4, "bf16", False), (300, 2, 4, 5, 3, "f32", True), (777, 1, 8, 32, 4, "bf16", True),
    (513, 2, 8, 16, 4, "f32", True), (100, 2, 1, 3, 2, "bf16", False), (200, 1, 2, 1, 1, "f32", False), (50, 2, 20, 32, 2, "f32", False), (90, 3, 100, 7, 7, "f32", True),
    (400, 2, 2, 8, 2, "bf16", False), (256, 2, 2, 16, 1, "bf16", True), (64, 1, 300, 2, 1, "bf16", False), (2500, 2, 4, 4, 2, "bf16", True), (33, 1, 1, 31, 4, "bf16", False),
]


def balance_inputs(N, S, H, E, k, t, padded, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + N)
    z = (torch.randn(N, S, H, E, generator=g, device="cuda") - 0.7 * torch.arange(E, device="cuda")).to(t)
    idx = torch.argsort(z.float(), dim=-1, descending=True, stable=True)[..., :k].permute(1, 0, 2, 3).int().contiguous()
    mask = (torch.rand(N, generator=g, device="cuda") < 0.7) if padded else None
    return z, idx, mask


def check_balance(z, idx, kind, coef, mask, gloss=None, got=None, dz=None):
    t = z.dtype
    got = b.sh_balance_loss(z, idx, kind=kind, coef=coef, mask=mask) if got is None else got
    dz = b.sh_balance_backward(z, got["slope"], mask=mask, gloss=None if gloss is None else torch.full((), gloss, device="cuda")) if dz is None else dz
    loss, counts, P, want = op.balance(host(z), idx.cpu().numpy(), kind, coef, None if mask is None else mask.cpu().numpy(), 1.0 if gloss is None else gloss)
    n, E = max(1, z.shape[0] if mask is None else int(mask.sum())), z.shape[3]
    assert np.array_equal(got["counts"].cpu().numpy(), counts) and got["counts"].dtype == torch.int32
    # p: the exponential 4 U, the difference in it half a step of the logits' range, a sum of at most 8 + 3 additions, a quotient and a product
    # (3 U); P: on top, a thread's additions (N / 592 rows at most) and those of a block's tokens (256 at most)
    zh = host(z)
    zf = zh[np.isfinite(zh)]
    p_u = (18 + (2 * np.abs(zf).max() if zf.size else 0.0)) * U
    P_u = p_u + (n / 592 + 256 + 2) * U
    close(got["prob"], P, P * P_u, torch.float32)
    with np.errstate(divide="ignore"):
        log = np.where(P > 0, np.abs(np.log(np.where(P > 0, P, 1.0))), 0.0)
    close(got["loss"], loss, coef * (P * (E if kind == "counts" else 1.0 + log) * P_u).sum(), torch.float32)
    # dz = p (c - sum p c) gloss / n with c centred: c within (E or log range) coef, off by U of that and, for the entropy, by P_u
    c = coef * (E if kind == "counts" else log.max(initial=0.0) + 1.0) * np.ones(1)
    with np.errstate(invalid="ignore"):
        e = np.exp(zh - np.where(np.isfinite(zh.max(-1, keepdims=True)), zh.max(-1, keepdims=True), 0.0))
        p = e / np.maximum(e.sum(-1, keepdims=True), 1e-300)
    close(dz, want, np.nan_to_num(p) * (2 * c * (p_u + 16 * U) + 2 * coef * P_u) * abs(1.0 if gloss is None else gloss) / n, t)
    return got, dz


@pytest.mark.parametrize("kind", ["counts", "entropy"])
@pytest.mark.parametrize("case", BALANCE)
def test_balance_and_its_gradient(case, kind):
    N, S, H, E, k, ty, padded = case
    z, idx, mask = balance_inputs(N, S, H, E, k, TYPES[ty], padded)
    got, dz = check_balance(z, idx, kind, 0.01, mask, gloss=3.0)
    if mask is not None:
        assert not dz[~mask].any()
    again = b.sh_balance_loss(z, idx, kind=kind, coef=0.01, mask=mask)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("kind", ["counts", "entropy"])
def test_balance_many_tokens(kind):
    z, idx, mask = balance_inputs(30000, 2, 2, 8, 2, torch.float32, True)
    check_balance(z, idx, kind, 1.0, mask)


@pytest.mark.parametrize("kind", ["counts", "entropy"])
@pytest.mark.parametrize("N,S,H,E,ty", [(40000, 1, 2, 4, "f32"), (9001, 2, 2, 16, "f32"), (9001, 1, 2, 31, "f32"), (70001, 1, 1, 3, "bf16"), (20003, 1, 2, 8, "bf16"), (9000, 1, 3, 16, "bf16"),
                                        (9001, 1, 1, 32, "bf16"), (9001, 1, 2, 20, "bf16"), (30, 2, 600, 8, "f32"), (3, 2, 40, 32, "bf16")])
def test_balance_of_two_launches(N, S, H, E, ty, kind):
    """Above the sizes of the kernel of one launch, every width of a row: against fp64 sums."""
    z, idx, mask = balance_inputs(N, S, H, E, min(3, E - 1), TYPES[ty], True)
    got = b.sh_balance_loss(z, idx, kind=kind, coef=0.1, mask=mask)
    dz = b.sh_balance_backward(z, got["slope"], mask=mask)
    n = int(mask.sum())
    p = torch.softmax(z.double(), -1) * mask[:, None, None, None]
    P = p.sum(0) / n
    picks = (idx.long()[..., None] == torch.arange(E, device="cuda")) & mask[None, :, None, None, None]
    counts = picks.sum((1, 3))
    assert torch.equal(got["counts"].long(), counts)
    f = counts.double() / counts.sum(-1, keepdim=True)
    c = 0.1 * E * f if kind == "counts" else 0.1 * torch.log(P)
    loss = (0.1 * E * (f * P).sum() if kind == "counts" else 0.1 * (P * torch.log(P)).sum()).item()
    want = p * (c - (p * c).sum(-1, keepdim=True)) / n
    # (p: 40 U, as above with logits of up to 8 and their differences; P: and a thread's additions, N / 444 rows at most, a block's 256)
    p_u = (18 + 2 * float(z.float().abs().max())) * U
    P_u = p_u + (N / 444 + 256 + 2) * U
    close(got["prob"], host(P), host(P) * P_u, torch.float32)
    log = float(torch.log(P).abs().max())
    close(got["loss"], loss, 0.1 * S * H * (E if kind == "counts" else 1 + log) * P_u, torch.float32)
    close(dz, host(want), host(p) * 0.1 * (2 * (E if kind == "counts" else 1 + log) * (p_u + 16 * U) + 2 * P_u) / n, TYPES[ty])


@pytest.mark.parametrize("N,S,H,E", [(2010, 2, 4, 2), (100000, 1, 2, 3), (4000, 1, 1, 4)])
def test_balance_of_nearly_balanced_gates(N, S, H, E):
    """The entropy's slope is what is left of ln P behind its mean: P has to be exact far below a rounding of its size a token."""
    g = torch.Generator(device="cuda").manual_seed(N)
    z = torch.randn(N, S, H, E, generator=g, device="cuda")
    idx = torch.zeros(S, N, H, 1, dtype=torch.int32, device="cuda")
    got = b.sh_balance_loss(z, idx, kind="entropy")
    dz = b.sh_balance_backward(z, got["slope"])
    p = torch.softmax(z.double(), -1)
    c = torch.log(p.mean(0))
    want = p * (c - (p * c).sum(-1, keepdim=True)) / N
    spread = float((c - c.mean(-1, keepdim=True)).square().mean().sqrt())
    # p: 30 U a token, by roundings of its own: six standard deviations of their mean 180 U / sqrt(N), beside blocks' sums rounded once each
    # (8 or more: U); as a share of the slope's spread, and 40 U of the products
    rel = float((dz.double() - want).norm() / want.norm())
    assert rel < (180 / np.sqrt(N) + 1) * U / spread + 40 * U, (rel, spread)


@pytest.mark.parametrize("kind", ["counts", "entropy"])
def test_balance_extreme_logits(kind):
    z, idx, mask = balance_inputs(64, 2, 2, 8, 2, torch.float32, False)
    z[:, 0, 0, 3] = -float("inf")                          # an expert that is switched off for everyone
    z[5, 1, 0] = -float("inf")                             # a row that is left with none
    z[:, 1, 1, 2:] = torch.finfo(torch.float32).min        # masks of the type's lowest value
    z[7, 0, 1] = 1e30
    idx[0, 3, 1, 0] = -1                                   # a slot without an expert, one that is none, the same twice
    idx[1, 4, 0, 1] = 99
    idx[1, 6, 0] = idx[1, 6, 0, :1]
    got = b.sh_balance_loss(z, idx, kind=kind, coef=1.0)
    dz = b.sh_balance_backward(z, got["slope"])
    loss, counts, P, want = op.balance(host(z), idx.cpu().numpy(), kind, 1.0)
    assert np.array_equal(got["counts"].cpu().numpy(), counts) and int(got["counts"].sum()) == 64 * 8 - 2
    assert np.abs(host(got["prob"]) - P).max() < 1e-6 and abs(float(got["loss"]) - loss) < 1e-5
    assert torch.isfinite(dz).all() and np.abs(host(dz) - want).max() < 1e-6
    assert not dz[5, 1, 0].any() and not dz[:, 0, 0, 3].any()


def test_balance_padding_may_hold_anything():
    z, idx, mask = balance_inputs(200, 2, 2, 8, 2, torch.float32, True)
    want = b.sh_balance_loss(z, idx, coef=1.0, mask=mask)
    dwant = b.sh_balance_backward(z, want["slope"], mask=mask)
    z[~mask] = float("nan")
    idx[:, ~mask] = 1 << 30
    got = b.sh_balance_loss(z, idx, coef=1.0, mask=mask.to(torch.uint8))
    dz = b.sh_balance_backward(z, got["slope"], mask=mask)
    assert all(torch.equal(got[n], want[n]) for n in want) and torch.equal(dz, dwant) and not dz[~mask].any()
    z[mask.nonzero()[3, 0], 1, 1, 2] = float("nan")        # ... and one that counts makes its gate's loss NaN, and no other gate's means
    got = b.sh_balance_loss(z, idx, coef=1.0, mask=mask)
    assert torch.isnan(got["loss"]) and torch.isnan(got["prob"][1, 1]).all() and torch.equal(got["prob"][0], want["prob"][0])


def test_balance_of_no_tokens():
    z, idx, mask = balance_inputs(40, 2, 2, 4, 2, torch.float32, False)
    none = torch.zeros(40, dtype=torch.bool, device="cuda")
    for args in ((z, idx, none), (z[:0], idx[:, :0].contiguous(), None)):
        got = b.sh_balance_loss(args[0], args[1], kind="entropy", mask=args[2])
        assert all(not got[n].any() for n in got)
        assert not b.sh_balance_backward(args[0], got["slope"], mask=args[2]).any()


def test_balance_strided_and_in_place():
    for E, t in ((8, torch.float32), (5, torch.float32), (8, torch.bfloat16)):
        z, idx, mask = balance_inputs(100, 2, 3, E, 2, t, True)
        wide = torch.full((100, 2 * 3 * E + 11), 5.0, device="cuda", dtype=t)
        view = wide[:, 3:3 + 6 * E].unflatten(1, (2, 3, E))
        view.copy_(z)
        got, want = b.sh_balance_loss(view, idx, mask=mask), b.sh_balance_loss(z, idx, mask=mask)
        assert all(torch.equal(got[n], want[n]) for n in want)
        dwant = b.sh_balance_backward(z, want["slope"], mask=mask)
        assert b.sh_balance_backward(view, got["slope"], mask=mask, out=view) is view
        assert torch.equal(view, dwant) and (wide[:, :3] == 5).all() and (wide[:, 3 + 6 * E:] == 5).all()


@pytest.mark.parametrize("ty", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 8), (5, 64), (4, 77), (2, 1030), (130, 40)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(rows, cols, ty, residual):
    t = TYPES[ty]
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    x, res = (torch.randn(rows, cols, generator=g, device="cuda").to(t) for _ in range(2))
    seed, offset = -123456789012345 + cols, (5 << 40) + rows
    rng = torch.tensor([seed, offset], device="cuda")
    for p in (0.0, 0.1, 0.5, 1.0):
        kept, scale = op.dropout_kept(rows, cols, seed, offset, p)
        y = b.sh_dropout(x, rng, p, residual=res if residual else None)
        r = host(res) if residual else np.zeros((rows, cols))
        want = np.where(kept, host(x) * scale, 0.0) + r
        close(y, want, 3 * U * (np.abs(host(x)) * scale + np.abs(r)), t)      # (the factor, the product, the sum)
        assert np.array_equal(host(y)[~kept], r[~kept])                       # what is dropped leaves the residual's bits


@pytest.mark.parametrize("ty", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(64, 17), (41, 23), (7, 1001), (300, 31), (9, 18), (5, 20), (1, 33), (2, 4095), (700, 19)])
def test_dropout_dense_rows_of_any_length(rows, cols, ty):
    # a thread's 16 values begin anywhere in a piece, end in the next row, and at the end of the matrix
    t = TYPES[ty]
    x, res = torch.randn(rows, cols, device="cuda").to(t), torch.randn(rows, cols, device="cuda").to(t)
    rng = torch.tensor([cols, 1 << 33], device="cuda")
    kept, scale = op.dropout_kept(rows, cols, cols, 1 << 33, 0.4)
    for r in (None, res):
        add = np.zeros((rows, cols)) if r is None else host(r)
        y = b.sh_dropout(x, rng, 0.4, residual=r)
        close(y, np.where(kept, host(x) * scale, 0.0) + add, 3 * U * (np.abs(host(x)) * scale + np.abs(add)), t)
        assert np.array_equal(host(y)[~kept], add[~kept])
    whole = torch.full((rows * cols + 32,), 9.0, device="cuda", dtype=t)                # what lies behind the last value stays
    out = whole[:rows * cols].view(rows, cols)
    assert torch.equal(b.sh_dropout(x, rng, 0.4, out=out), b.sh_dropout(x, rng, 0.4)) and (whole[rows * cols:] == 9).all()


@pytest.mark.parametrize("ty", ["f32", "bf16"])
@pytest.mark.parametrize("stride,cols", [(80, 77), (79, 77), (88, 80), (83, 40), (24, 9), (11, 5), (2008, 2001), (2003, 2001), (640, 513)])
def test_dropout_rows_apart(stride, cols, ty):
    # rows at vectors' addresses that end inside a piece, and rows anywhere: the same values as a dense matrix's
    t, rows = TYPES[ty], 37
    x, res = torch.randn(rows, cols, device="cuda").to(t), torch.randn(rows, cols, device="cuda").to(t)
    rng = torch.tensor([1, 2], device="cuda")
    want, plain = b.sh_dropout(x, rng, 0.3, residual=res), b.sh_dropout(x, rng, 0.3)
    wide = torch.full((rows, stride), 5.0, device="cuda", dtype=t)
    view = wide[:, :cols]
    view.copy_(x)
    assert torch.equal(b.sh_dropout(view, rng, 0.3), plain)
    assert b.sh_dropout(view, rng, 0.3, residual=res, out=view) is view
    assert torch.equal(view, want) and (wide[:, cols:] == 5).all()
    one = res[:1].expand(rows, cols)                                                        # one row for all of them
    assert torch.equal(b.sh_dropout(x, rng, 0.3, residual=one), b.sh_dropout(x, rng, 0.3, residual=one.contiguous()))
    assert torch.equal(b.sh_dropout(x[:1].expand(rows, cols), rng, 0.3), b.sh_dropout(x[:1].repeat(rows, 1), rng, 0.3))
    off = torch.empty(rows * cols + 1, device="cuda", dtype=t)[1:].view(rows, cols)         # dense, one value off alignment
    off.copy_(x)
    assert torch.equal(b.sh_dropout(off, rng, 0.3), plain)


def test_dropout_shapes_strides_and_places():
    rng = torch.tensor([3, 4], device="cuda")
    x, res = torch.randn(6, 10, 72, device="cuda"), torch.randn(6, 10, 72, device="cuda")
    want = b.sh_dropout(x, rng, 0.3, residual=res)
    assert want.shape == x.shape and torch.equal(b.sh_dropout(x.reshape(60, 72), rng, 0.3, residual=res.reshape(60, 72)).view_as(x), want)
    for pad in (8, 3):                                                        # rows apart: aligned or not
        wide = torch.full((60, 72 + pad), 5.0, device="cuda")
        wide[:, :72] = x.reshape(60, 72)
        b.sh_dropout(wide[:, :72], rng, 0.3, residual=res.reshape(60, 72), out=wide[:, :72])
        assert torch.equal(wide[:, :72], want.reshape(60, 72)) and (wide[:, 72:] == 5).all()
    place = res.clone()
    assert b.sh_dropout(x, rng, 0.3, residual=place, out=place) is place and torch.equal(place, want)
    assert b.sh_dropout(torch.zeros(0, 8, device="cuda"), rng, 0.3).shape == (0, 8)
    assert b.sh_dropout(torch.zeros(4, 0, device="cuda"), rng, 0.3).shape == (4, 0)
    line = torch.ones(100, device="cuda")
    assert torch.equal(b.sh_dropout(line, rng, 0.3), b.sh_dropout(line[None], rng, 0.3)[0])
    with pytest.raises(ValueError):
        b.sh_dropout(x.transpose(0, 1), rng, 0.3)
    with pytest.raises(b.SwitchHeadError, match="share an address"):
        b.sh_dropout(x[0], rng, 0.3, out=torch.zeros(1, 72, device="cuda").expand(10, 72))


def test_dropout_a_dropped_value_does_not_count():
    rng = torch.tensor([8, 9], device="cuda")
    x = torch.full((16, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    res = torch.randn(16, 64, device="cuda")
    kept, _ = op.dropout_kept(16, 64, 8, 9, 0.4)
    y = b.sh_dropout(x, rng, 0.4, residual=res).cpu().numpy()
    assert np.array_equal(y[~kept], res.cpu().numpy()[~kept]) and not np.isfinite(y[kept]).any()


def test_dropout_gradient_is_the_same_call():
    rng = torch.tensor([21, 22], device="cuda")
    x, dy = torch.randn(33, 100, device="cuda"), torch.randn(33, 100, device="cuda")
    # linear in x: <dropout(x), dy> = <x, dropout(dy)>, term by term up to the roundings of three products
    lhs, rhs = host(b.sh_dropout(x, rng, 0.25)) * host(dy), host(x) * host(b.sh_dropout(dy, rng, 0.25))
    assert np.abs(lhs - rhs).max() <= 4 * U * np.abs(lhs).max()
    h = 1.0                                                                   # (a difference of a linear map, at any step)
    diff = host(b.sh_dropout(x + h * dy, rng, 0.25)) - host(b.sh_dropout(x, rng, 0.25))
    assert np.abs(diff - host(b.sh_dropout(dy, rng, 0.25))).max() <= 8 * U * (np.abs(host(x)).max() + np.abs(host(dy)).max()) * 4 / 3


def test_dropout_rows_past_32_bits_of_elements():
    # 2^31 values and more: rows near the end have the bits their row number gives
    rows, cols = (1 << 18) + 5, 1 << 14
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    rng = torch.tensor([1, 2], device="cuda")
    b.sh_dropout(x, rng, 0.5, out=x)
    for r in (0, 131072, 262143, rows - 3):
        kept, _ = op.dropout_kept(3, 64, 1, 2, 0.5, first_row=r)
        assert np.array_equal(x[r:r + 3, :64].float().cpu().numpy() != 0, kept), r
    del x
    torch.cuda.empty_cache()


def test_captured_calls_replay_on_new_inputs():
    q, k = torch.randn(2, 40, 4, 64, device="cuda"), torch.randn(2, 40, 2, 64, device="cuda")
    dq, dk, gain = torch.randn_like(q), torch.randn_like(k), torch.ones(64, device="cuda")
    z, idx, _ = balance_inputs(80, 2, 2, 8, 2, torch.float32, False)
    large, lidx, _ = balance_inputs(9001, 1, 2, 16, 2, torch.bfloat16, False)
    x, rng = torch.randn(80, 128, device="cuda"), torch.tensor([1, 1], device="cuda")

    def calls():
        y = b.sh_qk_norm(q, k, gain, gain, rotated=64)
        back = b.sh_qk_norm_backward(q, k, dq, dk, gain, gain, rotated=64)
        got, more = b.sh_balance_loss(z, idx, kind="entropy"), b.sh_balance_loss(large, lidx)
        dz = b.sh_balance_backward(z, got["slope"], gloss=got["loss"])
        return [*y, *back.values(), *got.values(), dz, *more.values(), b.sh_dropout(x, rng, 0.5, residual=x), b.sh_dropout(x.view(-1)[:10001], rng, 0.5)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(calls())
    for turn in range(3):
        for a in (q, k, dq, dk, z, x, large):
            a.normal_()
        rng[1] += 1
        want = calls()
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(out, want)), turn


def test_two_calls_at_once():
    q, dq, g = torch.randn(4, 300, 6, 64, device="cuda"), torch.randn(4, 300, 6, 64, device="cuda"), torch.randn(64, device="cuda")
    z, idx, _ = balance_inputs(9001, 2, 2, 16, 3, torch.float32, False)
    x, rng = torch.randn(3000, 77, device="cuda"), torch.tensor([1, 1], device="cuda")

    def calls():
        back = b.sh_qk_norm_backward(q, q, dq, dq, g, g, rotated=64)
        got = b.sh_balance_loss(z, idx, kind="entropy")
        return [*back.values(), *got.values(), b.sh_balance_backward(z, got["slope"]), b.sh_dropout(x, rng, 0.5)]

    want = calls()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(calls())
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for out in outs for a, w in zip(out, want))


def test_on_another_stream():
    side = torch.cuda.Stream()
    x = torch.zeros(1 << 24, device="cuda").view(1 << 12, 1 << 12)
    rng = torch.tensor([1, 1], device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)                                   # (the call below has to come after these)
        y = b.sh_dropout(x, rng, 0.5)
    side.synchronize()
    assert set(y.unique().tolist()) == {0.0, 40.0}


def test_refusals_of_the_binding():
    q, k = torch.randn(2, 4, 2, 32, device="cuda"), torch.randn(2, 4, 1, 32, device="cuda")
    bad = [dict(k=k[:, :3]), dict(k=k.half()), dict(gq=torch.ones(31, device="cuda")), dict(gq=torch.ones(32, device="cuda").half()), dict(gk=torch.ones(32)),
           dict(positions=torch.zeros(2, 3, dtype=torch.int32, device="cuda")), dict(positions=torch.zeros(2, 4, device="cuda")), dict(q=q.transpose(2, 3)),
           dict(q_out=torch.empty(2, 4, 2, 32, device="cuda", dtype=torch.float16)), dict(k_out=k.cpu())]
    for kw in bad:
        args = dict(q=q, k=k, rotated=32)
        args.update(kw)
        with pytest.raises(ValueError):
            b.sh_qk_norm(args.pop("q"), args.pop("k"), args.pop("gq", None), args.pop("gk", None), **args)
    with pytest.raises(ValueError):
        b.sh_qk_norm_backward(q, k, q, None)
    for kw in (dict(rotated=33), dict(eps=0.0), dict(rotated=32, base=-1.0)):
        with pytest.raises(b.SwitchHeadError):
            b.sh_qk_norm(q, k, **kw)
    z, idx, mask = balance_inputs(20, 2, 2, 4, 2, torch.float32, True)
    for kw in (dict(idx=idx.long()), dict(idx=idx[:1]), dict(logits=z.half()), dict(logits=z.transpose(1, 2)), dict(mask=mask[:5]), dict(mask=mask.float()), dict(kind="none")):
        args = dict(logits=z, idx=idx, mask=mask)
        args.update(kw)
        with pytest.raises(ValueError):
            b.sh_balance_loss(args.pop("logits"), args.pop("idx"), **args)
    with pytest.raises(ValueError):
        b.sh_balance_backward(z, torch.zeros(2, 2, 5, device="cuda"))
    x, rng = torch.randn(4, 8, device="cuda"), torch.tensor([1, 2], device="cuda")
    for args in ((x, rng.int(), 0.1), (x, rng.cpu(), 0.1), (x.double(), rng, 0.1), (x, rng[:1], 0.1)):
        with pytest.raises(ValueError):
            b.sh_dropout(*args)
    with pytest.raises(ValueError):
        b.sh_dropout(x, rng, 0.1, residual=x[:3])
    with pytest.raises(b.SwitchHeadError):
        b.sh_dropout(x, rng, 1.1)
