"""The operators of a training step around the SwitchHead layer's projections and selection, as they are timed.

norm     queries and keys normalised per head and rotated by their position in the same pass, and the backward pass of that
balance  the balance loss of the gates with the per-expert counts, and its gradient with respect to the gate logits
dropout  dropout (with the residual sum) whose mask comes from a counter and is never stored

A case is one call (`balance` with its gradient: the two calls of a training step) over tensors that are on the GPU.  Sizes
are those of the repository's workloads (`paper_2312_07987_b200.inputs.CONFIGS`, `perf/cases.py`) and generic ones.
Where `own` is false the operators are computed in elementary torch operations, else by the library.
"""
import math

import torch

own = False

DEFAULTS = dict(op="norm", dtype="f32", direction="forward", batch=1, seq=64,
                q_heads=2, k_heads=2, d_head=32, rotated=32, halves=False, layout="bthd", positions="plain", q_scale=1.0, gains=True,
                sides=2, heads=2, experts=4, k=2, kind="counts", padded=False, zipf=0.0,
                cols=128, p=0.1, residual=False)
KEYS = dict(norm=("op", "dtype", "direction", "batch", "seq", "q_heads", "k_heads", "d_head", "rotated", "halves", "layout", "positions", "q_scale", "gains"),
            balance=("op", "dtype", "direction", "batch", "seq", "sides", "heads", "experts", "k", "kind", "padded", "zipf"),
            dropout=("op", "dtype", "direction", "batch", "seq", "cols", "p", "residual"))
TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)
BASE, EPS, COEF = 10000.0, 1e-6, 0.01


def _case(name=None, **kw):
    c = dict(DEFAULTS, **kw)
    c = {n: c[n] for n in KEYS[c["op"]]}
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token of each of 16 users far into their contexts: launches and their latency are all there is
        _case("norm_tokens_bf16", op="norm", dtype="bf16", batch=16, seq=1, q_heads=4, k_heads=4, d_head=128, rotated=128, layout="fused", positions="far"),
        # prompts of an odd length, a d_head that fits no vector of 16 bytes, in fp16, the layer's layout of queries and keys
        _case("norm_ragged_f16", op="norm", dtype="f16", batch=5, seq=777, q_heads=4, k_heads=4, d_head=100, rotated=100, layout="bhtd", q_scale=0.1),
        # long sequences with grouped heads out of one fused projection, half of the columns rotated
        _case("norm_long_bf16", op="norm", dtype="bf16", batch=4, seq=4096, q_heads=32, k_heads=8, d_head=128, rotated=64, halves=True, layout="fused"),
        # the gradients of a 47M-parameter model's training step
        _case("norm_grad_f32", op="norm", dtype="f32", direction="backward", batch=8, seq=256, q_heads=2, k_heads=2, d_head=76, rotated=76, layout="bhtd"),
        # ... and of a wide layer's over a long batch, in bf16
        _case("norm_grad_wide_bf16", op="norm", dtype="bf16", direction="backward", batch=8, seq=2048, q_heads=8, k_heads=8, d_head=128, rotated=128, halves=True),
        # the counts and the loss of a 262M-parameter model's batch, without the gradient (watched during evaluation)
        _case("balance_eval_f32", op="balance", dtype="f32", batch=16, seq=512, heads=4, experts=4, k=2),
        # a training step of a layer with many experts, unevenly routed, over a padded batch
        _case("balance_skew_f32", op="balance", dtype="f32", direction="both", batch=8, seq=2048, heads=8, experts=16, k=4, kind="entropy", padded=True, zipf=1.2),
        # the most experts a layer takes, one gate for both sides, a large batch, logits in bf16
        _case("balance_large_bf16", op="balance", dtype="bf16", direction="both", batch=128, seq=1024, sides=1, heads=8, experts=32, k=4),
        # the smallest layer's output
        _case("dropout_tiny_f32", op="dropout", dtype="f32", batch=1, seq=64, cols=128, residual=True),
        # the layer's output into the residual stream, as the 262M-parameter model's training step has it
        _case("dropout_residual_f32", op="dropout", dtype="f32", batch=16, seq=512, cols=1024, residual=True),
        # the gradient's way back through it
        _case("dropout_grad_bf16", op="dropout", dtype="bf16", direction="backward", batch=8, seq=2048, cols=2048, p=0.2),
        # a large batch of long sequences
        _case("dropout_long_bf16", op="dropout", dtype="bf16", batch=16, seq=4096, cols=2048, residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: an operator, then sizes over its range; the batch, then the sequence shrinks until it costs no more
    than the operator's largest listed case."""
    op = rng.choice(["norm", "norm", "balance", "dropout"])
    kw = dict(op=op, dtype=rng.choice(["f32", "bf16", "f16"]), seq=_log_int(rng, 1, 4096), batch=_log_int(rng, 1, 64))
    if op == "norm":
        d = rng.choice([32, 64, 76, 100, 112, 128, 128, 132, 168, 2 * rng.randint(4, 128)])
        kw.update(direction=rng.choice(["forward", "backward"]), k_heads=rng.choice([1, 2, 3, 4, 8]), d_head=d,
                  rotated=rng.choice([d, d, d, 0, 2 * rng.randint(1, d // 2)]), halves=rng.random() < 0.5, layout=rng.choice(["bthd", "bhtd", "fused"]),
                  positions=rng.choice(["plain", "plain", "packed", "far"]), q_scale=rng.choice([1.0, 1.0, 0.125]), gains=rng.random() < 0.85)
        kw["q_heads"] = kw["k_heads"] * rng.choice([1, 1, 2, 4])
    elif op == "balance":
        e = rng.choice([2, 3, 4, 5, 8, 16, 32])
        # (no fp16: a gradient of a mean over many tokens lies below its normal numbers; fewer selections than experts: else all are used alike and
        #  nothing is left of the gradient)
        kw.update(dtype=rng.choice(["f32", "f32", "bf16"]), direction=rng.choice(["forward", "both", "both"]), sides=rng.choice([1, 2, 2]), heads=rng.choice([1, 2, 3, 4, 8]), experts=e,
                  k=rng.randint(1, min(4, e - 1)), kind=rng.choice(["counts", "entropy"]), padded=rng.random() < 0.4, zipf=rng.choice([0.0, 0.0, 1.2]))
    else:
        kw.update(direction=rng.choice(["forward", "backward"]), cols=rng.choice([64 * rng.randint(1, 40), rng.randint(1, 2500)]), p=rng.choice([0.05, 0.1, 0.2, 0.5]))
        kw["residual"] = kw["direction"] == "forward" and rng.random() < 0.7
    c = _case(**kw)
    top = max(work(x)["bytes"] for x in listed() if x["op"] == op)
    while work(c)["bytes"] > top:
        if c["batch"] > 1:
            c["batch"] = max(1, c["batch"] * 3 // 4)
        else:
            c["seq"] = max(1, c["seq"] * 3 // 4)
    return c


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)


def _heads(c, g):
    """Queries and keys of drawn values in the case's layout, as views [B, T, H, D]."""
    B, T, D, n = c["batch"], c["seq"], c["d_head"], (c["q_heads"], c["k_heads"])
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(TYPES[c["dtype"]])
    if c["layout"] == "fused":           # the columns of one projection: queries, keys, values
        whole = normal(B, T, sum(n) + n[1], D)
        return whole[:, :, :n[0]], whole[:, :, n[0]:sum(n)]
    if c["layout"] == "bhtd":
        return tuple(normal(B, h, T, D).transpose(1, 2) for h in n)
    return tuple(normal(B, T, h, D) for h in n)


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    g = _generator(seed)
    B, T = c["batch"], c["seq"]
    s = dict(case=c)
    if c["op"] == "norm":
        s["q"], s["k"] = _heads(c, g)
        gain = lambda: 1.0 + 0.2 * torch.randn(c["d_head"], generator=g, device="cuda") if c["gains"] else None
        s["gq"], s["gk"] = gain(), gain()
        # (plain: token t at position t; packed: each row holds sequences one behind the other; far: one offset per row)
        t = torch.arange(T, device="cuda", dtype=torch.int32).expand(B, T)
        s["positions"] = None
        if c["positions"] == "far":
            s["positions"] = t + torch.randint(1 << 16, 1 << 20, (B, 1), generator=g, device="cuda", dtype=torch.int32)
        elif c["positions"] == "packed":
            cut = torch.randint(0, T, (B, 1), generator=g, device="cuda", dtype=torch.int32)
            s["positions"] = torch.where(t < cut, t, t - cut)
        if c["direction"] == "backward":
            s["dq"], s["dk"] = _heads(dict(c, layout="bthd"), g)
    elif c["op"] == "balance":
        N, S, H, E, k = B * T, c["sides"], c["heads"], c["experts"], c["k"]
        z = torch.randn(N, S, H, E, generator=g, device="cuda")
        if c["zipf"]:
            rank = torch.argsort(torch.rand(S, H, E, generator=g, device="cuda"), dim=-1).float() + 1
            z = z - c["zipf"] * torch.log(rank)
        s["z"] = z.to(TYPES[c["dtype"]])
        top = torch.argsort(s["z"].float(), dim=-1, descending=True, stable=True)[..., :k]
        s["idx"] = top.permute(1, 0, 2, 3).to(torch.int32).contiguous()
        s["mask"] = None
        if c["padded"]:
            length = torch.randint(1, T + 1, (B, 1), generator=g, device="cuda")
            s["mask"] = (torch.arange(T, device="cuda") < length).reshape(N)
        s["gloss"] = torch.full((), 1.0 + 0.001 * (int(seed) % 97), device="cuda")
    else:
        normal = lambda: torch.randn(B * T, c["cols"], generator=g, device="cuda").to(TYPES[c["dtype"]])
        s["x"] = normal()
        s["residual"] = normal() if c["residual"] else None
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device="cuda")      # the seed and the offset of this site and step
    return s


# The plain forms.

def _angles(c, positions, B, T):
    """cos and sin [B, T, 1, R / 2] of each position's angles, taken in 64 bits."""
    half = c["rotated"] // 2
    pos = torch.arange(T, device="cuda").expand(B, T) if positions is None else positions
    ang = pos.double()[..., None, None] * BASE ** (-2.0 * torch.arange(half, device="cuda").double() / max(1, c["rotated"]))
    return torch.cos(ang), torch.sin(ang)


def _turn(a, cos, sin, c):
    """The first `rotated` columns of a, pair by pair."""
    R = c["rotated"]
    if R == 0:
        return a
    if c["halves"]:
        x, y = a[..., :R // 2], a[..., R // 2:R]
        r = torch.cat([x * cos - y * sin, x * sin + y * cos], dim=-1)
    else:
        x, y = a[..., 0:R:2], a[..., 1:R:2]
        r = torch.stack([x * cos - y * sin, x * sin + y * cos], dim=-1).flatten(-2)
    return torch.cat([r, a[..., R:]], dim=-1) if R < a.shape[-1] else r


def _norm(x, gain, scale, cos, sin, c):
    f = x.float()
    n = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    if gain is not None:
        n = n * gain
    return (_turn(n, cos, sin, c) * scale).to(x.dtype)


def _norm_backward(x, dy, gain, scale, cos, sin, c):
    f = x.float()
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    n = f * r
    u = _turn(dy.float(), cos, -sin, c) * scale
    w = u if gain is None else u * gain
    dx = r * (w - n * (w * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), None if gain is None else (u * n).sum((0, 1, 2), dtype=torch.float64).float()


def _balance(s, c):
    z, idx, mask = s["z"], s["idx"].long(), s["mask"]
    N, S, H, E = z.shape
    p = torch.softmax(z.float(), dim=-1)
    chosen = (idx[..., None] == torch.arange(E, device="cuda")).sum(3)                     # [S, N, H, E]
    n = N
    if mask is not None:
        p = torch.where(mask[:, None, None, None], p, torch.zeros((), device="cuda"))
        chosen = chosen * mask[None, :, None, None]
        n = mask.sum()
    counts = chosen.sum(1)
    P = p.sum(0, dtype=torch.float64) / n
    f = counts.double() / counts.sum(-1, keepdim=True)
    if c["kind"] == "counts":
        loss, slope = COEF * E * (f * P).sum(), COEF * (E * f - 1.0)
    else:
        log = torch.log(P)
        loss, slope = COEF * (P * log).sum(), COEF * (log - log.mean(-1, keepdim=True))
    out = dict(loss=loss.float(), counts=counts.int(), prob=P.float())
    if c["direction"] == "both":
        slope = (slope / n).float()
        out["dz"] = (s["gloss"] * p * (slope - (p * slope).sum(-1, keepdim=True))).to(z.dtype)
    return out


def _philox(rows, blocks, rng):
    """Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3"): four words [rows, blocks] of 32 bits."""
    low = 0xFFFFFFFF
    seed, offset = rng[0], rng[1]
    ctr = [torch.arange(blocks, device="cuda").expand(rows, blocks), torch.arange(rows, device="cuda")[:, None].expand(rows, blocks), offset & low, (offset >> 32) & low]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = ctr[0] * 0xD2511F53, ctr[2] * 0xCD9E8D57
        ctr = [((b >> 32) & low) ^ ctr[1] ^ k0, b & low, ((a >> 32) & low) ^ ctr[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return ctr


def _dropout(s, c):
    x = s["x"]
    rows, cols = x.shape
    words = torch.stack(_philox(rows, (cols + 7) // 8, s["rng"]), dim=-1)
    bits = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, -1)[:, :cols]
    limit = int(round(c["p"] * 65536))
    y = torch.where(bits >= limit, x.float() * (65536.0 / (65536 - limit)), torch.zeros((), device="cuda"))
    return (y if s["residual"] is None else y + s["residual"].float()).to(x.dtype)


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "balance":
        return _balance(s, c)
    if c["op"] == "dropout":
        return _dropout(s, c)
    cos, sin = (a.float() for a in _angles(c, s["positions"], *s["q"].shape[:2]))
    if c["direction"] == "forward":
        return [_norm(s["q"], s["gq"], c["q_scale"], cos, sin, c), _norm(s["k"], s["gk"], 1.0, cos, sin, c)]
    q, k = _norm_backward(s["q"], s["dq"], s["gq"], c["q_scale"], cos, sin, c), _norm_backward(s["k"], s["dk"], s["gk"], 1.0, cos, sin, c)
    return dict(dq=q[0], dk=k[0], dgq=q[1], dgk=k[1])


def _run_own(s, c):
    from paper_2312_07987_b200 import binding
    if c["op"] == "norm":
        kw = dict(eps=EPS, base=BASE, rotated=c["rotated"], halves=c["halves"], positions=s["positions"], q_scale=c["q_scale"])
        if c["direction"] == "forward":
            return list(binding.sh_qk_norm(s["q"], s["k"], s["gq"], s["gk"], **kw))
        return binding.sh_qk_norm_backward(s["q"], s["k"], s["dq"], s["dk"], s["gq"], s["gk"], **kw)
    if c["op"] == "balance":
        got = binding.sh_balance_loss(s["z"], s["idx"], kind=c["kind"], coef=COEF, mask=s["mask"])
        out = dict(loss=got["loss"], counts=got["counts"], prob=got["prob"])
        if c["direction"] == "both":
            out["dz"] = binding.sh_balance_backward(s["z"], got["slope"], gloss=s["gloss"], mask=s["mask"])
        return out
    return binding.sh_dropout(s["x"], s["rng"], c["p"], residual=s["residual"])


def work(case):
    c = dict(DEFAULTS, **case)
    n, size = c["batch"] * c["seq"], TYPES[c["dtype"]].itemsize
    if c["op"] == "norm":
        values = n * (c["q_heads"] + c["k_heads"]) * c["d_head"]
        moved = 2 if c["direction"] == "forward" else 3
        return dict(bytes=values * size * moved + (0 if c["positions"] == "plain" else 4 * n), flops=values * (10 if moved == 2 else 20))
    if c["op"] == "balance":
        values, picks = n * c["sides"] * c["heads"] * c["experts"], n * c["sides"] * c["heads"] * c["k"]
        moved = 2 if c["direction"] == "both" else 1
        return dict(bytes=values * size * moved + 4 * picks + (n if c["padded"] else 0), flops=values * 6 * moved)
    values = n * c["cols"]
    return dict(bytes=values * size * (3 if c["residual"] else 2), flops=2 * values)


# The definitions in 64 bits.

def _exact_norm(s, c):
    D, R = c["d_head"], c["rotated"]
    B, T = s["q"].shape[:2]
    pos = (torch.arange(T, device="cuda").repeat(B, 1) if s["positions"] is None else s["positions"]).to(torch.float64)
    # each row's rotation as a complex factor per pair; pairs gathered by their columns
    i = torch.arange(R // 2, device="cuda")
    first, second = (i, i + R // 2) if c["halves"] else (2 * i, 2 * i + 1)
    factor = torch.polar(torch.ones(B, T, R // 2, device="cuda", dtype=torch.float64), pos[..., None] * torch.pow(torch.tensor(BASE, device="cuda", dtype=torch.float64), -2.0 * i.double() / max(R, 1)))[:, :, None, :]

    def rotate(a, by):
        out = a.clone()
        if R:
            pair = torch.complex(a[..., first], a[..., second]) * by
            out[..., first], out[..., second] = pair.real, pair.imag
        return out

    results = []
    for name, scale in (("q", c["q_scale"]), ("k", 1.0)):
        x = s[name].double()
        gain = torch.ones(D, device="cuda", dtype=torch.float64) if s["g" + name] is None else s["g" + name].double()
        length = torch.sqrt(torch.einsum("bthd,bthd->bth", x, x) / D + EPS)[..., None]
        if c["direction"] == "forward":
            results.append(scale * rotate(gain * x / length, factor))
            continue
        u = scale * rotate(s["d" + name].double(), factor.conj())
        along = torch.einsum("bthd,bthd->bth", u * gain, x)[..., None]
        results.append(u * gain / length - x * along / (D * length ** 3))
        results.append(None if s["g" + name] is None else torch.einsum("bthd,bthd->d", u, x / length))
    if c["direction"] == "forward":
        return results
    return dict(dq=results[0], dgq=results[1], dk=results[2], dgk=results[3])


def _exact_balance(s, c):
    z, E = s["z"].double(), c["experts"]
    keep = torch.ones(z.shape[0], dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    n = int(keep.sum())
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    P = torch.einsum("nshe,n->she", p, keep.double()) / n
    picks = s["idx"][:, keep].long()
    counts = torch.zeros(c["sides"], c["heads"], E, dtype=torch.int64, device="cuda")
    counts.scatter_add_(2, picks.permute(0, 2, 1, 3).reshape(c["sides"], c["heads"], -1), torch.ones_like(picks).permute(0, 2, 1, 3).reshape(c["sides"], c["heads"], -1))
    share = counts.double() / (n * c["k"])
    loss = COEF * E * (share * P).sum() if c["kind"] == "counts" else COEF * torch.special.xlogy(P, P).sum()
    out = dict(loss=loss, counts=counts.int(), prob=P)
    if c["direction"] == "both":
        slope = COEF * E * share if c["kind"] == "counts" else COEF * (torch.log(P) + 1.0)
        spread = slope - torch.einsum("nshe,she->nsh", p, slope)[..., None]
        out["dz"] = s["gloss"].double() / n * p * spread * keep[:, None, None, None]
    return out


def _exact_dropout(s, c):
    # the same counters, each word's products put together from halves of 16 bits
    rows, cols = s["x"].shape
    key = [int(v) & (2 ** 64 - 1) for v in s["rng"].tolist()]
    full = lambda v: torch.full((rows, -(-cols // 8)), v, dtype=torch.int64, device="cuda")
    w = [torch.arange(-(-cols // 8), device="cuda") + full(0), torch.arange(rows, device="cuda")[:, None] + full(0), full(key[1] % 2 ** 32), full(key[1] // 2 ** 32)]

    def product(a, m):
        lo, hi = (a % 65536) * m, (a // 65536) * m                       # both below 2^48
        mid = hi + lo // 65536
        return mid // 65536, (mid % 65536) * 65536 + lo % 65536

    for r in range(10):
        k0, k1 = (key[0] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (key[0] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = product(w[0], 0xD2511F53)
        h2, l2 = product(w[2], 0xCD9E8D57)
        w = [h2 ^ w[1] ^ k0, l2, h0 ^ w[3] ^ k1, l0]
    limit = math.floor(c["p"] * 65536 + 0.5)
    y = torch.zeros(rows, 8 * w[0].shape[1], dtype=torch.float64, device="cuda")
    x = torch.nn.functional.pad(s["x"].double(), (0, y.shape[1] - cols))
    for j in range(8):
        bits = w[j // 2] // 65536 if j % 2 else w[j // 2] % 65536
        y[:, j::8] = x[:, j::8] * (bits >= limit) * 65536 / (65536 - limit)
    y = y[:, :cols]
    return y if s["residual"] is None else y + s["residual"].double()


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    return (_exact_norm if c["op"] == "norm" else _exact_balance if c["op"] == "balance" else _exact_dropout)(s, c)
