"""A training step of the fp32 layer with norms of queries and keys, rotary positions, the balance loss and dropout in its own
passes (sh_set_qk_norm, sh_set_balance, sh_set_dropout), against the forward equations in fp64 and their automatic
differentiation; and the standalone operators around a plain pass against the same settings."""
import numpy as np
import pytest
import torch

from oracle import training_operators as op
from paper_2312_07987_b200 import binding, inputs

pytestmark = pytest.mark.gpu
TOL_Y, TOL_G = 1e-4, 2e-4          # max-abs error / RMS: the layer's own for outputs and for gradients (fp32 products, sums, atomics)
EPS = 1e-5
NAMES = ("Wq", "Wk", "Wv", "Wo", "Ws", "Wd")


def off(got, want):
    want = want.detach().numpy() if isinstance(want, torch.Tensor) else want
    return np.abs(got.detach().double().cpu().numpy() - want).max() / max(np.sqrt((want ** 2).mean()), 1e-30)


def reference(inp, G, causal=True, gains=None, base=None, balance=None, drop=None):
    """The layer's equations in fp64 (plain loops over heads and experts); gradients of sum(out G) + gloss loss."""
    c = inp.cfg
    B, T, M = inp.x.shape
    H, D, E, k, N = c.n_heads, c.d_head, c.n_experts, c.k, B * T
    leaf = lambda a: torch.tensor(np.asarray(a, dtype=np.float64), requires_grad=True)
    x, w = leaf(inp.x.reshape(N, M)), {n: leaf(getattr(inp, n)) for n in NAMES}
    gq, gk = (leaf(g) for g in gains) if gains is not None else (None, None)
    gate, loss, counts, probs = {}, torch.zeros((), dtype=torch.float64), [], []
    for side, W, bias in (("s", w["Ws"], inp.bias_s), ("d", w["Wd"], inp.bias_d)):
        z = torch.einsum("nm,hme->nhe", x, W) + (0 if bias is None else torch.tensor(bias, dtype=torch.float64))
        idx = torch.argsort(z.detach(), dim=2, descending=True, stable=True)[..., :k]
        gate[side] = torch.sigmoid(z) * torch.zeros_like(z).scatter(2, idx, 1.0)
        if balance is not None:
            kind, coef, mask, _ = balance
            keep = torch.ones(N, dtype=torch.float64) if mask is None else torch.tensor(mask, dtype=torch.float64)
            P = (torch.softmax(z, 2) * keep[:, None, None]).sum(0) / keep.sum()
            n = (torch.zeros_like(z).scatter(2, idx, 1.0) * keep[:, None, None]).sum(0)
            counts.append(n), probs.append(P)
            loss = loss + coef * (E * (n / n.sum(-1, keepdim=True) * P).sum() if kind == "counts" else (P * torch.log(P)).sum())
    seen = torch.ones(T, T, dtype=torch.bool).tril() if causal else torch.ones(T, T, dtype=torch.bool)
    ang = torch.arange(T, dtype=torch.float64)[:, None] * (base or 1.0) ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    y = torch.zeros(N, M, dtype=torch.float64)

    def finish(v, g):
        if gains is not None:
            v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * g
        if base is not None:
            a, b = v[..., 0::2], v[..., 1::2]
            v = torch.stack([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1).flatten(-2)
        return v

    for h in range(H):
        q, key = finish((x @ w["Wq"][h]).view(B, T, D), gq), finish((x @ w["Wk"][h]).view(B, T, D), gk)
        v = sum(gate["s"][:, h, e, None] * (x @ w["Wv"][h, e]) for e in range(E)).view(B, T, D)
        s = (q @ key.transpose(1, 2) / np.sqrt(D)).masked_fill(~seen, -np.inf)
        read = (torch.softmax(s, -1) @ v).reshape(N, D)
        for e in range(E):
            y = y + gate["d"][:, h, e, None] * (read @ w["Wo"][h, e])
    if drop is not None:
        kept, scale = drop
        y = y * torch.tensor(kept * scale)
    total = (y * torch.tensor(G.reshape(N, M), dtype=torch.float64)).sum() + (0 if balance is None else balance[3] * loss)
    wrt = [x] + [w[n] for n in NAMES] + ([gq, gk] if gains is not None else [])
    grads = dict(zip(["dx"] + ["d" + n for n in NAMES] + ["dgq", "dgk"], torch.autograd.grad(total, wrt)))
    grads["dx"] = grads["dx"].view(B, T, M)
    return dict(y=y.detach().view(B, T, M), loss=loss.detach(), counts=torch.stack(counts) if counts else None, prob=torch.stack(probs).detach() if probs else None, **grads)


def config(T, B, M, H, D, E, k):
    return inputs.LayerConfig("train", inputs.DTYPE_F32, B, T, M, H, D, E, k, seed=300 + T, zipf_bias=1.2 if E == 5 else 0.0)


def settings(cfg, what, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gains = [1 + 0.3 * torch.randn(cfg.d_head, generator=g, device="cuda") for _ in range(2)] if "norm" in what else None
    rng = torch.tensor([77 + seed, 1 << 35], device="cuda") if "dropout" in what else None
    mask = torch.rand(cfg.batch * cfg.seq, generator=g, device="cuda") < 0.8 if "mask" in what else None
    gloss = torch.full((), 500.0, device="cuda") if "balance" in what or "entropy" in what else None      # (a gradient that shows beside the task's)
    return gains, rng, mask, gloss


def check(cfg, what, causal=True):
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    layer.sh_set_causal(causal)
    x = binding.to_device(inp.x, cfg.dtype)
    G = np.random.default_rng(cfg.seed).standard_normal(inp.x.shape).astype(np.float32)
    gains, rng, mask, gloss = settings(cfg, what)
    p, kind = 0.2, "entropy" if "entropy" in what else "counts"
    if gains:
        layer.sh_set_qk_norm(*gains, eps=EPS)
    if "rope" in what:
        layer.sh_set_rope(10000.0)
    got = layer.sh_set_balance(kind, 0.02, mask, gloss) if gloss is not None else None
    if rng is not None:
        layer.sh_set_dropout(p, rng)
    for _ in range(2):                                     # (the second pass finds what the first left in the scratches)
        y = layer.sh_forward(x)
        back = layer.sh_backward(x, torch.from_numpy(G).cuda())
    torch.cuda.synchronize()
    assert layer.sh_last_status() == 0
    layer.sh_check_guards()
    N = cfg.batch * cfg.seq
    drop = op.dropout_kept(N, cfg.d_model, int(rng[0]), int(rng[1]), p) if rng is not None else None
    want = reference(inp, G, causal, [g.cpu() for g in gains] if gains else None, 10000.0 if "rope" in what else None,
                     (kind, 0.02, None if mask is None else mask.cpu().numpy(), 500.0) if gloss is not None else None, drop)
    assert off(y, want["y"]) < TOL_Y
    for n in [k for k in want if k.startswith("d")]:
        if not want[n].any():
            # one key: P = 1, and dS = P (dP - rowsum(dahat o ahat)) the difference of two fp32 sums of the same d_head products, taken in
            # two orders: 2 d_head U |dahat| |v| at most, which reaches these gradients through x and q or k - factors of dx's own terms
            assert float(back[n].abs().max()) < 4 * cfg.d_head * 2.0 ** -24 * float(want["dx"].abs().max()), n
            continue
        assert off(back[n], want[n]) < TOL_G, n
    if got:
        assert np.array_equal(got["counts"].cpu().numpy(), want["counts"].numpy())
        assert off(got["prob"], want["prob"]) < 1e-5 and abs(float(got["loss"]) - float(want["loss"])) < 1e-5 * abs(float(want["loss"])) + 1e-7
    layer.close()


ALL = ("norm", "rope", "entropy", "mask", "dropout")


@pytest.mark.parametrize("what", [("norm",), ("norm", "rope"), ("balance",), ("entropy", "mask"), ("dropout",), ALL])
def test_tiny(what):
    check(inputs.CONFIGS["tiny_f32"], what)


@pytest.mark.parametrize("shape,causal", [((70, 2, 128, 2, 40, 5, 3), True), ((33, 3, 64, 3, 64, 4, 1), False), ((150, 1, 192, 1, 132, 6, 2), True),
                                          ((340, 1, 128, 2, 76, 4, 2), True), ((1, 3, 64, 2, 32, 4, 2), True), ((17, 1, 64, 2, 16, 32, 4), True)])
def test_shapes(shape, causal):
    check(config(*shape), ALL, causal)


def test_odd_d_head_without_rotation():
    check(config(40, 2, 64, 2, 33, 4, 2), ("norm", "balance", "dropout"))


def test_settings_are_those_of_the_forward_pass_and_can_be_taken_back():
    cfg = inputs.CONFIGS["tiny_f32"]
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    G = torch.ones_like(x)
    plain, dplain = layer.sh_forward(x), layer.sh_backward(x, G)
    gains, rng, _, _ = settings(cfg, ("norm", "dropout"))
    layer.sh_set_qk_norm(*gains, eps=EPS)
    layer.sh_set_balance("counts", 0.1)
    layer.sh_set_dropout(0.3, rng)
    y = layer.sh_forward(x)
    dset = layer.sh_backward(x, G)
    assert not torch.equal(y, plain)
    layer.sh_set_qk_norm(eps=0.0)
    layer.sh_set_balance(None)
    layer.sh_set_dropout(0.0, None)
    torch.full((1 << 24,), float("nan"), device="cuda")    # (what memory that nobody holds has in it)
    again = layer.sh_backward(x, G)                        # still of the pass that was made
    for n in dset:
        assert float((again[n] - dset[n]).abs().max() / dset[n].abs().max()) < 1e-4, n
    back = layer.sh_forward(x)
    assert float((back - plain).abs().max() / plain.abs().max()) < 1e-5
    off_again = layer.sh_backward(x, G)
    assert set(off_again) == set(dplain)
    for n, w in dplain.items():
        assert float((off_again[n] - w).abs().max() / w.abs().max()) < 1e-4, n
    layer.close()


def test_other_gains_between_the_passes():
    cfg = inputs.CONFIGS["tiny_f32"]
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    G = torch.randn_like(x)
    gains, rng, _, _ = settings(cfg, ("norm", "dropout"))
    layer.sh_set_rope(10000.0)                             # (before the norms, which take it over)
    layer.sh_set_qk_norm(*gains, eps=EPS)
    layer.sh_set_dropout(0.3, rng)
    layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    layer.sh_forward(x)
    layer.sh_set_qk_norm(torch.zeros(cfg.d_head, device="cuda"), None, eps=EPS)
    layer.sh_set_dropout(0.9, torch.tensor([5, 5], device="cuda"))
    layer.sh_set_rope(0.0)
    for _ in range(8):
        torch.full((1 << 20,), float("nan"), device="cuda")
    got = layer.sh_backward(x, G)
    assert set(got) == set(want)
    for n in want:
        assert float((got[n] - want[n]).abs().max() / want[n].abs().max()) < 1e-4, n
    ref = reference(inp, G.cpu().numpy(), gains=[g.cpu() for g in gains], base=10000.0, drop=op.dropout_kept(64, cfg.d_model, int(rng[0]), int(rng[1]), 0.3))
    assert off(got["dgq"], ref["dgq"]) < TOL_G and off(got["dx"], ref["dx"]) < TOL_G
    layer.sh_configure(cfg.dtype, *inp.x.shape[:2])        # no settings any more
    layer.sh_set_weights(*[binding.to_device(a, cfg.dtype) for a in (inp.Wq, inp.Wk, inp.Wv, inp.Wo, inp.Ws, inp.Wd)])
    assert off(layer.sh_forward(x), reference(inp, G.cpu().numpy())["y"]) < TOL_Y
    assert "dgq" not in layer.sh_backward(x, G)
    layer.close()


def test_forward_only_settings_have_no_backward():
    cfg = inputs.CONFIGS["tiny_f32"]
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    layer.sh_set_qk_norm(eps=EPS, train=False)
    layer.sh_set_rope(10000.0)
    y = layer.sh_forward(x)
    with pytest.raises(binding.SwitchHeadError, match="NOT_CONFIGURED"):
        layer.sh_backward(x, torch.ones_like(x))
    ones = [np.ones(cfg.d_head)] * 2
    assert off(y, reference(inp, np.ones_like(inp.x), gains=ones, base=10000.0)["y"]) < TOL_Y
    layer.sh_set_qk_norm(eps=EPS)
    assert float((layer.sh_forward(x) - y).abs().max()) < 1e-5 * float(y.abs().max())
    layer.sh_backward(x, torch.ones_like(x))
    layer.sh_set_dropout(0.5, torch.tensor([1, 2], device="cuda"), train=False)
    layer.sh_forward(x)
    with pytest.raises(binding.SwitchHeadError, match="NOT_CONFIGURED"):
        layer.sh_backward(x, torch.ones_like(x))
    layer.close()


def test_standalone_operators_around_a_plain_pass():
    """The run of the operators as a user composes them: selections of sh_gate_topk, logits of their own, dropout with the residual."""
    cfg = config(70, 2, 128, 2, 40, 5, 3)
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    N, M = cfg.batch * cfg.seq, cfg.d_model
    rng = torch.tensor([5, 6], device="cuda")
    W = torch.stack([binding.to_device(w, cfg.dtype) for w in (inp.Ws, inp.Wd)])                          # [2, H, M, E]
    bias = torch.stack([torch.from_numpy(w).cuda() for w in (inp.bias_s, inp.bias_d)])
    z = (torch.einsum("nm,shme->nshe", x.view(N, M).double(), W.double()) + bias.double()).float()
    idx = layer.sh_gate_topk(x)[0]
    loss = binding.sh_balance_loss(z, idx, kind="entropy", coef=0.02)
    dz = binding.sh_balance_backward(z, loss["slope"])
    plain = layer.sh_forward(x)
    out = binding.sh_dropout(plain, rng, 0.2, residual=x)
    G = torch.randn_like(out)
    back = layer.sh_backward(x, binding.sh_dropout(G, rng, 0.2))
    dx = back["dx"].view(N, M) + G.view(N, M) + torch.einsum("nshe,shme->nm", dz, W)
    dWs = back["dWs"] + torch.einsum("nm,nhe->hme", x.view(N, M), dz[:, 0])
    Gn = G.cpu().numpy()
    want = reference(inp, Gn, balance=("entropy", 0.02, None, 1.0), drop=op.dropout_kept(N, M, 5, 6, 0.2))
    assert off(out, want["y"].numpy() + inp.x) < TOL_Y
    assert off(dx.view_as(x), want["dx"].numpy() + Gn) < TOL_G and off(dWs, want["dWs"]) < TOL_G
    # ... and as the layer's own settings
    got = layer.sh_set_balance("entropy", 0.02)
    layer.sh_set_dropout(0.2, rng)
    y = layer.sh_forward(x)
    own = layer.sh_backward(x, G)
    assert torch.equal(got["counts"], loss["counts"]) and abs(float(got["loss"]) - float(loss["loss"])) < 1e-5
    assert float((y + x - out).abs().max()) < 1e-4 * float(out.abs().max())
    assert float((own["dx"].view(N, M) + G.view(N, M) - dx).abs().max() / dx.abs().max()) < 1e-4
    layer.close()


def test_captured_training_step():
    cfg = config(70, 2, 128, 2, 40, 4, 2)
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    G = torch.randn_like(x)
    gains, rng, mask, gloss = settings(cfg, ALL)
    layer.sh_set_qk_norm(*gains, eps=EPS)
    layer.sh_set_rope(10000.0)
    got = layer.sh_set_balance("entropy", 0.02, mask, gloss)
    layer.sh_set_dropout(0.2, rng)
    step = lambda: (layer.sh_forward(x), layer.sh_backward(x, G))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, back = step()
    for turn in range(2):
        rng[1] += 1
        gains[0].mul_(1.1)
        G.normal_()
        graph.replay()
        y1, b1, l1 = y.clone(), {n: v.clone() for n, v in back.items()}, got["loss"].clone()
        y2, b2 = step()
        assert float((y1 - y2).abs().max()) < 1e-4 * float(y2.abs().max()) and torch.equal(l1, got["loss"])
        for n in b2:
            assert float((b1[n] - b2[n]).abs().max() / b2[n].abs().max()) < 1e-4, (turn, n)
    layer.close()


def test_cache_and_shared_selection():
    """Forward passes of layers without a backward: norms behind a cache, the balance loss of one gate for both sides."""
    cfg = config(60, 2, 128, 2, 40, 4, 2)
    inp = inputs.make_inputs(cfg)
    whole = binding.layer_from_inputs(inp)
    whole.sh_set_qk_norm(eps=EPS, train=False)
    x = binding.to_device(inp.x, cfg.dtype)
    want = whole.sh_forward(x)
    part = binding.layer_from_inputs(inp, cache_len=32)
    part.sh_set_qk_norm(eps=EPS, train=False)
    part.sh_set_dropout(0.5, torch.tensor([1, 2], device="cuda"), train=False)
    y = part.sh_forward(x)
    kept, scale = op.dropout_kept(2 * 28, cfg.d_model, 1, 2, 0.5)
    ref = want[:, 32:].reshape(56, -1).double().cpu().numpy() * kept * scale
    assert off(y.reshape(56, -1), ref) < TOL_Y
    one = binding.layer_from_inputs(inp, shared_selection=True)
    got = one.sh_set_balance("counts", 1.0)
    one.sh_forward(x)
    idx = one.sh_gate_topk(x)[0]
    z = torch.einsum("nm,hme->nhe", x.view(-1, cfg.d_model).double(), binding.to_device(inp.Ws, cfg.dtype).double())[:, None].float().contiguous()
    alone = binding.sh_balance_loss(z, idx[:1].contiguous())
    assert torch.equal(got["counts"], alone["counts"]) and torch.allclose(got["prob"], alone["prob"], atol=1e-5) and abs(float(got["loss"] - alone["loss"])) < 1e-4
    for l in (whole, part, one):
        l.close()


def test_refusals():
    cfg = inputs.CONFIGS["tiny_f32"]
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    ones = torch.ones(cfg.d_head, device="cuda")
    layer.sh_set_xl_positions(torch.zeros(cfg.n_heads, cfg.d_model, cfg.d_head, device="cuda"))
    with pytest.raises(binding.SwitchHeadError, match="relative-position"):
        layer.sh_set_qk_norm(ones, ones)
    layer.sh_set_xl_positions(None)
    layer.sh_set_qk_norm(ones, ones)
    with pytest.raises(binding.SwitchHeadError, match="relative-position"):
        layer.sh_set_xl_positions(torch.zeros(cfg.n_heads, cfg.d_model, cfg.d_head, device="cuda"))
    with pytest.raises(binding.SwitchHeadError, match="eps"):
        layer.sh_set_qk_norm(eps=-1.0)
    with pytest.raises(binding.SwitchHeadError, match="p must"):
        layer.sh_set_dropout(2.0, torch.tensor([1, 2], device="cuda"))
    layer.close()
    bf = binding.layer_from_inputs(inputs.make_inputs(inputs.CONFIGS["small_bf16"], batch=1))
    for call in (lambda: bf.sh_set_qk_norm(), lambda: bf.sh_set_balance("counts"), lambda: bf.sh_set_dropout(0.1, torch.tensor([1, 2], device="cuda"))):
        with pytest.raises(binding.SwitchHeadError, match="UNSUPPORTED"):
            call()
    bf.close()
