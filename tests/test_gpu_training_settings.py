"""Calls of the training operators and of the layer's training settings in combinations that their own tests do not make: inputs
whose rows overlap, settings switched between the passes, refused calls, a cache, and sizes above the small kernels' limits."""
import numpy as np
import pytest
import torch

from paper_2312_07987_b200 import binding, inputs
from tests import test_gpu_training_operators as given

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("strides", [(100, 1, 40, 1), (1, 1, 1, 1), (0, 3, 0, 1), (200, 8, 0, 1)])
def test_norm_of_rows_that_overlap(strides):
    """Inputs may share addresses (windows of one buffer, one row for all heads): what a copy of their own gives."""
    q = torch.randn(400, device="cuda").as_strided((2, 3, 2, 8), strides)
    dq = torch.randn(400, device="cuda").as_strided((2, 3, 2, 8), strides[2::-1] + (1,))
    gain = torch.randn(8, device="cuda")
    own, down = q.contiguous(), dq.contiguous()
    kw = dict(rotated=8, halves=True, q_scale=0.5)
    y, yk = binding.sh_qk_norm(q, q, gain, gain, **kw)
    want, wantk = binding.sh_qk_norm(own, own, gain, gain, **kw)
    assert y.stride(3) == yk.stride(3) == 1
    back, bwant = binding.sh_qk_norm_backward(q, q, dq, dq, gain, gain, **kw), binding.sh_qk_norm_backward(own, own, down, down, gain, gain, **kw)
    # Vectors are as wide as the addresses allow, so sums may go in another order.  A normalised value is at most sqrt(8) and its row's mean
    # magnitude at most 1; a result of either side is off by 40 roundings of these (sum, root, angle, products), a gradient by 80 of its terms
    # w (1 + sqrt(8)) / size, w the turned gradient times its gain, a gain's gradient by 100 of each of its 12 rows' terms.
    g, d = float(gain.abs().max()), 2 ** 0.5 * float(down.abs().max())
    size = float(own.square().mean(-1).sqrt().min())
    for got, ref, bound in ((y, want, 40 * 4 * g), (yk, wantk, 40 * 4 * g), (back["dq"], bwant["dq"], 80 * 4 * d * g / size), (back["dk"], bwant["dk"], 80 * 4 * d * g / size),
                            (back["dgq"], bwant["dgq"], 100 * 12 * 3 * d), (back["dgk"], bwant["dgk"], 100 * 12 * 3 * d)):
        assert float((got - ref).abs().max()) <= 2 * U * bound


def tiny_layer():
    inp = inputs.make_inputs(inputs.CONFIGS["tiny_f32"])
    return binding.layer_from_inputs(inp), binding.to_device(inp.x, inp.cfg.dtype)


def test_norms_switched_off_with_their_gains():
    """eps = 0 is off whatever else is given: a plain pass, and no gradients of gains that were not used."""
    layer, x = tiny_layer()
    G = torch.randn_like(x)
    plain, dplain = layer.sh_forward(x), layer.sh_backward(x, G)
    gains = [torch.full((layer.dims[2],), 1.5, device="cuda") for _ in range(2)]
    layer.sh_set_qk_norm(*gains)
    layer.sh_forward(x)
    assert {"dgq", "dgk"} < set(layer.sh_backward(x, G))
    layer.sh_set_qk_norm(*gains, eps=0.0)
    assert float((layer.sh_forward(x) - plain).abs().max() / plain.abs().max()) < 1e-5
    back = layer.sh_backward(x, G)
    assert set(back) == set(dplain)
    for n, w in dplain.items():
        assert float((back[n] - w).abs().max() / w.abs().max()) < 1e-4, n
    with pytest.raises(ValueError, match="eps"):
        layer.sh_set_qk_norm(*gains, eps=1e-46)
    layer.close()


def test_a_refused_pass_leaves_the_one_before_it():
    layer, x = tiny_layer()
    G, D = torch.randn_like(x), layer.dims[2]
    layer.sh_set_qk_norm(torch.rand(D, device="cuda"), None)
    layer.sh_set_balance("entropy", 0.1)
    layer.sh_set_dropout(0.3, torch.tensor([1, 2], device="cuda"))
    layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    layer.sh_set_qk_norm(None, torch.rand(D, device="cuda"))
    layer.sh_set_balance("counts", 0.1)
    layer.sh_set_dropout(0.6, torch.tensor([3, 4], device="cuda"))
    off = torch.empty(x.numel() + 1, device="cuda")[1:].view(x.shape)
    for call in (lambda: layer.sh_forward(off), lambda: layer.sh_forward(x, off), lambda: layer.sh_forward_timed(off, x), lambda: layer.sh_forward_stamped(off, x)):
        with pytest.raises(binding.SwitchHeadError, match="aligned"):
            call()
    for n in range(4, 25):
        torch.full((1 << n,), float("nan"), device="cuda")   # (what memory that nobody holds has in it)
    got = layer.sh_backward(x, G)
    assert set(got) == set(want) and "dgq" in got
    for n, w in want.items():
        assert float((got[n] - w).abs().max() / w.abs().max()) < 1e-4, n
    layer.close()


@pytest.mark.parametrize("later", ["rope", "rope and norms", "relative"])
def test_positions_switched_on_between_the_passes(later):
    """They are for the next forward pass: the one that was made had none, and is differentiated as it was."""
    layer, x = tiny_layer()
    G, (M, H, D, _, _) = torch.randn_like(x), layer.dims
    layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    plain = layer.sh_forward(x)
    if later == "relative":
        layer.sh_set_xl_positions(torch.randn(H, M, D, device="cuda"))
    else:
        layer.sh_set_rope(10000.0)
        if later == "rope and norms":
            layer.sh_set_qk_norm(torch.rand(D, device="cuda"), None)
    got = layer.sh_backward(x, G)
    assert set(got) == set(want)
    for n, w in want.items():
        assert float((got[n] - w).abs().max() / w.abs().max()) < 1e-4, n
    assert not torch.equal(layer.sh_forward(x), plain)
    if later == "rope and norms":
        assert "dgq" in layer.sh_backward(x, G)
    else:
        with pytest.raises(binding.SwitchHeadError, match="UNSUPPORTED"):
            layer.sh_backward(x, G)
    layer.close()


def test_rotation_of_norms_switched_on_behind_a_pass_without():
    """Norms in both passes, the rotation in the second only: each is differentiated as it was made."""
    layer, x = tiny_layer()
    G = torch.randn_like(x)
    layer.sh_set_qk_norm(torch.rand(layer.dims[2], device="cuda"), None)
    layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    layer.sh_set_rope(10000.0)
    got = layer.sh_backward(x, G)
    for n, w in want.items():
        assert float((got[n] - w).abs().max() / w.abs().max()) < 1e-4, n
    layer.sh_forward(x)
    turned = layer.sh_backward(x, G)
    assert float((turned["dWq"] - want["dWq"]).abs().max() / want["dWq"].abs().max()) > 1e-2
    layer.close()


def definition(z, idx, kind, coef, keep):
    """Loss, counts and probabilities of one side's gates in fp64: z [N, H, E], idx [N, H, k], keep [N]."""
    E, n = z.shape[2], int(keep.sum())
    P = (torch.softmax(z, -1) * keep[:, None, None]).sum(0) / n
    counts = ((idx.long()[..., None] == torch.arange(E, device=z.device)) & keep[:, None, None, None]).sum((0, 2))
    f = counts.double() / counts.sum(-1, keepdim=True)
    return coef * (E * (f * P).sum() if kind == "counts" else (P * torch.log(P)).sum()), counts, P


def layer_logits(inp, x):
    """The gates' logits [sides, N, H, E] in fp64, and how far the layer's fp32 sums over d_model may be from them."""
    N, M = inp.x.shape[0] * inp.x.shape[1], inp.cfg.d_model
    z, off = [], 0.0
    for W, bias in ((inp.Ws, inp.bias_s), (inp.Wd, inp.bias_d)):
        w, v = torch.from_numpy(np.asarray(W)).cuda().double(), x.view(N, M).double()
        z.append(torch.einsum("nm,hme->nhe", v, w) + (0 if bias is None else torch.from_numpy(bias).cuda().double()))
        off = max(off, float(torch.einsum("nm,hme->nhe", v.abs(), w.abs()).max()) * (M + 2) * U)
    return torch.stack(z), off


def check_statistics(got, want, kind, coef, z, off):
    """want: definition() of each side.  p is off by the logits' error twice (numerator and sum) and 18 roundings and those of its exponent, P by as much
    and 256 + N / 64 additions; the loss by that of its terms."""
    sides, N, H, E = z.shape
    assert torch.equal(got["counts"].long(), torch.stack([c for _, c, _ in want]))
    P = torch.stack([p for _, _, p in want])
    rel = 2 * off + (18 + 2 * float(z.abs().max()) + 256 + N / 64) * U
    assert float(((got["prob"].double() - P) / P).abs().max()) < rel
    scale = E if kind == "counts" else 1.0 + float(torch.log(P).abs().max())
    assert abs(float(got["loss"]) - float(sum(l for l, _, _ in want))) < coef * sides * H * scale * (rel + 4 * U)


@pytest.mark.parametrize("T,cache,B,H,E,k", [(60, 32, 2, 2, 4, 2), (40, 1, 3, 2, 5, 3), (33, 32, 2, 1, 8, 1), (1200, 500, 4, 8, 8, 2)])
@pytest.mark.parametrize("kind,masked", [("counts", False), ("entropy", True)])
def test_balance_behind_a_cache_counts_what_is_routed(T, cache, B, H, E, k, kind, masked):
    """The destination side has no tokens of the cache: its gates' counts, means and loss are the chunk's."""
    cfg = inputs.LayerConfig("cached", inputs.DTYPE_F32, B, T, 64, H, 32, E, k, seed=T)
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp, cache_len=cache)
    x = binding.to_device(inp.x, cfg.dtype)
    plain = layer.sh_forward(x)
    idx = layer.sh_gate_topk(x)[0]

    def some():
        m = torch.rand(B * T, device="cuda") < 0.6
        m[T - 1::T] = True                                   # (a chunk is never without a token)
        return m

    mask = some() if masked else None
    got = layer.sh_set_balance(kind, 0.1, mask)
    chunk = (torch.arange(T, device="cuda") >= cache).repeat(B)
    z, off = layer_logits(inp, x)

    def check():
        keep = torch.ones_like(chunk) if mask is None else mask
        check_statistics(got, [definition(z[0], idx[0], kind, 0.1, keep), definition(z[1], idx[1], kind, 0.1, keep & chunk)], kind, 0.1, z, off)

    y = layer.sh_forward(x)
    check()
    assert float((y - plain).abs().max()) < 1e-5 * float(plain.abs().max())
    layer.sh_check_guards()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.sh_forward(x, y)
    for t in got.values():
        t.zero_()
    if mask is not None:
        mask.copy_(some())                                   # (read by the pass, not before it)
    graph.replay()
    check()
    assert layer.sh_last_status() == 0
    layer.close()


def test_balance_of_a_shared_gate_behind_a_cache_counts_all():
    """One gate for both sides: its selections of the cached tokens serve their keys and values."""
    cfg = inputs.LayerConfig("cached", inputs.DTYPE_F32, 2, 50, 64, 2, 32, 4, 2, seed=5)
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp, shared_selection=True, cache_len=20)
    x = binding.to_device(inp.x, cfg.dtype)
    got = layer.sh_set_balance("counts", 0.1)
    layer.sh_forward(x)
    z, off = layer_logits(inp, x)
    keep = torch.ones(100, dtype=torch.bool, device="cuda")
    check_statistics(got, [definition(z[0], layer.sh_gate_topk(x)[0][0], "counts", 0.1, keep)], "counts", 0.1, z[:1], off)
    layer.close()


@pytest.mark.parametrize("kind,masked", [("counts", False), ("entropy", True)])
def test_balance_of_a_large_batch_in_the_layer(kind, masked):
    """More than 4096 tokens and 2^18 logits: the sort in blocks of 128 tokens, sums and loss in two launches out of the layer's scratch, and what
    sh_backward reads there; against the plain pass and the operators around it."""
    cfg = inputs.LayerConfig("large", inputs.DTYPE_F32, 9, 500, 64, 4, 32, 16, 3, seed=11, zipf_bias=1.2)
    N, H, E = 4500, 4, 16
    assert binding.lib.sh_balance_workspace_bytes(N, 2, H, E) > 0
    inp = inputs.make_inputs(cfg)
    layer = binding.layer_from_inputs(inp)
    x = binding.to_device(inp.x, cfg.dtype)
    G = torch.randn_like(x)
    mask = torch.rand(N, device="cuda") < 0.8 if masked else None
    gloss = torch.full((), 3e4, device="cuda")               # (a gradient that shows beside the task's)
    z, off = layer_logits(inp, x)
    idx = layer.sh_gate_topk(x)[0]
    zt = z.permute(1, 0, 2, 3).float().contiguous()
    alone = binding.sh_balance_loss(zt, idx, kind=kind, coef=0.1, mask=mask)
    dz = binding.sh_balance_backward(zt, alone["slope"], mask=mask, gloss=gloss)
    plain = layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    W = torch.stack([binding.to_device(w, cfg.dtype) for w in (inp.Ws, inp.Wd)])
    d = dz.double()
    share = dict(dx=torch.einsum("nshe,shme->nm", d, W.double()).view_as(x), dWs=torch.einsum("nm,nhe->hme", x.view(N, 64).double(), d[:, 0]),
                 dWd=torch.einsum("nm,nhe->hme", x.view(N, 64).double(), d[:, 1]))
    got = layer.sh_set_balance(kind, 0.1, mask, gloss)

    def check(y, back):
        keep = torch.ones(N, dtype=torch.bool, device="cuda") if mask is None else mask
        check_statistics(got, [definition(z[s], idx[s], kind, 0.1, keep) for s in range(2)], kind, 0.1, z, off)
        assert float((y - plain).abs().max()) < 1e-5 * float(plain.abs().max())
        for n, w in want.items():
            w = w.double() + share.get(n, 0.0)
            assert float((back[n].double() - w).abs().max() / w.square().mean().sqrt()) < 2e-4, n
            if n in share:                                   # (a loss that did not reach a gradient would be seen)
                assert float(share[n].abs().max() / w.square().mean().sqrt()) > 1e-2, n

    step = lambda: (layer.sh_forward(x), layer.sh_backward(x, G))
    for _ in range(2):
        check(*step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for t in (*got.values(), out[0], *out[1].values()):
        t.fill_(7)
    graph.replay()
    check(*out)
    assert layer.sh_last_status() == 0
    layer.sh_check_guards()
    layer.close()


@pytest.mark.parametrize("heads", [(1, 0), (12, 1), (3, 8)])
def test_gain_gradients_of_many_rows(heads):
    """Sums of one sign over hundreds of millions of rows (one row that all share): what a row gives times their number.  A thread's fp32 sum is of 512
    rows, joined in 32 bits over 32 groups of a block and the launches, beyond the blocks in 64."""
    B, T = 32, (1 << 27) // (32 * sum(heads)) + 3
    g = torch.Generator(device="cuda").manual_seed(3)
    row, drow = (torch.rand(1, 1, 1, 2, generator=g, device="cuda") + 0.3 for _ in range(2))
    gain = torch.tensor([0.7, 1.3], device="cuda")
    q, dq = (t.expand(B, T, heads[0], 2) for t in (row, drow))
    k, dk = (t.expand(B, T, heads[1], 2) if heads[1] else None for t in (row, drow))
    outs = []
    for _ in range(2):
        back = binding.sh_qk_norm_backward(q, k, dq, dk, gain, gain if heads[1] else None)
        one = binding.sh_qk_norm_backward(row, None, drow, None, gain)
        outs.append([back["dgq"]] + ([back["dgk"]] if heads[1] else []))
        assert all((back[n] == one["dq"]).all() for n in ("dq", "dk") if back[n] is not None)
        del back
    share = row.double() * drow.double() / torch.sqrt(row.double().square().mean(-1, keepdim=True) + 1e-6)
    # (a row's share: the sum of squares, root, two products: 10 U; 37 launches at most)
    for dg, n in zip(outs[0], heads):
        want = share.view(2) * (B * T * n)
        assert float(((dg.double() - want) / want).abs().max()) < (10 + 512 + 32 + 40) * U, (dg, want)
    assert all(torch.equal(a, c) for a, c in zip(*outs))
    torch.cuda.empty_cache()


def test_balance_of_tokens_that_share_their_logits():
    """The mean of one row's p over 2^28 tokens is p: a thread adds 256 of them in 32 bits, a launch of the sums is rounded once."""
    N = (1 << 28) + 12345
    g = torch.Generator(device="cuda").manual_seed(4)
    row = torch.randn(1, 1, 1, 4, generator=g, device="cuda")
    idx = torch.randint(-1, 5, (1, N, 1, 1), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.rand(N, generator=g, device="cuda") < 0.9
    got = binding.sh_balance_loss(row.expand(N, 1, 1, 4), idx, mask=mask)
    counts = torch.stack([((idx.view(-1) == e) & mask).sum() for e in range(4)])
    assert torch.equal(got["counts"].view(4).long(), counts)
    p = torch.softmax(row.double(), -1).view(4)
    off = float(((got["prob"].view(4).double() - p) / p).abs().max())
    assert off < (18 + 2 * float(row.abs().max()) + 256 + 12) * U, off
    del idx, mask
    torch.cuda.empty_cache()


@pytest.mark.parametrize("S,H,E,ty", [(2, 4, 32, torch.bfloat16), (1, 3, 20, torch.float32)])
def test_balance_sums_of_several_launches(S, H, E, ty):
    """Tokens of their own logits, selections and mask, more than one launch of the sums takes: every token counts once."""
    N, chunk = 6000007, 500000
    g = torch.Generator(device="cuda").manual_seed(E)
    z = torch.empty(N, S, H, E, dtype=ty, device="cuda").normal_(generator=g)
    idx = torch.randint(-1, E, (S, N, H, 2), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.rand(N, generator=g, device="cuda") < 0.5
    got, again = (binding.sh_balance_loss(z, idx, kind="entropy", mask=mask) for _ in range(2))
    assert all(torch.equal(got[n], again[n]) for n in got)
    P, counts = torch.zeros(S, H, E, dtype=torch.float64, device="cuda"), torch.zeros(S, H, E, dtype=torch.int64, device="cuda")
    for t in range(0, N, chunk):
        m = mask[t:t + chunk]
        P += (torch.softmax(z[t:t + chunk].double(), -1) * m[:, None, None, None]).sum(0)
        picks = torch.where(m[None, :, None, None], idx[:, t:t + chunk], -1).permute(0, 2, 1, 3).reshape(S, H, -1)
        counts += torch.stack([(picks == e).sum(-1) for e in range(E)], -1)
    P /= mask.sum()
    assert torch.equal(got["counts"].long(), counts)
    off = (18 + 2 * float(z.abs().max()) + 256 + 8) * U
    assert float(((got["prob"].double() - P) / P).abs().max()) < off
    loss = float((P * torch.log(P)).sum())
    assert abs(float(got["loss"]) - loss) < S * H * (1 + float(torch.log(P).abs().max())) * off
    del z, idx
    torch.cuda.empty_cache()


def test_memory_of_settings_waits_for_the_stream_of_their_passes():
    """Set on one stream, used by passes on another: let go of while these wait to run, it is nobody else's yet."""
    layer, x = tiny_layer()
    G = torch.randn_like(x)
    layer.sh_forward(x)
    want = layer.sh_backward(x, G)
    gains = [torch.rand(layer.dims[2], device="cuda") for _ in range(2)]
    for turn in range(2):
        layer.sh_set_qk_norm(*[g.clone() for g in gains])
        layer.sh_set_balance("counts")
        layer.sh_set_dropout(0.2, torch.tensor([1, 2], device="cuda"))
        if turn == 0:
            layer.sh_forward(x)
            first = layer.sh_backward(x, G)
            torch.cuda.synchronize()
            continue
        own = [t for kept in layer._settings.values() for t in kept if isinstance(t, torch.Tensor)]
        places = {t.untyped_storage().data_ptr() for t in own}
        sizes = [t.untyped_storage().nbytes() for t in own]
        del own
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(400_000_000)                   # (a fifth of a second)
            layer.sh_forward(x)
            got = layer.sh_backward(x, G)
        layer.sh_set_qk_norm(eps=0.0)
        layer.sh_set_balance(None)
        layer.sh_set_dropout(0.0, None)
        with torch.cuda.stream(side):
            layer.sh_forward(x)
            plain = layer.sh_backward(x, G)
        others = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
        assert not side.query() and not places & {t.untyped_storage().data_ptr() for t in others}
    side.synchronize()
    for a, w in ((got, first), (plain, want)):
        assert set(a) == set(w)
        for n in w:
            assert float((a[n] - w[n]).abs().max() / w[n].abs().max()) < 1e-4, n
    layer.close()


@pytest.mark.parametrize("ty", ["f32", "f16"])
@pytest.mark.parametrize("D,R,halves", [(132, 132, True), (140, 140, True), (188, 100, True), (130, 130, False), (166, 60, False), (190, 190, False), (194, 194, False)])
def test_norm_of_wide_heads_in_vectors_of_two(D, R, halves, ty):
    for B, T, Hq, Hk in ((1, 1, 1, 1), (3, 17, 5, 2)):
        given.test_norm_and_its_gradients((B, T, Hq, Hk, D, R, halves, "bthd", ty, 0.5), "packed")


def test_a_captured_step_outlives_its_settings():
    """Replayed after its settings have been switched off and their names taken by others, it still is the step that was captured."""
    layer, x = tiny_layer()
    G = torch.randn_like(x)
    layer.sh_set_qk_norm(torch.rand(layer.dims[2], device="cuda"), torch.rand(layer.dims[2], device="cuda"))
    layer.sh_set_balance("entropy", 0.1)
    layer.sh_set_dropout(0.2, torch.tensor([1, 2], device="cuda"))
    want = layer.sh_forward(x).clone(), layer.sh_backward(x, G)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = layer.sh_forward(x), layer.sh_backward(x, G)
    layer.sh_set_qk_norm(eps=0.0)
    layer.sh_set_balance(None)
    layer.sh_set_dropout(0.0, None)
    plain = layer.sh_forward(x).clone()
    held = [torch.full((1 << n,), float("nan"), device="cuda") for n in range(4, 22) for _ in range(4)]
    for _ in range(2):
        graph.replay()
        assert float((got[0] - want[0]).abs().max() / want[0].abs().max()) < 1e-5
        assert set(got[1]) == set(want[1]) and "dgk" in got[1]
        for n, w in want[1].items():
            assert float((got[1][n] - w).abs().max() / w.abs().max()) < 1e-4, n
        assert all(bool(h.isnan().all()) for h in held)
        assert float((layer.sh_forward(x) - plain).abs().max() / plain.abs().max()) < 1e-5
    layer.close()
