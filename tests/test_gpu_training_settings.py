"""Calls of the training operators and of the layer's training settings in combinations that their own tests do not make: inputs
whose rows overlap, settings switched between the passes, refused calls, a cache, and sizes above the small kernels' limits."""
import pytest
import torch

from paper_2312_07987_b200 import binding, inputs

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
