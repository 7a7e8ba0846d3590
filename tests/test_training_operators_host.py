"""Host-side checks of the training operators that need no GPU: refused arguments are refused before any CUDA call, with a
reason; the packed arguments have the header's layout."""
import pytest
import torch

from paper_2312_07987_b200 import binding as b

HEADS = ("data", "batch_stride", "token_stride", "head_stride")
NORM = ("gq", "gk", "positions", "base", "dtype", "batch", "seq", "q_heads", "k_heads", "d_head", "rotated", "halves", "positions_64", "eps", "q_scale", "reserved")
BACKWARD = ("dgq", "dgk", "workspace", "workspace_bytes")
BALANCE = ("n_tokens", "token_stride", "dtoken_stride", "logits", "idx", "mask", "gloss", "loss", "prob", "slope", "counts", "dlogits", "workspace", "workspace_bytes",
           "dtype", "kind", "sides", "n_heads", "n_experts", "k", "coef", "reserved")
DROPOUT = ("x", "residual", "y", "rng", "rows", "cols", "x_stride", "residual_stride", "y_stride", "p", "dtype", "reserved")
PTR = 0x1000          # never used as an address: each call below is refused


def norm_args(heads=None, backward=False, **kw):
    h = {n: dict(data=PTR, batch_stride=256, token_stride=64, head_stride=32) for n in ("q", "k", "q_out", "k_out", "dq", "dk")}
    for n, v in (heads or {}).items():
        h[n].update(v)
    f = dict(gq=0, gk=0, dgq=0, dgk=0, positions=0, workspace=0, workspace_bytes=0, base=10000.0, dtype=b.SH_F32, batch=2, seq=4, q_heads=2, k_heads=2, d_head=32, rotated=32,
             halves=0, positions_64=0, eps=1e-6, q_scale=1.0, reserved=0)
    f.update(kw)
    fields = [h[n][m] for n in list(h)[:4] for m in HEADS] + [f[n] for n in NORM]
    if not backward:
        return b._QK_NORM.pack(*fields)
    return b._QK_NORM_BACKWARD.pack(*fields, *[h[n][m] for n in ("dq", "dk") for m in HEADS], *[f[n] for n in BACKWARD])


@pytest.mark.parametrize("kw,heads,code,frag", [
    (dict(dtype=3), {}, -1, "dtype"), (dict(batch=-1), {}, -1, "batch"), (dict(seq=-1), {}, -1, "seq"), (dict(d_head=0), {}, -1, "d_head"),
    (dict(d_head=257), {}, -1, "d_head"), (dict(rotated=3), {}, -1, "rotated"), (dict(rotated=34), {}, -1, "rotated"), (dict(rotated=-2), {}, -1, "rotated"),
    (dict(d_head=33, rotated=32), {}, -2, "even d_head"), (dict(base=0.0), {}, -1, "base"), (dict(base=float("nan")), {}, -1, "base"), (dict(eps=0.0), {}, -1, "eps"),
    (dict(eps=float("nan")), {}, -1, "eps"), (dict(q_scale=float("inf")), {}, -1, "q_scale"), (dict(q_heads=-1), {}, -1, "heads"), ({}, dict(k=dict(data=0)), -1, "k and k_out"),
    ({}, dict(q_out=dict(data=0)), -1, "q_out"), ({}, dict(k_out=dict(token_stride=0)), -1, "share an address"), ({}, dict(q_out=dict(head_stride=0)), -1, "share an address"),
    ({}, dict(q=dict(data=PTR + 2)), -1, "aligned to 4"), (dict(gq=PTR + 2), {}, -1, "gains"), (dict(positions=PTR + 4, positions_64=1), {}, -1, "positions"),
])
def test_norm_refusals(kw, heads, code, frag):
    for fn, backward in ((b.lib.sh_qk_norm, False), (b.lib.sh_qk_norm_backward, True)):
        assert fn(norm_args(heads, backward, **kw), None) == code
        assert frag in b.sh_last_error()


def test_norm_backward_refusals():
    fn = b.lib.sh_qk_norm_backward
    assert fn(norm_args(dict(dq=dict(data=0)), True), None) == -1 and "dq" in b.sh_last_error()
    assert fn(norm_args(None, True, dgq=PTR), None) == -4 and "workspace" in b.sh_last_error()
    need = b.lib.sh_qk_norm_workspace_bytes(32)
    assert need > 0 and b.lib.sh_qk_norm_workspace_bytes(0) == 0 and b.lib.sh_qk_norm_workspace_bytes(257) == 0
    assert fn(norm_args(None, True, dgq=PTR, workspace=PTR + 8, workspace_bytes=need), None) == -4
    assert fn(norm_args(None, True, dgk=PTR, workspace=PTR, workspace_bytes=need - 1), None) == -4 and "too small" in b.sh_last_error()
    for f in (b.lib.sh_qk_norm, fn, b.lib.sh_balance_loss, b.lib.sh_balance_backward, b.lib.sh_dropout):
        assert f(None, None) == -1 and "NULL" in b.sh_last_error()


def test_norm_of_no_rows_needs_no_device():
    assert b.lib.sh_qk_norm(norm_args(batch=0), None) == 0
    assert b.lib.sh_qk_norm(norm_args(seq=0, rotated=0), None) == 0


def balance_args(**kw):
    f = dict(n_tokens=1 << 20, token_stride=16, dtoken_stride=16, logits=PTR, idx=PTR, mask=0, gloss=0, loss=PTR, prob=PTR, slope=PTR, counts=PTR, dlogits=PTR, workspace=PTR,
             workspace_bytes=1 << 30, dtype=b.SH_F32, kind=0, sides=2, n_heads=2, n_experts=4, k=2, coef=1.0, reserved=0)
    f.update(kw)
    return b._BALANCE.pack(*[f[n] for n in BALANCE])


@pytest.mark.parametrize("kw,code,frag", [
    (dict(dtype=b.SH_F16), -1, "dtype"), (dict(n_tokens=-1), -1, "n_tokens"), (dict(sides=0), -1, "sides"), (dict(n_heads=0), -1, "n_heads"), (dict(n_experts=33), -1, "n_experts"),
    (dict(sides=256, n_heads=256), -2, "65535"), (dict(logits=0), -1, "logits"), (dict(k=0), -1, "k must"), (dict(k=5), -1, "k must"), (dict(n_tokens=1 << 30), -2, "2^31"),
    (dict(kind=2), -1, "kind"), (dict(coef=float("nan")), -1, "coef"), (dict(idx=0), -1, "idx"), (dict(loss=0), -1, "loss"), (dict(counts=0), -1, "counts"),
    (dict(logits=PTR + 2), -1, "logits"), (dict(idx=PTR + 1), -1, "idx"), (dict(prob=PTR + 2), -1, "prob"), (dict(workspace=0), -4, "workspace"), (dict(workspace=PTR + 16), -4, "256"), (dict(workspace_bytes=100), -4, "too small"),
])
def test_balance_refusals(kw, code, frag):
    assert b.lib.sh_balance_loss(balance_args(**kw), None) == code
    assert frag in b.sh_last_error()


@pytest.mark.parametrize("kw,frag", [(dict(slope=0), "slope"), (dict(dlogits=0), "dlogits"), (dict(dtoken_stride=0), "share an address"), (dict(dtype=7), "dtype"), (dict(logits=0), "logits"), (dict(dlogits=PTR + 2), "dlogits"), (dict(gloss=PTR + 1), "gloss")])
def test_balance_backward_refusals(kw, frag):
    assert b.lib.sh_balance_backward(balance_args(**kw), None) == -1
    assert frag in b.sh_last_error()


def test_balance_workspace():
    need = lambda n, *a: b.lib.sh_balance_workspace_bytes(n, *a)
    assert need(1 << 20, 2, 8, 16) > need(1 << 20, 2, 2, 4) > 0 and need(1, 2, 40, 32) > 0
    assert need(1, 2, 2, 4) == 0                            # few rows: one launch without a workspace
    assert need(8, 0, 8, 16) == 0 and need(8, 1, 1, 33) == 0


@pytest.mark.parametrize("kw,code,frag", [
    (dict(dtype=5), -1, "dtype"), (dict(rows=-1), -1, "rows"), (dict(cols=-1), -1, "cols"), (dict(cols=1 << 31), -2, "cols"), (dict(rows=(1 << 32) + 1), -2, "rows"), (dict(p=-0.1), -1, "p must"),
    (dict(p=1.5), -1, "p must"), (dict(p=float("nan")), -1, "p must"), (dict(x=0), -1, "x, y"), (dict(y=0), -1, "x, y"), (dict(rng=0), -1, "rng"), (dict(rng=PTR + 4), -1, "rng"), (dict(x=PTR + 2), -1, "aligned"),
    (dict(residual=PTR + 1), -1, "aligned"),
    (dict(y_stride=0), -1, "share an address"),
])
def test_dropout_refusals(kw, code, frag):
    f = dict(x=PTR, residual=0, y=PTR, rng=PTR, rows=4, cols=64, x_stride=64, residual_stride=64, y_stride=64, p=0.1, dtype=b.SH_F32, reserved=0)
    f.update(kw)
    assert b.lib.sh_dropout(b._DROPOUT.pack(*[f[n] for n in DROPOUT]), None) == code
    assert frag in b.sh_last_error()


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 4, 2, 32)
    with pytest.raises(ValueError, match="CUDA"):
        b.sh_qk_norm(x, x)
    with pytest.raises(ValueError, match="CUDA"):
        b.sh_balance_loss(x, torch.zeros(4, 2, 2, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        b.sh_balance_backward(x, x)
    with pytest.raises(ValueError, match="CUDA"):
        b.sh_dropout(x, torch.zeros(2, dtype=torch.int64), 0.1)


def configured(dtype=b.SH_F32, **kw):
    import ctypes
    h = ctypes.c_void_p(b.lib.sh_create(128, 2, 32, 4, 2) if not kw else b.lib.sh_create_moe_qk(128, 2, 32, 4, 2, 1, 1, 0))
    assert b.lib.sh_configure(h, dtype, 2, 64) == 0
    return h


def test_layer_settings_refusals():
    lib, P = b.lib, PTR * 16
    bare = configured()
    assert lib.sh_training_scratch_bytes(None, 0) == 0
    assert lib.sh_set_qk_norm(None, None, None, 1e-6, None, None, None, 0) == -1
    for call in (lambda h: lib.sh_set_qk_norm(h, None, None, 1e-6, None, None, None, 0), lambda h: lib.sh_set_balance(h, 0, 1.0, None, P, P, P, None, P, 1 << 30),
                 lambda h: lib.sh_set_dropout(h, 0.1, P, None, 0)):
        assert call(bare) == -3 and "workspace" in b.sh_last_error()                  # no workspace yet
        bf = configured(b.SH_BF16)
        assert lib.sh_set_workspace(bf, P, lib.sh_workspace_bytes(bf)) == 0
        assert call(bf) == -2 and "fp32" in b.sh_last_error()
        lib.sh_destroy(bf)
    assert lib.sh_set_workspace(bare, P, lib.sh_workspace_bytes(bare)) == 0
    need = [lib.sh_training_scratch_bytes(bare, i) for i in range(4)]
    assert all(n > 0 for n in need[:3]) and need[3] == 0
    norm = lambda gq=None, gk=None, eps=1e-6, dgq=None, dgk=None, s=None, n=0: lib.sh_set_qk_norm(bare, gq, gk, eps, dgq, dgk, s, n)
    for args, code, frag in ((dict(eps=-1.0), -1, "eps"), (dict(eps=float("nan")), -1, "eps"), (dict(gq=P + 2), -1, "aligned"), (dict(dgq=P), -1, "scratch"),
                             (dict(s=P + 8, n=1 << 30), -4, "256"), (dict(s=P, n=need[0] - 1), -4, "too small")):
        assert norm(**args) == code and frag in b.sh_last_error(), args
    assert norm(s=P, n=need[0]) == 0 and norm(eps=0.0) == 0
    bal = lambda kind=0, coef=1.0, loss=P, counts=P, prob=P, s=P, n=1 << 30: lib.sh_set_balance(bare, kind, coef, None, loss, counts, prob, None, s, n)
    for args, code, frag in ((dict(kind=5), -1, "kind"), (dict(coef=float("inf")), -1, "coef"), (dict(loss=None), -1, "loss"), (dict(counts=P + 1), -1, "aligned"),
                             (dict(s=None), -4, "scratch"), (dict(n=need[1] - 1), -4, "too small")):
        assert bal(**args) == code and frag in b.sh_last_error(), args
    assert bal() == 0 and bal(loss=None, s=None) == 0
    drop = lambda p=0.1, rng=P, s=None, n=0: lib.sh_set_dropout(bare, p, rng, s, n)
    for args, code, frag in ((dict(p=1.1), -1, "p must"), (dict(p=float("nan")), -1, "p must"), (dict(rng=P + 4), -1, "rng"), (dict(s=P + 1, n=1 << 30), -4, "256"),
                             (dict(s=P, n=need[2] - 1), -4, "too small")):
        assert drop(**args) == code and frag in b.sh_last_error(), args
    assert drop(s=P, n=need[2]) == 0 and drop(rng=None) == 0
    moe = configured(moe=True)
    assert lib.sh_set_workspace(moe, P, lib.sh_workspace_bytes(moe)) == 0
    assert lib.sh_set_qk_norm(moe, None, None, 1e-6, None, None, None, 0) == -2 and "experts" in b.sh_last_error()
    lib.sh_destroy(moe)
    lib.sh_destroy(bare)
