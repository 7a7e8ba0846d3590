"""What the binding does around the training operators and the layer's training settings, without a GPU."""
import os
import subprocess
import sys
import types

import pytest
import torch

from paper_2312_07987_b200 import binding as b
from tests import test_training_operators_host as given


@pytest.mark.parametrize("shape,strides", [((2, 3, 2, 8), (100, 1, 40, 1)), ((3, 4, 2, 16), (4, 12, 1, 1)), ((2, 3, 2, 8), (0, 1, 0, 1)), ((2, 3, 2, 8), (1, 1, 1, 1)),
                                           ((2, 3, 2, 8), (48, 8, 24, 1)), ((2, 3, 2, 1), (6, 2, 1, 5)), ((2, 0, 2, 8), (0, 1, 0, 1)), ((1, 1, 1, 2), (7, 7, 7, 1))])
def test_outputs_of_heads_have_dense_rows_of_their_own(shape, strides):
    t = torch.zeros(1000).as_strided(shape, strides)
    out, (at, *_, ) = b._heads_like(t)
    assert out.shape == t.shape and out.dtype == t.dtype and at == out.data_ptr()
    assert out.stride(3) == 1 or shape[3] == 1
    if out.numel():
        places = torch.zeros(out.untyped_storage().nbytes() // 4, dtype=torch.int32)
        places.as_strided(out.shape, out.stride()).fill_(1)
        assert int(places.sum()) == out.numel()              # no two elements at one address


def test_outputs_of_heads_keep_the_order_of_dimensions():
    for t in (torch.zeros(2, 5, 3, 8), torch.zeros(2, 3, 5, 8).transpose(1, 2)):
        out, fields = b._heads_like(t)
        assert out.stride() == t.stride() and fields == (out.data_ptr(), *t.stride()[:3])


class OnDevice(torch.Tensor):
    """A host tensor that passes for one on the device: what calls it is a stand-in for the library."""
    is_cuda = True
    used = ()

    def record_stream(self, stream):
        self.used += (stream.cuda_stream,)


def device_tensor(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def layer(monkeypatch):
    """A Layer over a library that notes its calls, and refuses those whose name is in layer.refuse."""
    one = object.__new__(b.Layer)
    one.handle, one.dense, one.shared_selection, one.dims = None, False, False, (128, 2, 32, 4, 2)
    one.workspace, one.dtype, one.batch, one.seq, one.seq_out = torch.empty(1), b.SH_F32, 2, 8, 8
    one._settings, one._of_forward, one._captured = {}, {}, {}
    one.calls, one.refuse = [], set()
    for name in ("sh_set_qk_norm", "sh_set_balance", "sh_set_dropout", "sh_set_rope", "sh_forward", "sh_forward_timed", "sh_forward_stamped", "sh_backward"):
        monkeypatch.setattr(b.lib, name, lambda *a, name=name: one.calls.append((name, a)) or (-1 if name in one.refuse else 0))
    monkeypatch.setattr(b.lib, "sh_training_scratch_bytes", lambda *a: 64)
    monkeypatch.setattr(b, "_stream", lambda: None)
    one.stream = types.SimpleNamespace(cuda_stream=0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: one.stream)
    one.capturing = False
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: one.capturing)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: None)
    return one


@pytest.mark.parametrize("train", [True, False])
def test_norms_that_are_off_have_no_gradients(layer, train):
    gains = device_tensor(32), device_tensor(32)
    layer.sh_set_qk_norm(*gains)
    assert len(layer._settings["qk_norm"]) == 5
    layer.sh_set_qk_norm(*gains, eps=0.0, train=train)
    assert layer.calls[-1] == ("sh_set_qk_norm", (None, None, None, 0.0, None, None, None, 0))
    x = device_tensor(2, 8, 128)
    layer.sh_forward(x)
    assert "qk_norm" not in layer._of_forward and set(layer.sh_backward(x, x)) == {"dx", "dWq", "dWk", "dWv", "dWo", "dWs", "dWd"}


@pytest.mark.parametrize("eps", [1e-46, -1e-60, 5e-324])
def test_an_eps_that_rounds_to_zero_is_refused(layer, eps):
    layer.sh_set_qk_norm(device_tensor(32), None)
    had, calls = dict(layer._settings), len(layer.calls)
    with pytest.raises(ValueError, match="eps"):
        layer.sh_set_qk_norm(device_tensor(32), None, eps=eps)
    assert layer._settings == had and len(layer.calls) == calls


@pytest.mark.parametrize("name", ["sh_forward", "sh_forward_timed", "sh_forward_stamped"])
def test_a_refused_pass_leaves_the_one_before_it(layer, name):
    """Its tensors live on, and sh_backward's gradients of gains are its own."""
    gq, x = device_tensor(32), device_tensor(2, 8, 128)
    layer.sh_set_qk_norm(gq)
    rng = device_tensor(2, dtype=torch.int64)
    layer.sh_set_dropout(0.1, rng)
    layer.sh_forward(x)
    of_pass = dict(layer._settings)
    assert layer._of_forward == of_pass
    layer.sh_set_qk_norm(None, device_tensor(32))
    layer.sh_set_dropout(0.5, device_tensor(2, dtype=torch.int64))
    layer.refuse = {name}
    with pytest.raises(b.SwitchHeadError):
        getattr(layer, name)(x, x)
    assert layer._of_forward is not layer._settings and all(layer._of_forward[n] is of_pass[n] for n in of_pass)
    assert "dgq" in layer.sh_backward(x, x) and "dgk" not in layer.sh_backward(x, x)
    layer.refuse = set()
    getattr(layer, name)(x, x)
    assert layer._of_forward == layer._settings and "dgk" in layer.sh_backward(x, x)


WITHOUT = """
import torch
names = {n: getattr(torch._C, n) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream") if hasattr(torch._C, n)}
for n in names:
    delattr(torch._C, n)
from paper_2312_07987_b200 import binding as b
for n, f in names.items():                                   # (torch.cuda's functions call them)
    setattr(torch._C, n, f)
assert b._current_device is torch.cuda.current_device and b._raw_stream is not names.get("_cuda_getCurrentRawStream")
"""


def run_without_private_names(more=""):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", WITHOUT + more], check=True, cwd=root, timeout=300)


def test_the_binding_needs_no_private_names_of_torch():
    run_without_private_names("""
class Stream:
    cuda_stream = 77
torch.cuda.current_stream = lambda device: Stream if device == 3 else None
assert b._raw_stream(3) == 77
""")


@pytest.mark.gpu
def test_calls_without_private_names_of_torch():
    run_without_private_names("""
x, rng = torch.ones(64, 64, device="cuda"), torch.tensor([1, 2], device="cuda")
side = torch.cuda.Stream()
side.wait_stream(torch.cuda.current_stream())
with torch.cuda.stream(side):
    assert b._raw_stream(0) == side.cuda_stream
    y = b.sh_dropout(x, rng, 0.5)
side.synchronize()
assert torch.equal(y, b.sh_dropout(x, rng, 0.5)) and set(y.unique().tolist()) == {0.0, 2.0}
""")


@pytest.mark.parametrize("stride", [1, 31, -31])
@pytest.mark.parametrize("which", ["batch_stride", "token_stride", "head_stride"])
def test_heads_of_an_output_that_overlap_are_refused(which, stride):
    for fn, backward in ((b.lib.sh_qk_norm, False), (b.lib.sh_qk_norm_backward, True)):
        for out in ("q_out", "k_out"):
            assert fn(given.norm_args({out: {which: stride}}, backward), None) == -1 and "share an address" in b.sh_last_error()
    # (a dimension of one has no stride)
    size = dict(batch_stride=dict(batch=1), token_stride=dict(seq=1), head_stride=dict(q_heads=1, k_heads=1))[which]
    fn = b.lib.sh_qk_norm
    assert fn(given.norm_args(dict(q_out={which: stride}, k=dict(data=0)), **size), None) == -1 and "k and k_out" in b.sh_last_error()


def test_other_outputs_that_overlap_are_refused():
    for stride in (15, 1, -15):                              # sides * heads * experts = 16
        assert b.lib.sh_balance_backward(given.balance_args(dtoken_stride=stride), None) == -1 and "share an address" in b.sh_last_error()
    f = dict(x=given.PTR, residual=0, y=given.PTR, rng=given.PTR, rows=4, cols=64, x_stride=64, residual_stride=64, y_stride=63, p=0.1, dtype=b.SH_F32, reserved=0)
    for stride in (63, 1, -63):
        f["y_stride"] = stride
        assert b.lib.sh_dropout(b._DROPOUT.pack(*[f[n] for n in given.DROPOUT]), None) == -1 and "share an address" in b.sh_last_error()


def test_settings_want_tensors_of_the_layer_s_device(layer):
    """Their pointers are kept, and read by kernels on that device."""
    gain, rng, mask, one = device_tensor(32), device_tensor(2, dtype=torch.int64), device_tensor(16, dtype=torch.bool), device_tensor(1)
    calls = (lambda: layer.sh_set_qk_norm(gain), lambda: layer.sh_set_qk_norm(None, gain), lambda: layer.sh_set_balance("counts", mask=mask),
             lambda: layer.sh_set_balance("counts", gloss=one), lambda: layer.sh_set_dropout(0.1, rng))
    for call in calls:
        call()
    layer.calls.clear()
    layer.workspace = types.SimpleNamespace(device=torch.device("cuda", 1))
    for call in calls:
        with pytest.raises(AssertionError):
            call()
    assert not layer.calls


def test_settings_note_the_streams_of_their_passes(layer):
    gain, rng, mask, x = device_tensor(32), device_tensor(2, dtype=torch.int64), device_tensor(16, dtype=torch.bool), device_tensor(2, 8, 128)
    layer.sh_set_qk_norm(gain)
    layer.sh_set_dropout(0.1, rng)
    layer.sh_set_balance("counts", mask=mask)
    for n, call in ((5, layer.sh_forward), (5, layer.sh_forward), (6, lambda x: layer.sh_backward(x, x)), (7, lambda x: layer.sh_forward_timed(x, x)), (8, lambda x: layer.sh_forward_stamped(x, x))):
        layer.stream.cuda_stream = n
        call(x)
    assert all(t.used == (5, 6, 7, 8) for t in (gain, rng, mask))      # once each
    layer.sh_set_dropout(0.2, device_tensor(2, dtype=torch.int64))
    layer.stream.cuda_stream = 9
    layer.sh_backward(x, x)                                            # of the pass before: with the tensors it had
    assert rng.used == (5, 6, 7, 8, 9) and layer._settings["dropout"][0].used == ()


@pytest.mark.parametrize("backward", [False, True])
def test_settings_of_a_captured_pass_live_on(layer, backward):
    """A replay uses them, whatever has been set since."""
    x = device_tensor(2, 8, 128)
    layer.sh_set_qk_norm(device_tensor(32))
    layer.sh_set_dropout(0.1, device_tensor(2, dtype=torch.int64))
    of_pass = list(layer._settings.values())
    if backward:
        layer.sh_forward(x)
    assert not layer._captured
    layer.capturing = True
    layer.sh_backward(x, x) if backward else layer.sh_forward(x)
    layer.capturing = False
    layer.sh_set_qk_norm(eps=0.0)
    layer.sh_set_dropout(0.0, None)
    layer.sh_forward(x)
    assert len(layer._captured) == 2 and all(any(k is kept for k in layer._captured.values()) for kept in of_pass)
