"""ctypes binding of libswitchhead.so: argument marshalling only.

Every step of the forward pass runs in the library's CUDA kernels; torch is used here for
device memory and streams.  Function names mirror the C ABI (include/switchhead.h).
There is no CPU fallback: if the library cannot be loaded, importing this module fails.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from typing import Optional

import numpy as np
import torch

from . import build as _build

SH_F32, SH_BF16, SH_F16 = 0, 1, 2
SH_BALANCE = dict(counts=0, entropy=1)
SH_OK = 0
ERROR_NAMES = {-1: "SH_ERR_INVALID_ARG", -2: "SH_ERR_UNSUPPORTED", -3: "SH_ERR_NOT_CONFIGURED",
               -4: "SH_ERR_WORKSPACE", -5: "SH_ERR_CUDA", -6: "SH_ERR_TIMEOUT", -7: "SH_ERR_BOUNDS"}
BUF = dict(Q=0, K=1, V=2, AHAT=3, IDX=4, GATE=5, OFFSETS=6, LISTS=7)

EXPORTS = ["sh_create", "sh_create_shared", "sh_create_moe_qk", "sh_create_dense", "sh_configure", "sh_configure_xl", "sh_workspace_bytes", "sh_set_workspace",
           "sh_set_weights", "sh_set_causal", "sh_set_rope", "sh_set_xl_positions", "sh_forward", "sh_backward", "sh_forward_timed", "sh_forward_stamped", "sh_gate_topk",
           "sh_noalloc_gate_topk", "sh_debug_buffer", "sh_last_status", "sh_status_block", "sh_clear_status", "sh_check_guards",
           "sh_selftest", "sh_set_output_f16", "sh_is_debug_build", "sh_launch_count", "sh_last_error", "sh_destroy",
           "sh_qk_norm", "sh_qk_norm_backward", "sh_qk_norm_workspace_bytes", "sh_balance_loss", "sh_balance_backward",
           "sh_balance_workspace_bytes", "sh_dropout", "sh_training_scratch_bytes", "sh_set_qk_norm", "sh_set_balance", "sh_set_dropout"]
STAMP_KERNELS = ["gate", "sort", "qk_a", "qk_b", "v", "attn", "o"]


def _load() -> ctypes.CDLL:
    path = os.environ.get("SWITCHHEAD_LIB") or _build.LIB_PATH     # a custom build of the library
    if not os.path.exists(path):
        path = _build.build()
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.sh_create.restype = vp
    lib.sh_create.argtypes = [i32] * 5
    lib.sh_create_shared.restype = vp
    lib.sh_create_shared.argtypes = [i32] * 5
    lib.sh_create_moe_qk.restype = vp
    lib.sh_create_moe_qk.argtypes = [i32] * 8
    lib.sh_create_dense.restype = vp
    lib.sh_create_dense.argtypes = [i32] * 3
    lib.sh_configure.restype = i32
    lib.sh_configure.argtypes = [vp, i32, i32, i32]
    lib.sh_configure_xl.restype = i32
    lib.sh_configure_xl.argtypes = [vp, i32, i32, i32, i32]
    lib.sh_workspace_bytes.restype = sz
    lib.sh_workspace_bytes.argtypes = [vp]
    lib.sh_set_workspace.restype = i32
    lib.sh_set_workspace.argtypes = [vp, vp, sz]
    lib.sh_set_weights.restype = i32
    lib.sh_set_weights.argtypes = [vp] * 10
    lib.sh_forward.restype = i32
    lib.sh_forward.argtypes = [vp, vp, vp, vp]
    lib.sh_backward.restype = i32
    lib.sh_backward.argtypes = [vp] * 11
    lib.sh_forward_timed.restype = i32
    lib.sh_forward_timed.argtypes = [vp, vp, vp, vp, ctypes.POINTER(ctypes.c_float)]
    lib.sh_forward_stamped.restype = i32
    lib.sh_forward_stamped.argtypes = [vp, vp, vp, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.sh_status_block.restype = i32
    lib.sh_status_block.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
    lib.sh_clear_status.restype = i32
    lib.sh_clear_status.argtypes = [vp, vp]
    lib.sh_check_guards.restype = i32
    lib.sh_check_guards.argtypes = [vp, vp]
    lib.sh_selftest.restype = i32
    lib.sh_selftest.argtypes = [vp, i32, ctypes.c_uint64, vp]
    lib.sh_is_debug_build.restype = i32
    lib.sh_is_debug_build.argtypes = []
    lib.sh_gate_topk.restype = i32
    lib.sh_gate_topk.argtypes = [vp] * 7
    lib.sh_noalloc_gate_topk.restype = i32
    lib.sh_noalloc_gate_topk.argtypes = [i32] * 6 + [vp] * 8
    lib.sh_set_causal.restype = i32
    lib.sh_set_causal.argtypes = [vp, i32]
    lib.sh_set_xl_positions.restype = i32
    lib.sh_set_xl_positions.argtypes = [vp, vp, vp, vp, vp]
    lib.sh_set_rope.restype = i32
    lib.sh_set_rope.argtypes = [vp, ctypes.c_double, vp]
    lib.sh_debug_buffer.restype = i32
    lib.sh_debug_buffer.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(sz)]
    lib.sh_last_status.restype = i32
    lib.sh_last_status.argtypes = [vp, vp]
    lib.sh_set_output_f16.restype = i32
    lib.sh_set_output_f16.argtypes = [vp, i32]
    lib.sh_launch_count.restype = i32
    lib.sh_launch_count.argtypes = [vp]
    lib.sh_last_error.restype = ctypes.c_char_p
    lib.sh_last_error.argtypes = []
    for name in ("sh_qk_norm", "sh_qk_norm_backward", "sh_balance_loss", "sh_balance_backward", "sh_dropout"):
        getattr(lib, name).restype = i32
        getattr(lib, name).argtypes = [ctypes.c_char_p, vp]      # a packed struct of arguments; the stream
    lib.sh_qk_norm_workspace_bytes.restype = sz
    lib.sh_qk_norm_workspace_bytes.argtypes = [i32]
    lib.sh_balance_workspace_bytes.restype = sz
    lib.sh_balance_workspace_bytes.argtypes = [ctypes.c_int64] + [i32] * 3
    lib.sh_training_scratch_bytes.restype = sz
    lib.sh_training_scratch_bytes.argtypes = [vp, i32]
    lib.sh_set_qk_norm.restype = i32
    lib.sh_set_qk_norm.argtypes = [vp, vp, vp, ctypes.c_float, vp, vp, vp, sz]
    lib.sh_set_balance.restype = i32
    lib.sh_set_balance.argtypes = [vp, i32, ctypes.c_float] + [vp] * 6 + [sz]
    lib.sh_set_dropout.restype = i32
    lib.sh_set_dropout.argtypes = [vp, ctypes.c_double, vp, vp, sz]
    lib.sh_destroy.restype = None
    lib.sh_destroy.argtypes = [vp]
    return lib


lib = _load()


class SwitchHeadError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        msg = lib.sh_last_error().decode()
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {msg}")


def _check(code: int) -> None:
    if code != SH_OK:
        raise SwitchHeadError(code)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def sh_last_error() -> str:
    return lib.sh_last_error().decode()


class _Kept(tuple):
    """The tensors of a training setting.  They were made on the stream that was current then; the passes may run on others."""

    def used_on(self, stream) -> None:
        """Their memory is not given to anybody before what `stream` holds now and later, until they are let go of, is done."""
        streams = self.__dict__.setdefault("streams", set())
        if stream.cuda_stream not in streams:
            streams.add(stream.cuda_stream)
            for t in self:
                for one in t.values() if isinstance(t, dict) else (t,):
                    if one is not None:
                        one.record_stream(stream)


class Layer:
    """Owns one sh_layer handle plus the torch tensors that back its workspace."""

    def __init__(self, d_model: int, n_heads: int, d_head: int, n_experts: int = 1, k: int = 1,
                 dense: bool = False, shared_selection: bool = False, moe_q: bool = False, moe_k: bool = False):
        self.dense = dense
        self.shared_selection = shared_selection
        self.dims = (d_model, n_heads, d_head, n_experts, k)
        if dense:
            h = lib.sh_create_dense(d_model, n_heads, d_head)
        elif moe_q or moe_k:
            h = lib.sh_create_moe_qk(d_model, n_heads, d_head, n_experts, k, int(moe_q), int(moe_k), int(shared_selection))
        elif shared_selection:
            h = lib.sh_create_shared(d_model, n_heads, d_head, n_experts, k)
        else:
            h = lib.sh_create(d_model, n_heads, d_head, n_experts, k)
        if not h:
            raise SwitchHeadError(-1)
        self.handle = ctypes.c_void_p(h)
        self.workspace = None
        self.dtype = None
        self.batch = self.seq = 0
        self._settings, self._of_forward, self._captured = {}, {}, {}

    def sh_configure(self, dtype: int, batch: int, seq: int, device="cuda", cache_len: int = 0) -> None:
        """cache_len > 0: Transformer-XL context (sh_configure_xl): x is [B, cache_len + seq, M], out [B, seq, M]."""
        if cache_len:
            _check(lib.sh_configure_xl(self.handle, dtype, batch, seq, cache_len))
        else:
            _check(lib.sh_configure(self.handle, dtype, batch, seq))
        # (self.seq: tokens per sequence the layer sees, cache included; self.seq_out: rows of out per sequence)
        self.dtype, self.batch, self.seq, self.seq_out = dtype, batch, cache_len + seq, seq
        nbytes = lib.sh_workspace_bytes(self.handle)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self._settings = {}                                # tensors that the training settings read and write, by setting ...
        self._of_forward = {}                              # ... those of the last forward pass, which sh_backward differentiates ...
        self._captured = {}                                # ... and those of captured passes
        _check(lib.sh_set_workspace(self.handle, ctypes.c_void_p(self._ws_ptr), nbytes))

    def sh_set_weights(self, Wq, Wk, Wv, Wo, Ws=None, Wd=None, bias_s=None, bias_d=None) -> None:
        ts = [Wq, Wk, Wv, Wo, Ws, Wd, bias_s, bias_d]
        for t in ts:
            assert t is None or (t.is_cuda and t.is_contiguous())
        _check(lib.sh_set_weights(self.handle, *[_ptr(t) for t in ts], _stream()))
        torch.cuda.current_stream().synchronize()   # the source tensors may now be released

    def sh_set_causal(self, causal: bool) -> None:
        _check(lib.sh_set_causal(self.handle, 1 if causal else 0))

    def sh_set_xl_positions(self, Wr, u=None, v=None) -> None:
        """Transformer-XL relative-position term (fp32 layers): Wr [H, M, D], u, v [H, D] fp32 device tensors; None switches it off."""
        for t in (Wr, u, v):
            assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == torch.float32)
        _check(lib.sh_set_xl_positions(self.handle, _ptr(Wr), _ptr(u), _ptr(v), _stream()))
        torch.cuda.current_stream().synchronize()   # the source tensors may now be released

    def sh_set_rope(self, base: float) -> None:
        _check(lib.sh_set_rope(self.handle, float(base), _stream()))

    def _scratch(self, which: int):
        """A scratch of a training setting, and its bytes."""
        n = lib.sh_training_scratch_bytes(self.handle, which)
        return torch.empty(n, dtype=torch.uint8, device=self.workspace.device) if n else None, n

    def _mine(self, t: Optional[torch.Tensor]) -> bool:
        """Whether a tensor that the passes will read is on the layer's device (without a workspace the call itself is refused)."""
        return t is None or (t.is_cuda and (self.workspace is None or t.device == self.workspace.device))

    def sh_set_qk_norm(self, gq=None, gk=None, eps: float = 1e-6, train: bool = True) -> None:
        """Q and K normalised per head between projection and attention (fp32 layers), gains gq, gk [d_head] fp32 device tensors or None;
        eps = 0 switches it off.  train: sh_backward returns dgq and dgk of the gains that are given."""
        D = self.dims[2]
        for g in (gq, gk):
            assert self._mine(g) and (g is None or (g.is_contiguous() and g.dtype == torch.float32 and tuple(g.shape) == (D,)))
        if ctypes.c_float(eps).value == 0.0:               # (as the call takes it; off: no gains, so no gradients of them)
            if eps != 0.0:
                raise ValueError(f"eps must be 0 (off) or at least fp32's smallest positive value: got {eps}")
            _check(lib.sh_set_qk_norm(self.handle, None, None, 0.0, None, None, None, 0))
            self._settings.pop("qk_norm", None)
            return
        grads = [torch.empty_like(g) if g is not None and train else None for g in (gq, gk)]
        scratch, n = self._scratch(0) if train else (None, 0)
        _check(lib.sh_set_qk_norm(self.handle, _ptr(gq), _ptr(gk), eps, _ptr(grads[0]), _ptr(grads[1]), _ptr(scratch), n))
        self._settings["qk_norm"] = _Kept((*grads, gq, gk, scratch))

    def sh_set_balance(self, kind: Optional[str], coef: float = 0.01, mask: Optional[torch.Tensor] = None, gloss: Optional[torch.Tensor] = None) -> Optional[dict]:
        """sh_forward also gives the balance loss of its gates (fp32 layers): returns the tensors it writes, {loss, counts, prob}; sh_backward
        adds gloss times its gradient to the gates'.  kind: "counts", "entropy", or None to switch it off.  mask [batch * seq] bool: tokens that count (those of
        a cache among them; the destination side's gates count the chunk's tokens only)."""
        if kind is None:
            _check(lib.sh_set_balance(self.handle, 0, 0.0, *([None] * 6), 0))
            self._settings.pop("balance", None)
            return None
        dev, (_, H, _, E, _) = self.workspace.device, self.dims
        assert self._mine(mask) and self._mine(gloss), "mask and gloss must be on the layer's device"
        assert mask is None or (mask.is_contiguous() and mask.dtype in (torch.bool, torch.uint8) and mask.numel() == self.batch * self.seq)
        assert gloss is None or (gloss.dtype == torch.float32 and gloss.numel() == 1)
        sides = 1 if self.shared_selection else 2
        out = dict(loss=torch.empty((), device=dev), counts=torch.empty((sides, H, E), dtype=torch.int32, device=dev), prob=torch.empty((sides, H, E), device=dev))
        scratch, n = self._scratch(1)
        _check(lib.sh_set_balance(self.handle, SH_BALANCE[kind], coef, _ptr(mask), _ptr(out["loss"]), _ptr(out["counts"]), _ptr(out["prob"]), _ptr(gloss), _ptr(scratch), n))
        self._settings["balance"] = _Kept((mask, gloss, out, scratch))
        return out

    def sh_set_dropout(self, p: float, rng: Optional[torch.Tensor], train: bool = True) -> None:
        """Dropout of sh_forward's output (fp32 layers); rng: a device tensor of two int64, seed and offset, which the passes read (None: off)."""
        assert self._mine(rng) and (rng is None or rng.dtype == torch.int64 and rng.is_contiguous() and rng.numel() == 2)
        scratch, n = self._scratch(2) if train and rng is not None else (None, 0)
        _check(lib.sh_set_dropout(self.handle, p, _ptr(rng), _ptr(scratch), n))
        self._settings["dropout"] = _Kept((rng, scratch))

    def sh_set_output_f16(self, enable: bool) -> None:
        """sh_forward writes fp16 instead of fp32 from now on (bf16 storage configuration only)."""
        _check(lib.sh_set_output_f16(self.handle, 1 if enable else 0))
        self.out_dtype = torch.float16 if enable else torch.float32

    def _of_this_pass(self) -> None:
        """The settings' tensors belong to the pass that has been made (a refused one leaves the pass before it, which keeps its own)."""
        self._of_forward = dict(self._settings)
        self._used_by_a_pass()

    def _used_by_a_pass(self) -> None:
        if self._of_forward:
            stream = torch.cuda.current_stream()
            for kept in self._of_forward.values():
                kept.used_on(stream)
            if torch.cuda.is_current_stream_capturing():   # (a replay uses them whatever has been set since: kept until the next sh_configure)
                self._captured.update({id(kept): kept for kept in self._of_forward.values()})

    def sh_forward(self, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        assert x.is_cuda and x.is_contiguous()
        if out is None:
            out = torch.empty((x.shape[0], self.seq_out, x.shape[2]), dtype=getattr(self, "out_dtype", torch.float32), device=x.device)
        assert out.dtype == getattr(self, "out_dtype", torch.float32), "out must have the layer's output dtype (see sh_set_output_f16)"
        _check(lib.sh_forward(self.handle, _ptr(x), _ptr(out), _stream()))
        self._of_this_pass()
        return out

    def sh_forward_timed(self, x: torch.Tensor, out: torch.Tensor):
        """Returns the six stage times in ms: gate+sort, qk, v, attention, o, total."""
        ms = (ctypes.c_float * 6)()
        _check(lib.sh_forward_timed(self.handle, _ptr(x), _ptr(out), _stream(), ms))
        self._of_this_pass()
        return list(ms)

    def sh_forward_stamped(self, x: torch.Tensor, out: torch.Tensor):
        """One forward pass launched as sh_forward launches it; returns {kernel: (resident, start, end)} in
        nanoseconds of the device clock for the kernels that ran (see STAMP_KERNELS)."""
        n = len(STAMP_KERNELS)
        buf = (ctypes.c_uint64 * (3 * n))()
        _check(lib.sh_forward_stamped(self.handle, _ptr(x), _ptr(out), _stream(), buf))
        self._of_this_pass()
        return {name: (buf[i], buf[n + i], buf[2 * n + i]) for i, name in enumerate(STAMP_KERNELS) if buf[2 * n + i] != 0}

    def sh_status_block(self):
        w = (ctypes.c_int32 * 16)()
        _check(lib.sh_status_block(self.handle, w, _stream()))
        return list(w)

    def sh_clear_status(self) -> None:
        _check(lib.sh_clear_status(self.handle, _stream()))

    def sh_check_guards(self) -> None:
        _check(lib.sh_check_guards(self.handle, _stream()))

    def sh_selftest(self, which: int, arg: int) -> None:
        _check(lib.sh_selftest(self.handle, which, arg, _stream()))

    def sh_backward(self, x: torch.Tensor, dout: torch.Tensor) -> dict:
        """Gradients of sum(out * dout) with respect to x and every weight (fp32 configuration; call sh_forward(x) first), and of the gains of
        sh_set_qk_norm (dgq, dgk)."""
        d_model, H, D, E, k = self.dims
        dev = x.device
        z = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)
        g = dict(dx=z(self.batch, self.seq, d_model), dWq=z(H, d_model, D), dWk=z(H, d_model, D), dWv=z(H, E, d_model, D),
                 dWo=z(H, E, D, d_model), dWs=z(H, d_model, E), dWd=z(H, d_model, E))
        _check(lib.sh_backward(self.handle, _ptr(x), _ptr(dout), *[_ptr(g[n]) for n in ("dx", "dWq", "dWk", "dWv", "dWo", "dWs", "dWd")], _stream()))
        self._used_by_a_pass()
        for name, grad in zip(("dgq", "dgk"), self._of_forward.get("qk_norm", ())):
            if grad is not None:
                g[name] = grad.clone()
        return g

    def sh_gate_topk(self, x: torch.Tensor):
        d_model, H, D, E, k = self.dims
        N = self.batch * self.seq
        dev = x.device
        idx = torch.empty((2, N, H, k), dtype=torch.int32, device=dev)
        gate = torch.empty((2, N, H, k), dtype=torch.float32, device=dev)
        offsets = torch.empty((2, H, E + 1), dtype=torch.int32, device=dev)
        lists = torch.empty((2, H, N * k), dtype=torch.int32, device=dev)
        _check(lib.sh_gate_topk(self.handle, _ptr(x), _ptr(idx), _ptr(gate), _ptr(offsets), _ptr(lists), _stream()))
        return idx, gate, offsets, lists

    def sh_debug_buffer(self, name: str) -> torch.Tensor:
        """Copy of an intermediate buffer as a torch tensor (Q, K, V [B,H,T,D]; AHAT [N,H,D])."""
        p, n = ctypes.c_void_p(), ctypes.c_size_t()
        _check(lib.sh_debug_buffer(self.handle, BUF[name], ctypes.byref(p), ctypes.byref(n)))
        off = p.value - self.workspace.data_ptr()
        raw = self.workspace[off:off + n.value].clone()
        d_model, H, D, E, k = self.dims
        if name in ("Q", "K", "V", "AHAT"):
            t = raw.view(torch.float32 if self.dtype == SH_F32 else torch.float16)
            # d_head is stored padded with zero columns (64 / 128 on the bf16 path, 32 / 64 / 128 on fp32)
            Dp = (64 if D <= 64 else 128 if D <= 128 else 256) if self.dtype != SH_F32 else (32 if D <= 32 else 64 if D <= 64 else 128 if D <= 128 else 256)
            t = t.view(self.batch, H, self.seq, Dp) if name != "AHAT" else t.view(self.batch * self.seq, H, Dp)
            return t[..., :D]
        return raw.view(torch.float32 if name == "GATE" else torch.int32)

    def sh_last_status(self) -> int:
        return lib.sh_last_status(self.handle, _stream())

    def sh_launch_count(self) -> int:
        return lib.sh_launch_count(self.handle)

    def close(self) -> None:
        if self.handle:
            lib.sh_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sh_noalloc_gate_topk(dtype: int, x: torch.Tensor, w_gate: torch.Tensor, bias: Optional[torch.Tensor],
                         n_heads: int, n_experts: int, k: int):
    """Gate + top-k + bucket sort without a layer handle or workspace (see switchhead.h).
    x [N, M]; w_gate [2*H*E, M] (one row per gate column); returns idx, gate, offsets, lists.
    The output tensors are allocated here, by torch, before the call; the call itself allocates nothing."""
    N, M = x.shape
    dev = x.device
    idx = torch.empty((2, N, n_heads, k), dtype=torch.int32, device=dev)
    gate = torch.empty((2, N, n_heads, k), dtype=torch.float32, device=dev)
    offsets = torch.empty((2, n_heads, n_experts + 1), dtype=torch.int32, device=dev)
    lists = torch.empty((2, n_heads, N * k), dtype=torch.int32, device=dev)
    _check(lib.sh_noalloc_gate_topk(dtype, N, M, n_heads, n_experts, k, _ptr(x), _ptr(w_gate), _ptr(bias),
                                    _ptr(idx), _ptr(gate), _ptr(offsets), _ptr(lists), _stream()))
    return idx, gate, offsets, lists


# The operators of a training step (switchhead.h).  Their arguments are one C struct, packed here field by field: small calls
# are bound by what happens on the host.
_QK_NORM_FIELDS = "P3q" * 4 + "3Pd9i2fi"
_QK_NORM = struct.Struct(_QK_NORM_FIELDS)
_QK_NORM_BACKWARD = struct.Struct(_QK_NORM_FIELDS + "P3q" * 2 + "3PQ")
_BALANCE = struct.Struct("3q10PQ6ifi")
_DROPOUT = struct.Struct("4P5qd2i")
_DTYPES = {torch.float32: SH_F32, torch.bfloat16: SH_BF16, torch.float16: SH_F16}
_NO_HEADS = (0, 0, 0, 0)


# (torch.cuda's own make objects first: 2 us of a 10 us call; they serve where a torch has not these names, which are not public)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _launch(fn, packed: bytes, device: int) -> None:
    """The call on the tensors' device and on the stream that is current there."""
    if device == _current_device():
        rc = fn(packed, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(packed, _raw_stream(device))
    if rc != SH_OK:
        raise SwitchHeadError(rc)


def _heads(name: str, t: torch.Tensor, q: torch.Tensor, shape) -> tuple:
    """The fields of one sh_heads: t [B, T, heads, d_head] of q's type and device, the last dimension dense."""
    s = t.stride()
    if t.shape != shape or t.dtype != q.dtype or t.get_device() != q.get_device() or (s[3] != 1 and shape[3] > 1):
        raise ValueError(f"{name} must be [batch, seq, heads, d_head] = {tuple(shape)} of {q.dtype} on {q.device}, its last dimension "
                         f"dense: got {tuple(t.shape)}, {t.dtype}, {t.device}, strides {tuple(s)}")
    return t.data_ptr(), s[0], s[1], s[2]


def _dense_f32(name: str, t: torch.Tensor, like: torch.Tensor, shape) -> int:
    if t.dtype != torch.float32 or t.shape != shape or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor {tuple(shape)} on {like.device}: got {tuple(t.shape)}, {t.dtype}, {t.device}")
    return t.data_ptr()


def _heads_like(t: torch.Tensor) -> tuple:
    """An output for t [B, T, heads, d_head] and its fields: t's order of dimensions, but the last one dense (for an input whose rows overlap -
    windows of one buffer, say - empty_like may put another dimension innermost)."""
    out = torch.empty_like(t)
    s = out.stride()
    if s[3] != 1 and t.shape[3] > 1:
        out = torch.empty_like(t, memory_format=torch.contiguous_format)
        s = out.stride()
    return out, (out.data_ptr(), s[0], s[1], s[2])


def _qk_norm_fields(q, k, q_out, k_out, gq, gk, eps, base, rotated, halves, positions, q_scale) -> tuple:
    """The fields of sh_qk_norm_args.  An output that is None is made here; returns (fields, q_out, k_out)."""
    code = _DTYPES.get(q.dtype)
    if code is None or q.dim() != 4 or not q.is_cuda:
        raise ValueError(f"q must be a CUDA tensor [batch, seq, heads, d_head] of fp32, bf16 or fp16: got {tuple(q.shape)}, {q.dtype}, {q.device}")
    shape = q.shape
    B, T, H, D = shape
    s = q.stride()
    if s[3] != 1 and D > 1:
        raise ValueError(f"q's last dimension must be dense: got strides {s}")
    hq = (q.data_ptr(), s[0], s[1], s[2])
    if q_out is None:
        q_out, oq = _heads_like(q)
    else:
        oq = _heads("the output for q", q_out, q, shape)
    if k is None:
        K, hk, ok = 0, _NO_HEADS, _NO_HEADS
    else:
        ks = k.shape
        K = ks[2] if len(ks) == 4 else 0
        hk = _heads("k", k, q, (B, T, K, D))
        if k_out is None:
            k_out, ok = _heads_like(k)
        else:
            ok = _heads("the output for k", k_out, q, ks)
    pos = wide = 0
    if positions is not None:
        wide = positions.dtype == torch.int64
        if positions.shape != shape[:2] or not (wide or positions.dtype == torch.int32) or positions.get_device() != q.get_device() or not positions.is_contiguous():
            raise ValueError(f"positions must be a contiguous int32 or int64 tensor {(B, T)} on {q.device}: got {tuple(positions.shape)}, {positions.dtype}, {positions.device}")
        pos = positions.data_ptr()
    return (*hq, *hk, *oq, *ok, 0 if gq is None else _dense_f32("gq", gq, q, (D,)), 0 if gk is None else _dense_f32("gk", gk, q, (D,)), pos, base,
            code, B, T, H, K, D, rotated, halves, wide, eps, q_scale, 0), q_out, k_out


def sh_qk_norm(q: torch.Tensor, k: Optional[torch.Tensor], gq: Optional[torch.Tensor] = None, gk: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
               base: float = 10000.0, rotated: int = 0, halves: bool = False, positions: Optional[torch.Tensor] = None, q_scale: float = 1.0,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Queries and keys normalised per head and rotated by their position, in one pass.  q, k [batch, seq, heads, d_head] in any strides
    with a dense last dimension (columns of a fused projection, transposed views); k may be None.  gq, gk [d_head] fp32 gains.
    q_out, k_out: where the results go (q and k themselves are allowed).  Returns (q_out, k_out)."""
    fields, q_out, k_out = _qk_norm_fields(q, k, q_out, k_out, gq, gk, eps, base, rotated, halves, positions, q_scale)
    _launch(lib.sh_qk_norm, _QK_NORM.pack(*fields), q.get_device())
    return q_out, k_out


@functools.lru_cache(maxsize=None)
def _qk_norm_workspace_bytes(d_head: int) -> int:
    return lib.sh_qk_norm_workspace_bytes(d_head)


@functools.lru_cache(maxsize=4096)
def _balance_shape(tokens: int, sides: int, heads: int, experts: int):
    """Shape and strides of a dense [sides, heads, experts], bytes of the workspace."""
    return (sides, heads, experts), (heads * experts, experts, 1), lib.sh_balance_workspace_bytes(tokens, sides, heads, experts)


def sh_qk_norm_backward(q: torch.Tensor, k: Optional[torch.Tensor], dq: torch.Tensor, dk: Optional[torch.Tensor], gq: Optional[torch.Tensor] = None,
                        gk: Optional[torch.Tensor] = None, *, eps: float = 1e-6, base: float = 10000.0, rotated: int = 0, halves: bool = False,
                        positions: Optional[torch.Tensor] = None, q_scale: float = 1.0) -> dict:
    """Gradients of sh_qk_norm(q, k, gq, gk, ...) from those of its outputs, dq and dk: {dq, dk} with respect to its inputs, and of the
    gains that were given (dgq, dgk [d_head] fp32, summed over tokens and heads; None where there is no gain)."""
    if dq is None or (dk is None) != (k is None):
        raise ValueError("dq and, with k, dk must be given")
    fields, out_q, out_k = _qk_norm_fields(q, k, None, None, gq, gk, eps, base, rotated, halves, positions, q_scale)
    dgq = None if gq is None else torch.empty_like(gq)
    dgk = None if gk is None else torch.empty_like(gk)
    ws, nbytes = None, 0
    if gq is not None or gk is not None:
        nbytes = _qk_norm_workspace_bytes(q.shape[3])
        ws = (gk if gq is None else gq).new_empty(nbytes // 4)
    _launch(lib.sh_qk_norm_backward, _QK_NORM_BACKWARD.pack(*fields, *_heads("dq", dq, q, q.shape), *(_NO_HEADS if k is None else _heads("dk", dk, q, k.shape)),
                                                            0 if dgq is None else dgq.data_ptr(), 0 if dgk is None else dgk.data_ptr(),
                                                            0 if ws is None else ws.data_ptr(), nbytes), q.get_device())
    return dict(dq=out_q, dk=out_k, dgq=dgq, dgk=dgk)


def _logits(name: str, z: torch.Tensor) -> None:
    """[N, sides, heads, experts] with a token's gates dense."""
    s, st = z.shape, z.stride()
    if (z.dim() != 4 or z.dtype not in (torch.float32, torch.bfloat16) or not z.is_cuda
            or not ((s[3] == 1 or st[3] == 1) and (s[2] == 1 or st[2] == s[3]) and (s[1] == 1 or st[1] == s[2] * s[3]))):
        raise ValueError(f"{name} must be a CUDA tensor [tokens, sides, heads, experts] of fp32 or bf16, a token's gates dense: got {tuple(s)}, {z.dtype}, {z.device}, strides {z.stride()}")


def _token_mask(mask: Optional[torch.Tensor], z: torch.Tensor) -> int:
    if mask is None:
        return 0
    if mask.dtype not in (torch.bool, torch.uint8) or mask.shape != z.shape[:1] or mask.get_device() != z.get_device() or not mask.is_contiguous():
        raise ValueError(f"mask must be a contiguous bool or uint8 tensor [{z.shape[0]}] on {z.device}: got {tuple(mask.shape)}, {mask.dtype}, {mask.device}")
    return mask.data_ptr()


def sh_balance_loss(logits: torch.Tensor, idx: torch.Tensor, *, kind: str = "counts", coef: float = 1.0, mask: Optional[torch.Tensor] = None) -> dict:
    """Balance loss of the gates with the per-expert counts.  logits [N, sides, heads, experts] fp32 or bf16; idx [sides, N, heads, k] int32 (the
    selections, as sh_gate_topk gives them); mask [N]: tokens that count.  Returns {loss, counts, prob, slope}: loss a scalar, the others
    [sides, heads, experts]; slope is what sh_balance_backward takes."""
    _logits("logits", logits)
    N, S, H, E = logits.shape
    if idx.dtype != torch.int32 or idx.dim() != 4 or idx.shape[:3] != (S, N, H) or idx.get_device() != logits.get_device() or not idx.is_contiguous():
        raise ValueError(f"idx must be a contiguous int32 tensor [sides, tokens, heads, k] on {logits.device}: got {tuple(idx.shape)}, {idx.dtype}, {idx.device}")
    if kind not in SH_BALANCE:
        raise ValueError(f"kind must be one of {sorted(SH_BALANCE)}: got {kind!r}")
    dev = logits.device
    shape, strides, nbytes = _balance_shape(N, S, H, E)
    prob = torch.empty_strided(shape, strides, dtype=torch.float32, device=dev)
    loss = prob.new_empty(())
    slope = torch.empty_like(prob)
    counts = torch.empty_like(prob, dtype=torch.int32)
    ws = prob.new_empty((nbytes + 3) // 4) if nbytes else None
    _launch(lib.sh_balance_loss, _BALANCE.pack(N, logits.stride(0), 0, logits.data_ptr(), idx.data_ptr(), _token_mask(mask, logits), 0, loss.data_ptr(),
                                               prob.data_ptr(), slope.data_ptr(), counts.data_ptr(), 0, ws.data_ptr() if nbytes else 0, nbytes,
                                               _DTYPES[logits.dtype], SH_BALANCE[kind], S, H, E, idx.shape[3], coef, 0), logits.get_device())
    return dict(loss=loss, counts=counts, prob=prob, slope=slope)


def sh_balance_backward(logits: torch.Tensor, slope: torch.Tensor, *, gloss: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of the balance loss with respect to the logits, times gloss (a device scalar, the gradient of the loss); slope and mask: of the
    sh_balance_loss call.  out: where it goes (logits itself is allowed)."""
    _logits("logits", logits)
    N, S, H, E = logits.shape
    if out is None:
        out = torch.empty_like(logits) if logits.is_contiguous() else torch.empty_like(logits, memory_format=torch.contiguous_format)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.get_device() != logits.get_device():
        raise ValueError("out must have the shape, type and device of logits")
    else:
        _logits("out", out)
    _launch(lib.sh_balance_backward, _BALANCE.pack(N, logits.stride(0), out.stride(0), logits.data_ptr(), 0, _token_mask(mask, logits),
                                                   0 if gloss is None else _dense_f32("gloss", gloss, logits, ()), 0, 0, _dense_f32("slope", slope, logits, (S, H, E)), 0,
                                                   out.data_ptr(), 0, 0, _DTYPES[logits.dtype], 0, S, H, E, 1, 0.0, 0), logits.get_device())
    return out


def _rows(name: str, t: torch.Tensor, x: torch.Tensor) -> int:
    """The row stride of a matrix of x's shape (leading dimensions flattened)."""
    if t.shape != x.shape or t.dtype != x.dtype or t.get_device() != x.get_device():
        raise ValueError(f"{name} must have the shape, type and device of x")
    if t.is_contiguous():
        return t.shape[-1]
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        return t.stride(0)
    raise ValueError(f"{name} must be contiguous, or a matrix with dense rows")


def sh_dropout(x: torch.Tensor, rng: torch.Tensor, p: float, *, residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x) over rows of x's last dimension, fp32, bf16 or fp16.  rng: a device tensor of two int64, the seed and the offset (another
    offset for every site and step); the mask follows from them alone, so sh_dropout(dy, rng, p) is the gradient's way back.
    out may be x or residual."""
    if x.dtype not in _DTYPES or not x.is_cuda or x.dim() < 1:
        raise ValueError(f"x must be a CUDA tensor [..., columns] of fp32, bf16 or fp16: got {tuple(x.shape)}, {x.dtype}, {x.device}")
    if rng.dtype != torch.int64 or rng.shape != (2,) or rng.get_device() != x.get_device() or not rng.is_contiguous():
        raise ValueError(f"rng must be a contiguous int64 tensor [2] on {x.device}: got {tuple(rng.shape)}, {rng.dtype}, {rng.device}")
    if out is None:
        out = torch.empty_like(x) if x.is_contiguous() else torch.empty_like(x, memory_format=torch.contiguous_format)
    cols = x.shape[-1]
    _launch(lib.sh_dropout, _DROPOUT.pack(x.data_ptr(), 0 if residual is None else residual.data_ptr(), out.data_ptr(), rng.data_ptr(),
                                          x.numel() // cols if cols else 0, cols, _rows("x", x, x), 0 if residual is None else _rows("residual", residual, x),
                                          _rows("out", out, x), p, _DTYPES[x.dtype], 0), x.get_device())
    return out


def to_device(a: Optional[np.ndarray], dtype: int, device="cuda") -> Optional[torch.Tensor]:
    """Host array (fp32 values already representable in the storage type) -> device tensor."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    if dtype == SH_BF16:
        t = t.to(torch.bfloat16)
    return t.to(device).contiguous()


def layer_from_inputs(inp, batch=None, seq=None, device="cuda", shared_selection=False, cache_len=0) -> "Layer":
    """Create, configure and load a Layer from a LayerInputs record (see inputs.py).
    shared_selection: the source gate (Ws, bias_s) serves both sides; Wd and bias_d are not used.
    cache_len: the first cache_len tokens of every sequence of inp.x are a Transformer-XL cache."""
    cfg = inp.cfg
    B, T = inp.x.shape[0], inp.x.shape[1]
    # (Wq / Wk given per expert, [H, E, M, D]: a layer with query / key experts)
    L = Layer(cfg.d_model, cfg.n_heads, cfg.d_head, cfg.n_experts, cfg.k, shared_selection=shared_selection,
              moe_q=inp.Wq.ndim == 4, moe_k=inp.Wk.ndim == 4)
    L.sh_configure(cfg.dtype, B, T - cache_len, device=device, cache_len=cache_len)
    dv = lambda a: to_device(a, cfg.dtype, device)
    bias = lambda a: None if a is None else torch.from_numpy(a).to(device)
    L.sh_set_weights(dv(inp.Wq), dv(inp.Wk), dv(inp.Wv), dv(inp.Wo), dv(inp.Ws),
                     None if shared_selection else dv(inp.Wd),
                     bias(inp.bias_s), None if shared_selection else bias(inp.bias_d))
    return L
