"""Configurations and scratch of the sequence mixers over packed sequences
(bcmt_attn_*, bcmt_linattn_*), for callers that hold torch tensors.

Allocation and argument checks only: the arithmetic runs in the library's HIP
kernels.  The C ABI takes bare pointers, so every tensor is checked here
against the configuration: type, extent, row stride, contiguity and device.
An object belongs to the device that it was made for and keeps one workspace:
its calls must be ordered (one stream, or streams that wait for each other),
and a captured graph replays in that workspace.
"""

import torch

from . import bcmt as abi
from .layer import TORCH_DTYPE


class _Mixer:
    def _setup(self, cfg, validate, dtype, device):
        st = validate(cfg)
        if st != abi.BCMT_OK:
            raise abi.BcmtError(st, validate.__name__)
        self.cfg, self.dtype = cfg, dtype
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self._torch_dtype = TORCH_DTYPE[dtype]

    def _scratch(self, n):
        return torch.empty(max(256, n), dtype=torch.uint8, device=self.device)

    def _rows(self, name, t, rows, width, ld):
        """A tensor of `rows` rows of `width` elements (in any shape that
        flattens to it), `ld` elements apart (0: dense)."""
        if not isinstance(t, torch.Tensor) or t.dtype != self._torch_dtype or t.device != self.device:
            raise ValueError(f"{name}: a {self._torch_dtype} tensor on {self.device} is wanted")
        if t.dim() < 2 or t.shape[0] != rows or t.numel() != rows * width:
            raise ValueError(f"{name}: {rows} rows of {width} elements are wanted, got {tuple(t.shape)}")
        if rows > 1 and t.stride(0) != (ld or width):
            raise ValueError(f"{name}: row stride {ld or width} is wanted, got {t.stride(0)}")
        n = 1
        for d in range(t.dim() - 1, 0, -1):
            if t.shape[d] > 1 and t.stride(d) != n:
                raise ValueError(f"{name}: the elements of a row must be contiguous")
            n *= t.shape[d]

    def _array(self, name, t, shape, dtype, optional=False):
        if t is None and optional:
            return
        if (not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape)
                or not t.is_contiguous() or t.device != self.device):
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on "
                             f"{self.device} is wanted")

    def _on(self, stream):
        """The caller's stream, or the current one of this object's device."""
        if stream is None:
            return torch.cuda.current_stream(self.device)
        return stream


class PackedAttention(_Mixer):
    """Causal attention with grouped heads over `nseq` sequences in `total`
    rows; `cu` (int32 [nseq + 1], on the device) holds where each begins."""

    def __init__(self, total, nseq, H, Hkv, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0,
                 ldo=0, device="cuda"):
        self._setup(abi.make_attn_config(total, nseq, H, Hkv, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_attn_validate, dtype, device)
        self.ws = None

    def _check(self, q, k, v, cu, o):
        c = self.cfg
        self._rows("q", q, c.total, c.H * c.dh, c.ldq)
        self._rows("k", k, c.total, c.Hkv * c.dh, c.ldk)
        self._rows("v", v, c.total, c.Hkv * c.dh, c.ldv)
        self._rows("o", o, c.total, c.H * c.dh, c.ldo)
        self._array("cu", cu, (c.nseq + 1,), torch.int32)

    def new_output(self):
        c = self.cfg
        return torch.empty((c.total, c.ldo or c.H * c.dh), dtype=self._torch_dtype,
                           device=self.device)[:, :c.H * c.dh]

    def new_lse(self):
        return torch.empty((self.cfg.H, self.cfg.total), dtype=torch.float32, device=self.device)

    def forward(self, q, k, v, cu, o, lse=None, stream=None):
        self._check(q, k, v, cu, o)
        self._array("lse", lse, (self.cfg.H, self.cfg.total), torch.float32, optional=True)
        with torch.cuda.device(self.device):
            abi.bcmt_attn_forward(self.cfg, q, k, v, cu, o, lse, stream=self._on(stream))

    def backward(self, q, k, v, cu, o, lse, dO, dq, dk, dv, stream=None):
        c = self.cfg
        self._check(q, k, v, cu, o)
        self._array("lse", lse, (c.H, c.total), torch.float32)
        self._rows("dO", dO, c.total, c.H * c.dh, c.ldo)
        self._rows("dq", dq, c.total, c.H * c.dh, c.ldq)
        self._rows("dk", dk, c.total, c.Hkv * c.dh, c.ldk)
        self._rows("dv", dv, c.total, c.Hkv * c.dh, c.ldv)
        if self.ws is None:
            self.ws = self._scratch(abi.bcmt_attn_workspace_bytes(c))
        with torch.cuda.device(self.device):
            abi.bcmt_attn_backward(c, q, k, v, cu, o, lse, dO, dq, dk, dv, self.ws,
                                   stream=self._on(stream))


class AttentionDecoder(_Mixer):
    """Attention for one token per sequence against caches of `slots` slots of
    `cap` positions, [slots, cap, Hkv, dh] or with the strides cs, ct, ch."""

    def __init__(self, B, slots, cap, H, Hkv, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0,
                 ldo=0, cs=0, ct=0, ch=0, device="cuda"):
        self._setup(abi.make_attn_decode_config(B, slots, cap, H, Hkv, dh, dtype, scale, ldq, ldk,
                                                ldv, ldo, cs, ct, ch),
                    abi.bcmt_attn_decode_validate, dtype, device)
        self.ws = self._scratch(abi.bcmt_attn_decode_workspace_bytes(self.cfg))

    def new_cache(self):
        """A dense cache for keys or values."""
        c = self.cfg
        return torch.zeros((c.slots, c.cap, c.Hkv, c.dh), dtype=self._torch_dtype,
                           device=self.device)

    def _cache(self, name, t):
        c = self.cfg
        shape = (c.slots, c.cap, c.Hkv, c.dh)
        if not isinstance(t, torch.Tensor) or t.dtype != self._torch_dtype or t.device != self.device:
            raise ValueError(f"{name}: a {self._torch_dtype} tensor on {self.device} is wanted")
        want = (c.cs or c.cap * c.Hkv * c.dh, c.ct or c.Hkv * c.dh, c.ch or c.dh, 1)
        if tuple(t.shape) != shape or any(n > 1 and s != w for n, s, w in
                                          zip(shape, t.stride(), want)):
            raise ValueError(f"{name}: shape {shape} with strides {want} is wanted, got "
                             f"{tuple(t.shape)} with {t.stride()}")

    def step(self, q, k, v, slot, length, kcache, vcache, o, stream=None):
        c = self.cfg
        self._rows("q", q, c.B, c.H * c.dh, c.ldq)
        self._rows("k", k, c.B, c.Hkv * c.dh, c.ldk)
        self._rows("v", v, c.B, c.Hkv * c.dh, c.ldv)
        self._rows("o", o, c.B, c.H * c.dh, c.ldo)
        self._array("slot", slot, (c.B,), torch.int32, optional=True)
        self._array("length", length, (c.B,), torch.int32)
        self._cache("kcache", kcache)
        self._cache("vcache", vcache)
        with torch.cuda.device(self.device):
            abi.bcmt_attn_decode(c, q, k, v, slot, length, kcache, vcache, o, self.ws,
                                 stream=self._on(stream))


class LinearAttention(_Mixer):
    """Linear attention with one decay per head over `nseq` sequences in
    `total` rows; states are float32 [nseq, H, dh, dh]."""

    def __init__(self, total, nseq, H, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0, ldo=0,
                 device="cuda"):
        self._setup(abi.make_linattn_config(total, nseq, H, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_linattn_validate, dtype, device)
        self.ws = self._scratch(abi.bcmt_linattn_workspace_bytes(self.cfg, abi.BCMT_PASS_FORWARD))
        self.ws_bwd = None

    def new_state(self):
        """Zero states: empty histories."""
        c = self.cfg
        return torch.zeros((c.nseq, c.H, c.dh, c.dh), dtype=torch.float32, device=self.device)

    def _check(self, q, k, v, gamma, cu):
        c = self.cfg
        w = c.H * c.dh
        self._rows("q", q, c.total, w, c.ldq)
        self._rows("k", k, c.total, w, c.ldk)
        self._rows("v", v, c.total, w, c.ldv)
        self._array("gamma", gamma, (c.H,), torch.float32)
        self._array("cu", cu, (c.nseq + 1,), torch.int32)

    def _state(self, name, t):
        c = self.cfg
        self._array(name, t, (c.nseq, c.H, c.dh, c.dh), torch.float32, optional=True)

    def forward(self, q, k, v, gamma, cu, o, S_in=None, S_out=None, stream=None):
        c = self.cfg
        self._check(q, k, v, gamma, cu)
        self._rows("o", o, c.total, c.H * c.dh, c.ldo)
        self._state("S_in", S_in)
        self._state("S_out", S_out)
        with torch.cuda.device(self.device):
            abi.bcmt_linattn_forward(c, q, k, v, gamma, cu, S_in, o, S_out, self.ws,
                                     stream=self._on(stream))

    def backward(self, q, k, v, gamma, cu, dO, dq, dk, dv, S_in=None, dS_out=None, dS_in=None,
                 dgamma=None, stream=None):
        c = self.cfg
        w = c.H * c.dh
        self._check(q, k, v, gamma, cu)
        self._rows("dO", dO, c.total, w, c.ldo)
        self._rows("dq", dq, c.total, w, c.ldq)
        self._rows("dk", dk, c.total, w, c.ldk)
        self._rows("dv", dv, c.total, w, c.ldv)
        for name, t in (("S_in", S_in), ("dS_out", dS_out), ("dS_in", dS_in)):
            self._state(name, t)
        self._array("dgamma", dgamma, (c.H,), torch.float32, optional=True)
        if self.ws_bwd is None:
            self.ws_bwd = self._scratch(abi.bcmt_linattn_workspace_bytes(c, abi.BCMT_PASS_BACKWARD))
        with torch.cuda.device(self.device):
            abi.bcmt_linattn_backward(c, q, k, v, gamma, cu, S_in, dO, dS_out, dq, dk, dv, dS_in,
                                      dgamma, self.ws_bwd, stream=self._on(stream))


class LinearAttentionDecoder(_Mixer):
    """Linear attention for one token per sequence on a pool of states
    [slots, H, dh, dh] (float32)."""

    def __init__(self, B, slots, H, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0, ldo=0,
                 device="cuda"):
        self._setup(abi.make_linattn_step_config(B, slots, H, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_linattn_step_validate, dtype, device)

    def new_state(self):
        c = self.cfg
        return torch.zeros((c.slots, c.H, c.dh, c.dh), dtype=torch.float32, device=self.device)

    def step(self, q, k, v, gamma, slot, S_in, S_out, o, stream=None):
        c = self.cfg
        w = c.H * c.dh
        for name, t, ld in (("q", q, c.ldq), ("k", k, c.ldk), ("v", v, c.ldv), ("o", o, c.ldo)):
            self._rows(name, t, c.B, w, ld)
        self._array("gamma", gamma, (c.H,), torch.float32)
        self._array("slot", slot, (c.B,), torch.int32, optional=True)
        self._array("S_in", S_in, (c.slots, c.H, c.dh, c.dh), torch.float32)
        self._array("S_out", S_out, (c.slots, c.H, c.dh, c.dh), torch.float32)
        with torch.cuda.device(self.device):
            abi.bcmt_linattn_step(c, q, k, v, gamma, slot, S_in, S_out, o, stream=self._on(stream))
