"""Configurations and scratch of the sequence mixers over packed sequences
(bcmt_attn_*, bcmt_linattn_*), for callers that hold torch tensors.

Allocation and argument checks only: the arithmetic runs in the library's HIP
kernels.  The C ABI takes bare pointers, so every tensor is checked here
against the configuration: type, extent, row stride, contiguity and device.
An object belongs to the device that it was made for.  Where a call needs a
workspace, the object keeps one for every stream that it is called on, allocated
on that stream at the first such call: torch's allocator orders memory by the
stream that it was allocated on, so neither an earlier nor a later owner of the
memory can meet the kernels.  A captured graph replays in the workspace of the
stream that it was captured on: graphs captured on one stream must not replay at
the same time, and the object must outlive them.
"""

import ctypes

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
        self._index = self.device.index
        self._torch_dtype = TORCH_DTYPE[dtype]
        self._ref = ctypes.byref(cfg)
        self._lib = abi.lib()

    def _stream(self, stream):
        """The address of the caller's stream, or of the current one of this
        object's device (the address alone: 0.1 us, the stream object 1.1)."""
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def _scratch(self, held, n, s):
        """(address, bytes) of the workspace of stream s, kept in `held`."""
        ws = held.get(s)
        if ws is None:
            on = torch.cuda.ExternalStream(s, device=self.device) if s else \
                torch.cuda.default_stream(self.device)
            with torch.cuda.stream(on):
                ws = held[s] = torch.empty(max(256, n), dtype=torch.uint8, device=self.device)
        return ws.data_ptr(), ws.numel()

    def _rows(self, name, t, rows, width, ld):
        """The address of a tensor of `rows` rows of `width` elements (in any
        shape that flattens to it), `ld` elements apart (0: dense)."""
        if not isinstance(t, torch.Tensor) or t.dtype != self._torch_dtype or \
                t.get_device() != self._index:
            raise ValueError(f"{name}: a {self._torch_dtype} tensor on {self.device} is wanted")
        if t.dim() < 2 or t.shape[0] != rows or t.numel() != rows * width:
            raise ValueError(f"{name}: {rows} rows of {width} elements are wanted, got {tuple(t.shape)}")
        if ld in (0, width) and t.is_contiguous():
            return t.data_ptr()
        if rows > 1 and t.stride(0) != (ld or width):
            raise ValueError(f"{name}: row stride {ld or width} is wanted, got {t.stride(0)}")
        n = 1
        for d in range(t.dim() - 1, 0, -1):
            if t.shape[d] > 1 and t.stride(d) != n:
                raise ValueError(f"{name}: the elements of a row must be contiguous")
            n *= t.shape[d]
        return t.data_ptr()

    def _array(self, name, t, shape, dtype, optional=False):
        """The address of a contiguous tensor of this shape and type."""
        if t is None and optional:
            return None
        if (not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape
                or t.get_device() != self._index or not t.is_contiguous()):
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on "
                             f"{self.device} is wanted")
        return t.data_ptr()

    def _call(self, fn, s, *args):
        """Enqueues on stream s; this object's device is the current one for the call."""
        if torch.cuda.current_device() == self._index:
            st = fn(self._ref, *args, s)
        else:
            with torch.cuda.device(self._index):
                st = fn(self._ref, *args, s)
        if st != abi.BCMT_OK:
            raise abi.BcmtError(st, fn.__name__)


class PackedAttention(_Mixer):
    """Causal attention with grouped heads over `nseq` sequences in `total`
    rows; `cu` (int32 [nseq + 1], on the device) holds where each begins."""

    def __init__(self, total, nseq, H, Hkv, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0,
                 ldo=0, device="cuda"):
        self._setup(abi.make_attn_config(total, nseq, H, Hkv, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_attn_validate, dtype, device)
        self._ws, self._ws_bytes = {}, abi.bcmt_attn_workspace_bytes(self.cfg)
        self._total, self._nseq, self._H = total, nseq, H
        self._wq, self._wk = H * dh, Hkv * dh
        self._ld = ldq, ldk, ldv, ldo

    def _inputs(self, q, k, v, cu):
        n, (ldq, ldk, ldv, _) = self._total, self._ld
        return (self._rows("q", q, n, self._wq, ldq), self._rows("k", k, n, self._wk, ldk),
                self._rows("v", v, n, self._wk, ldv),
                self._array("cu", cu, (self._nseq + 1,), torch.int32))

    def new_output(self):
        return torch.empty((self._total, self._ld[3] or self._wq), dtype=self._torch_dtype,
                           device=self.device)[:, :self._wq]

    def new_lse(self):
        return torch.empty((self._H, self._total), dtype=torch.float32, device=self.device)

    def forward(self, q, k, v, cu, o, lse=None, stream=None):
        self._call(self._lib.bcmt_attn_forward, self._stream(stream), *self._inputs(q, k, v, cu),
                   self._rows("o", o, self._total, self._wq, self._ld[3]),
                   self._array("lse", lse, (self._H, self._total), torch.float32, True))

    def backward(self, q, k, v, cu, o, lse, dO, dq, dk, dv, stream=None):
        n, wq, wk, (ldq, ldk, ldv, ldo) = self._total, self._wq, self._wk, self._ld
        args = (*self._inputs(q, k, v, cu), self._rows("o", o, n, wq, ldo),
                self._array("lse", lse, (self._H, n), torch.float32),
                self._rows("dO", dO, n, wq, ldo), self._rows("dq", dq, n, wq, ldq),
                self._rows("dk", dk, n, wk, ldk), self._rows("dv", dv, n, wk, ldv))
        s = self._stream(stream)
        self._call(self._lib.bcmt_attn_backward, s, *args,
                   *self._scratch(self._ws, self._ws_bytes, s))


class AttentionDecoder(_Mixer):
    """Attention for one token per sequence against caches of `slots` slots of
    `cap` positions, [slots, cap, Hkv, dh] or with the strides cs, ct, ch."""

    def __init__(self, B, slots, cap, H, Hkv, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0,
                 ldo=0, cs=0, ct=0, ch=0, device="cuda"):
        self._setup(abi.make_attn_decode_config(B, slots, cap, H, Hkv, dh, dtype, scale, ldq, ldk,
                                                ldv, ldo, cs, ct, ch),
                    abi.bcmt_attn_decode_validate, dtype, device)
        self._ws, self._ws_bytes = {}, abi.bcmt_attn_decode_workspace_bytes(self.cfg)
        self._B, self._wq, self._wk = B, H * dh, Hkv * dh
        self._ld = ldq, ldk, ldv, ldo
        self._shape = (slots, cap, Hkv, dh)
        self._strides = (cs or cap * Hkv * dh, ct or Hkv * dh, ch or dh, 1)

    def new_cache(self):
        """A dense cache for keys or values."""
        return torch.zeros(self._shape, dtype=self._torch_dtype, device=self.device)

    def _cache(self, name, t):
        if not isinstance(t, torch.Tensor) or t.dtype != self._torch_dtype or \
                t.get_device() != self._index:
            raise ValueError(f"{name}: a {self._torch_dtype} tensor on {self.device} is wanted")
        shape, want = self._shape, self._strides
        if t.shape != shape or (t.stride() != want and any(
                n > 1 and s != w for n, s, w in zip(shape, t.stride(), want))):
            raise ValueError(f"{name}: shape {shape} with strides {want} is wanted, got "
                             f"{tuple(t.shape)} with {t.stride()}")
        return t.data_ptr()

    def step(self, q, k, v, slot, length, kcache, vcache, o, stream=None):
        n, wq, wk, (ldq, ldk, ldv, ldo) = self._B, self._wq, self._wk, self._ld
        s = self._stream(stream)
        self._call(self._lib.bcmt_attn_decode, s, self._rows("q", q, n, wq, ldq),
                   self._rows("k", k, n, wk, ldk), self._rows("v", v, n, wk, ldv),
                   self._array("slot", slot, (n,), torch.int32, True),
                   self._array("length", length, (n,), torch.int32),
                   self._cache("kcache", kcache), self._cache("vcache", vcache),
                   self._rows("o", o, n, wq, ldo), *self._scratch(self._ws, self._ws_bytes, s))


class LinearAttention(_Mixer):
    """Linear attention with one decay per head over `nseq` sequences in
    `total` rows; states are float32 [nseq, H, dh, dh]."""

    def __init__(self, total, nseq, H, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0, ldo=0,
                 device="cuda"):
        self._setup(abi.make_linattn_config(total, nseq, H, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_linattn_validate, dtype, device)
        self._ws, self._ws_bwd = {}, {}
        self._ws_bytes, self._ws_bwd_bytes = (
            abi.bcmt_linattn_workspace_bytes(self.cfg, p)
            for p in (abi.BCMT_PASS_FORWARD, abi.BCMT_PASS_BACKWARD))
        self._total, self._nseq, self._H, self._w = total, nseq, H, H * dh
        self._ld = ldq, ldk, ldv, ldo
        self._shape = (nseq, H, dh, dh)

    def new_state(self):
        """Zero states: empty histories."""
        return torch.zeros(self._shape, dtype=torch.float32, device=self.device)

    def _inputs(self, q, k, v, gamma, cu):
        n, w, (ldq, ldk, ldv, _) = self._total, self._w, self._ld
        return (self._rows("q", q, n, w, ldq), self._rows("k", k, n, w, ldk),
                self._rows("v", v, n, w, ldv),
                self._array("gamma", gamma, (self._H,), torch.float32),
                self._array("cu", cu, (self._nseq + 1,), torch.int32))

    def _state(self, name, t):
        return self._array(name, t, self._shape, torch.float32, True)

    def forward(self, q, k, v, gamma, cu, o, S_in=None, S_out=None, stream=None):
        s = self._stream(stream)
        self._call(self._lib.bcmt_linattn_forward, s, *self._inputs(q, k, v, gamma, cu),
                   self._state("S_in", S_in), self._rows("o", o, self._total, self._w, self._ld[3]),
                   self._state("S_out", S_out), *self._scratch(self._ws, self._ws_bytes, s))

    def backward(self, q, k, v, gamma, cu, dO, dq, dk, dv, S_in=None, dS_out=None, dS_in=None,
                 dgamma=None, stream=None):
        n, w, (ldq, ldk, ldv, ldo) = self._total, self._w, self._ld
        args = (*self._inputs(q, k, v, gamma, cu), self._state("S_in", S_in),
                self._rows("dO", dO, n, w, ldo), self._state("dS_out", dS_out),
                self._rows("dq", dq, n, w, ldq), self._rows("dk", dk, n, w, ldk),
                self._rows("dv", dv, n, w, ldv), self._state("dS_in", dS_in),
                self._array("dgamma", dgamma, (self._H,), torch.float32, True))
        s = self._stream(stream)
        self._call(self._lib.bcmt_linattn_backward, s, *args,
                   *self._scratch(self._ws_bwd, self._ws_bwd_bytes, s))


class LinearAttentionDecoder(_Mixer):
    """Linear attention for one token per sequence on a pool of states
    [slots, H, dh, dh] (float32)."""

    def __init__(self, B, slots, H, dh, dtype="bf16", scale=None, ldq=0, ldk=0, ldv=0, ldo=0,
                 device="cuda"):
        self._setup(abi.make_linattn_step_config(B, slots, H, dh, dtype, scale, ldq, ldk, ldv, ldo),
                    abi.bcmt_linattn_step_validate, dtype, device)
        self._B, self._H, self._w = B, H, H * dh
        self._ld = ldq, ldk, ldv, ldo
        self._shape = (slots, H, dh, dh)

    def new_state(self):
        return torch.zeros(self._shape, dtype=torch.float32, device=self.device)

    def step(self, q, k, v, gamma, slot, S_in, S_out, o, stream=None):
        n, w, (ldq, ldk, ldv, ldo) = self._B, self._w, self._ld
        self._call(self._lib.bcmt_linattn_step, self._stream(stream), self._rows("q", q, n, w, ldq),
                   self._rows("k", k, n, w, ldk), self._rows("v", v, n, w, ldv),
                   self._array("gamma", gamma, (self._H,), torch.float32),
                   self._array("slot", slot, (n,), torch.int32, True),
                   self._array("S_in", S_in, self._shape, torch.float32),
                   self._array("S_out", S_out, self._shape, torch.float32),
                   self._rows("o", o, n, w, ldo))
