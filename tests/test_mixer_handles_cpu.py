"""The handles of the packed-sequence mixers without a GPU: what they allocate, and
on which stream.  The library's entry points and torch's streams are stand-ins
that write down what reaches them."""

import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2608_13578_amd import bcmt as abi
from paper_2608_13578_amd import mixers

CURRENT, OTHER = 0x1000, 0x2000


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(abi.LIB_PATH):
        from paper_2608_13578_amd.build import build
        build()


@pytest.fixture
def gpu(monkeypatch):
    """allocated: {address: the stream that was current}; calls: (entry, arguments)."""
    log = SimpleNamespace(allocated={}, calls=[], current=[CURRENT])
    empty = torch.empty

    def on_stream(*a, device=None, **kw):
        t = empty(*a, **kw)
        log.allocated[t.data_ptr()] = log.current[-1]
        return t

    @contextlib.contextmanager
    def stream(s):
        log.current.append(s.cuda_stream)
        yield
        log.current.pop()

    class Entries:
        def __getattr__(self, name):
            def entry(*args):
                log.calls.append((name, args))
                return abi.BCMT_OK
            entry.__name__ = name
            return entry

    def handle(made):
        made._lib = Entries()
        return made

    log.handle = handle
    monkeypatch.setattr(torch, "empty", on_stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream",
                        lambda s, device=None: SimpleNamespace(cuda_stream=s))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d=None: SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: log.current[-1],
                        raising=False)
    for check in ("_rows", "_array", "_cache"):  # (the tensors are of no account here)
        for c in (mixers._Mixer, mixers.AttentionDecoder):
            if check in vars(c):
                monkeypatch.setattr(c, check, lambda self, *a: 16)
    return log


CALLS = {  # a handle, its call, the tensors of one call
    "attention gradient": (lambda: mixers.PackedAttention(500, 2, 4, 2, 64, device="cuda:0"), "backward", 10),
    "decode": (lambda: mixers.AttentionDecoder(2, 3, 5000, 4, 2, 64, device="cuda:0"), "step", 8),
    "linear": (lambda: mixers.LinearAttention(500, 2, 4, 64, device="cuda:0"), "forward", 6),
    "linear gradient": (lambda: mixers.LinearAttention(500, 2, 4, 64, device="cuda:0"), "backward", 9),
}


@pytest.mark.parametrize("name", CALLS)
def test_workspace_is_allocated_on_the_stream_of_the_call(gpu, name):
    """On any other stream, the memory could still be in use by work of its last
    owner, and go to a next owner before the kernels are done."""
    make, call, n = CALLS[name]
    d = gpu.handle(make())
    seen = {}
    for stream in (None, OTHER, SimpleNamespace(cuda_stream=OTHER), 0, None, OTHER):
        getattr(d, call)(*[None] * n, stream=stream)
        _, args = gpu.calls[-1]
        ws, nbytes, s = args[-3:]
        want = CURRENT if stream is None else getattr(stream, "cuda_stream", stream)
        assert s == want
        assert gpu.allocated[ws] == want
        assert nbytes > 256  # (a size that needs scratch)
        assert seen.setdefault(s, ws) == ws  # kept from call to call
    assert len(set(seen.values())) == 3  # calls on different streams share none
