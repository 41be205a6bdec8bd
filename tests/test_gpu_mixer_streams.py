"""Calls of the packed-sequence mixers with a stream of the caller's, the first ones of
their handles among them, and with memory that was in use on another stream."""

import math

import pytest
import torch

from test_gpu_mixers import i32, normal, offsets, rng
from test_gpu_parity import say, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

LENS, H, HKV, DH = [200, 1, 333, 130], 4, 2, 64
CAP = 3000  # (in several parts, which lie in the workspace)


def setup(dtype, seed):
    """(inputs, offsets, outputs by name)."""
    cu = offsets(LENS)
    g, total, n = rng(seed), cu[-1], len(LENS)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]

    def new(*shape):
        return normal(g, *shape, dtype=dtype).to(dt).cuda()

    x = {m: new(total, H, DH) for m in ("q", "do", "k2", "v2")}
    x.update({m: new(total, HKV, DH) for m in ("k", "v")})
    x.update(q1=new(n, H, DH), k1=new(n, HKV, DH), v1=new(n, HKV, DH), kc=new(n, CAP, HKV, DH),
             vc=new(n, CAP, HKV, DH), gamma=torch.tensor([0.8, 0.9, 0.99, 1.0], device="cuda"),
             length=i32([CAP - 1, 0, 700, 2000]))
    return x, i32(cu)


def outputs(x):
    out = {m: torch.zeros_like(x[y]) for m, y in (
        ("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"), ("y", "q"), ("eq", "q"), ("ek", "k2"),
        ("ev", "v2"), ("o1", "q1"))}
    out.update(lse=torch.zeros(H, x["q"].shape[0], device="cuda"), dgamma=torch.zeros(H, device="cuda"),
               S=torch.zeros(len(LENS), H, DH, DH, device="cuda"))
    return out


def handles(x, dtype):
    from paper_2608_13578_amd import mixers
    total, n = x["q"].shape[0], len(LENS)
    return (mixers.PackedAttention(total, n, H, HKV, DH, dtype),
            mixers.AttentionDecoder(n, n, CAP, H, HKV, DH, dtype),
            mixers.LinearAttention(total, n, H, DH, dtype))


def calls(made, x, c, out, stream):
    att, dec, lin = made
    att.forward(x["q"], x["k"], x["v"], c, out["o"], out["lse"], stream=stream)
    att.backward(x["q"], x["k"], x["v"], c, out["o"], out["lse"], x["do"], out["dq"], out["dk"],
                 out["dv"], stream=stream)
    lin.forward(x["q"], x["k2"], x["v2"], x["gamma"], c, out["y"], None, out["S"], stream=stream)
    lin.backward(x["q"], x["k2"], x["v2"], x["gamma"], c, x["do"], out["eq"], out["ek"], out["ev"],
                 None, None, None, out["dgamma"], stream=stream)
    dec.step(x["q1"], x["k1"], x["v1"], None, x["length"], x["kc"], x["vc"], out["o1"], stream=stream)


def plain(x, c, dtype):
    out = outputs(x)
    calls(handles(x, dtype), x, c, out, None)
    torch.cuda.synchronize()
    return out


def same(got, want):
    for n in want:
        assert torch.equal(got[n], want[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_calls_on_a_given_stream(torch_cuda, dtype):
    """The stream as an object and as an address; memory that the current stream has
    just given back, and still writes, is not the workspace's."""
    say(f"given stream {dtype}")
    x, c = setup(dtype, 1)
    want = plain(x, c, dtype)
    s = torch.cuda.Stream()
    slow = torch.randn(4096, 4096, device="cuda")
    for stream in (s, s.cuda_stream):
        out, made = outputs(x), handles(x, dtype)
        torch.cuda.synchronize()
        for _ in range(20):  # work before the writes
            slow = slow @ slow * 1e-2
        held = [torch.empty(1 << k, dtype=torch.uint8, device="cuda") for k in range(9, 25)]
        for t in held:
            t.fill_(0xff)
        del t, held
        calls(made, x, c, out, stream)  # reads nothing that the current stream still writes
        torch.cuda.synchronize()
        same(out, want)


def test_handles_on_several_streams_at_once(torch_cuda):
    """One handle on two streams that do not wait for each other."""
    x, c = setup("bf16", 2)
    y, _ = setup("bf16", 3)
    want = plain(x, c, "bf16"), plain(y, c, "bf16")
    made = handles(x, "bf16")
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs = outputs(x), outputs(y)
    torch.cuda.synchronize()
    for _ in range(10):
        for s, z, out in zip(streams, (x, y), outs):
            calls(made, z, c, out, s)
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        same(out, w)


def test_first_calls_inside_a_capture(torch_cuda):
    """The first calls of the handles are captured; the graph replays between eager
    calls of the same handles, which have a workspace of their own."""
    x, c = setup("bf16", 4)
    want = plain(x, c, "bf16")
    made, out, eager = handles(x, "bf16"), outputs(x), outputs(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(made, x, c, out, None)
    for _ in range(4):
        for t in out.values():
            t.fill_(math.nan)
        calls(made, x, c, eager, None)
        graph.replay()
        calls(made, x, c, eager, None)
        torch.cuda.synchronize()
        same(out, want)
        same(eager, want)
