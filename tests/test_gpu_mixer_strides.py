"""Row strides of the packed-sequence mixers wider than the rows, of outputs too: the
columns between two rows keep what they held."""

import math

import pytest
import torch

import mixer_reference as ref
from test_gpu_mixers import DT, dev, i32, normal, offsets, rng
from test_gpu_parity import say, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = [(t, d) for t in ("bf16", "f32") for d in (16, 32, 64, 128)]
GAP = 24  # columns behind a row: a multiple of 16 bytes in both types
FILL = 7.0


class Columns:
    """Arrays of the given widths side by side in the rows of one, with a gap behind
    each; `ld` its row stride."""

    def __init__(self, rows, widths, dtype, fill):
        self.ld = sum(widths) + GAP * len(widths)
        self.all = torch.full((rows, self.ld), fill, dtype=DT[dtype], device="cuda")
        at = 0
        self.parts, self.gaps = [], []
        for w in widths:
            self.parts.append(self.all[:, at:at + w])
            self.gaps.append(self.all[:, at + w:at + w + GAP])
            at += w + GAP

    def put(self, *xs):
        for p, x in zip(self.parts, xs):
            p.copy_(x.reshape(x.shape[0], -1).to(p.dtype))
        return self.parts

    def untouched(self):
        return all(bool((x == FILL).all()) for x in self.gaps)


@pytest.mark.parametrize("dtype,dh", TYPES)
def test_attention(torch_cuda, dtype, dh):
    from paper_2608_13578_amd.mixers import PackedAttention
    H, Hkv, lens, lead, behind = 6, 2, [150, 1, 0, 99], 2, 3
    cu = offsets(lens, lead)
    total = cu[-1] + behind
    say(f"attention {dtype} {dh}")
    g = rng(41)
    q, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(2))
    k, v = (normal(g, total, Hkv, dh, dtype=dtype) for _ in range(2))
    want = ref.attention(q, k, v, cu, dh ** -0.5, dtype, do)
    w, wk = H * dh, Hkv * dh
    ins, grads = Columns(total, (w, wk, wk), dtype, math.nan), Columns(total, (w, wk, wk), dtype, FILL)
    up, out = Columns(total, (w,), dtype, math.nan), Columns(total, (w,), dtype, FILL)
    qd, kd, vd = ins.put(q, k, v)
    (dod,), (o,) = up.put(do), out.parts
    att = PackedAttention(total, len(lens), H, Hkv, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld,
                          ldo=out.ld)
    lse = att.new_lse()
    assert att.new_output().stride() == o.stride()
    att.forward(qd, kd, vd, i32(cu), o, lse)
    att.backward(qd, kd, vd, i32(cu), o, lse, dod, *grads.parts)
    torch.cuda.synchronize()
    rows = list(range(cu[0], cu[-1]))
    for n, x in zip(("o", "dq", "dk", "dv"), (o, *grads.parts)):
        ref.within(n, x, want[n], rows)
        assert bool((x[:lead] == FILL).all()) and bool((x[cu[-1]:] == FILL).all()), n
    assert out.untouched() and grads.untouched()


@pytest.mark.parametrize("dtype,dh", TYPES)
def test_linear_attention(torch_cuda, dtype, dh):
    from paper_2608_13578_amd.mixers import LinearAttention
    H, lens, lead, behind = 3, [150, 1, 0, 199], 2, 3
    cu = offsets(lens, lead)
    total = cu[-1] + behind
    say(f"linear attention {dtype} {dh}")
    g = rng(42)
    q, k, v, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(4))
    S0, R1 = (normal(g, len(lens), H, dh, dh) for _ in range(2))
    gam = torch.tensor([0.8, 0.97, 1.0])
    want = ref.linear(q, k, v, gam.double(), cu, dh ** -0.5, dtype, S0, do, R1)
    w = H * dh
    ins, grads = (Columns(total, (w, w, w), dtype, f) for f in (math.nan, FILL))
    up, out = Columns(total, (w,), dtype, math.nan), Columns(total, (w,), dtype, FILL)
    qd, kd, vd = ins.put(q, k, v)
    (dod,), (o,) = up.put(do), out.parts
    lin = LinearAttention(total, len(lens), H, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld, ldo=out.ld)
    S, dS, dg = lin.new_state(), lin.new_state(), torch.zeros(H, device="cuda")
    args = (qd, kd, vd, gam.cuda(), i32(cu))
    lin.forward(*args, o, S0.float().cuda(), S)
    lin.backward(*args, dod, *grads.parts, S0.float().cuda(), R1.float().cuda(), dS, dg)
    torch.cuda.synchronize()
    rows = list(range(cu[0], cu[-1]))
    for n, x in zip(("o", "dq", "dk", "dv"), (o, *grads.parts)):
        ref.within(n, x, want[n], rows)
        assert bool((x[:lead] == FILL).all()) and bool((x[cu[-1]:] == FILL).all()), n
    for n, x in (("S", S), ("dS", dS), ("dgamma", dg)):
        ref.within(n, x, want[n])
    assert out.untouched() and grads.untouched()


@pytest.mark.parametrize("cap", [70, 5000])
@pytest.mark.parametrize("dtype,dh", TYPES)
def test_single_tokens(torch_cuda, dtype, dh, cap):
    """The projection's row of a token read in place; outputs in rows with a gap."""
    from paper_2608_13578_amd.mixers import AttentionDecoder, LinearAttentionDecoder
    H, Hkv, lens = 6, 2, [cap - 1, 33, 0, -1]
    B, w, wk = len(lens), H * dh, Hkv * dh
    say(f"single tokens {dtype} {dh} {cap}")
    g = rng(43)
    q = normal(g, B, H, dh, dtype=dtype)
    k, v = (normal(g, B, Hkv, dh, dtype=dtype) for _ in range(2))
    kc, vc = (normal(g, B, cap, Hkv, dh, dtype=dtype) for _ in range(2))
    ins, out = Columns(B, (w, wk, wk), dtype, math.nan), Columns(B, (w,), dtype, FILL)
    (o,) = out.parts
    d = AttentionDecoder(B, B, cap, H, Hkv, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld, ldo=out.ld)
    d.step(*ins.put(q, k, v), None, i32(lens), dev(kc, dtype), dev(vc, dtype), o)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        if n < 0:
            assert bool((o[b] == 0).all())
            continue
        ref.within(f"o[{b}]", o[b], ref.token(q[b], torch.cat([kc[b, :n], k[b][None]]),
                                              torch.cat([vc[b, :n], v[b][None]]), dh ** -0.5, dtype))
    assert out.untouched()

    k, v = (normal(g, B, H, dh, dtype=dtype) for _ in range(2))
    gam, S0 = torch.linspace(0.5, 1.0, H), normal(g, B, H, dh, dh)
    ins, out = Columns(B, (w, w, w), dtype, math.nan), Columns(B, (w,), dtype, FILL)
    (o,) = out.parts
    d = LinearAttentionDecoder(B, B, H, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld, ldo=out.ld)
    S = S0.float().cuda()
    d.step(*ins.put(q, k, v), gam.cuda(), i32([3, 1, -1, 0]), S, S, o)
    torch.cuda.synchronize()
    for b, s in enumerate((3, 1, -1, 0)):
        if s < 0:
            assert bool((o[b] == 0).all())
            continue
        r = ref.linear(q[b:b + 1], k[b:b + 1], v[b:b + 1], gam.double(), [0, 1], dh ** -0.5, dtype,
                       S0[s:s + 1])
        ref.within("o", o[b:b + 1], r["o"])
        ref.within("S", S[s:s + 1], r["S"])
    assert torch.equal(S[2].double().cpu(), S0[2]) and out.untouched()
