"""Every array that the packed-sequence entry points write lies between guards, before
and behind, and so does their scratch; offsets, slots and lengths are out of range.
The calls go through the binding, with scratch of exactly the stated size."""

import pytest
import torch

import mixer_reference as ref
from test_gpu_mixers import DT, dev, i32, normal, rng
from test_gpu_parity import say, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

PAD = 1 << 16  # bytes on both sides: more than 64 rows of any array here
MARK = 0x5a


class Guarded:
    """Arrays of device memory between marked bytes."""

    def __init__(self):
        self.held = []

    def new(self, shape, dtype):
        n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
        room = torch.full((n + 2 * PAD,), MARK, dtype=torch.uint8, device="cuda")
        self.held.append((room, n))
        t = room[PAD:PAD + n].view(dtype).view(shape)
        t.zero_()
        return t

    def put(self, x):
        t = self.new(x.shape, x.dtype)
        t.copy_(x)
        return t

    def scratch(self, n):
        return self.new((n,), torch.uint8) if n else None

    def check(self):
        torch.cuda.synchronize()
        for room, n in self.held:
            assert bool((room[:PAD] == MARK).all()) and bool((room[PAD + n:] == MARK).all())


TYPES = [("bf16", 64), ("f32", 16), ("bf16", 128), ("f32", 64)]
# offsets, and what they are clamped to where that is in order
OFFSETS = [([0, 300, 301, 700], [0, 300, 301, 700]),
           ([-5, 200, 2000000000, 2147483647], [0, 200, 700, 700]),
           ([-2147483648, -64, 333, 2147483647], [0, 0, 333, 700]),
           ([0, 500, 50, 700], None), ([0, 1 << 30, 5, -7], None), ([700, 0, 700, 0], None),
           ([2147483647, -2147483648, 2147483647, -2147483648], None)]


@pytest.mark.parametrize("dtype,dh", TYPES)
def test_attention(torch_cuda, dtype, dh):
    from paper_2608_13578_amd import bcmt as abi
    total, H, Hkv, n = 700, 4, 2, 3
    g, G = rng(31), Guarded()
    q, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(2))
    k, v = (normal(g, total, Hkv, dh, dtype=dtype) for _ in range(2))
    qd, kd, vd, dod = (dev(x, dtype) for x in (q, k, v, do))
    o, dq = (G.new((total, H, dh), DT[dtype]) for _ in range(2))
    dk, dv = (G.new((total, Hkv, dh), DT[dtype]) for _ in range(2))
    lse = G.new((H, total), torch.float32)
    cfg = abi.make_attn_config(total, n, H, Hkv, dh, dtype)
    ws = G.scratch(abi.bcmt_attn_workspace_bytes(cfg))
    outs = dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)

    def run(cu):
        c = i32(cu)
        abi.bcmt_attn_forward(cfg, qd, kd, vd, c, o, lse)
        abi.bcmt_attn_backward(cfg, qd, kd, vd, c, o, lse, dod, dq, dk, dv, ws)
        G.check()
        return {m: x.clone() for m, x in outs.items()}

    for cu, clamped in OFFSETS:
        say(f"attention {dtype} {dh} {cu}")
        got = run(cu)
        if clamped is None:
            continue
        want = ref.attention(q, k, v, clamped, dh ** -0.5, dtype, do)
        for m, x in got.items():
            ref.within(m, x, want[m])
        for m, x in run(clamped).items():
            assert torch.equal(x, got[m]), m


@pytest.mark.parametrize("dtype,dh", TYPES)
def test_linear_attention(torch_cuda, dtype, dh):
    from paper_2608_13578_amd import bcmt as abi
    total, H, n = 700, 3, 3
    g, G = rng(32), Guarded()
    q, k, v, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(4))
    S0, R1 = (normal(g, n, H, dh, dh) for _ in range(2))
    gam = torch.tensor([0.8, 0.97, 1.0])
    qd, kd, vd, dod = (dev(x, dtype) for x in (q, k, v, do))
    s_in, ds_out, gamma = S0.float().cuda(), R1.float().cuda(), gam.cuda()
    o, dq, dk, dv = (G.new((total, H, dh), DT[dtype]) for _ in range(4))
    S, dS = (G.new((n, H, dh, dh), torch.float32) for _ in range(2))
    dg = G.new((H,), torch.float32)
    cfg = abi.make_linattn_config(total, n, H, dh, dtype)
    ws, ws_bwd = (G.scratch(abi.bcmt_linattn_workspace_bytes(cfg, p))
                  for p in (abi.BCMT_PASS_FORWARD, abi.BCMT_PASS_BACKWARD))
    outs = dict(o=o, S=S, dq=dq, dk=dk, dv=dv, dS=dS, dgamma=dg)

    def run(cu):
        c = i32(cu)
        abi.bcmt_linattn_forward(cfg, qd, kd, vd, gamma, c, s_in, o, S, ws)
        abi.bcmt_linattn_backward(cfg, qd, kd, vd, gamma, c, s_in, dod, ds_out, dq, dk, dv, dS, dg,
                                  ws_bwd)
        G.check()
        return {m: x.clone() for m, x in outs.items()}

    for cu, clamped in OFFSETS:
        say(f"linear attention {dtype} {dh} {cu}")
        got = run(cu)
        if clamped is None:
            continue
        want = ref.linear(q, k, v, gam.double(), clamped, dh ** -0.5, dtype, S0, do, R1)
        for m, x in got.items():
            ref.within(m, x, want[m])
        for m, x in run(clamped).items():
            assert torch.equal(x, got[m]), m


OUTSIDE = [-1, 3, 1 << 30, 2147483647, -2147483648]


@pytest.mark.parametrize("cap", [90, 5000])
@pytest.mark.parametrize("dtype,dh", TYPES)
def test_single_tokens(torch_cuda, dtype, dh, cap):
    """Slots and lengths out of range among good ones."""
    from paper_2608_13578_amd import bcmt as abi
    slots, H, Hkv = 3, 4, 2
    slot = [2, *OUTSIDE, 1, 1, 0]
    length = [cap - 1, 0, 1, 2, 3, 4, cap, -7, 2147483647]
    B = len(slot)
    say(f"single tokens {dtype} {dh} {cap}")
    g, G = rng(33), Guarded()
    q = normal(g, B, H, dh, dtype=dtype)
    k, v = (normal(g, B, Hkv, dh, dtype=dtype) for _ in range(2))
    kc, vc = (normal(g, slots, cap, Hkv, dh, dtype=dtype) for _ in range(2))
    qd, kd, vd = (dev(x, dtype) for x in (q, k, v))
    kcd, vcd = (G.put(dev(x, dtype)) for x in (kc, vc))
    before = kcd.clone(), vcd.clone()
    o = G.new((B, H, dh), DT[dtype])
    o.fill_(7.0)
    cfg = abi.make_attn_decode_config(B, slots, cap, H, Hkv, dh, dtype)
    ws = G.scratch(abi.bcmt_attn_decode_workspace_bytes(cfg))
    abi.bcmt_attn_decode(cfg, qd, kd, vd, i32(slot), i32(length), kcd, vcd, o, ws)
    G.check()
    want = ref.token(q[0], torch.cat([kc[2, :cap - 1], k[0][None]]),
                     torch.cat([vc[2, :cap - 1], v[0][None]]), dh ** -0.5, dtype)
    ref.within("o", o[0], want)
    assert bool((o[1:] == 0).all())
    before[0][2, cap - 1], before[1][2, cap - 1] = kd[0], vd[0]
    assert torch.equal(kcd, before[0]) and torch.equal(vcd, before[1])

    k2, v2 = (normal(g, B, H, dh, dtype=dtype) for _ in range(2))
    gam = torch.tensor([0.5, 0.8, 0.97, 1.0])
    S0 = normal(g, slots, H, dh, dh)
    s_in = S0.float().cuda()
    S = G.new((slots, H, dh, dh), torch.float32)
    S.fill_(7.0)
    o.fill_(7.0)
    slot = [2, *OUTSIDE, -2, 0]
    cfg = abi.make_linattn_step_config(len(slot), slots, H, dh, dtype)
    m = len(slot)
    abi.bcmt_linattn_step(cfg, qd[:m], dev(k2[:m], dtype), dev(v2[:m], dtype), gam.cuda(), i32(slot),
                          s_in, S, o[:m])
    G.check()
    for b in (0, m - 1):
        r = ref.linear(q[b:b + 1], k2[b:b + 1], v2[b:b + 1], gam.double(), [0, 1], dh ** -0.5, dtype,
                       S0[slot[b]:slot[b] + 1])
        ref.within("o", o[b:b + 1], r["o"])
        ref.within("S", S[slot[b]:slot[b] + 1], r["S"])
    assert bool((o[1:m - 1] == 0).all()) and bool((o[m:] == 7.0).all()) and bool((S[1] == 7.0).all())
