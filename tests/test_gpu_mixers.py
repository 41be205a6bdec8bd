"""Attention and linear attention over packed sequences on the GPU, against the
64-bit references of mixer_reference.py and their element-wise bounds."""

import math

import pytest
import torch

import mixer_reference as ref
from test_gpu_parity import say, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype="f32", std=1.0):
    """Host values representable in the type, as float64."""
    return (torch.randn(shape, generator=g) * std).to(DT[dtype]).double()


def dev(x, dtype):
    return x.to(DT[dtype]).cuda()


def offsets(lens, lead=0):
    cu = [lead]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Fused:
    """q, k, v as columns of one array, or as three dense ones."""

    def __init__(self, total, H, Hkv, dh, dtype, fused, fill=None):
        w = (H * dh, Hkv * dh, Hkv * dh)
        make = torch.zeros if fill is None else (lambda *s, **k: torch.full(s[0], fill, **k))
        kw = dict(dtype=DT[dtype], device="cuda")
        if fused:
            self.ld = sum(w)
            self.parts = make((total, sum(w)), **kw).split(w, dim=1)
        else:
            self.ld = 0
            self.parts = [make((total, x), **kw) for x in w]

    def set(self, *xs):
        for p, x in zip(self.parts, xs):
            p.copy_(x.reshape(x.shape[0], -1).to(p.dtype))
        return self.parts


ATTN = [
    # dtype, dh, H, Hkv, lengths, rows before, rows behind, fused, factor of q
    ("bf16", 64, 4, 2, [1, 63, 64, 65, 0, 130], 0, 0, True, 1.0),
    ("bf16", 64, 3, 1, [127, 128, 129, 257], 5, 7, False, 1.0),
    ("bf16", 128, 4, 1, [200, 1, 77], 3, 1, True, 1.0),
    ("bf16", 128, 2, 2, [513], 0, 9, False, 6.0),
    ("bf16", 32, 5, 5, [33, 31, 300], 0, 2, True, 1.0),
    ("bf16", 16, 8, 8, [16, 17, 0, 0, 200], 1, 0, False, 4.0),
    ("bf16", 64, 16, 1, [190], 0, 0, False, 1.0),
    ("f32", 64, 4, 2, [1, 63, 64, 65, 0, 130], 2, 3, True, 1.0),
    ("f32", 128, 2, 1, [70, 129], 0, 5, False, 1.0),
    ("f32", 32, 3, 3, [257, 2], 4, 0, True, 6.0),
    ("f32", 16, 8, 2, [100, 1, 1, 65], 0, 1, False, 1.0),
    ("bf16", 64, 2, 1, [1] * 150, 0, 0, False, 1.0),
    ("f32", 64, 1, 1, [1], 0, 0, False, 1.0),
    ("bf16", 64, 12, 4, [700, 300], 0, 0, True, 1.0),
]


def attn_inputs(case, seed=0):
    dtype, dh, H, Hkv, lens, lead, behind, fused, f = case
    cu = offsets(lens, lead)
    total = cu[-1] + behind
    g = rng(seed)
    q = normal(g, total, H, dh, dtype=dtype)
    q = (q * f).to(DT[dtype]).double()
    k, v, do = (normal(g, total, h, dh, dtype=dtype) for h in (Hkv, Hkv, H))
    return cu, total, q, k, v, do


@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"{c[0]}-dh{c[1]}-H{c[2]}.{c[3]}-{sum(c[4])}rows")
def test_attention(torch_cuda, case):
    from paper_2608_13578_amd.mixers import PackedAttention
    dtype, dh, H, Hkv, lens, lead, behind, fused, f = case
    say(f"attention {case}")
    cu, total, q, k, v, do = attn_inputs(case)
    want = ref.attention(q, k, v, cu, dh ** -0.5, dtype, do)
    ins = Fused(total, H, Hkv, dh, dtype, fused)
    qd, kd, vd = ins.set(q, k, v)
    outside = list(range(cu[0])) + list(range(cu[-1], total))
    for x in (qd, kd, vd):  # rows of no sequence are not read
        x[outside] = math.nan
    grads = Fused(total, H, Hkv, dh, dtype, fused, fill=7.0)
    dq, dk, dv = grads.parts
    att = PackedAttention(total, len(lens), H, Hkv, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld)
    o = torch.full((total, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((H, total), 7.0, device="cuda")
    dod = dev(do, dtype)
    dod[outside] = math.nan
    c = i32(cu)

    def run():
        att.forward(qd, kd, vd, c, o, lse)
        att.backward(qd, kd, vd, c, o, lse, dod, dq, dk, dv)
        torch.cuda.synchronize()

    run()
    rows = list(range(cu[0], cu[-1]))
    worst = {"o": ref.within("o", o, want["o"], rows)}
    worst["lse"] = ref.within("lse", lse.T, (want["lse"][0].T, want["lse"][1].T), rows)
    for n, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        worst[n] = ref.within(n, x, want[n], rows)
        assert bool((x[outside] == 7.0).all()), n  # and not written
    assert bool((o[outside] == 7.0).all()) and bool((lse[:, outside] == 7.0).all())
    say("  of the bounds: " + ", ".join(f"{n} {x:.2f}" for n, x in worst.items()))
    first = [x.clone() for x in (o, lse, dq, dk, dv)]
    run()
    for x, y in zip(first, (o, lse, dq, dk, dv)):
        assert torch.equal(x, y)
    o2 = torch.zeros_like(o)
    att.forward(qd, kd, vd, c, o2)  # without lse
    torch.cuda.synchronize()
    assert torch.equal(o2[rows], o[rows])


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 32), ("bf16", 128), ("bf16", 16)])
def test_attention_values_that_are_not_finite(torch_cuda, dtype, dh):
    """An infinite or NaN key or value changes no row that does not see it."""
    from paper_2608_13578_amd.mixers import PackedAttention
    case = (dtype, dh, 2, 1, [150, 90, 40], 0, 0, False, 1.0)
    cu, total, q, k, v, do = attn_inputs(case, 3)
    want = ref.attention(q, k, v, cu, dh ** -0.5, dtype)
    qd, kd, vd = (dev(x, dtype) for x in (q, k, v))
    at = 100  # in the first sequence
    vd[at] = math.inf
    vd[150 + 89, 0, 3] = math.nan  # the second one's last row
    kd[260, 0, 0] = math.nan       # in the third
    att = PackedAttention(total, 3, 2, 1, dh, dtype)
    o = torch.zeros_like(qd)
    att.forward(qd, kd, vd, i32(cu), o)
    torch.cuda.synchronize()
    clean = list(range(at)) + list(range(150, 239)) + list(range(240, 260))
    ref.within("o", o, want["o"], clean)
    assert not bool(torch.isfinite(o[at:150].float()).any())
    last = o[239].float()
    assert bool(torch.isnan(last[:, 3]).all()) and bool(torch.isfinite(last[:, :3]).all())
    assert bool(torch.isnan(o[260:].float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_first_scores_minus_infinity(torch_cuda, dtype):
    """Scores of -inf at the start of a row (no weight) leave later ones as they are."""
    from paper_2608_13578_amd.mixers import PackedAttention
    dh, n = 64, 150
    g = rng(5)
    q, k, v = (normal(g, n, 1, dh, dtype=dtype) for _ in range(3))
    q[:, 0, 0] = 1.0
    kinf = k.clone()
    kinf[:70, 0, 0] = -math.inf
    want = ref.attention(q[70:], k[70:], v[70:], [0, n - 70], dh ** -0.5, dtype)
    o = torch.zeros(n, 1, dh, dtype=DT[dtype], device="cuda")
    PackedAttention(n, 1, 1, 1, dh, dtype).forward(dev(q, dtype), dev(kinf, dtype), dev(v, dtype),
                                                   i32([0, n]), o)
    torch.cuda.synchronize()
    ref.within("o", o[70:], want["o"])


def test_offsets_out_of_order_stay_inside(torch_cuda):
    """Offsets outside the arrays or out of order are clamped: rows of the
    sequences that are in order come out, and nothing outside is written."""
    from paper_2608_13578_amd.mixers import LinearAttention, PackedAttention
    total, H, dh = 300, 2, 64
    g = rng(1)
    q, k, v = (normal(g, total, H, dh, dtype="bf16") for _ in range(3))
    guard = torch.full((total + 64, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    for cu in ([0, 100, 50, 300], [0, 1 << 30, 5, -7], [-5, 200, 2000000000, 2147483647]):
        c = i32(cu)
        o = guard[:total]
        ins = [dev(x, "bf16") for x in (q, k, v)]
        PackedAttention(total, 3, H, H, dh).forward(*ins, c, o)
        LinearAttention(total, 3, H, dh).forward(*ins, torch.full((H,), 0.9, device="cuda"), c, o)
        torch.cuda.synchronize()
        assert bool((guard[total:] == 7.0).all())


DECODE = [
    # dtype, dh, B, slots, cap, H, Hkv, lengths (-1, cap: inactive), head-major cache
    ("bf16", 64, 5, 7, 700, 8, 2, [0, 1, 31, 32, 699], False),
    ("bf16", 128, 3, 3, 1000, 8, 1, [999, 500, -1], True),
    ("bf16", 64, 2, 2, 64, 40, 2, [63, 33], False),
    ("bf16", 16, 3, 4, 300, 8, 8, [299, 128, 127], False),
    ("bf16", 32, 2, 5, 130, 6, 3, [129, 64], True),
    ("f32", 64, 3, 4, 400, 4, 4, [399, 400, 17], False),
    ("f32", 128, 2, 2, 200, 6, 2, [199, 3], False),
    ("f32", 16, 2, 2, 90, 4, 1, [89, 0], True),
    ("bf16", 64, 1, 1, 1, 2, 2, [0], False),
    ("bf16", 64, 64, 64, 300, 16, 8, [(37 * b) % 300 for b in range(64)], False),
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"{c[0]}-dh{c[1]}-B{c[2]}-cap{c[4]}-H{c[5]}.{c[6]}")
def test_attention_decode(torch_cuda, case):
    from paper_2608_13578_amd.mixers import AttentionDecoder
    dtype, dh, B, slots, cap, H, Hkv, lens, head_major = case
    say(f"decode {case}")
    g = rng(2)
    q, k, v = (normal(g, B, h, dh, dtype=dtype) for h in (H, Hkv, Hkv))
    kc, vc = (normal(g, slots, cap, Hkv, dh, dtype=dtype) for _ in range(2))
    slot = torch.randperm(slots, generator=g)[:B].tolist()
    kd, vd = dev(kc, dtype), dev(vc, dtype)
    for b, n in enumerate(lens):  # rows behind the token hold anything
        if 0 <= n < cap:
            kd[slot[b], n:] = math.nan
            vd[slot[b], n:] = math.inf
    strides = {}
    if head_major:  # [slots, Hkv, cap, dh]
        kd, vd = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kd, vd))
        strides = dict(cs=Hkv * cap * dh, ct=dh, ch=cap * dh)
    before = kd.clone(), vd.clone()
    o = torch.full((B, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    d = AttentionDecoder(B, slots, cap, H, Hkv, dh, dtype, **strides)
    args = (dev(q, dtype), dev(k, dtype), dev(v, dtype), i32(slot), i32(lens), kd, vd)
    d.step(*args, o)
    d.step(*args, o)  # the same call again changes nothing
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        s = slot[b]
        if not 0 <= n < cap:
            assert bool((o[b] == 0).all())
            continue
        kk, vv = torch.cat([kc[s, :n], k[b][None]]), torch.cat([vc[s, :n], v[b][None]])
        qq = torch.zeros(n + 1, H, dh, dtype=torch.float64)
        qq[n] = q[b]
        want = ref.attention(qq, kk, vv, [0, n + 1], dh ** -0.5, dtype)["o"]
        ref.within(f"o[{b}]", o[b], (want[0][n], want[1][n]))
        before[0][s, n], before[1][s, n] = args[1][b], args[2][b]
    for x, y in zip((kd, vd), before):
        assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))


def test_attention_decode_slots_outside_the_pool(torch_cuda):
    from paper_2608_13578_amd.mixers import AttentionDecoder
    B, slots, cap, H, dh = 4, 2, 50, 2, 64
    g = rng(4)
    q, k, v = (dev(normal(g, B, H, dh, dtype="bf16"), "bf16") for _ in range(3))
    d = AttentionDecoder(B, slots, cap, H, H, dh)
    kc, vc = d.new_cache(), d.new_cache()
    o = torch.full((B, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    d.step(q, k, v, i32([1, -1, 2, 1 << 30]), i32([0, 0, 0, 0]), kc, vc, o)
    torch.cuda.synchronize()
    assert torch.equal(o[0], v[0]) and bool((o[1:] == 0).all())
    assert torch.equal(kc[1, 0], k[0]) and float(kc[0].abs().max()) == 0
    # no slots: sequence b in slot b
    d2 = AttentionDecoder(2, 2, cap, H, H, dh)
    d2.step(q[:2], k[:2], v[:2], None, i32([0, 3]), kc, vc, o[:2])
    torch.cuda.synchronize()
    assert torch.equal(kc[0, 0], k[0]) and torch.equal(kc[1, 3], k[1])


def test_offsets_past_32_bits(torch_cuda):
    """Caches and rows further apart than 2^32 bytes."""
    from paper_2608_13578_amd.mixers import AttentionDecoder, LinearAttention, PackedAttention
    dh, cap, slots = 64, 40, 3
    cs = (1 << 31) + 8  # elements
    room = torch.empty((slots - 1) * cs + cap * dh, dtype=torch.bfloat16, device="cuda")
    kd, vd = (room.as_strided((slots, cap // 2, 1, dh), (cs, 2 * dh, dh, 1), i * dh) for i in (0, 1))
    g = rng(6)
    kc, vc = (normal(g, slots, cap // 2, 1, dh, dtype="bf16") for _ in range(2))
    kd.copy_(dev(kc, "bf16"))
    vd.copy_(dev(vc, "bf16"))
    q, k, v = (normal(g, slots, 1, dh, dtype="bf16") for _ in range(3))
    o = torch.zeros(slots, 1, dh, dtype=torch.bfloat16, device="cuda")
    d = AttentionDecoder(slots, slots, cap // 2, 1, 1, dh, cs=cs, ct=2 * dh, ch=dh)
    d.step(dev(q, "bf16"), dev(k, "bf16"), dev(v, "bf16"), None, i32([19, 5, 12]), kd, vd, o)
    torch.cuda.synchronize()
    for b, n in enumerate((19, 5, 12)):
        qq = torch.zeros(n + 1, 1, dh, dtype=torch.float64)
        qq[n] = q[b]
        want = ref.attention(qq, torch.cat([kc[b, :n], k[b][None]]), torch.cat([vc[b, :n], v[b][None]]),
                             [0, n + 1], dh ** -0.5, "bf16")["o"]
        ref.within("o", o[b], (want[0][n], want[1][n]))
    del kd, vd
    total, ld = 200, 1 << 24
    x = room.as_strided((total, 3, dh), (ld, dh, 1))
    q, k, v = (normal(g, total, 1, dh, dtype="bf16") for _ in range(3))
    for i, y in enumerate((q, k, v)):
        x[:, i:i + 1].copy_(dev(y, "bf16"))
    o = torch.zeros(total, 1, dh, dtype=torch.bfloat16, device="cuda")
    parts = [x[:, i] for i in range(3)]
    PackedAttention(total, 1, 1, 1, dh, ldq=ld, ldk=ld, ldv=ld).forward(*parts, i32([0, total]), o)
    torch.cuda.synchronize()
    ref.within("o", o, ref.attention(q, k, v, [0, total], dh ** -0.5, "bf16")["o"])
    LinearAttention(total, 1, 1, dh, ldq=ld, ldk=ld, ldv=ld).forward(
        *parts, torch.full((1,), 0.95, device="cuda"), i32([0, total]), o)
    torch.cuda.synchronize()
    gam = torch.full((1,), 0.95).double()
    ref.within("o", o, ref.linear(q, k, v, gam, [0, total], dh ** -0.5, "bf16")["o"])


LINEAR = [
    # dtype, dh, decays, lengths, rows before, rows behind, fused, states
    ("bf16", 64, [0.9, 0.999, 1.0], [1, 63, 64, 65, 0, 130], 0, 0, True, True),
    ("bf16", 64, [0.0, 0.5], [700], 3, 5, False, True),
    ("bf16", 64, [0.97], [300, 513, 1, 0, 257], 0, 0, False, False),
    ("bf16", 128, [0.99, 0.8], [129, 600], 2, 0, True, True),
    ("bf16", 32, [0.3, 0.95, 0.9995], [40, 400], 0, 3, False, True),
    ("bf16", 16, [0.9] * 5, [1, 2, 300, 17], 0, 0, True, True),
    ("f32", 64, [0.9, 0.999, 1.0], [1, 63, 64, 65, 0, 130], 1, 2, False, True),
    ("f32", 128, [0.97], [300], 0, 0, True, True),
    ("f32", 32, [0.0, 0.99], [600, 1], 0, 0, False, True),
    ("f32", 16, [0.5, 1.0], [100, 0, 290], 0, 7, True, True),
    ("f32", 64, [0.9], [1], 0, 0, False, False),
    ("bf16", 64, [0.9, 0.99], [1, 2, 3] * 60, 0, 0, False, True),
]


@pytest.mark.parametrize("case", LINEAR, ids=lambda c: f"{c[0]}-dh{c[1]}-H{len(c[2])}-{sum(c[3])}rows")
def test_linear_attention(torch_cuda, case):
    from paper_2608_13578_amd.mixers import LinearAttention
    dtype, dh, decays, lens, lead, behind, fused, states = case
    say(f"linear attention {dtype} {dh} {len(decays)} heads {lens}")
    H, cu, scale = len(decays), offsets(lens, lead), dh ** -0.5
    total = cu[-1] + behind
    g = rng(7)
    q, k, v, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(4))
    gam = torch.tensor(decays, dtype=torch.float32)
    S_in = normal(g, len(lens), H, dh, dh) if states else None
    dS_out = normal(g, len(lens), H, dh, dh) if states else None
    want = ref.linear(q, k, v, gam.double(), cu, scale, dtype, S_in, do, dS_out)
    ins = Fused(total, H, H, dh, dtype, fused)
    qd, kd, vd = ins.set(q, k, v)
    outside = list(range(cu[0])) + list(range(cu[-1], total))
    dod = dev(do, dtype)
    for x in (qd, kd, vd, dod):
        x[outside] = math.nan
    dq, dk, dv = Fused(total, H, H, dh, dtype, fused, fill=7.0).parts
    la = LinearAttention(total, len(lens), H, dh, dtype, ldq=ins.ld, ldk=ins.ld, ldv=ins.ld)
    o = torch.full((total, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    sin = dev(S_in, "f32") if states else None
    dso = dev(dS_out, "f32") if states else None
    S, dS = la.new_state(), la.new_state()
    dg = torch.empty(H, device="cuda")
    gd, c = gam.cuda(), i32(cu)
    rows = list(range(cu[0], cu[-1]))

    def check():
        torch.cuda.synchronize()
        worst = {"o": ref.within("o", o, want["o"], rows), "S": ref.within("S", S, want["S"])}
        for n, x in (("dq", dq), ("dk", dk), ("dv", dv)):
            worst[n] = ref.within(n, x, want[n], rows)
            assert bool((x[outside] == 7.0).all()), n
        worst["dS"] = ref.within("dS", dS, want["dS"])
        worst["dgamma"] = ref.within("dgamma", dg, want["dgamma"])
        assert bool((o[outside] == 7.0).all())
        say("  of the bounds: " + ", ".join(f"{n} {x:.2f}" for n, x in worst.items()))

    la.forward(qd, kd, vd, gd, c, o, sin, S)
    la.backward(qd, kd, vd, gd, c, dod, dq, dk, dv, sin, dso, dS, dg)
    check()
    first = [x.clone() for x in (o, S, dq, dk, dv, dS, dg)]
    la.forward(qd, kd, vd, gd, c, o, sin, S)
    la.backward(qd, kd, vd, gd, c, dod, dq, dk, dv, sin, dso, dS, dg)
    torch.cuda.synchronize()
    for x, y in zip(first, (o, S, dq, dk, dv, dS, dg)):
        assert torch.equal(x, y)
    if states:  # the states in place
        S, dS = sin.clone(), dso.clone()
        la.forward(qd, kd, vd, gd, c, o, S, S)
        la.backward(qd, kd, vd, gd, c, dod, dq, dk, dv, sin, dS, dS, dg)
        torch.cuda.synchronize()
        for x, y in zip(first, (o, S, dq, dk, dv, dS, dg)):
            assert torch.equal(x, y)
    # without states and decay gradient wanted
    o2 = torch.zeros_like(o)
    la.forward(qd, kd, vd, gd, c, o2, sin)
    d2 = [torch.zeros((total, H, dh), dtype=DT[dtype], device="cuda") for _ in range(3)]
    la2 = LinearAttention(total, len(lens), H, dh, dtype)
    la2.backward(*(x.reshape(total, H, dh).contiguous() for x in (qd, kd, vd)), gd, c, dod, *d2, sin, dso)
    torch.cuda.synchronize()
    assert torch.equal(o2[rows], o[rows])
    for x, y in zip(d2, (dq, dk, dv)):
        assert torch.equal(x[rows].reshape(-1), y[rows].reshape(-1))


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 32)])
def test_linear_attention_values_that_are_not_finite(torch_cuda, dtype, dh):
    from paper_2608_13578_amd.mixers import LinearAttention
    n, H, at = 400, 2, 150
    g = rng(8)
    q, k, v = (normal(g, n, H, dh, dtype=dtype) for _ in range(3))
    gam = torch.tensor([0.9, 0.99])
    want = ref.linear(q, k, v, gam.double(), [0, n], dh ** -0.5, dtype)
    qd, kd, vd = (dev(x, dtype) for x in (q, k, v))
    vd[at] = math.inf
    o = torch.zeros_like(qd)
    LinearAttention(n, 1, H, dh, dtype).forward(qd, kd, vd, gam.cuda(), i32([0, n]), o)
    torch.cuda.synchronize()
    ref.within("o", o, want["o"], list(range(at)))
    assert not bool(torch.isfinite(o[at].float()).any())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 16), ("bf16", 128)])
def test_linear_attention_by_pieces_and_tokens(torch_cuda, dtype, dh):
    """A prompt in pieces on carried states, then single tokens on a pool of
    states, against the whole sequence."""
    from paper_2608_13578_amd.mixers import LinearAttention, LinearAttentionDecoder
    H, lens, cuts = 3, [330, 200], (0, 90, 91, 180)
    g = rng(9)
    B, n = len(lens), max(lens)
    q, k, v = (normal(g, B, n, H, dh, dtype=dtype) for _ in range(3))
    gam = torch.tensor([0.7, 0.98, 1.0])
    gd = gam.cuda()
    la = [LinearAttention(B * (b - a), B, H, dh, dtype) for a, b in zip(cuts, cuts[1:])]
    S = torch.zeros(B, H, dh, dh, device="cuda")
    got = torch.zeros(B, n, H, dh, dtype=DT[dtype], device="cuda")
    for m, a, b in zip(la, cuts, cuts[1:]):
        x = [dev(t[:, a:b].reshape(-1, H, dh), dtype) for t in (q, k, v)]
        o = torch.empty_like(x[0])
        m.forward(*x, gd, i32([0, b - a, 2 * (b - a)]), o, S, S)
        got[:, a:b] = o.reshape(B, b - a, H, dh)
    slots = 5
    pool = torch.full((slots, H, dh, dh), 3.0, device="cuda")
    place = [3, 1]
    pool[place] = S
    step = LinearAttentionDecoder(B, slots, H, dh, dtype)
    for t in range(cuts[-1], n):
        live = [place[b] if t < lens[b] else -1 for b in range(B)]
        x = [dev(y[:, t].contiguous(), dtype) for y in (q, k, v)]
        o = torch.full_like(x[0], 7.0)
        step.step(*x, gd, i32(live), pool, pool, o)
        got[:, t] = o
    torch.cuda.synchronize()
    for b in range(B):
        w = ref.linear(q[b, :lens[b]], k[b, :lens[b]], v[b, :lens[b]], gam.double(), [0, lens[b]],
                       dh ** -0.5, dtype)
        ref.within("o", got[b, :lens[b]], w["o"])
        ref.within("S", pool[place[b]], (w["S"][0][0], w["S"][1][0]))
        assert bool((got[b, lens[b]:] == 0).all())
    assert bool((pool[[0, 2, 4]] == 3.0).all())


@pytest.mark.parametrize("dtype,dh", [(t, d) for t in ("bf16", "f32") for d in (16, 32, 64, 128)])
def test_linear_attention_step(torch_cuda, dtype, dh):
    from paper_2608_13578_amd.mixers import LinearAttentionDecoder
    B, slots, H = 7, 9, 3
    g = rng(10)
    q, k, v = (normal(g, B, H, dh, dtype=dtype) for _ in range(3))
    S = normal(g, slots, H, dh, dh)
    gam = torch.tensor([0.0, 0.9, 1.0])
    slot = [4, -1, 0, 9, 8, 2, 1 << 30]
    d = LinearAttentionDecoder(B, slots, H, dh, dtype, scale=0.3)
    sd = S.float().cuda()
    out = torch.full_like(sd, 7.0)
    o = torch.full((B, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    args = [dev(x, dtype) for x in (q, k, v)]
    d.step(*args, gam.cuda(), i32(slot), sd, out, o)
    inplace, o2 = sd.clone(), torch.empty_like(o)
    d.step(*args, gam.cuda(), i32(slot), inplace, inplace, o2)
    torch.cuda.synchronize()
    assert torch.equal(o, o2)
    for b, s in enumerate(slot):
        if not 0 <= s < slots:
            assert bool((o[b] == 0).all())
            continue
        w = ref.linear(q[b][None], k[b][None], v[b][None], gam.double(), [0, 1], 0.3, dtype,
                       S_in=S[s][None])
        ref.within("o", o[b], w["o"])
        ref.within("S", out[s], w["S"])
        assert torch.equal(out[s], inplace[s])
    for s in set(range(slots)) - set(slot):
        assert bool((out[s] == 7.0).all()) and torch.equal(inplace[s], sd[s])


def test_gradients_against_differences(torch_cuda):
    """Float32 gradients against central differences of the forward passes."""
    from paper_2608_13578_amd.mixers import LinearAttention, PackedAttention
    H, Hkv, dh, cu = 2, 1, 16, [0, 37, 90]
    g = rng(11)
    total = cu[-1]
    x = {n: normal(g, total, h, dh) for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("do", H))}
    d = {n: normal(g, *x[n].shape) for n in ("q", "k", "v")}
    d = {n: t / t.norm() for n, t in d.items()}
    c = i32(cu)
    f = lambda t: t.float().cuda()  # noqa: E731
    att = PackedAttention(total, 2, H, Hkv, dh, "f32")

    def loss(q, k, v):
        o = torch.empty(total, H, dh, device="cuda")
        att.forward(f(q), f(k), f(v), c, o)
        return float((o.double().cpu() * x["do"]).sum())

    o, lse = torch.empty(total, H, dh, device="cuda"), att.new_lse()
    att.forward(f(x["q"]), f(x["k"]), f(x["v"]), c, o, lse)
    grads = [torch.empty_like(f(x[n])) for n in "qkv"]
    att.backward(f(x["q"]), f(x["k"]), f(x["v"]), c, o, lse, f(x["do"]), *grads)
    # the loss is a sum of 2880 terms of size 1 whose outputs err by about
    # 2^-20: 2^-14 on the loss (they do not all add), 2^-9 over the 2 h of the
    # quotient; the third derivative adds h^2 = 2^-10 of the gradient's size
    h = 2.0 ** -5
    for n, got in zip("qkv", grads):
        a = {m: x[m] + (h * d[m] if m == n else 0) for m in "qkv"}
        b = {m: x[m] - (h * d[m] if m == n else 0) for m in "qkv"}
        num = (loss(**a) - loss(**b)) / (2 * h)
        val = float((got.double().cpu() * d[n]).sum())
        size = float(got.double().norm())
        assert abs(num - val) <= 2.0 ** -9 + 2.0 ** -9 * max(1.0, size), (n, num, val)

    kk, vv = normal(g, total, H, dh), normal(g, total, H, dh)
    y = {"q": x["q"], "k": kk, "v": vv, "gamma": torch.tensor([0.6, 0.95], dtype=torch.float64)}
    la = LinearAttention(total, 2, H, dh, "f32")

    def lloss(q, k, v, gamma):
        o = torch.empty(total, H, dh, device="cuda")
        la.forward(f(q), f(k), f(v), f(gamma), c, o)
        return float((o.double().cpu() * x["do"]).sum())

    dd = {"q": d["q"], "k": normal(g, *kk.shape), "v": normal(g, *vv.shape),
          "gamma": torch.tensor([0.6, -0.8], dtype=torch.float64)}
    dd = {n: t / t.norm() for n, t in dd.items()}
    grads = {n: torch.empty_like(f(y[n])) for n in y}
    la.backward(f(y["q"]), f(y["k"]), f(y["v"]), f(y["gamma"]), c, f(x["do"]), grads["q"],
                grads["k"], grads["v"], dgamma=grads["gamma"])
    # linear in q, k and v: no truncation; outputs of size ~10 err by 2^-18,
    # 2^-12 on the loss, 2^-8 over 2 h; the decays, with h = 2^-10, lose 2^-3 to
    # rounding and h^2 times a third derivative of up to 2^13 to truncation
    for n, h, tol in (("q", 2.0 ** -5, 2.0 ** -8), ("k", 2.0 ** -5, 2.0 ** -8),
                      ("v", 2.0 ** -5, 2.0 ** -8), ("gamma", 2.0 ** -10, 2.0 ** -2)):
        a = {m: y[m] + (h * dd[m] if m == n else 0) for m in y}
        b = {m: y[m] - (h * dd[m] if m == n else 0) for m in y}
        num = (lloss(**a) - lloss(**b)) / (2 * h)
        val = float((grads[n].double().cpu() * dd[n]).sum())
        assert abs(num - val) <= tol * (1 + 2.0 ** -4 * float(grads[n].double().norm())), (n, num, val)


def _everything(seed=12):
    """Handles, inputs and one pass through all entry points, as a decoder
    that mixes both would make it."""
    from paper_2608_13578_amd import mixers
    H, Hkv, dh, lens = 4, 2, 64, [200, 1, 333]
    cu = offsets(lens)
    total, n = cu[-1], len(lens)
    g = rng(seed)
    t = {"q": normal(g, total, H, dh), "k": normal(g, total, Hkv, dh), "v": normal(g, total, Hkv, dh),
         "k2": normal(g, total, H, dh), "v2": normal(g, total, H, dh), "do": normal(g, total, H, dh),
         "q1": normal(g, n, H, dh), "k1": normal(g, n, Hkv, dh), "v1": normal(g, n, Hkv, dh),
         "k3": normal(g, n, H, dh), "v3": normal(g, n, H, dh)}
    x = {m: dev(y, "bf16") for m, y in t.items()}
    t = {m: y.double().cpu() for m, y in x.items()}  # the values as they are rounded
    x["gamma"] = torch.tensor([0.8, 0.9, 0.99, 1.0], device="cuda")
    c = i32(cu)
    att = mixers.PackedAttention(total, n, H, Hkv, dh)
    dec = mixers.AttentionDecoder(n, n, 400, H, Hkv, dh)
    lin = mixers.LinearAttention(total, n, H, dh)
    step = mixers.LinearAttentionDecoder(n, n, H, dh)
    kc, vc = dec.new_cache(), dec.new_cache()
    for b, (i, j) in enumerate(zip(cu, cu[1:])):
        kc[b, :j - i], vc[b, :j - i] = x["k"][i:j], x["v"][i:j]
    length = i32(lens)
    out = {m: torch.zeros_like(x[y]) for m, y in (
        ("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"), ("y", "q"), ("dq2", "q"), ("dk2", "k2"),
        ("dv2", "v2"), ("o1", "q1"), ("y1", "q1"))}
    out.update(lse=att.new_lse(), S=lin.new_state(), S1=lin.new_state(), dS=lin.new_state(),
               dgamma=torch.zeros(H, device="cuda"))

    def run():
        # attention, linear attention over its output, both backward, a token
        att.forward(x["q"], x["k"], x["v"], c, out["o"], out["lse"])
        lin.forward(out["o"], x["k2"], x["v2"], x["gamma"], c, out["y"], None, out["S"])
        lin.backward(out["o"], x["k2"], x["v2"], x["gamma"], c, x["do"], out["dq2"], out["dk2"],
                     out["dv2"], None, None, out["dS"], out["dgamma"])
        att.backward(x["q"], x["k"], x["v"], c, out["o"], out["lse"], out["dq2"], out["dq"],
                     out["dk"], out["dv"])
        dec.step(x["q1"], x["k1"], x["v1"], None, length, kc, vc, out["o1"])
        step.step(out["o1"], x["k3"], x["v3"], x["gamma"], None, out["S"], out["S1"], out["y1"])

    return run, out, t, cu


def test_together(torch_cuda):
    """Attention feeding linear attention, forward and backward, then a token,
    against autograd in 64 bits through both."""
    run, out, t, cu = _everything()
    run()
    torch.cuda.synchronize()
    H, Hkv, dh = 4, 2, 64
    gam = torch.tensor([0.8, 0.9, 0.99, 1.0]).double().requires_grad_()
    leaf = {m: t[m].clone().requires_grad_() for m in ("q", "k", "v", "k2", "v2")}
    o = torch.zeros_like(t["q"])
    parts = []
    for a, b in zip(cu, cu[1:]):
        K, V = (leaf[m][a:b].repeat_interleave(H // Hkv, 1).transpose(0, 1) for m in "kv")
        z = leaf["q"][a:b].transpose(0, 1) @ K.transpose(1, 2) / 8
        z = z.masked_fill(~torch.ones(b - a, b - a, dtype=torch.bool).tril(), -math.inf)
        oo = torch.softmax(z, -1) @ V
        e = torch.arange(b - a).double()
        lag = e[:, None] - e[None, :]
        D = torch.where(lag >= 0, gam[:, None, None] ** lag.clamp(min=0), torch.zeros(()).double())
        y = (D * (oo @ leaf["k2"][a:b].transpose(0, 1).transpose(1, 2)) / 8) @ leaf["v2"][a:b].transpose(0, 1)
        parts.append((oo.transpose(0, 1), y.transpose(0, 1)))
    o, y = (torch.cat(p) for p in zip(*parts))
    grads = torch.autograd.grad((y * t["do"]).sum(), [*leaf.values(), gam])
    want = dict(zip(("dq", "dk", "dv", "dk2", "dv2", "dgamma"), grads), o=o, y=y)
    # relative in the 2-norm: every result passes at most five roundings to
    # bf16 one after another (o, its score or state, the gradient handed on,
    # the weight's gradient, the result), each at most 2^-8 of what it rounds;
    # sums add no correlated error
    for n, w in want.items():
        got = out[n].double().cpu().reshape(w.shape)
        rel = float((got - w.detach()).norm() / w.detach().norm())
        say(f"  {n}: {rel:.2e}")
        assert rel <= 5 * 2.0 ** -8, (n, rel)
    # the token's attention equals a prompt one longer
    for b, (a, e) in enumerate(zip(cu, cu[1:])):
        m = e - a
        q = torch.cat([t["q"][a:e], t["q1"][b][None]])
        k, v = (torch.cat([t[x][a:e], t[x + "1"][b][None]]) for x in "kv")
        w = ref.attention(q, k, v, [0, m + 1], dh ** -0.5, "bf16")["o"]
        ref.within("o1", out["o1"][b], (w[0][m], w[1][m]))


def test_captured_and_replayed(torch_cuda):
    """All entry points in one graph, replayed between eager passes of others."""
    run, out, _, _ = _everything()
    other, _, _, _ = _everything(13)
    run()
    torch.cuda.synchronize()
    want = {n: x.clone() for n, x in out.items()}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        for x in out.values():
            x.zero_()
        other()
        graph.replay()
        other()
        torch.cuda.synchronize()
        for n, x in out.items():
            assert torch.equal(x, want[n]), n


def test_on_another_stream(torch_cuda):
    run, out, _, _ = _everything()
    run()
    torch.cuda.synchronize()
    want = {n: x.clone() for n, x in out.items()}
    for x in out.values():
        x.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    for n, x in out.items():
        assert torch.equal(x, want[n]), n


def test_tensors_that_do_not_fit_are_refused(torch_cuda):
    from paper_2608_13578_amd import mixers
    from paper_2608_13578_amd.bcmt import BcmtError
    att = mixers.PackedAttention(10, 1, 2, 1, 64)
    q, k, v, o = (torch.zeros(10, h, 64, dtype=torch.bfloat16, device="cuda") for h in (2, 1, 1, 2))
    c = i32([0, 10])
    att.forward(q, k, v, c, o)
    for bad in ((q.float(), k, v, c, o), (q[:9], k, v, c, o), (q, k.cpu(), v, c, o),
                (q, k, v, c.long(), o), (q, k, v, i32([0, 5, 10]), o), (q, k, v, c, o[:, :1]),
                (q.transpose(1, 2), k, v, c, o), (torch.zeros(20, 2, 64, dtype=q.dtype, device="cuda")[::2], k, v, c, o)):
        with pytest.raises(ValueError):
            att.forward(*bad)
    with pytest.raises(BcmtError):
        att.forward(q, k, v, c, q)  # the output over an input
    dec = mixers.AttentionDecoder(2, 3, 8, 2, 1, 64)
    kc, vc = dec.new_cache(), dec.new_cache()
    with pytest.raises(ValueError):
        dec.step(q[:2], k[:2], v[:2], None, i32([0, 0]), kc.transpose(0, 1), vc, o[:2])
    with pytest.raises(BcmtError):
        dec.step(q[:2], k[:2], v[:2], None, i32([0, 0]), kc, kc, o[:2])
    lin = mixers.LinearAttention(10, 1, 2, 64)
    with pytest.raises(ValueError):
        lin.forward(q, q.clone(), q.clone(), torch.ones(3, device="cuda"), c, o)
    with pytest.raises(ValueError):
        lin.forward(q, q.clone(), q.clone(), torch.ones(2, device="cuda"), c, o,
                    torch.zeros(1, 2, 64, 32, device="cuda"))


# Batches with workgroups for the whole chip several times over, where the kernels
# take more waves a workgroup and split no group of heads, or only in part.
ATTN_MANY = [
    ("bf16", 64, 16, 4, [(37 * i) % 131 for i in range(220)], 0, 0, True, 1.0),
    ("bf16", 32, 16, 16, [(53 * i) % 301 for i in range(64)], 1, 2, False, 1.0),
    ("bf16", 16, 32, 8, [(29 * i) % 71 for i in range(200)], 0, 3, False, 4.0),
    ("bf16", 128, 16, 2, [(41 * i) % 140 for i in range(220)], 2, 0, False, 1.0),
    ("bf16", 64, 16, 1, [(29 * i) % 71 for i in range(90)], 0, 0, False, 1.0),
    ("f32", 64, 8, 4, [(23 * i) % 61 for i in range(150)], 0, 1, True, 1.0),
]


@pytest.mark.parametrize("case", ATTN_MANY,
                         ids=lambda c: f"{c[0]}-dh{c[1]}-H{c[2]}.{c[3]}-{len(c[4])}sequences")
def test_attention_of_many_sequences(torch_cuda, case):
    test_attention(torch_cuda, case)


LONG_CACHES = [
    # dtype, dh, cap, H, Hkv, lengths
    ("bf16", 64, 20000, 4, 2, [19999]),
    ("bf16", 16, 9000, 3, 1, [8999, 300]),
    ("bf16", 32, 9000, 2, 2, [4500, 9000]),
    ("bf16", 128, 70001, 1, 1, [70000]),
    ("f32", 128, 5000, 2, 1, [4321, 0]),
    ("f32", 32, 6000, 2, 2, [5999]),
    ("bf16", 64, 2000, 8, 2, [1999, 700, -1]),
    ("bf16", 128, 1500, 40, 2, [1499, -1, 0]),
    ("f32", 64, 1200, 2, 2, [1199, 1200, 5]),
]


@pytest.mark.parametrize("case", LONG_CACHES, ids=lambda c: f"{c[0]}-dh{c[1]}-cap{c[2]}")
def test_attention_decode_of_long_caches(torch_cuda, case):
    """Caches in many parts, joined by more lanes."""
    from paper_2608_13578_amd.mixers import AttentionDecoder
    dtype, dh, cap, H, Hkv, lens = case
    say(f"decode {case}")
    g, B = rng(13), len(lens)
    q, k, v = (normal(g, B, h, dh, dtype=dtype) for h in (H, Hkv, Hkv))
    kc, vc = (normal(g, B, cap, Hkv, dh, dtype=dtype) for _ in range(2))
    d = AttentionDecoder(B, B, cap, H, Hkv, dh, dtype)
    o = torch.full((B, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    args = (dev(q, dtype), dev(k, dtype), dev(v, dtype), None, i32(lens), dev(kc, dtype), dev(vc, dtype))
    d.step(*args, o)
    again = torch.empty_like(o)
    d.step(*args, again)
    torch.cuda.synchronize()
    assert torch.equal(o, again)
    for b, n in enumerate(lens):
        if not 0 <= n < cap:
            assert bool((o[b] == 0).all())
            continue
        ref.within(f"o[{b}]", o[b], ref.token(q[b], torch.cat([kc[b, :n], k[b][None]]),
                                              torch.cat([vc[b, :n], v[b][None]]), dh ** -0.5, dtype))


def test_gradients_with_rows_far_apart(torch_cuda):
    """Rows more than 2^25 bytes apart, gradients among them."""
    from paper_2608_13578_amd.mixers import LinearAttention, PackedAttention
    dh, total, ld = 64, 150, (1 << 24) + 64
    room = torch.empty((total - 1) * ld + 6 * dh, dtype=torch.bfloat16, device="cuda")
    parts = [room.as_strided((total, dh), (ld, 1), i * dh) for i in range(6)]
    g, cu, scale = rng(14), [0, 81, 150], dh ** -0.5
    q, k, v, do = (normal(g, total, 1, dh, dtype="bf16") for _ in range(4))
    for p, x in zip(parts, (q, k, v)):
        p.copy_(dev(x[:, 0], "bf16"))
    ins, grads, c, dod = parts[:3], parts[3:], i32(cu), dev(do, "bf16")
    o = torch.empty(total, 1, dh, dtype=torch.bfloat16, device="cuda")
    att = PackedAttention(total, 2, 1, 1, dh, ldq=ld, ldk=ld, ldv=ld)
    lse = att.new_lse()
    att.forward(*ins, c, o, lse)
    att.backward(*ins, c, o, lse, dod, *grads)
    torch.cuda.synchronize()
    want = ref.attention(q, k, v, cu, scale, "bf16", do)
    for n, x in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        ref.within(n, x, want[n])
    la = LinearAttention(total, 2, 1, dh, ldq=ld, ldk=ld, ldv=ld)
    gam = torch.tensor([0.97])
    la.forward(*ins, gam.cuda(), c, o)
    la.backward(*ins, gam.cuda(), c, dod, *grads)
    torch.cuda.synchronize()
    want = ref.linear(q, k, v, gam.double(), cu, scale, "bf16", None, do)
    for n, x in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        ref.within(n, x, want[n])


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 32), ("bf16", 128)])
def test_linear_attention_with_a_negative_scale(torch_cuda, dtype, dh):
    from paper_2608_13578_amd.mixers import LinearAttention
    H, cu, scale = 2, [0, 300, 377], -0.7
    g, total = rng(15), 377
    q, k, v, do = (normal(g, total, H, dh, dtype=dtype) for _ in range(4))
    gam = torch.tensor([0.9, 0.99])
    want = ref.linear(q, k, v, gam.double(), cu, scale, dtype, None, do)
    la = LinearAttention(total, 2, H, dh, dtype, scale=scale)
    x = [dev(t, dtype) for t in (q, k, v, do)]
    o, dq, dk, dv = (torch.empty_like(x[0]) for _ in range(4))
    S, dS, dg = la.new_state(), la.new_state(), torch.empty(H, device="cuda")
    la.forward(*x[:3], gam.cuda(), i32(cu), o, None, S)
    la.backward(*x[:3], gam.cuda(), i32(cu), x[3], dq, dk, dv, None, None, dS, dg)
    torch.cuda.synchronize()
    for n, y in (("o", o), ("S", S), ("dq", dq), ("dk", dk), ("dv", dv), ("dS", dS), ("dgamma", dg)):
        ref.within(n, y, want[n])


def test_states_past_32_bits(torch_cuda):
    """A pool of states of more than 2^33 bytes."""
    from paper_2608_13578_amd.mixers import LinearAttentionDecoder
    H, dh, slots = 16, 128, 8200
    pool = torch.empty(slots, H, dh, dh, device="cuda")
    g = rng(16)
    slot = [slots - 1, 0, slots // 2 + 5]
    S = normal(g, 3, H, dh, dh)
    pool[slot] = S.float().cuda()
    q, k, v = (normal(g, 3, H, dh, dtype="bf16") for _ in range(3))
    gam = torch.linspace(0.5, 1.0, H)
    o = torch.empty(3, H, dh, dtype=torch.bfloat16, device="cuda")
    LinearAttentionDecoder(3, slots, H, dh).step(*(dev(x, "bf16") for x in (q, k, v)), gam.cuda(),
                                                 i32(slot), pool, pool, o)
    torch.cuda.synchronize()
    for b, s in enumerate(slot):
        w = ref.linear(q[b][None], k[b][None], v[b][None], gam.double(), [0, 1], dh ** -0.5, "bf16",
                       S_in=S[b][None])
        ref.within("o", o[b], w["o"])
        ref.within("S", pool[s], w["S"])


def test_two_streams_at_once(torch_cuda):
    """Objects of their own on streams of their own: the same bits as in turn."""
    from paper_2608_13578_amd import mixers
    H, Hkv, dh, cu = 8, 2, 64, [0, 700, 1500, 1501, 2400]
    g, total, n = rng(17), 2400, 4
    q, do, k2, v2 = (dev(normal(g, total, H, dh, dtype="bf16"), "bf16") for _ in range(4))
    k, v = (dev(normal(g, total, Hkv, dh, dtype="bf16"), "bf16") for _ in range(2))
    gam, c = torch.linspace(0.8, 1.0, H, device="cuda"), i32(cu)

    def make():
        att, la = mixers.PackedAttention(total, n, H, Hkv, dh), mixers.LinearAttention(total, n, H, dh)
        outs = [torch.empty_like(x) for x in (q, q, k, v, q, q, q, q)]
        return att, la, outs, att.new_lse(), torch.empty(H, device="cuda")

    def run(att, la, outs, lse, dg):
        o, dq, dk, dv, y, eq, ek, ev = outs
        att.forward(q, k, v, c, o, lse)
        la.forward(q, k2, v2, gam, c, y)
        att.backward(q, k, v, c, o, lse, do, dq, dk, dv)
        la.backward(q, k2, v2, gam, c, do, eq, ek, ev, dgamma=dg)

    sets = [make() for _ in range(3)]
    run(*sets[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s, x in zip(streams, sets[1:]):
            with torch.cuda.stream(s):
                run(*x)
    torch.cuda.synchronize()
    for x in sets[1:]:
        for a, b in zip(sets[0][2] + [sets[0][3], sets[0][4]], x[2] + [x[3], x[4]]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 16), ("bf16", 128), ("f32", 128)])
def test_attention_of_short_sequences_with_values_that_are_not_finite(torch_cuda, dtype, dh):
    """As above, where one team of waves takes all keys of a workgroup's queries."""
    from paper_2608_13578_amd.mixers import PackedAttention
    lens = [150] + [30] * 20
    cu, total, q, k, v, do = attn_inputs((dtype, dh, 2, 1, lens, 0, 0, False, 1.0), 18)
    want = ref.attention(q, k, v, cu, dh ** -0.5, dtype)
    qd, kd, vd = (dev(x, dtype) for x in (q, k, v))
    vd[100, 0, 5] = -math.inf
    vd[cu[3] + 7] = math.nan
    att = PackedAttention(total, len(lens), 2, 1, dh, dtype)
    o = torch.zeros_like(qd)
    att.forward(qd, kd, vd, i32(cu), o)
    torch.cuda.synchronize()
    hit = list(range(cu[3] + 7, cu[4]))
    clean = [t for t in range(total) if t not in hit and not 100 <= t < 150]
    ref.within("o", o, want["o"], clean)
    assert not bool(torch.isfinite(o[hit].float()).any())
    assert bool((o[100:150, :, 5] == -math.inf).all())
    rest = [c for c in range(dh) if c != 5]
    ref.within("o", o[100:150][:, :, rest], tuple(x[100:150][:, :, rest] for x in want["o"]))


# Heads for the whole chip, so that a segment of a sequence holds several chunks.
LINEAR_MANY = [
    ("bf16", 64, 96, [500, 120], 0, 0, True, True),
    ("bf16", 32, 193, [300, 70], 1, 0, False, True),
    ("bf16", 16, 380, [300, 1, 70], 0, 2, False, False),
    ("bf16", 128, 48, [400, 130], 0, 0, False, True),
    ("f32", 64, 50, [500, 0, 120], 0, 0, False, True),
    ("f32", 16, 190, [300, 70], 2, 1, True, True),
    ("f32", 128, 48, [400, 130], 0, 0, False, False),
    ("bf16", 64, 520, [150, 50], 0, 0, False, True),  # no sequence is cut
    ("f32", 32, 520, [150, 50], 0, 0, False, True),
]


@pytest.mark.parametrize("case", LINEAR_MANY, ids=lambda c: f"{c[0]}-dh{c[1]}-H{c[2]}-{sum(c[3])}rows")
def test_linear_attention_of_many_heads(torch_cuda, case):
    dtype, dh, H, *rest = case
    test_linear_attention(torch_cuda, (dtype, dh, [0.8 + 0.2 * i / (H - 1) for i in range(H)], *rest))


# Long sequences of few heads: several workgroups take the queries of the same keys.
ATTN_LONG = [
    ("bf16", 64, 1, 1, [2117], 0, 3, False, 1.0),
    ("bf16", 128, 2, 2, [1201], 1, 0, True, 1.0),
    ("bf16", 32, 3, 1, [1500, 1130], 0, 0, False, 1.0),
    ("f32", 128, 1, 1, [1203], 0, 0, False, 1.0),
    ("f32", 16, 2, 1, [1100], 2, 1, True, 1.0),
]


@pytest.mark.parametrize("case", ATTN_LONG, ids=lambda c: f"{c[0]}-dh{c[1]}-H{c[2]}.{c[3]}-{sum(c[4])}rows")
def test_attention_of_long_sequences(torch_cuda, case):
    test_attention(torch_cuda, case)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("f32", 16), ("bf16", 128)])
def test_gradients_of_offsets_out_of_order_stay_inside(torch_cuda, dtype, dh):
    """Nothing outside the arrays is written, and correct offsets after it give
    what they gave before."""
    from paper_2608_13578_amd.mixers import LinearAttention, PackedAttention
    total, H, n = 700, 4, 3
    g = rng(19)
    q, k, v, do = (dev(normal(g, total, H, dh, dtype=dtype), dtype) for _ in range(4))
    k2, v2 = (x[:, :2].contiguous() for x in (k, v))
    gam = torch.full((H,), 0.9, device="cuda")
    att = PackedAttention(total, n, H, 2, dh, dtype)
    la = LinearAttention(total, n, H, dh, dtype)
    guards = [torch.full((total + 64, h, dh), 7.0, dtype=DT[dtype], device="cuda")
              for h in (H, H, 2, 2, H, H, H)]
    o, dq, dk, dv, eq, ek, ev = (x[:total] for x in guards)
    lse, dg = torch.zeros(H, total, device="cuda"), torch.zeros(H, device="cuda")
    S = la.new_state()

    def run(cu):
        c = i32(cu)
        att.forward(q, k2, v2, c, o, lse)
        att.backward(q, k2, v2, c, o, lse, do, dq, dk, dv)
        la.backward(q, k, v, gam, c, do, eq, ek, ev, S, None, None, dg)
        torch.cuda.synchronize()
        return [x.clone() for x in (o, dq, dk, dv, eq, ek, ev, dg)]

    first = run([0, 300, 301, 700])
    for cu in ([0, 500, 50, 700], [0, 1 << 30, 5, -7], [-5, 200, 2000000000, 2147483647], [700, 0, 700, 0]):
        run(cu)
        for x in guards:
            assert bool((x[total:] == 7.0).all())
    for x, y in zip(first, run([0, 300, 301, 700])):
        assert torch.equal(x, y)
