"""The packed-sequence mixers at the largest numbers of workgroups that their
configurations allow, against the 64-bit references."""

import pytest
import torch

import mixer_reference as ref
from test_gpu_mixers import DT, i32
from test_gpu_parity import say, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

TOP = (1 << 23) - 1  # (total / 64 + nseq) H and, of single tokens, B H


def values(seed, dtype, *shape):
    """Device values of the type."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


def chosen(cu, lens, ids):
    """Rows of these sequences, and their offsets when they are packed alone."""
    rows = [r for s in ids for r in range(cu[s], cu[s + 1])]
    alone = [0]
    for s in ids:
        alone.append(alone[-1] + lens[s])
    return rows, alone


def batch(H):
    """As many sequences as there can be, and as many rows as these heads leave."""
    nseq = 65535
    total = (TOP // H - nseq) * 64 + 63
    lens = [i % 2 for i in range(nseq)]
    lens[40000] = 700
    lens[3], lens[65534] = 65, 130
    for s in range(nseq - 2, 0, -1):  # the rest of the rows, if they are fewer
        if sum(lens) <= total - 5:
            break
        lens[s] = 0 if lens[s] == 1 and s % 4 == 1 else lens[s]
    cu = torch.tensor([0] + lens).cumsum(0).tolist()
    assert cu[-1] <= total
    return nseq, total, lens, cu, [0, 1, 3, 7, 8, 39999, 40000, 40003, 65527, 65533, 65534]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_most_sequences(torch_cuda, dtype):
    """127 heads of 65535 sequences, attention and linear attention with their gradients."""
    from paper_2608_13578_amd.mixers import LinearAttention, PackedAttention
    H, dh = 127, 16
    nseq, total, lens, cu, ids = batch(H)
    say(f"{dtype}: {total} rows of {nseq} sequences, {H} heads")
    q, k, v, do = (values(i, dtype, total, H, dh) for i in range(4))
    gam = torch.linspace(0.8, 1.0, H, device="cuda")
    c, behind = i32(cu), slice(cu[-1], total)
    o, dq, dk, dv, y, eq, ek, ev = (torch.full_like(q, 7.0) for _ in range(8))
    lse = torch.full((H, total), 7.0, device="cuda")
    att = PackedAttention(total, nseq, H, H, dh, dtype)
    lin = LinearAttention(total, nseq, H, dh, dtype)
    att.forward(q, k, v, c, o, lse)
    att.backward(q, k, v, c, o, lse, do, dq, dk, dv)
    lin.forward(q, k, v, gam, c, y)
    lin.backward(q, k, v, gam, c, do, eq, ek, ev)
    torch.cuda.synchronize()
    rows, alone = chosen(cu, lens, ids)
    heads = [0, 1, 64, 126]
    host = [x[rows][:, heads].double().cpu() for x in (q, k, v, do)]
    want = ref.attention(*host[:3], alone, dh ** -0.5, dtype, host[3])
    for n, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.within(n, x[rows][:, heads], want[n])
        assert bool((x[behind] == 7.0).all()), n
    ref.within("lse", lse[heads][:, rows], want["lse"])
    want = ref.linear(*host[:3], gam[heads].double().cpu(), alone, dh ** -0.5, dtype, None, host[3])
    for n, x in (("o", y), ("dq", eq), ("dk", ek), ("dv", ev)):
        ref.within(n, x[rows][:, heads], want[n])
        assert bool((x[behind] == 7.0).all()), n
    # every sequence of one row, without a reference: its only weight p is its own sum, so
    # that p v / p has three roundings of float32, which bfloat16 does not see
    one = torch.tensor([cu[s] for s in range(nseq) if lens[s] == 1], device="cuda")
    off = (o[one].double() - v[one].double()).abs()
    assert bool((off <= (0.0 if dtype == "bf16" else 4 * ref.E) * v[one].double().abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_most_decoded_sequences(torch_cuda, dtype):
    from paper_2608_13578_amd.mixers import AttentionDecoder
    B, cap, dh = 65535, 6, 16
    say(f"{dtype}: {B} sequences")
    q, k, v = (values(i, dtype, B, 1, dh) for i in range(3))
    kc, vc = (values(i, dtype, B, cap, 1, dh) for i in (3, 4))
    lens = [b % cap for b in range(B)]
    length, r = i32(lens), torch.arange(B, device="cuda")
    o = torch.full_like(q, 7.0)
    AttentionDecoder(B, B, cap, 1, 1, dh, dtype).step(q, k, v, None, length, kc, vc, o)
    torch.cuda.synchronize()
    assert torch.equal(kc[r, length.long()], k) and torch.equal(vc[r, length.long()], v)
    for b in (*range(12), 32768, *range(B - 12, B)):
        n = lens[b] + 1
        ref.within(f"o[{b}]", o[b], ref.token(q[b].double().cpu(), kc[b, :n].double().cpu(),
                                              vc[b, :n].double().cpu(), dh ** -0.5, dtype))
    # a sequence without a history returns its value
    assert torch.equal(o[::cap], v[::cap])


def test_most_states(torch_cuda):
    """One token of as many sequences as there can be, in place."""
    from paper_2608_13578_amd.mixers import LinearAttentionDecoder
    B, dh = TOP, 16
    say(f"{B} states")
    q, k, v = (values(i, "f32", B, 1, dh) for i in range(3))
    S = values(3, "f32", B, 1, dh, dh)
    gam = torch.full((1,), 0.9, device="cuda")
    ids = [0, 1, 2, B // 2, B - 2, B - 1]
    before = S[ids].double()
    o = torch.full_like(q, 7.0)
    LinearAttentionDecoder(B, B, 1, dh, "f32").step(q, k, v, gam, None, S, S, o)
    torch.cuda.synchronize()
    qq, kk, vv = (x[ids, 0].double() for x in (q, k, v))
    new = float(gam[0]) * before[:, 0] + kk[:, :, None] * vv[:, None, :]
    mag = float(gam[0]) * before[:, 0].abs() + (kk[:, :, None] * vv[:, None, :]).abs()
    # a product and a fused sum, or two products and a sum: three roundings
    assert bool(((S[ids][:, 0].double() - new).abs() <= 3 * ref.E * mag).all())
    want = (qq[:, :, None] * new).sum(1) * dh ** -0.5
    most = (qq.abs()[:, :, None] * mag).sum(1) * dh ** -0.5
    # the state's three, a product, 16 sums and the scale
    assert bool(((o[ids, 0].double() - want).abs() <= 22 * ref.E * most).all())
    # no state is left out: every output against the products in float32 (each side
    # makes at most 18 roundings of them)
    for a in range(0, B, 1 << 21):
        e = min(B, a + (1 << 21))
        want = (q[a:e, 0, :, None] * S[a:e, 0]).sum(1) * dh ** -0.5
        most = (q[a:e, 0, :, None] * S[a:e, 0]).abs().sum(1) * dh ** -0.5
        assert bool(((o[a:e, 0] - want).abs() <= 40 * ref.E * most).all())
