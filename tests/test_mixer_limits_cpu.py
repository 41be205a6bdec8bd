"""Sizes of the packed-sequence entry points on both sides of their limits, without a
GPU: fake device addresses do, since every refusal comes before any HIP call."""

import pytest

from paper_2608_13578_amd import bcmt as abi


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(abi.LIB_PATH):
        from paper_2608_13578_amd.build import build
        build()
    return abi.lib()


MAKE = {
    "attn": (abi.make_attn_config, dict(total=1000, nseq=3, H=8, Hkv=2, dh=64), ()),
    "decode": (abi.make_attn_decode_config, dict(B=4, slots=8, cap=100, H=8, Hkv=2, dh=64),
               ("cs", "ct", "ch")),
    "linear": (abi.make_linattn_config, dict(total=1000, nseq=3, H=4, dh=64), ()),
    "step": (abi.make_linattn_step_config, dict(B=4, slots=8, H=4, dh=64), ()),
}


@pytest.mark.parametrize("name", MAKE)
def test_sizes_that_a_configuration_cannot_hold(name):
    """They are refused, not cut off to the bits that fit."""
    make, sizes, more = MAKE[name]
    for n, x in sizes.items():
        for big in ((1 << 32) + x, (1 << 31), -(1 << 31) - 1):
            with pytest.raises(ValueError, match=n):
                make(**{**sizes, n: big})
        assert getattr(make(**{**sizes, n: (1 << 31) - 1}), n) == (1 << 31) - 1
    for n in ("ldq", "ldk", "ldv", "ldo", *more):
        for big in ((1 << 64) + 512, 1 << 63):
            with pytest.raises(ValueError, match=n):
                make(**sizes, **{n: big})
        assert getattr(make(**sizes, **{n: (1 << 63) - 1}), n) == (1 << 63) - 1


INVALID, UNSUPPORTED, OK = abi.BCMT_ERR_INVALID, abi.BCMT_ERR_UNSUPPORTED, abi.BCMT_OK
CHECK = {"attn": abi.bcmt_attn_validate, "decode": abi.bcmt_attn_decode_validate,
         "linear": abi.bcmt_linattn_validate, "step": abi.bcmt_linattn_step_validate}
TOP = (1 << 23) - 1  # (total / 64 + nseq) H and, of single tokens, B H


def both_sides(name, inside, outside, code):
    make, sizes, _ = MAKE[name]
    for change, want in ((inside, OK), (outside, code)):
        kw = {**sizes, **change}
        if name in ("attn", "decode") and "H" in change and "Hkv" not in change:
            kw["Hkv"] = kw["H"]
        assert CHECK[name](make(**kw)) == want, kw


@pytest.mark.parametrize("name", ["attn", "linear"])
def test_rows_and_sequences(name):
    for H, nseq in ((1, 1), (16, 3), (127, 65535), (12, 100), (65535, 1)):
        total = (TOP // H - nseq) * 64 + 63  # the last row before the bound
        both_sides(name, dict(total=total, nseq=nseq, H=H, dh=16),
                   dict(total=total + 1, nseq=nseq, H=H, dh=16), UNSUPPORTED)
    both_sides(name, dict(nseq=65535, H=1), dict(nseq=65536, H=1), UNSUPPORTED)
    both_sides(name, dict(H=65535, nseq=1), dict(H=65536, nseq=1), UNSUPPORTED)
    both_sides(name, dict(ldq=1 << 28, ldo=1 << 28), dict(ldq=(1 << 28) + 8), INVALID)


def test_decode():
    for B, H, Hkv in ((65535, 1, 1), (8191, 64, 8), (4095, 32, 16), (4095, 17 * 8, 8), (1, 65535, 1)):
        nh = -(-(H // Hkv) // 16)
        assert B * Hkv * nh <= 65535 < (B + 1) * Hkv * nh or B == 1
        both_sides("decode", dict(B=B, H=H, Hkv=Hkv),
                   dict(B=65535 // (Hkv * nh) + 1, H=H, Hkv=Hkv), UNSUPPORTED)
    both_sides("decode", dict(H=65535, B=1), dict(H=65536, B=1, Hkv=1), UNSUPPORTED)
    both_sides("decode", dict(cap=1 << 30, slots=1), dict(cap=(1 << 30) + 1, slots=1), UNSUPPORTED)
    both_sides("decode", dict(slots=1 << 30), dict(slots=(1 << 30) + 1), UNSUPPORTED)
    # extents: 8 slots, 100 positions, 2 heads: 8 cs + 100 * 64 + 2 * 64 = 10^18
    top = (10 ** 18 - 102 * 64) // 8
    both_sides("decode", dict(cs=top, ct=64, ch=64), dict(cs=top + 1000, ct=64, ch=64), INVALID)
    both_sides("decode", dict(cs=64, ct=64, ch=64), dict(cs=64, ct=64, ch=56), INVALID)
    both_sides("decode", dict(slots=1 << 20, cap=1 << 30), dict(slots=1 << 30, cap=1 << 30), INVALID)
    both_sides("decode", dict(ldk=1 << 28), dict(ldk=(1 << 28) + 8), INVALID)


def test_step():
    for H in (1, 12, 128, 65535):
        both_sides("step", dict(B=TOP // H, H=H), dict(B=TOP // H + 1, H=H), UNSUPPORTED)
    both_sides("step", dict(H=65535, B=1), dict(H=65536, B=1), UNSUPPORTED)
    both_sides("step", dict(slots=1 << 30), dict(slots=(1 << 30) + 1), UNSUPPORTED)
    both_sides("step", dict(ldv=1 << 28), dict(ldv=(1 << 28) + 8), INVALID)
