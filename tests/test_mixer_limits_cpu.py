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
