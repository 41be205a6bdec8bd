"""Refusals of the packed-sequence entry points: every bad argument is an error
before any HIP call, so fake device addresses do."""

import ctypes

import pytest

from paper_2608_13578_amd import bcmt as abi

A = 1 << 40
MB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(abi.LIB_PATH):
        from paper_2608_13578_amd.build import build
        build()
    return abi.lib()


INVALID, UNSUPPORTED = abi.BCMT_ERR_INVALID, abi.BCMT_ERR_UNSUPPORTED


def attn(**kw):
    return abi.make_attn_config(**{**dict(total=1000, nseq=3, H=8, Hkv=2, dh=64), **kw})


def dec(**kw):
    return abi.make_attn_decode_config(**{**dict(B=4, slots=8, cap=100, H=8, Hkv=2, dh=64), **kw})


def lin(**kw):
    return abi.make_linattn_config(**{**dict(total=1000, nseq=3, H=4, dh=64), **kw})


def step(**kw):
    return abi.make_linattn_step_config(**{**dict(B=4, slots=8, H=4, dh=64), **kw})


COMMON = [
    (dict(), 0), (dict(dtype="f32"), 0), (dict(dh=16), 0), (dict(dh=32), 0), (dict(dh=128), 0),
    (dict(dh=8), UNSUPPORTED), (dict(dh=256), UNSUPPORTED), (dict(dh=0, scale=1.0), INVALID),
    (dict(H=0), INVALID), (dict(H=70000, dh=16), UNSUPPORTED),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(ldq=1536), 0), (dict(ldq=100), INVALID), (dict(ldo=-512), INVALID),
    (dict(ldq=516), INVALID), (dict(ldq=516, dtype="f32"), 0), (dict(ldv=1 << 30), INVALID),
]


@pytest.mark.parametrize("make,check", [(attn, abi.bcmt_attn_validate), (dec, abi.bcmt_attn_decode_validate),
                                        (lin, abi.bcmt_linattn_validate), (step, abi.bcmt_linattn_step_validate)])
def test_configurations(make, check):
    for kw, code in COMMON:
        if "H" in kw and make in (attn, dec):
            kw = dict(kw, Hkv=max(kw["H"], 1))
        assert check(make(**kw)) == code, kw
    c = make()
    c.dtype = 7
    assert check(c) == INVALID
    raw = {attn: "bcmt_attn_validate", dec: "bcmt_attn_decode_validate",
           lin: "bcmt_linattn_validate", step: "bcmt_linattn_step_validate"}[make]
    assert getattr(abi.lib(), raw)(None) == INVALID


@pytest.mark.parametrize("check,c,code", [
    (abi.bcmt_attn_validate, dict(total=0), INVALID), (abi.bcmt_attn_validate, dict(nseq=0), INVALID),
    (abi.bcmt_attn_validate, dict(Hkv=3), INVALID), (abi.bcmt_attn_validate, dict(Hkv=16), INVALID),
    (abi.bcmt_attn_validate, dict(Hkv=0), INVALID), (abi.bcmt_attn_validate, dict(scale=0.0), INVALID),
    (abi.bcmt_attn_validate, dict(scale=-1.0), INVALID), (abi.bcmt_attn_validate, dict(ldk=64), INVALID),
    (abi.bcmt_attn_validate, dict(total=(1 << 30) + 1, H=1, Hkv=1, dh=16), UNSUPPORTED),
    (abi.bcmt_attn_validate, dict(total=1 << 30), UNSUPPORTED),
    (abi.bcmt_attn_validate, dict(nseq=65536), UNSUPPORTED),
])
def test_attention_sizes(check, c, code):
    assert check(attn(**c)) == code
    if code:
        assert abi.bcmt_attn_workspace_bytes(attn(**c)) == 0


@pytest.mark.parametrize("c,code", [
    (dict(B=0), INVALID), (dict(slots=0), INVALID), (dict(cap=0), INVALID), (dict(Hkv=3), INVALID),
    (dict(scale=0.0), INVALID), (dict(cs=12800, ct=128, ch=64), 0), (dict(cs=12800, ct=64, ch=6400), 0),
    (dict(cs=12800, ct=128), INVALID), (dict(cs=12800, ct=32, ch=64), INVALID),
    (dict(cs=12801, ct=128, ch=64), INVALID), (dict(cs=1 << 60, ct=128, ch=64), INVALID),
    (dict(B=65536), UNSUPPORTED), (dict(cap=(1 << 30) + 1), UNSUPPORTED),
    (dict(slots=(1 << 30) + 1), UNSUPPORTED),
])
def test_decode_sizes(c, code):
    assert abi.bcmt_attn_decode_validate(dec(**c)) == code
    assert (abi.bcmt_attn_decode_workspace_bytes(dec(**c)) == 0) == bool(code)


@pytest.mark.parametrize("c,code", [
    (dict(total=0), INVALID), (dict(nseq=0), INVALID), (dict(scale=-1.0), 0), (dict(scale=0.0), 0),
    (dict(nseq=65536), UNSUPPORTED), (dict(total=(1 << 30) + 1, H=1, dh=16), UNSUPPORTED),
])
def test_linear_sizes(c, code):
    assert abi.bcmt_linattn_validate(lin(**c)) == code
    assert abi.bcmt_linattn_workspace_bytes(lin(), 9) == 0
    if code:
        assert abi.bcmt_linattn_workspace_bytes(lin(**c), abi.BCMT_PASS_BACKWARD) == 0


def test_step_sizes():
    assert abi.bcmt_linattn_step_validate(step(B=0)) == INVALID
    assert abi.bcmt_linattn_step_validate(step(slots=0)) == INVALID
    assert abi.bcmt_linattn_step_validate(step(slots=(1 << 30) + 1)) == UNSUPPORTED
    assert abi.bcmt_linattn_step_validate(step(B=1 << 30)) == UNSUPPORTED


def call(name, cfg, names, **kw):
    """Calls an entry point with distinct far apart addresses; kw replaces some."""
    args = []
    for i, n in enumerate(names):
        if n == "ws_bytes":
            args.append(kw.get(n, 1 << 40))
        elif n == "stream":
            args.append(None)
        else:
            args.append(kw[n] if n in kw else A + (i + 1) * 64 * MB)
    return getattr(abi.lib(), name)(ctypes.byref(cfg), *args)


AF = ("q", "k", "v", "cu", "o", "lse", "stream")
AB = ("q", "k", "v", "cu", "o", "lse", "dO", "dq", "dk", "dv", "ws", "ws_bytes", "stream")
AD = ("q", "k", "v", "slot", "length", "kc", "vc", "o", "ws", "ws_bytes", "stream")
LF = ("q", "k", "v", "gamma", "cu", "S_in", "o", "S_out", "ws", "ws_bytes", "stream")
LB = ("q", "k", "v", "gamma", "cu", "S_in", "dO", "dS_out", "dq", "dk", "dv", "dS_in", "dgamma", "ws",
      "ws_bytes", "stream")
LS = ("q", "k", "v", "gamma", "slot", "S_in", "S_out", "o", "stream")
ENTRIES = [("bcmt_attn_forward", attn, AF, {"lse"}), ("bcmt_attn_backward", attn, AB, set()),
           ("bcmt_attn_decode", dec, AD, {"slot"}), ("bcmt_linattn_forward", lin, LF, {"S_in", "S_out"}),
           ("bcmt_linattn_backward", lin, LB, {"S_in", "dS_out", "dS_in", "dgamma"}),
           ("bcmt_linattn_step", step, LS, {"slot"})]


@pytest.mark.parametrize("name,make,names,optional", ENTRIES, ids=[e[0] for e in ENTRIES])
def test_pointers(name, make, names, optional):
    pointers = [n for n in names if n not in ("ws_bytes", "stream")]
    for n in pointers:
        if n not in optional:
            assert call(name, make(), names, **{n: None}) == INVALID, n
        at = A + (names.index(n) + 1) * 64 * MB
        assert call(name, make(), names, **{n: at + 2}) == INVALID, n  # aligned to nothing
        if n not in ("cu", "lse", "slot", "length", "gamma", "dgamma"):
            assert call(name, make(), names, **{n: at + 8}) == INVALID, n
    assert call(name, make(dh=24), names) == UNSUPPORTED
    assert call(name, make(B=0) if make in (dec, step) else make(total=0), names) == INVALID
    if "ws" in names:
        assert call(name, make(), names, ws_bytes=0) == abi.BCMT_ERR_WORKSPACE


def place(names, n):
    return A + (names.index(n) + 1) * 64 * MB


@pytest.mark.parametrize("name,make,names,outs", [
    ("bcmt_attn_forward", attn, AF, ("o", "lse")), ("bcmt_attn_backward", attn, AB, ("dq", "dk", "dv", "ws")),
    ("bcmt_attn_decode", dec, AD, ("o", "kc", "vc", "ws")),
    ("bcmt_linattn_forward", lin, LF, ("o", "S_out", "ws")),
    ("bcmt_linattn_backward", lin, LB, ("dq", "dk", "dv", "dS_in", "dgamma", "ws")),
    ("bcmt_linattn_step", step, LS, ("o", "S_out"))], ids=["af", "ab", "ad", "lf", "lb", "ls"])
def test_outputs_over_other_arrays(name, make, names, outs):
    cfg = make()
    for n in outs:
        for m in names:
            if m in ("ws_bytes", "stream", n):
                continue
            got = call(name, cfg, names, **{n: place(names, m)})
            # states may advance in place
            if (n, m) in (("S_out", "S_in"), ("dS_in", "dS_out")):
                continue  # (would be accepted and enqueue: not called here)
            assert got == INVALID, (n, m)


def test_columns_of_one_array_do_not_meet():
    """dq, dk, dv as columns of one array pass the checks up to the workspace's
    size; shifted by a head they meet."""
    w = (8 + 2 * 2) * 64
    cfg = attn(ldq=w, ldk=w, ldv=w)
    base = A + (1 << 34)
    cols = dict(dq=base, dk=base + 2 * 8 * 64, dv=base + 2 * 10 * 64)
    assert call("bcmt_attn_backward", cfg, AB, ws_bytes=0, **cols) == abi.BCMT_ERR_WORKSPACE
    cols["dk"] -= 2 * 64
    assert call("bcmt_attn_backward", cfg, AB, ws_bytes=0, **cols) == INVALID
    # the last head of a row must not reach into the next row's first column
    cols = dict(dq=base, dk=base + 2 * 8 * 64, dv=base + 2 * 11 * 64)
    assert call("bcmt_attn_backward", cfg, AB, ws_bytes=0, **cols) == INVALID


def test_dense_caches_past_62_bits():
    assert abi.bcmt_attn_decode_validate(dec(slots=1 << 30, cap=1 << 30)) == INVALID
    assert abi.bcmt_attn_decode_workspace_bytes(dec(slots=1 << 30, cap=1 << 30)) == 0
    assert abi.bcmt_attn_decode_validate(dec(slots=1 << 20, cap=1 << 20)) == abi.BCMT_OK
