"""Measured cases of the sequence mixers over packed sequences.

Two operators, each with its pass over whole prompts, its gradients and its
form for single tokens:

  attention         causal softmax attention; query heads share key/value
                    heads in groups; sequences of any lengths lie one after
                    another in the rows of the arrays (`cu` holds the first
                    row of each and the end of the last)
  linear attention  S_t = g S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t with a
                    decay g for each head, over the same packed rows

  attn_fwd       a prompt through attention
  attn_train     attention forward and backward
  attn_decode    one token per sequence against key/value caches
  lin_fwd        a prompt through linear attention, with its states
  lin_train      linear attention forward and backward
  lin_step       one token per sequence against a pool of states

`run` computes the plain form in 32 bits from elementary operations, or, where
`own` is true, calls the library.  Inputs are drawn on the GPU from the seed:
queries, keys, values and upstream gradients N(0, 1), decays 1 - 2^-u with u
spread over 1.5 to 9, states N(0, 1).
"""

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases


def _case(name, op, lens, H, Hkv, dh, dtype="bf16", fused=False, states=False, dgamma=False):
    return {"name": name, "op": op, "lens": lens, "H": H, "Hkv": Hkv, "dh": dh, "dtype": dtype,
            "fused": fused, "states": states, "dgamma": dgamma}


def _steps(name, op, B, slots, cap, H, Hkv, dh, dtype="bf16"):
    return {"name": name, "op": op, "B": B, "slots": slots, "cap": cap, "H": H, "Hkv": Hkv,
            "dh": dh, "dtype": dtype}


def listed():
    return [
        # A handful of short prompts of a serving batch, read in place from
        # the fused projection: launches and latency.
        _case("attn_fwd_prompts", "attn_fwd", "37,1,200,64,129", 12, 4, 64, fused=True),
        # Long documents through wide heads, eight queries to a key head.
        _case("attn_fwd_long", "attn_fwd", "8192,5001,1791,1400", 16, 2, 128),
        # The paper's heads of 16 in float32, an empty sequence among them.
        _case("attn_train_f32", "attn_train", "1024,511,257,1,0,303", 8, 8, 16, "f32"),
        # A training batch of documents at GPT-2-small width.
        _case("attn_train_batch", "attn_train", "2048,1000,1,1500,777,2048,513,305", 12, 4, 64,
              fused=True),
        # One conversation, one token: latency alone.
        _steps("attn_decode_one", "attn_decode", 1, 1, 1024, 12, 12, 64),
        # A full serving batch over long caches; some sequences are short,
        # more slots than sequences.
        _steps("attn_decode_batch", "attn_decode", 32, 40, 8192, 32, 8, 128),
        # Short prompts continued from their states, in float32.
        _case("lin_fwd_prompts", "lin_fwd", "129,64,1,0,200", 8, 8, 32, "f32", states=True),
        # Contexts of the library's longest benchmark, states kept.
        _case("lin_fwd_long", "lin_fwd", "65536,40000,25536", 16, 16, 64, states=True),
        # A training batch with trained decays and carried states.
        _case("lin_train_batch", "lin_train", "2048,1000,1,1500,777,2048,513,305", 12, 12, 64,
              fused=True, states=True, dgamma=True),
        # Long documents through wide heads, decays fixed.
        _case("lin_train_long", "lin_train", "16384,9000,7384", 16, 16, 128),
        # One conversation, one token: latency alone.
        _steps("lin_step_one", "lin_step", 1, 1, 0, 12, 12, 64),
        # A full serving batch.
        _steps("lin_step_batch", "lin_step", 128, 160, 0, 32, 32, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn_fwd", "attn_train", "attn_decode", "lin_fwd", "lin_train", "lin_step"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    dh = rng.choice((16, 32, 64, 64, 128))
    Hkv = rng.choice((1, 2, 3, 4, 8))
    H = Hkv * rng.choice((1, 2, 3, 4, 8))
    H = min(H, 16 // Hkv * Hkv) if op.startswith("attn") else rng.choice((1, 2, 5, 8, 12, 16))
    if op.startswith("lin"):
        Hkv = H
    if op in ("attn_decode", "lin_step"):
        cap = _log(rng, 16, 8192) if op == "attn_decode" else 0
        B = _log(rng, 1, 32 if cap > 2048 else 128)
        return _steps("", op, B, B + rng.randrange(5), cap, H, Hkv, dh, dtype)
    top = {"attn_fwd": 4096, "attn_train": 2048, "lin_fwd": 32768, "lin_train": 8192}[op]
    total = _log(rng, 64, 2 * top)
    lens, left = [], total
    while left > 0 and len(lens) < 12:
        n = min(left, top, _log(rng, 1, top))
        lens.append(n)
        left -= n
    if rng.random() < 0.3:
        lens.insert(rng.randrange(len(lens) + 1), 0)
    return _case("", op, ",".join(map(str, lens)), H, Hkv, dh, dtype, fused=rng.random() < 0.5,
                 states=op.startswith("lin") and rng.random() < 0.5,
                 dgamma=op == "lin_train" and rng.random() < 0.5)


def _lens(c):
    return [int(n) for n in c["lens"].split(",")]


def _cached(c):
    """Tokens in each sequence's cache before the call: spread over the capacity."""
    return [(b * 2654435761 + 300) % c["cap"] for b in range(c["B"])]


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, H, Hkv, dh = TYPES[c["dtype"]], c["H"], c["Hkv"], c["dh"]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)

    s = {"case": c}
    if c["op"].startswith("lin"):
        u = torch.linspace(1.5, 9.0, H, device="cuda") if H > 1 else torch.full((1,), 5.0, device="cuda")
        s["gamma"] = 1.0 - torch.exp2(-(u + 0.3 * torch.rand(H, generator=g, device="cuda")))
    if c["op"] in ("attn_decode", "lin_step"):
        B = c["B"]
        s.update(q=normal(B, H, dh), k=normal(B, Hkv, dh), v=normal(B, Hkv, dh))
        s["slot"] = torch.randperm(c["slots"], generator=g, device="cuda")[:B].to(torch.int32)
        if c["op"] == "attn_decode":
            s["length"] = torch.tensor(_cached(c), dtype=torch.int32, device="cuda")
            s["kcache"] = normal(c["slots"], c["cap"], Hkv, dh)
            s["vcache"] = normal(c["slots"], c["cap"], Hkv, dh)
        else:
            s["S_in"] = normal(c["slots"], H, dh, dh, dtype=torch.float32)
            s["S_out"] = torch.zeros_like(s["S_in"])
        if own:
            s["plan"] = _plan(c, 0, 0)
        return s
    lens = _lens(c)
    total, n = sum(lens), len(lens)
    if c["fused"]:
        qkv = normal(total, (H + 2 * Hkv) * dh)
        s["q"], s["k"], s["v"] = qkv.split([H * dh, Hkv * dh, Hkv * dh], dim=1)
    else:
        s["q"], s["k"], s["v"] = normal(total, H * dh), normal(total, Hkv * dh), normal(total, Hkv * dh)
    cu = [0]
    for m in lens:
        cu.append(cu[-1] + m)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    s["longest"] = max(lens)
    if c["op"].endswith("train"):
        s["do"] = normal(total, H * dh)
    if c["states"]:
        s["S_in"] = normal(n, H, dh, dh, dtype=torch.float32)
        if c["op"].endswith("train"):
            s["dS_out"] = normal(n, H, dh, dh, dtype=torch.float32)
    if own:
        s["plan"] = _plan(c, total, n)
    return s


def _plan(c, total, n):
    """The library's handle (configuration and workspace) that a program keeps."""
    from paper_2608_13578_amd import mixers
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    if c["op"] == "attn_decode":
        return mixers.AttentionDecoder(c["B"], c["slots"], c["cap"], H, Hkv, dh, dtype=c["dtype"])
    if c["op"] == "lin_step":
        return mixers.LinearAttentionDecoder(c["B"], c["slots"], H, dh, dtype=c["dtype"])
    ld = (H + 2 * Hkv) * dh if c["fused"] else 0
    if c["op"].startswith("attn"):
        return mixers.PackedAttention(total, n, H, Hkv, dh, dtype=c["dtype"], ldq=ld, ldk=ld, ldv=ld)
    return mixers.LinearAttention(total, n, H, dh, dtype=c["dtype"], ldq=ld, ldk=ld, ldv=ld)


# ------------------------------------------------------------------ one pass


def run(state):
    return (_run_own if own else _run_plain)(state)


def _grads_like(s):
    """Gradients in the layout of the inputs: one array for a fused projection."""
    c = s["case"]
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    if c["fused"]:
        d = torch.empty((s["q"].shape[0], (H + 2 * Hkv) * dh), dtype=s["q"].dtype, device="cuda")
        return (*d.split([H * dh, Hkv * dh, Hkv * dh], dim=1),)
    return torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])


def _run_own(s):
    c, p = s["case"], s["plan"]
    op, q, k, v = c["op"], s["q"], s["k"], s["v"]
    o = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    if op == "attn_decode":
        p.step(q, k, v, s["slot"], s["length"], s["kcache"], s["vcache"], o)
        return {"o": o, "kcache": s["kcache"], "vcache": s["vcache"]}
    if op == "lin_step":
        p.step(q, k, v, s["gamma"], s["slot"], s["S_in"], s["S_out"], o)
        return {"o": o, "S": s["S_out"]}
    cu = s["cu"]
    if op == "attn_fwd":
        p.forward(q, k, v, cu, o)
        return {"o": o}
    if op == "attn_train":
        lse = torch.empty((c["H"], q.shape[0]), dtype=torch.float32, device="cuda")
        p.forward(q, k, v, cu, o, lse)
        dq, dk, dv = _grads_like(s)
        p.backward(q, k, v, cu, o, lse, s["do"], dq, dk, dv)
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    S_in = s.get("S_in")
    S = torch.empty_like(S_in) if S_in is not None else None
    p.forward(q, k, v, s["gamma"], cu, o, S_in, S)
    out = {"o": o}
    if S is not None:
        out["S"] = S
    if op == "lin_train":
        dq, dk, dv = _grads_like(s)
        dS = torch.empty_like(S_in) if S_in is not None else None
        dg = torch.empty_like(s["gamma"]) if c["dgamma"] else None
        p.backward(q, k, v, s["gamma"], cu, s["do"], dq, dk, dv, S_in, s.get("dS_out"), dS, dg)
        out.update(dq=dq, dk=dk, dv=dv)
        if dS is not None:
            out["dS"] = dS
        if dg is not None:
            out["dgamma"] = dg
    return out


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "attn_decode":
        return _plain_decode(s)
    if op == "lin_step":
        i = s["slot"].long()
        q, k, v = (s[x].float() for x in "qkv")
        S = s["gamma"][None, :, None, None] * s["S_in"][i] + k[..., :, None] * v[..., None, :]
        o = (q[..., None, :] @ S)[..., 0, :] * c["dh"] ** -0.5
        s["S_out"][i] = S
        return {"o": o.to(s["q"].dtype), "S": s["S_out"]}
    return _plain_attention(s) if op.startswith("attn") else _plain_linear(s)


# Packed rows as [sequences, longest, heads, dh] and back.


def _places(s, longest):
    cu = s["cu"].long()
    total = s["q"].shape[0]
    at = torch.arange(longest, device="cuda")
    rows = cu[:-1, None] + at
    there = rows < cu[1:, None]
    r = torch.arange(total, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), r, right=True)
    return rows.clamp(max=total - 1), there, seq * longest + r - cu[seq]


def _pad(x, heads, places):
    rows, there, _ = places
    x = x.float().reshape(x.shape[0], heads, -1)
    return torch.where(there[..., None, None], x[rows], 0.0).transpose(1, 2)


def _pack(x, places):
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0] * x.shape[1], -1)[places[2]]


def _plain_attention(s):
    c = s["case"]
    H, Hkv, dh, L = c["H"], c["Hkv"], c["dh"], s["longest"]
    G, scale, dt = H // Hkv, c["dh"] ** -0.5, s["q"].dtype
    places = _places(s, L)
    q = _pad(s["q"], H, places)
    k = _pad(s["k"], Hkv, places).repeat_interleave(G, 1)
    v = _pad(s["v"], Hkv, places).repeat_interleave(G, 1)
    at = torch.arange(L, device="cuda")
    z = (q @ k.transpose(-1, -2)) * scale
    z = z.masked_fill(at[None, :] > at[:, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    del z
    p = p / p.sum(-1, keepdim=True)
    o = p @ v
    out = {"o": _pack(o, places).to(dt)}
    if c["op"] == "attn_train":
        do = _pad(s["do"], H, places)

        def shared(d):  # the gradient of a key/value head adds its queries'
            n = d.shape[0]
            return _pack(d.reshape(n, Hkv, G, L, dh).sum(2), places).to(dt)

        out["dv"] = shared(p.transpose(-1, -2) @ do)
        ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) * scale
        out["dk"] = shared(ds.transpose(-1, -2) @ q)
        out["dq"] = _pack(ds @ k, places).to(dt)
    return out


def _plain_decode(s):
    c = s["case"]
    H, Hkv, dh, B = c["H"], c["Hkv"], c["dh"], c["B"]
    i, n = s["slot"].long(), s["length"].long()
    s["kcache"][i, n] = s["k"]
    s["vcache"][i, n] = s["v"]
    q = s["q"].float().reshape(B, Hkv, H // Hkv, dh)
    k = s["kcache"][i].float().transpose(1, 2)
    v = s["vcache"][i].float().transpose(1, 2)
    z = (q @ k.transpose(-1, -2)) * dh ** -0.5
    later = torch.arange(c["cap"], device="cuda")[None, :] > n[:, None]
    z = z.masked_fill(later[:, None, None, :], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    o = (p @ v) / p.sum(-1, keepdim=True)
    return {"o": o.reshape(B, H, dh).to(s["q"].dtype), "kcache": s["kcache"], "vcache": s["vcache"]}


def _power(g, e):
    """g[h]^e[...] as [h, ...], the power taken in 64 bits."""
    return torch.pow(g.double().reshape(-1, *([1] * e.dim())), e.double()).float()


def _plain_linear(s):
    """Chunks of 128 tokens: products inside a chunk, and the states before
    the chunks from a product over chunks."""
    c = s["case"]
    H, dh, dt, C = c["H"], c["dh"], s["q"].dtype, 128
    train = c["op"] == "lin_train"
    L = -(-s["longest"] // C) * C
    places = _places(s, L)
    n = s["cu"].shape[0] - 1
    nc = L // C
    leaves = [_pad(s[x], H, places) for x in "qkv"] + [s["gamma"].detach().clone()]
    S_in = s.get("S_in")
    if S_in is not None:
        leaves.append(S_in.detach().clone())
    with torch.set_grad_enabled(train):
        for x in leaves:
            x.requires_grad_(train)
        q, k, v, g = leaves[:4]
        S0 = leaves[4] if S_in is not None else None
        qc, kc, vc = (x.reshape(n, H, nc, C, dh) for x in (q, k, v))
        t = torch.arange(C, device="cuda")
        ch = torch.arange(nc, device="cuda")
        lag = t[:, None] - t[None, :]
        D = torch.where(lag >= 0, _power(g, lag.clamp(min=0)), 0.0)
        o = ((qc @ kc.transpose(-1, -2)) * D[None, :, None]) @ vc
        add = (kc * _power(g, C - 1 - t)[None, :, None, :, None]).transpose(-1, -2) @ vc
        lag = ch[:, None] - 1 - ch[None, :]
        E = torch.where(lag >= 0, _power(g, C * lag.clamp(min=0)), 0.0)
        S = (E[None] @ add.reshape(n, H, nc, dh * dh)).reshape(n, H, nc, dh, dh)
        if S0 is not None:
            S = S + _power(g, C * ch)[None, :, :, None, None] * S0[:, :, None]
        o = o + (qc @ S) * _power(g, t + 1)[None, :, None, :, None]
        o = o.reshape(n, H, L, dh) * dh ** -0.5
        out = {"o": _pack(o, places).detach().to(dt)}
        ends, grads = [o], []
        if train:
            grads = [_pad(s["do"], H, places)]
        if S0 is not None:
            m = (s["cu"][1:] - s["cu"][:-1]).long()
            left = m[:, None] - 1 - torch.arange(L, device="cuda")[None, :]
            w = torch.where(left >= 0, _power(g, left.clamp(min=0)), 0.0).transpose(0, 1)
            S1 = (k * w[..., None]).transpose(-1, -2) @ v
            S1 = S1 + _power(g, m).transpose(0, 1)[..., None, None] * S0
            out["S"] = S1.detach()
            ends.append(S1)
            grads.append(s.get("dS_out"))
        if train:
            want = leaves if c["dgamma"] else leaves[:3] + leaves[4:]
            got = list(torch.autograd.grad(ends, want, grads))
            for x in ("dq", "dk", "dv"):
                out[x] = _pack(got.pop(0), places).to(dt)
            if c["dgamma"]:
                out["dgamma"] = got.pop(0)
            if S0 is not None:
                out["dS"] = got.pop(0)
    return out


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "lin_step":
        return {"bytes": c["B"] * H * (8 * dh * dh + 4 * dh * es), "flops": c["B"] * H * 5 * dh * dh}
    if c["op"] == "attn_decode":
        seen = sum(n + 1 for n in _cached(c))
        return {"bytes": (seen * 2 * Hkv + c["B"] * (2 * H + 2 * Hkv)) * dh * es,
                "flops": seen * H * 4 * dh}
    lens = _lens(c)
    total = sum(lens)
    if c["op"].startswith("attn"):
        pairs = sum(n * (n + 1) // 2 for n in lens)
        b, f = total * (2 * H + 2 * Hkv) * dh * es, pairs * H * 4 * dh
        if c["op"] == "attn_train":  # + q, k, v, o, do read and dq, dk, dv written
            b += total * (4 * H + 4 * Hkv) * dh * es + 8 * total * H
            f += pairs * H * 10 * dh
        return {"bytes": b, "flops": f}
    b, f = total * H * 4 * dh * es, total * H * 4 * dh * dh
    states = len(lens) * H * dh * dh * 4 if c["states"] else 0
    b += 2 * states
    if c["op"] == "lin_train":  # + q, k, v, do read and dq, dk, dv written
        b += total * H * 7 * dh * es + 3 * states
        f += total * H * 10 * dh * dh
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    scale = 1.0 / math.sqrt(dh)
    if c["op"] == "attn_decode":
        o = torch.zeros((c["B"], H, dh), dtype=torch.float64, device="cuda")
        slot = s["slot"].tolist()
        for b, n in enumerate(_cached(c)):
            s["kcache"][slot[b], n] = s["k"][b]
            s["vcache"][slot[b], n] = s["v"][b]
            for h in range(H):
                kk = s["kcache"][slot[b], :n + 1, h * Hkv // H].double()
                vv = s["vcache"][slot[b], :n + 1, h * Hkv // H].double()
                w = torch.softmax(kk @ s["q"][b, h].double() * scale, 0)
                o[b, h] = w @ vv
        return {"o": o, "kcache": None, "vcache": None}
    if c["op"] == "lin_step":
        g = s["gamma"].double()
        S = torch.zeros(s["S_in"].shape, dtype=torch.float64, device="cuda")
        o = torch.zeros((c["B"], H, dh), dtype=torch.float64, device="cuda")
        for b, i in enumerate(s["slot"].tolist()):
            S[i] = g[:, None, None] * s["S_in"][i].double() + torch.einsum(
                "hi,hj->hij", s["k"][b].double(), s["v"][b].double())
            o[b] = scale * torch.einsum("hi,hij->hj", s["q"][b].double(), S[i])
        return {"o": o, "S": S}
    cu = [0]
    for m in _lens(c):
        cu.append(cu[-1] + m)
    return (_exact_attention if c["op"].startswith("attn") else _exact_linear)(c, s, cu, scale)


def _exact_attention(c, s, cu, scale):
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    total = cu[-1]
    train = c["op"] == "attn_train"
    if sum((b - a) ** 2 for a, b in zip(cu, cu[1:])) * H * dh * (14 if train else 4) > 1e14:
        return None

    def zeros(h):
        return torch.zeros((total, h, dh), dtype=torch.float64, device="cuda")

    q, k, v = (s[x].reshape(total, -1, dh) for x in "qkv")
    o, dq, dk, dv = zeros(H), zeros(H), zeros(Hkv), zeros(Hkv)
    for a, b in zip(cu, cu[1:]):
        for h in range(H):
            j = h // (H // Hkv)
            for t in range(a, b, 2048):  # rows of queries at a time
                e = min(b, t + 2048)
                qq, kk, vv = q[t:e, h].double(), k[a:e, j].double(), v[a:e, j].double()
                seen = torch.ones((e - t, e - a), dtype=torch.bool, device="cuda").tril(t - a)
                w = torch.softmax(torch.where(seen, scale * qq @ kk.T, -math.inf), 1)
                o[t:e, h] = w @ vv
                if train:
                    d = s["do"].reshape(total, H, dh)[t:e, h].double()
                    dv[a:e, j] += w.T @ d
                    x = d @ vv.T
                    x = w * (x - (w * x).sum(1, keepdim=True)) * scale
                    dq[t:e, h] = x @ kk
                    dk[a:e, j] += x.T @ qq
    out = {"o": o.reshape(total, -1)}
    if train:
        out.update(dq=dq.reshape(total, -1), dk=dk.reshape(total, -1), dv=dv.reshape(total, -1))
    return out


def _exact_linear(c, s, cu, scale):
    """Token by token, all sequences and heads abreast; a sequence that has
    ended keeps its state."""
    H, dh = c["H"], c["dh"]
    n, total, longest = len(cu) - 1, cu[-1], s["longest"]
    train = c["op"] == "lin_train"
    if longest > 200000:
        return None
    lens = torch.tensor(_lens(c), device="cuda")
    start = torch.tensor(cu[:-1], device="cuda")
    q, k, v = (s[x].reshape(total, H, dh) for x in "qkv")
    do = s["do"].reshape(total, H, dh) if train else None
    g = s["gamma"].double()[None, :, None, None]
    S = s["S_in"].double() if "S_in" in s else torch.zeros((n, H, dh, dh), dtype=torch.float64, device="cuda")
    dot = torch.zeros_like(S)  # dS / dg
    o, dq, dk, dv = (torch.zeros((total + 1, H, dh), dtype=torch.float64, device="cuda") for _ in range(4))
    dg = torch.zeros(H, dtype=torch.float64, device="cuda")
    zero = torch.zeros((1, H, dh), dtype=q.dtype, device="cuda")
    qz, kz, vz = (torch.cat([x, zero]) for x in (q, k, v))
    dz = torch.cat([do, zero]) if train else None
    lasting = min(int(x) for x in lens.tolist())
    for t in range(longest):
        r = torch.where(t < lens, start + t, total)
        f = g if t < lasting else torch.where((t < lens)[:, None, None, None], g, 1.0)
        kt, vt, qt = kz[r].double(), vz[r].double(), qz[r].double()
        if c["dgamma"]:
            dot = f * dot + (S if t < lasting else torch.where((t < lens)[:, None, None, None], S, 0.0))
        S = torch.addcmul(f * S, kt[..., :, None], vt[..., None, :])
        o[r] = scale * (qt[..., None, :] @ S)[..., 0, :]
        if train:
            dt = dz[r].double()
            dq[r] = scale * (S @ dt[..., None])[..., 0]
            if c["dgamma"]:
                dg += scale * ((qt[..., None, :] @ dot)[..., 0, :] * dt).sum((0, 2))
    out = {"o": o[:total].reshape(total, -1)}
    if c["states"]:
        out["S"] = S
    if train:
        R = s["dS_out"].double() if "dS_out" in s else torch.zeros_like(S)
        if c["dgamma"]:
            dg += (R * dot).sum((0, 2, 3))
            out["dgamma"] = dg
        for t in reversed(range(longest)):
            r = torch.where(t < lens, start + t, total)
            R = torch.addcmul(R, scale * qz[r].double()[..., :, None], dz[r].double()[..., None, :])
            dk[r] = (R @ vz[r].double()[..., None])[..., 0]
            dv[r] = (kz[r].double()[..., None, :] @ R)[..., 0, :]
            R = (g if t < lasting else torch.where((t < lens)[:, None, None, None], g, 1.0)) * R
        out.update({x: y[:total].reshape(total, -1) for x, y in (("dq", dq), ("dk", dk), ("dv", dv))})
        if c["states"]:
            out["dS"] = R
    return out
