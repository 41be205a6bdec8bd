"""Packed attention and linear attention in 64 bits on the CPU, with error bounds.

Every function returns its outputs and, for each, a bound on the error that a
correct kernel may make, element by element.  `u` is half a step of the
compute type (2^-8 for bfloat16, 2^-24 for float32) and E = 2^-24 half a step
of float32.  What is counted:

  - each product's operand that is rounded to the type: u of its magnitude
    (softmax weights, their gradients, decayed scores, states as an operand);
  - the output's own rounding: u of its magnitude;
  - float32 sums of n terms: n E of the sum of magnitudes, and the relative
    error of an exponential or a power, E times its exponent's size.

The sums of magnitudes are formed in 64 bits beside the values.
"""

import math

import torch

E = 2.0 ** -24


def unit(dtype):
    return 2.0 ** -8 if dtype == "bf16" else E


def sequences(cu):
    return [(a, b) for a, b in zip(cu, cu[1:])]


def attention(q, k, v, cu, scale, dtype, do=None):
    """q, do [total, H, dh], k, v [total, Hkv, dh] float64; rows outside the
    sequences stay zero.  {name: (value, bound)}."""
    total, H, dh = q.shape
    Hkv = k.shape[1]
    G, u = H // Hkv, unit(dtype)
    res = {n: [torch.zeros_like(q), torch.zeros_like(q)] for n in ("o", "dq")}
    res.update({n: [torch.zeros_like(k), torch.zeros_like(k)] for n in ("dk", "dv")})
    res["lse"] = [torch.zeros(H, total, dtype=q.dtype), torch.zeros(H, total, dtype=q.dtype)]
    for a, b in sequences(cu):
        n = b - a
        if n == 0:
            continue
        seen = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(H):
            j = h // G
            Q, K, V = q[a:b, h], k[a:b, j], v[a:b, j]
            z = scale * Q @ K.T
            zabs = scale * Q.abs() @ K.abs().T
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[:, None])
            o = p @ V
            # relative error of a weight: the score's sum, the exponent, the
            # float32 sum of the weights
            zmax = torch.where(seen, zabs, torch.zeros_like(z)).amax(1)
            ep = E * ((dh + 8) * (zabs + zmax[:, None]) + 4 * lse.abs()[:, None] + n + 16)
            pa = p * (u + ep)
            eo = pa @ V.abs() + (n + 64) * E * (p @ V.abs()) + u * o.abs()
            res["o"][0][a:b, h], res["o"][1][a:b, h] = o, eo
            res["lse"][0][h, a:b] = lse
            res["lse"][1][h, a:b] = E * ((dh + 8) * zmax + 4 * lse.abs() + n + 16)
            if do is None:
                continue
            D = do[a:b, h]
            dv = p.T @ D
            res["dv"][0][a:b, j] += dv
            res["dv"][1][a:b, j] += pa.T @ D.abs() + (n + 64) * E * (p.T @ D.abs())
            dp = D @ V.T
            delta = (D * o).sum(1, keepdim=True)
            dz = p * (dp - delta)
            # delta comes from the rounded o
            ed = (D.abs() * eo).sum(1, keepdim=True) + (dh + 8) * E * (D * o).abs().sum(1, keepdim=True)
            edp = (dh + 8) * E * D.abs() @ V.abs().T
            ez = dz.abs() * (u + ep) + p * (1 + u) * (ed + edp)
            m = dz.abs() + ez
            res["dq"][0][a:b, h] = scale * dz @ K
            res["dq"][1][a:b, h] = scale * (ez @ K.abs() + (n + 64) * E * (m @ K.abs()))
            res["dk"][0][a:b, j] += scale * dz.T @ Q
            res["dk"][1][a:b, j] += scale * (ez.T @ Q.abs() + (n + 64) * G * E * (m.T @ Q.abs()))
    for n in ("dq", "dk", "dv"):
        res[n][1] += u * (res[n][0].abs() + res[n][1])
    return {n: tuple(x) for n, x in res.items()}


def token(q, k, v, scale, dtype):
    """The last row of a sequence: q [H, dh], k, v [n, Hkv, dh].  (value, bound) as
    of `attention`."""
    (H, dh), (n, Hkv, _), u = q.shape, k.shape, unit(dtype)
    val, bound = torch.zeros_like(q), torch.zeros_like(q)
    for h in range(H):
        K, V = k[:, h * Hkv // H], v[:, h * Hkv // H]
        z, zabs = scale * K @ q[h], scale * K.abs() @ q[h].abs()
        lse = torch.logsumexp(z, 0)
        p = torch.exp(z - lse)
        ep = E * ((dh + 8) * (zabs + zabs.max()) + 4 * lse.abs() + n + 16)
        val[h] = p @ V
        bound[h] = (p * (u + ep)) @ V.abs() + (n + 64) * E * (p @ V.abs()) + u * val[h].abs()
    return val, bound


def linear(q, k, v, gamma, cu, scale, dtype, S_in=None, do=None, dS_out=None):
    """q, k, v, do [total, H, dh], gamma [H], states [nseq, H, dh, dh], float64.
    {name: (value, bound)} from the quadratic form."""
    total, H, dh = q.shape
    u, ns = unit(dtype), len(cu) - 1
    zero = torch.zeros(ns, H, dh, dh, dtype=q.dtype)
    S0 = zero if S_in is None else S_in
    R1 = zero if dS_out is None else dS_out
    res = {n: [torch.zeros_like(q), torch.zeros_like(q)] for n in ("o", "dq", "dk", "dv")}
    res.update({n: [torch.zeros_like(zero), torch.zeros_like(zero)] for n in ("S", "dS")})
    res["dgamma"] = [torch.zeros(H, dtype=q.dtype), torch.zeros(H, dtype=q.dtype)]
    A = scale if scale >= 0 else -scale
    for s, (a, b) in enumerate(sequences(cu)):
        n = b - a
        for h in range(H):
            g = float(gamma[h])

            def power(e):
                return torch.where(e == 0, torch.ones_like(e), torch.as_tensor(g, dtype=q.dtype) ** e)

            t = torch.arange(n, dtype=q.dtype)
            lag = t[:, None] - t[None, :]
            D = torch.where(lag >= 0, power(lag.clamp(min=0)), torch.zeros_like(lag))
            first, left = power(t + 1), power(n - 1 - t)
            # a power's exponent is e log2 g: its error is E of that, and no
            # larger than n |log2 g| E where the power matters (0 is exact)
            f = E * (2 * n * (abs(math.log2(g)) if g > 0 else 0.0) + 2 * n + 200)
            Q, K, V = q[a:b, h], k[a:b, h], v[a:b, h]
            S, R = S0[s, h], R1[s, h]
            o = scale * ((D * (Q @ K.T)) @ V + first[:, None] * (Q @ S))
            oa = A * ((D * (Q.abs() @ K.abs().T)) @ V.abs() + first[:, None] * (Q.abs() @ S.abs()))
            res["o"][0][a:b, h], res["o"][1][a:b, h] = o, (u + f) * oa + u * o.abs()
            gn = float(power(torch.tensor(float(n), dtype=q.dtype)))
            res["S"][0][s, h] = (K * left[:, None]).T @ V + gn * S
            res["S"][1][s, h] = f * ((K.abs() * left[:, None]).T @ V.abs() + gn * S.abs())
            if do is None:
                continue
            d = do[a:b, h]
            dov, qk = d @ V.T, Q @ K.T
            dova, qka = d.abs() @ V.abs().T, Q.abs() @ K.abs().T
            for name, val, mag in (
                    ("dq", scale * ((D * dov) @ K + first[:, None] * (d @ S.T)),
                     A * ((D * dova) @ K.abs() + first[:, None] * (d.abs() @ S.abs().T))),
                    ("dk", scale * (D * dov).T @ Q + left[:, None] * (V @ R.T),
                     A * (D * dova).T @ Q.abs() + left[:, None] * (V.abs() @ R.abs().T)),
                    ("dv", scale * (D * qk).T @ d + left[:, None] * (K @ R),
                     A * (D * qka).T @ d.abs() + left[:, None] * (K.abs() @ R.abs()))):
                res[name][0][a:b, h] = val
                res[name][1][a:b, h] = (u + f) * mag + u * val.abs()
            res["dS"][0][s, h] = scale * (Q * first[:, None]).T @ d + gn * R
            res["dS"][1][s, h] = f * (A * (Q.abs() * first[:, None]).T @ d.abs() + gn * R.abs())
            # d/dg g^e = e g^(e-1)
            dD = torch.where(lag >= 1, lag * power((lag - 1).clamp(min=0)), torch.zeros_like(lag))
            df = (t + 1) * power(t)
            dl = torch.where(n - 1 - t >= 1, (n - 1 - t) * power((n - 2 - t).clamp(min=0)),
                             torch.zeros_like(t))
            dn = n * float(power(torch.tensor(max(n - 1.0, 0.0), dtype=q.dtype))) if n else 0.0
            val = (scale * ((dD * qk * dov).sum() + (df[:, None] * (Q @ S) * d).sum())
                   + (R * (dn * S + (K * dl[:, None]).T @ V)).sum())
            mag = (A * ((dD * qka * dova).sum() + (df[:, None] * (Q.abs() @ S.abs()) * d.abs()).sum())
                   + (R.abs() * (dn * S.abs() + (K.abs() * dl[:, None]).T @ V.abs())).sum())
            res["dgamma"][0][h] += val
            res["dgamma"][1][h] += 2 * f * mag
    return {n: tuple(x) for n, x in res.items()}


def within(name, got, ref, rows=None):
    """Asserts |got - value| <= bound element by element (exact zeros too)."""
    val, bound = ref
    x = got.detach().cpu().double().reshape(val.shape)
    if rows is not None:
        x, val, bound = x[rows], val[rows], bound[rows]
    assert bool(torch.isfinite(x).all()), f"{name}: not finite"
    over = (x - val).abs() - bound
    worst = float(over.max()) if over.numel() else 0.0
    ratio = float(((x - val).abs() / bound.clamp(min=1e-300)).max()) if over.numel() else 0.0
    assert worst <= 0.0, f"{name}: error up to {ratio:.3f} of its bound"
    return ratio
