"""The operators' definitions in float64, with bounds on what float32 and bf16 roundings can move.

A rounding to bf16 moves a value by at most 2^-8 of it, one to float32 by at most 2^-24."""
import math

import torch

F64 = torch.float64
BF, F = 2.0 ** -8, 2.0 ** -24
# Results of the exponential, and operands and products of the matrix unit, below the normal range of 2^-126
# become 0: each is off by at most that.
TINY = 2.0 ** -126


# ----------------------------------------------------------------------------- token log probabilities

def logprobs(z, y=None, top=0):
    """dict of float64 lse, logp, entropy, top_ids, top_logp; empty rows and absent targets as documented."""
    z = z.to(F64)
    V = z.shape[1]
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    empty = (z == -math.inf).all(1)
    lp[empty] = -math.inf
    p = lp.exp()
    r = {"lse": lse, "entropy": -torch.where(p == 0, 0.0, p * lp).sum(1)}
    if y is not None:
        r["logp"] = lp.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
        r["logp"] = torch.where(y < 0, 0.0, torch.where(y >= V, math.nan, r["logp"]))
    if top:
        r["top_ids"] = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
        r["top_logp"] = lp.gather(1, r["top_ids"])
    return r


def logprobs_gradient(z, y=None, ids=None, dlogp=None, dentropy=None, dtop=None):
    """(gradient, bound on the float32 errors before the rounding to the output type)."""
    z = z.to(F64)
    T, V = z.shape
    r = logprobs(z)
    lp = z - r["lse"][:, None]
    empty = (r["lse"] == -math.inf)[:, None]
    p = torch.where(empty, 0.0, lp.exp())
    c = torch.zeros(T, dtype=F64, device=z.device)
    e = torch.zeros_like(z)

    def put(cols, g):
        ok = (cols >= 0) & (cols < V)
        g = torch.where(ok, g, 0.0)
        e.scatter_add_(1, cols.clamp(0, V - 1), g)
        return g.sum(1)

    if dlogp is not None:
        c += put(y[:, None], dlogp.to(F64)[:, None])
    if dtop is not None:
        c += put(ids, dtop.to(F64))
    dh = torch.zeros(T, 1, dtype=F64, device=z.device) if dentropy is None else dentropy.to(F64)[:, None]
    inner = torch.where(p == 0, 0.0, lp + r["entropy"][:, None])
    g = torch.where(empty, 0.0, -p * (c[:, None] + dh * inner) + e)
    # p = e^(z - lse): the exponent is off by the roundings of z - lse, of lse and of the entropy
    rel = lse_bound(V, r["lse"])[:, None] + 4 * F * (1 + torch.where(p == 0, 0.0, lp).abs())
    bound = p * (rel + 16 * F) * (c.abs()[:, None] + dh.abs() * (inner.abs() + 1)) + p * dh.abs() * rel * 4
    return g, bound + 70 * F * (e.abs() + p * c.abs()[:, None])


def lse_bound(V, lse):
    """A sum of V exponentials in float32 by at least 256 partial sums, and the rounding of the result."""
    return (V / 256 + 64) * F + 4 * F * torch.where(torch.isfinite(lse), lse, 0.0).abs()


# ----------------------------------------------------------------------------- packed attention

def attention(q, k, v, cu, do=None, scale=None):
    """dict name -> (float64 value, bound): o, lse and, with do, dq, dk, dv.  Rows outside every sequence are 0.
    Bounds: P and dS rounded to bf16 as operands, O as the backward reads it, and the outputs; float32 sums."""
    T, H, hd = q.shape
    G = k.shape[1]
    scale = 1 / math.sqrt(hd) if scale is None else scale
    x = {n: t.to(F64) for n, t in (("q", q), ("k", k), ("v", v))}
    r = {n: (torch.zeros(s, dtype=F64, device=q.device), torch.zeros(s, dtype=F64, device=q.device)) for n, s in
         (("o", q.shape), ("lse", (H, T)), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    ends = [int(c) for c in cu]
    for a, b in zip(ends[:-1], ends[1:]):
        if a == b:
            continue
        keep = torch.ones((b - a, b - a), dtype=torch.bool, device=q.device).tril()
        for h in range(H):
            g = h * G // H
            Q, K, V = x["q"][a:b, h], x["k"][a:b, g], x["v"][a:b, g]
            S = (Q @ K.t() * scale).masked_fill(~keep, -math.inf)
            lse = torch.logsumexp(S, 1)
            P = (S - lse[:, None]).exp()
            # float32: scores of hd products, their exponent, sums of b - a terms
            eS = (hd * F * (Q.abs() @ K.abs().t()) * scale + 8 * F * (1 + S.abs().masked_fill(~keep, 0)))
            eL = (b - a + 16) * F + eS.amax(1) + 4 * F * lse.abs()
            eP = P * (eS + eL[:, None]) + TINY * keep
            O = P @ V
            eO = (P * BF + eP) @ V.abs() + (b - a) * F * (P @ V.abs())
            r["o"][0][a:b, h], r["o"][1][a:b, h] = O, eO + BF * (O.abs() + eO)
            r["lse"][0][h, a:b], r["lse"][1][h, a:b] = lse, eL
            if do is None:
                continue
            D = do[a:b, h].to(F64)
            dP = D @ V.t()
            delta = (O * D).sum(1)
            eD = (r["o"][1][a:b, h] * D.abs()).sum(1) + hd * F * (O * D).abs().sum(1)
            dS = P * (dP - delta[:, None])
            edP = hd * F * (D.abs() @ V.abs().t())
            edS = P * (edP + eD[:, None]) + eP * (dP - delta[:, None]).abs() + dS.abs() * BF + TINY * keep
            n = (b - a + 8) * F
            for name, val, err, i in (("dq", dS @ K * scale, (edS + n * dS.abs()) @ K.abs() * scale, h),
                                      ("dk", dS.t() @ Q * scale, (edS + n * dS.abs()).t() @ Q.abs() * scale, g),
                                      ("dv", P.t() @ D, (P * (BF + n) + eP).t() @ D.abs(), g)):
                r[name][0][a:b, i] += val
                r[name][1][a:b, i] += err
    for name in ("dq", "dk", "dv"):
        r[name] = (r[name][0], r[name][1] + BF * (r[name][0].abs() + r[name][1]) + TINY)
    return r


# ----------------------------------------------------------------------------- 8-bit product

def quantize_rows(x):
    """(codes as float64, float32 scales)."""
    x = x.to(F64)
    s = (x.abs().amax(1) / 127).to(torch.float32)
    bad = ~torch.isfinite(x).all(1)
    s[bad] = math.nan
    ok = (s > 0)[:, None]
    q = torch.where(ok, x / s.to(F64)[:, None], 0.0).round().clamp(-127, 127)
    return q, s


def linear(xq, sx, wq, sw, bias=None):
    """(float64 value, bound of its float32 evaluation)."""
    y = xq.to(F64) @ wq.to(F64).t() * sx.to(F64)[:, None] * sw.to(F64)
    b = torch.zeros_like(sw, dtype=F64) if bias is None else bias.to(F64)
    return y + b, 5 * F * (y.abs() + b.abs()) + 2.0 ** -149


def close(got, want, bound, name=""):
    """Whether got (any float type) is within bound of want everywhere, NaN and infinities in the same places."""
    got = got.to(F64)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{name}: infinities"
    off = torch.where(fine, (got - want).abs() - bound, -1.0)
    if off.numel():
        i = int(off.argmax())
        assert float(off.flatten()[i]) <= 0, (
            f"{name}: {float(got.flatten()[i])} is {float((got - want).abs().flatten()[i])} off "
            f"{float(want.flatten()[i])}, bound {float((bound + torch.zeros_like(want)).flatten()[i])} (entry {i})")
