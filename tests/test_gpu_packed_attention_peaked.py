"""Gradients of packed attention where softmax rows have one large entry and many keys: dS is then a small difference
beside delta, and delta formed from the bf16 output alone would drown it."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu
BF16, F64, F = torch.bfloat16, torch.float64, ref.F


def gradients(q, k, v, cu, do):
    """dict name -> (float64 value, bound) of dq and dk.  The delta of dK is that of the row's dS, in float32; that of
    dQ is off by at most 2^-9 of the sum of |dS| over the row (as formed: 1 / (1 - 2^-9) of the true one) and float32;
    dS is rounded to bf16 as operand; the output is rounded once."""
    T, H, hd = q.shape
    G, scale = k.shape[1], 1 / math.sqrt(q.shape[2])
    x = [t.to(F64) for t in (q, k, v, do)]
    r = {n: (torch.zeros(t.shape, dtype=F64, device=q.device), torch.zeros(t.shape, dtype=F64, device=q.device))
         for n, t in (("dq", q), ("dk", k))}
    ends = [int(c) for c in cu]
    for a, b in zip(ends[:-1], ends[1:]):
        keep = torch.ones((b - a, b - a), dtype=torch.bool, device=q.device).tril()
        n = (b - a + 16) * F
        for h in range(H):
            g = h * G // H
            Q, K, V, D = x[0][a:b, h], x[1][a:b, g], x[2][a:b, g], x[3][a:b, h]
            S = (Q @ K.t() * scale).masked_fill(~keep, -math.inf)
            lse = torch.logsumexp(S, 1)
            P = (S - lse[:, None]).exp()
            eS = hd * F * (Q.abs() @ K.abs().t()) * scale + 8 * F * (1 + S.abs().masked_fill(~keep, 0))
            eP = P * (eS + (n + eS.masked_fill(~keep, 0).amax(1) + 4 * F * lse.abs())[:, None]) + ref.TINY * keep
            dP = D @ V.t()
            delta = (P * dP).sum(1)
            dS = P * (dP - delta[:, None])
            edP = hd * F * (D.abs() @ V.abs().t())
            wide = dP.abs() + delta.abs()[:, None]
            narrow = ((eP + n * P) * wide + P * edP).sum(1) * 2  # float32: delta and the sum of a row of dS
            for name, left in (("dq", 1.01 * 2.0 ** -9 * dS.abs().sum(1)), ("dk", 0.0)):
                e = P * (edP + (narrow + left)[:, None]) + eP * (dP - delta[:, None]).abs() + ref.TINY * keep
                e = e + (ref.BF + n) * (dS.abs() + e)
                if name == "dq":
                    r[name][0][a:b, h], r[name][1][a:b, h] = dS @ K * scale, e @ K.abs() * scale
                else:
                    r[name][0][a:b, g] += dS.t() @ Q * scale
                    r[name][1][a:b, g] += e.t() @ Q.abs() * scale
    return {n: (w, e + ref.BF * (w.abs() + e) + ref.TINY) for n, (w, e) in r.items()}


def make(lens, H, G, hd, sink, spread, device="cuda", seed=0):
    """Queries along a direction that is each sequence's first key; without a sink, that key twice as long as others."""
    g = torch.Generator(device=device).manual_seed(seed)
    T = sum(lens)
    randn = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
    cu = torch.tensor([0] + lens, device=device).cumsum(0).to(torch.int32)
    d = randn(hd)
    d = d / d.norm()
    q, k = randn(T, H, hd) * spread + sink * d, randn(T, G, hd)
    first = cu[:-1].long()
    k[first] = sink * d if sink else 2 * k[first]
    return q.to(BF16), k.to(BF16), randn(T, G, hd).to(BF16), randn(T, H, hd).to(BF16), cu


# one wave group a tile and two, every channel class
CASES = [([600], 4, 2, 64), ([600, 130], 4, 2, 96), ([700], 4, 2, 128), ([300], 2, 1, 256),
         ([2000, 1000, 2000], 16, 2, 64),
         ([2000, 1000, 2000], 16, 8, 128)]


@pytest.mark.parametrize("lens,H,G,hd", CASES, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("sink,spread", [(0.0, 1.3), (0.0, 2.5), (9.0, 1.0), (12.0, 1.0)])
def test_rows_with_a_large_entry_behind_the_first_tile(rq, ctx, lens, H, G, hd, sink, spread):
    print(f"[gpu-case] peaked attention {lens} {H}/{G} x {hd}, sink {sink}, spread {spread}", flush=True)
    q, k, v, do, cu = make(lens, H, G, hd, sink, spread)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    dq, dk, _ = rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)
    want = gradients(q, k, v, cu, do)
    ref.close(dq, *want["dq"], "dq")
    ref.close(dk, *want["dk"], "dk")
