"""Token log probabilities, entropy, alternatives and their gradient against the float64 definition."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 7), (3, 64), (2, 1000), (5, 4099), (33, 32003), (1, 128256), (257, 2051), (600, 515), (40, 151936), (1, 700001), (3, 1100003)]


def make(T, V, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((T, V), generator=g, device="cuda") * 3
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    z[torch.arange(T, device="cuda"), y] += 5
    return z.to(dtype), y, g


def check_forward(r, z, y, top):
    want = ref.logprobs(z, y, top)
    tol = ref.lse_bound(z.shape[1], want["lse"])
    ref.close(r.lse, want["lse"], tol, "lse")
    if y is not None:
        ref.close(r.logp, want["logp"], tol + 4 * ref.F * want["logp"].abs().nan_to_num(0, 0, 0), "logp")
    if r.entropy is not None:
        # log S - U / S: both sums to the bound of S, U's terms at most 0.37 V + |U|
        ref.close(r.entropy, want["entropy"], 2 * tol + 3 * tol * (1 + want["entropy"] + math.log(z.shape[1])), "entropy")
    if top:
        assert torch.equal(r.top_ids, want["top_ids"])
        ref.close(r.top_logp, want["top_logp"],
                  tol[:, None] + 4 * ref.F * want["top_logp"].abs().nan_to_num(0, 0, 0), "top_logp")
    return want


def check_gradient(rq, ctx, z, y, scores, g, inplace=False, ld=None):
    T, V = z.shape
    dlogp = torch.randn(T, generator=g, device="cuda")
    dent = torch.randn(T, generator=g, device="cuda") if scores.entropy is not None else None
    dtop = torch.randn(scores.top_ids.shape, generator=g, device="cuda") if scores.top_ids is not None else None
    want, bound = ref.logprobs_gradient(z, y, scores.top_ids, dlogp, dent, dtop)
    if z.dtype == torch.bfloat16:
        bound = bound + ref.BF * (want.abs() + bound) + 2.0 ** -133
    bound = bound + 2.0 ** -120  # what falls below the normal range is 0
    src = z.clone() if inplace else z
    got = rq.token_logprobs_backward(ctx, src, y, scores, dlogp=dlogp, dentropy=dent, dtop=dtop,
                                     out=src if inplace else None)
    ref.close(got, want, bound, "dlogits")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V", SIZES)
def test_scores_and_gradient(rq, ctx, T, V, dtype):
    print(f"[gpu-case] logprobs {T}x{V} {dtype}", flush=True)
    z, y, g = make(T, V, dtype)
    for top in sorted({0, 1, min(V, 5), min(V, 20), min(V, 64)}):
        r = rq.token_logprobs(ctx, z, y, top=top, entropy=True)
        check_forward(r, z, y, top)
        if top in (0, min(V, 5)):
            check_gradient(rq, ctx, z, y, r, g, inplace=top == 0)
    bare = rq.token_logprobs(ctx, z)
    assert bare.logp is None and bare.entropy is None
    check_forward(bare, z, None, 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(6, 5003), (520, 1537)])
def test_masks_infinities_and_ties(rq, ctx, T, V, dtype):
    """Masked tokens, the type's lowest value, an empty row, one token left, NaN, +infinity, all equal, targets
    that are absent, masked or out of range."""
    z, y, g = make(T, V, dtype, 1)
    low = torch.finfo(dtype).min
    z[0, V // 3:] = -math.inf
    y[0] = 1
    z[1] = low
    z[1, 11:17] = 0.0
    y[1] = V - 1
    z[2] = -math.inf
    z[3] = 0.25
    y[3] = -100
    z[4] = -math.inf
    z[4, V - 2] = 3.0
    y[4] = V - 2
    z[5] = low
    y[5] = V
    top = 9
    r = rq.token_logprobs(ctx, z, y, top=top, entropy=True)
    want = check_forward(r, z, y, top)
    assert float(r.lse[2]) == float(r.logp[2]) == -math.inf and float(r.entropy[2]) == 0
    assert torch.equal(r.top_ids[2], torch.arange(top, device="cuda")) and torch.equal(r.top_ids[3], r.top_ids[2])
    assert float(want["logp"][3]) == 0 and math.isnan(float(r.logp[5]))
    y[5] = -1
    r = rq.token_logprobs(ctx, z, y, top=top, entropy=True)
    check_gradient(rq, ctx, z, y, r, g)
    y[5] = V
    got = rq.token_logprobs_backward(ctx, z, y, r, dlogp=torch.ones(T, device="cuda"))
    assert torch.isnan(got[5]).all() and torch.isfinite(got[:5]).all()
    assert (got[2] == 0).all() and (got[3] == 0).all()
    for bad in (math.nan, math.inf):
        z[0, 7] = bad
        r = rq.token_logprobs(ctx, z, y, top=top, entropy=True)
        assert torch.isnan(torch.stack([r.lse[0], r.logp[0], r.entropy[0]])).all() and torch.isnan(r.top_logp[0]).all()
        assert ((r.top_ids >= 0) & (r.top_ids < V)).all() and torch.isfinite(r.logp[1]) and torch.isfinite(r.lse[3])


def test_many_ties_and_sorted_rows(rq, ctx):
    """Few distinct values, ascending and descending rows, the best columns all in one stretch: the
    alternatives are those of a stable sort."""
    V = 70001
    j = torch.arange(V, device="cuda", dtype=torch.float32)
    z = torch.stack([(j * 7 % 3), j / V, -j / V, torch.where(j == V - 1, 1.0, 0.0), (j // 64 % 17),
                     torch.where((j > 5000) & (j < 5100), 9 - j / V, -j / V), torch.where(j % 256 == 3, 2.0, 1.0),
                     torch.where(j < 100, -0.0, 0.0)])
    for dtype in (torch.float32, torch.bfloat16):
        for rows in (z, z.repeat(80, 1)):
            x = rows.to(dtype)
            r = rq.token_logprobs(ctx, x, None, top=64)
            assert torch.equal(r.top_ids, torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :64])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (8, 8), (0, 1)])
def test_strided_and_unaligned_rows(rq, ctx, dtype, offset, pad):
    T, V = 5, 3001
    z, y, g = make(T, V + offset + pad, dtype, 2)
    z = z[:, offset:offset + V]
    y = y % V
    r = rq.token_logprobs(ctx, z, y, top=5, entropy=True)
    check_forward(r, z, y, 5)
    check_gradient(rq, ctx, z, y, r, g)
    out = torch.full((T, V + 7), 5.0, device="cuda", dtype=dtype)
    rq.token_logprobs_backward(ctx, z, y, r, dlogp=torch.ones(T, device="cuda"), out=out[:, 3:3 + V])
    assert (out[:, :3] == 5).all() and (out[:, 3 + V:] == 5).all()


def test_repeated_columns_receive_the_sum(rq, ctx):
    """Alternatives given by the caller that name a column twice, the target, or nothing."""
    z, y, g = make(3, 400, torch.float32, 3)
    y[:] = 17
    r = rq.token_logprobs(ctx, z, y, top=4, entropy=True)
    r.top_ids = torch.tensor([[17, 17, 5, 5], [3, 3, 3, 3], [-1, 400, 17, 0]], device="cuda")
    check_gradient(rq, ctx, z, y, r, g)


def test_gradient_against_differences(rq, ctx):
    """d/de of sum w logp + sum u entropy along a direction, by central differences of the float64 definition;
    their error is e^2 times a third derivative of order 1."""
    z, y, g = make(7, 900, torch.float32, 4)
    w, u = torch.randn(7, generator=g, device="cuda"), torch.randn(7, generator=g, device="cuda")
    d = torch.randn((7, 900), generator=g, device="cuda", dtype=torch.float64)
    r = rq.token_logprobs(ctx, z, y, entropy=True)
    got = (rq.token_logprobs_backward(ctx, z, y, r, dlogp=w, dentropy=u).double() * d).sum()

    def f(x):
        s = ref.logprobs(x, y)
        return (s["logp"] * w.double()).sum() + (s["entropy"] * u.double()).sum()
    e = 1e-4
    diff = (f(z.double() + e * d) - f(z.double() - e * d)) / (2 * e)
    _, bound = ref.logprobs_gradient(z, y, None, w, u)
    assert abs(float(got - diff)) <= float((bound * d.abs()).sum()) + 1e-5 * (1 + abs(float(diff)))


def test_long_rows_far_apart(rq, ctx):
    """Rows whose offsets pass 2^31 elements."""
    V, ld = 1000, 1 << 30
    buf = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((3, V), (ld, 1))
    z.copy_(torch.randn(3, V, device="cuda"))
    y = torch.tensor([0, 5, 999], device="cuda")
    r = rq.token_logprobs(ctx, z, y, top=3, entropy=True)
    check_forward(r, z, y, 3)
    check_gradient(rq, ctx, z, y, r, torch.Generator(device="cuda").manual_seed(1))


def test_no_rows(rq, ctx):
    z = torch.empty((0, 50), device="cuda")
    r = rq.token_logprobs(ctx, z, torch.empty(0, dtype=torch.int64, device="cuda"), top=2, entropy=True)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 2)
    assert rq.token_logprobs_backward(ctx, z, None, r).shape == (0, 50)


@pytest.mark.parametrize("T", [1, 300])
def test_captured_and_replayed(rq, T):
    """Two graphs of one context, replayed in turn with new logits and eager work between."""
    V = 20011
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = rq.Context(stream)
        z, y, g = make(T, V, torch.bfloat16, 5)
        w = torch.randn(T, generator=g, device="cuda")

        def run(top):
            r = rq.token_logprobs(c, z, y, top=top, entropy=True)
            return [r.logp, r.lse, r.entropy, r.top_ids, r.top_logp, rq.token_logprobs_backward(c, z, y, r, dlogp=w)]
        run(3)
        stream.synchronize()
        graphs = []
        for top in (3, 20):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                graphs.append((graph, top, run(top)))
            graph = None
        for i in range(3):
            z.copy_(torch.randn((T, V), generator=g, device="cuda"))
            for graph, top, out in graphs:
                graph.replay()
            stream.synchronize()
            torch.randn(1 << 16, device="cuda").sum().item()
            for graph, top, out in graphs:
                for a, b in zip(out, run(top)):
                    assert torch.equal(a, b), (i, top)
        stream.synchronize()
        c.close()
