"""Packed causal attention, forward and backward, against the float64 definition with bounds counted from its
roundings."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

LENS = [[1], [2], [31, 1, 0, 33], [64], [127, 129], [0, 0, 5, 0], [257], [700, 3, 128, 0, 1, 500],
        [1] * 70, [5] * 130 + [200]]


def make(lens, H, G, hd, seed=0, behind=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lens) + behind
    r = lambda n, s=1.0: (torch.randn((T, n, hd), generator=g, device="cuda") * s).to(BF16)  # noqa: E731
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    return r(H, 1.5 * spread), r(G, spread), r(G), r(H), cu


def check(rq, ctx, q, k, v, do, cu, scale=None, backward=True):
    want = ref.attention(q, k, v, cu, do, scale)
    o, lse = rq.packed_attention(ctx, q, k, v, cu, scale=scale)
    n = int(cu[-1])
    ref.close(o[:n], want["o"][0][:n], want["o"][1][:n], "o")
    ref.close(lse[:, :n], want["lse"][0][:, :n], want["lse"][1][:, :n], "lse")
    if backward:
        for name, got in zip(("dq", "dk", "dv"), rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do, scale=scale)):
            ref.close(got[:n], want[name][0][:n], want[name][1][:n], name)
    return o, lse


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", LENS, ids=lambda x: f"{len(x)}x{max(x)}")
def test_lengths(rq, ctx, lens, hd):
    print(f"[gpu-case] packed attention {lens[:8]} hd {hd}", flush=True)
    check(rq, ctx, *make(lens, 4, 2, hd))


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (6, 2), (8, 1), (5, 1)])
@pytest.mark.parametrize("hd", [8, 32, 72, 96, 120, 160, 192, 256])
def test_heads(rq, ctx, H, G, hd):
    print(f"[gpu-case] packed attention heads {H}/{G} x {hd}", flush=True)
    check(rq, ctx, *make([40, 150, 1], H, G, hd, 1))


@pytest.mark.parametrize("hd", [64, 88, 96, 104, 128])
@pytest.mark.parametrize("lens", [[900], [900] + [5] * 150], ids=["few", "many"])
def test_head_sizes_in_few_and_many_tiles(rq, ctx, lens, hd):
    check(rq, ctx, *make(lens, 4, 1, hd, 5))


@pytest.mark.parametrize("scale", [0.01, 0.5])
def test_scales_and_wide_scores(rq, ctx, scale):
    """Flat and saturated softmaxes."""
    check(rq, ctx, *make([300], 2, 1, 64, 2, spread=3.0), scale=scale)


def test_one_long_sequence(rq, ctx):
    check(rq, ctx, *make([4099], 2, 1, 128, 3))


def test_rows_behind_the_last_sequence_stay(rq, ctx):
    q, k, v, do, cu = make([100, 60], 4, 2, 64, 4, behind=37)
    n = 160
    q[n:], k[n:], v[n:], do[n:] = math.nan, math.nan, math.nan, math.nan
    out = torch.full_like(q, 7.0)
    _, lse = rq.packed_attention(ctx, q, k, v, cu, out=out)
    grads = rq.packed_attention_backward(ctx, q, k, v, cu, out, lse, do, dq=torch.full_like(q, 7.0),
                                         dk=torch.full_like(k, 7.0), dv=torch.full_like(v, 7.0))
    want = ref.attention(q, k, v, cu, do)
    for name, got in zip(("o", "dq", "dk", "dv"), (out, *grads)):
        assert (got[n:] == 7).all(), name
        ref.close(got[:n], want[name][0][:n], want[name][1][:n], name)


def test_a_sequence_does_not_see_its_neighbours(rq, ctx):
    """Each sequence gives what it gives alone (to the sum of both bounds: the order of its sums goes by the size
    of the call), and a NaN in one leaves the others' bits as they were."""
    lens = [70, 200, 1, 33]
    q, k, v, do, cu = make(lens, 4, 2, 128, 5)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    grads = rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)
    want = ref.attention(q, k, v, cu, do)
    a = 0
    for n in lens:
        rows = slice(a, a + n)
        one = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        part = [t[rows].contiguous() for t in (q, k, v, do)]
        o1, l1 = rq.packed_attention(ctx, *part[:3], one)
        ref.close(l1, lse[:, rows].double(), 2 * want["lse"][1][:, rows], "lse")
        alone = (o1, *rq.packed_attention_backward(ctx, *part[:3], one, o1, l1, part[3]))
        for name, x, y in zip(("o", "dq", "dk", "dv"), alone, (o, *grads)):
            ref.close(x, y[rows].double(), 2 * want[name][1][rows], name)
        a += n
    for t in (q, k, v, do):
        t[100] = math.nan
    o2, l2 = rq.packed_attention(ctx, q, k, v, cu)
    g2 = rq.packed_attention_backward(ctx, q, k, v, cu, o2, l2, do)
    for x, y in zip((o, *grads), (o2, *g2)):
        assert torch.equal(x[:70], y[:70]) and torch.equal(x[270:], y[270:])
        assert torch.isnan(y[100].float()).any()


def test_strided_rows(rq, ctx):
    """q, k and v (and their gradients) as slices of one projection's output."""
    H, G, hd = 4, 2, 64
    lens = [33, 90]
    w = (H + 2 * G) * hd
    g = torch.Generator(device="cuda").manual_seed(6)
    qkv = torch.randn((123, w + 8), generator=g, device="cuda").to(BF16)[:, :w]
    cut = lambda t: (t[:, :H * hd].unflatten(1, (H, hd)), t[:, H * hd:(H + G) * hd].unflatten(1, (G, hd)),  # noqa: E731
                     t[:, (H + G) * hd:].unflatten(1, (G, hd)))
    q, k, v = cut(qkv)
    cu = torch.tensor([0, 33, 123], dtype=torch.int32, device="cuda")
    do = torch.randn((123, H, hd), generator=g, device="cuda").to(BF16)
    o, lse = check(rq, ctx, q, k, v, do, cu)
    grads = torch.full((123, w + 8), 3.0, dtype=BF16, device="cuda")
    dq, dk, dv = cut(grads[:, :w])
    rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do, dq=dq, dk=dk, dv=dv)
    ref2 = rq.packed_attention_backward(ctx, q.contiguous(), k.contiguous(), v.contiguous(), cu, o, lse, do)
    for a, b in zip((dq, dk, dv), ref2):
        assert torch.equal(a, b)
    assert (grads[:, w:] == 3).all()


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_a_single_key_has_no_gradient(rq, ctx, hd):
    """The softmax over one key is constant: dQ of every sequence's first token and dK of sequences of one
    token are 0, to the bit."""
    q, k, v, do, cu = make([1, 40, 1, 1, 200], 4, 2, hd, 11)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    dq, dk, dv = rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)
    assert (dq[cu[:-1].long()] == 0).all() and (dk[[0, 41, 42]] == 0).all()
    assert torch.equal(o[0], v[0].repeat_interleave(2, 0)) and (dk[1] != 0).any()


def test_peaked_rows_keep_their_gradient(rq, ctx):
    """Few keys and saturated rows, where dS is a small difference: relative to its 2-norm dQ and dK keep the
    roundings of dS and of the output (each 2^-8 at most, evenly spread: 2^-8 / sqrt(3)), within a factor of 2."""
    q, k, v, do, cu = make([2] * 40 + [5] * 20 + [17] * 6, 4, 2, 96, 12)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    want = ref.attention(q, k, v, cu, do)
    for name, got in zip(("dq", "dk"), rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)):
        off = (got.double() - want[name][0]).norm() / want[name][0].norm()
        assert off <= 2 * math.sqrt(2 / 3) * ref.BF, (name, float(off))


def test_gradients_against_differences(rq, ctx):
    """The gradients along a direction against central differences of the float64 definition."""
    q, k, v, do, cu = make([45, 20], 4, 2, 64, 7)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    grads = rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)
    want = ref.attention(q, k, v, cu, do)
    g = torch.Generator(device="cuda").manual_seed(8)
    e = 1e-4
    for i, name in enumerate(("dq", "dk", "dv")):
        d = torch.randn(grads[i].shape, generator=g, device="cuda", dtype=torch.float64)

        def f(s):
            x = [t.double() for t in (q, k, v)]
            x[i] = x[i] + s * d
            return (ref.attention(*x, cu)["o"][0] * do.double()).sum()
        diff = float((f(e) - f(-e)) / (2 * e))
        got = float((grads[i].double() * d).sum())
        assert abs(got - diff) <= float((want[name][1] * d.abs()).sum()) + 1e-5 * (1 + abs(diff)), name


def test_the_same_bits_again(rq, ctx):
    q, k, v, do, cu = make([900, 300], 8, 2, 128, 9)
    runs = []
    for _ in range(3):
        o, lse = rq.packed_attention(ctx, q, k, v, cu)
        runs.append((o, lse, *rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_rows_far_apart(rq, ctx):
    """Rows whose offsets pass 2^31 elements: q, k, v, dO and the gradients in columns of one wide array."""
    T, H, G, hd, ld = 140, 2, 1, 64, 1 << 24
    buf = torch.empty(T * ld, dtype=BF16, device="cuda")
    at = lambda c, n: buf.as_strided((T, n, hd), (ld, hd, 1), c)  # noqa: E731
    q, k, v, do, cu = make([9, 131], H, G, hd, 13)
    wide = [at(1024 * i, t.shape[1]) for i, t in enumerate((q, k, v, do))]
    for w, t in zip(wide, (q, k, v, do)):
        w.copy_(t)
    o, lse = check(rq, ctx, *wide, cu)
    out, grads = at(8192, H), [at(9216 + 1024 * i, n) for i, n in enumerate((H, G, G))]
    rq.packed_attention(ctx, *wide[:3], cu, out=out)
    rq.packed_attention_backward(ctx, *wide[:3], cu, out, lse, wide[3], dq=grads[0], dk=grads[1], dv=grads[2])
    assert torch.equal(out, o)
    for a, b in zip(grads, rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do)):
        assert torch.equal(a, b)


def test_offsets_that_lie(rq, ctx):
    """Offsets outside the arrays or in a wrong order are cut to them: no meaning, no access outside, and what
    lies outside every cut sequence stays."""
    q, k, v, do, _ = make([64], 2, 1, 64, 10)
    for cu in ([-5, 1000], [0, 40, 20, 64], [70, 90], [0, 2 ** 31 - 1], [-2 ** 31, 10]):
        c = torch.tensor(cu, dtype=torch.int64).to(torch.int32).cuda()
        o, lse = rq.packed_attention(ctx, q, k, v, c)
        rq.packed_attention_backward(ctx, q, k, v, c, o, lse, do)
    torch.cuda.synchronize()


def test_nothing_to_do(rq, ctx):
    q, k, v, do, cu = make([0], 2, 1, 64)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)
    q, k, v, do, _ = make([9], 2, 1, 64)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 2.0)
    rq.packed_attention(ctx, q, k, v, none, out=out)
    assert (out == 2).all()


def test_captured_and_replayed(rq):
    """Graphs of two lengths of one context, the offsets changed between replays."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = rq.Context(stream)
        graphs = []
        for n in (300, 1000):
            q, k, v, do, _ = make([n], 4, 2, 128, n)
            cu = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")

            def run(q=q, k=k, v=v, do=do, cu=cu):
                o, lse = rq.packed_attention(c, q, k, v, cu)
                return (o, lse, *rq.packed_attention_backward(c, q, k, v, cu, o, lse, do))
            run()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = run()
            graphs.append((graph, run, out, cu, n))
        for i in range(3):
            for graph, run, out, cu, n in graphs:
                cu[1] = (n // 3, 0, n - 1)[i]
                q.normal_()
                graph.replay()
            stream.synchronize()
            torch.randn(1 << 16, device="cuda").sum().item()
            for graph, run, out, cu, n in graphs:
                assert all(torch.equal(a, b) for a, b in zip(out, run())), (i, n)
        stream.synchronize()
        c.close()
