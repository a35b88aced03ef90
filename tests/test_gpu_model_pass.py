"""The operators in a row, as a program uses them: projections quantized per row by the layer sweep and run in
8-bit integers, packed attention, a head, the tokens' log probabilities, the gradient back through the head and
the attention, and the Stage-0 accumulators on what arrives at a projection's output.  Every stage is checked
against its float64 definition on the inputs it was given."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu
BF16, F64 = torch.bfloat16, torch.float64


def close_linear(y, xq, sx, w8, sw, name):
    want, bound = ref.linear(xq, sx, w8, sw)
    ref.close(y, want, bound + ref.BF * (want.abs() + bound), name)


@pytest.mark.parametrize("lens", [[40, 1, 87], [200, 0, 56]])
def test_score_and_differentiate_a_quantized_block(rq, ctx, lens):
    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    d, H, G, hd, V, T = 128, 4, 2, 64, 1003, sum(lens)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    calib = randn(512, d).to(BF16)

    def quantized(rows, cols, X):
        """Integer weights of a module quantized per row, and their scales."""
        W = (randn(rows, cols) / math.sqrt(cols)).to(BF16).float()
        r = rq.quantize_layer(ctx, W, X, X, qp=rq.qparams(bits=4, group=0, sym=True), bgd=rq.bgd_params(steps=1, lr=1e-4))
        w8 = (r.codes.to(torch.int16) - r.zeros.to(torch.int16)).to(torch.int8)
        sw = r.scales[:, 0].contiguous()
        assert torch.equal(w8.float() * sw[:, None], r.W_hat)
        return w8, sw

    wqkv = [quantized(n * hd, d, calib) for n in (H, G, G)]
    wo = quantized(d, H * hd, randn(512, H * hd).to(BF16))
    head = (randn(V, d) * 0.5).to(BF16)
    x = randn(T, d).to(BF16)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    targets[0] = -1  # the first token has no prediction

    # forward
    xq, sx = rq.quantize_rows_i8(ctx, x)
    qkv = torch.empty((T, (H + 2 * G) * hd), dtype=BF16, device="cuda")  # one buffer, as the attention reads it
    cuts = (slice(0, H * hd), slice(H * hd, (H + G) * hd), slice((H + G) * hd, (H + 2 * G) * hd))
    for (w8, sw), cut in zip(wqkv, cuts):
        rq.linear_i8(ctx, xq, sx, w8, sw, out=qkv[:, cut])
        close_linear(qkv[:, cut], xq, sx, w8, sw, "projection")
    q, k, v = (qkv[:, c].unflatten(1, (-1, hd)) for c in cuts)
    o, lse = rq.packed_attention(ctx, q, k, v, cu)
    oq, so = rq.quantize_rows_i8(ctx, o.flatten(1))
    h = rq.linear_i8(ctx, oq, so, *wo)
    close_linear(h, oq, so, *wo, "output projection")
    logits = (h.float() @ head.float().t()).to(BF16)
    s = rq.token_logprobs(ctx, logits, targets, top=5, entropy=True)

    # the mean negative log probability, and its gradient
    w = -torch.ones(T, device="cuda") / (T - 1)
    dlogits = rq.token_logprobs_backward(ctx, logits, targets, s, dlogp=w)
    dh = dlogits.float() @ head.float()
    do = ((dh.to(BF16).float() @ (wo[0].float() * wo[1][:, None]))).to(BF16).unflatten(1, (H, hd))
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = (dqkv[:, c].unflatten(1, (-1, hd)) for c in cuts)
    rq.packed_attention_backward(ctx, q, k, v, cu, o, lse, do, dq=dq, dk=dk, dv=dv)

    # Stage 0 on the gradients at the query projection's output
    G_out = dq.flatten(1).contiguous()
    F_acc = torch.zeros((H * hd, H * hd), dtype=F64, device="cuda")
    rq.fisher_accum(ctx, G_out, F_acc)
    sal = rq.saliency(ctx, G_out, 2)

    # against the definitions
    att = ref.attention(q, k, v, cu, do)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.close(got, *att[name], name)
    want = ref.logprobs(logits, targets, 5)
    tol = ref.lse_bound(V, want["lse"])
    ref.close(s.lse, want["lse"], tol, "lse")
    ref.close(s.logp, want["logp"], tol + 4 * ref.F * want["logp"].abs(), "logp")
    assert float(s.logp[0]) == 0 and torch.equal(s.top_ids, want["top_ids"])
    grad, bound = ref.logprobs_gradient(logits, targets, None, w)
    ref.close(dlogits, grad, bound + ref.BF * (grad.abs() + bound) + ref.TINY, "dlogits")
    assert (dlogits[0] == 0).all()
    gd = G_out.to(F64)
    ref.close(F_acc, gd.t() @ gd, 2 * T * ref.F * (gd.abs().t() @ gd.abs()) + ref.TINY, "fisher")
    # squares and sums in float64, stored in float32
    halves = gd.square().unflatten(1, (2, -1)).sum(2).t()
    ref.close(sal, halves, 2 * ref.F * halves + 2.0 ** -149, "saliency")


def test_one_token_after_another(rq, ctx):
    """A batch of one token through a projection and its scores: the rows of the prompt's."""
    g = torch.Generator(device="cuda").manual_seed(5)
    T, n, m, V = 70, 512, 384, 20000
    w, sw = rq.quantize_rows_i8(ctx, torch.randn((m, n), generator=g, device="cuda"))
    x = torch.randn((T, n), generator=g, device="cuda").to(BF16)
    whole = rq.linear_i8(ctx, *rq.quantize_rows_i8(ctx, x), w, sw)
    logits = torch.randn((T, V), generator=g, device="cuda").to(BF16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    scores = rq.token_logprobs(ctx, logits, y, top=3, entropy=True)
    for t in (0, 33, 69):
        one = rq.linear_i8(ctx, *rq.quantize_rows_i8(ctx, x[t:t + 1]), w, sw)
        assert torch.equal(one[0], whole[t])
        s = rq.token_logprobs(ctx, logits[t:t + 1], y[t:t + 1], top=3, entropy=True)
        assert torch.equal(s.top_ids[0], scores.top_ids[t])
        tol = ref.lse_bound(V, s.lse.double())
        assert (s.lse - scores.lse[t]).abs() <= 2 * tol and (s.logp - scores.logp[t]).abs() <= 2 * tol + 1e-6


def test_another_stream(rq):
    """A context on a stream that is not current: its outputs are that stream's, its inputs' memory is not given
    out again before it is through with them."""
    side = torch.cuda.Stream()
    c = rq.Context(side)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((300, 512), generator=g, device="cuda").to(BF16)
    w, sw = torch.randint(-127, 128, (256, 512), generator=g, device="cuda").to(torch.int8), torch.rand(256, generator=g, device="cuda")
    logits = torch.randn((64, 30000), generator=g, device="cuda")
    q = torch.randn((300, 4, 64), generator=g, device="cuda").to(BF16)
    cu = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    here = rq.Context()
    want = (rq.linear_i8(here, *rq.quantize_rows_i8(here, x), w, sw), rq.token_logprobs(here, logits, top=2).lse,
            *rq.packed_attention(here, q, q, q, cu))
    copies = [t.clone() for t in (x, logits, q)]
    torch.cuda.synchronize()
    got = (rq.linear_i8(c, *rq.quantize_rows_i8(c, copies[0]), w, sw), rq.token_logprobs(c, copies[1], top=2).lse,
           *rq.packed_attention(c, copies[2], copies[2], copies[2], cu))
    del copies
    junk = [torch.full((300, 512), 9.0, device="cuda") for _ in range(20)]  # would land in the freed memory
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    del junk
    c.close()
    here.close()


def test_two_contexts_at_once(rq):
    """Two contexts on streams of their own, the same inputs and no wait between their calls."""
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((500, 1000), generator=g, device="cuda").to(BF16)
    w, sw = torch.randint(-127, 128, (900, 1000), generator=g, device="cuda").to(torch.int8), torch.rand(900, generator=g, device="cuda")
    logits = torch.randn((3, 600000), generator=g, device="cuda")  # rows in stretches
    y = torch.tensor([5, 599999, -1], device="cuda")
    q = torch.randn((700, 4, 96), generator=g, device="cuda").to(BF16)
    cu = torch.tensor([0, 100, 700], dtype=torch.int32, device="cuda")
    ones = torch.ones(3, device="cuda")

    def run(c):
        s = rq.token_logprobs(c, logits, y, top=7, entropy=True)
        o, lse = rq.packed_attention(c, q, q, q, cu)
        return [rq.linear_i8(c, *rq.quantize_rows_i8(c, x), w, sw), s.lse, s.entropy, s.top_ids,
                rq.token_logprobs_backward(c, logits, y, s, dlogp=ones, dentropy=ones), o, lse,
                *rq.packed_attention_backward(c, q, q, q, cu, o, lse, q)]

    torch.cuda.synchronize()
    contexts = [rq.Context(torch.cuda.Stream()) for _ in range(2)]
    want = run(contexts[0])
    torch.cuda.synchronize()
    got = [[run(c) for c in contexts] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for outs in pair:
            for a, b in zip(outs, want):
                assert torch.equal(a, b)
    for c in contexts:
        c.close()
