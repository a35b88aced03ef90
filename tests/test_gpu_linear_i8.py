"""Row quantization to 8 bits and the integer product, against exact arithmetic."""
import math

import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32, I8 = torch.bfloat16, torch.float32, torch.int8


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(rows, n, g, pad=0, offset=0):
    c = torch.randint(-127, 128, (rows, n + pad + offset), generator=g, device="cuda").to(I8)
    return c[:, offset:offset + n]


def check(rq, ctx, xq, sx, wq, sw, bias=None, dtype=BF16, out=None):
    y = rq.linear_i8(ctx, xq, sx, wq, sw, bias=bias, dtype=dtype, out=out)
    want, bound = ref.linear(xq, sx, wq, sw, bias)
    if y.dtype == BF16:
        bound = bound + ref.BF * (want.abs() + bound)
    ref.close(y, want, bound, "y")
    return y


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,n", [(1, 1), (1, 4096), (3, 15), (7, 1352), (2, 14336), (130, 257), (5, 33001), (9, 16), (3, 20001), (2, 32768)])
def test_codes_and_scales_are_those_of_exact_quotients(rq, ctx, T, n, dtype):
    x = (torch.randn((T, n), generator=gen(n), device="cuda") * torch.exp(torch.randn(n, generator=gen(1), device="cuda"))).to(dtype)
    q, s = rq.quantize_rows_i8(ctx, x)
    wq, ws = ref.quantize_rows(x)
    assert torch.equal(s, ws) and torch.equal(q.double(), wq)
    assert q.stride(0) % 16 == 0 or T == 1


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_quotients_at_a_half_zeros_tiny_and_bad_rows(rq, ctx, dtype):
    """Rows of multiples of half a step around scales whose quotients round, all zeros, subnormal rows, huge rows
    and rows with NaN or infinities."""
    h = torch.arange(-254, 255, device="cuda", dtype=torch.float64) / 2
    rows = [h * s for s in (1.0, 0.3, 1 / 3, 7e-5, 1e30, 2.0 ** 100 / 127 * 1.1, 2.0 ** -120, 2.0 ** -130, 2.0 ** -148)]
    rows += [torch.zeros_like(h), h * 0 + 2.0 ** -149, h * 1e-40, h * 2.6e36]
    x = torch.stack(rows).to(dtype)
    # values next to a half-step of the float32 scale
    s = (x.double().abs().amax(1) / 127).float().double()
    near = (h * s[:, None]).to(dtype)
    near = torch.where(near.abs() <= x.abs().amax(1, keepdim=True), near, x)
    for r in (x, torch.cat([x, near, torch.nextafter(near.float(), near.float() * 2).to(dtype)], 1)):
        q, s = rq.quantize_rows_i8(ctx, r)
        wq, ws = ref.quantize_rows(r)
        assert torch.equal(s, ws)
        assert torch.equal(q.double(), wq), (q.double() - wq).abs().max()
    bad = torch.randn((4, 40), device="cuda").to(dtype)
    bad[0, 3], bad[1, 39], bad[2, 0] = math.nan, math.inf, -math.inf
    q, s = rq.quantize_rows_i8(ctx, bad)
    assert torch.isnan(s[:3]).all() and torch.isfinite(s[3]) and (q[:3] == 0).all()
    y = rq.linear_i8(ctx, q, s, torch.ones((3, 40), dtype=I8, device="cuda"), torch.ones(3, device="cuda"))
    assert torch.isnan(y[:3].float()).all() and torch.isfinite(y[3].float()).all()


@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 33, 64, 65, 128, 300])
@pytest.mark.parametrize("n,m", [(64, 64), (4096, 512), (1352, 1000), (17, 5), (1, 1), (2000, 77), (14336, 40), (80, 12300), (144, 6200)])
def test_products(rq, ctx, T, n, m):
    print(f"[gpu-case] linear_i8 {T}x{n}x{m}", flush=True)
    g = gen(T * 7 + n)
    pad = -n % 16
    xq, wq = codes(T, n, g, pad), codes(m, n, g, pad)
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    bias = torch.randn(m, generator=g, device="cuda") * 1000
    check(rq, ctx, xq, sx, wq, sw)
    check(rq, ctx, xq, sx, wq, sw, bias, F32)


@pytest.mark.parametrize("T,n,m", [(700, 1024, 900), (513, 4096, 1100), (2049, 192, 300), (1030, 2000, 520), (1280, 64, 4096)])
def test_large_products(rq, ctx, T, n, m):
    g = gen(T)
    xq, wq = codes(T, n, g, -n % 16), codes(m, n, g, -n % 16)
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    bias = torch.randn(m, generator=g, device="cuda") * 1000
    check(rq, ctx, xq, sx, wq, sw, bias)
    check(rq, ctx, xq, sx, wq, sw, None, F32)


@pytest.mark.parametrize("T,m", [(66, 1000), (90, 4000), (250, 3900), (300, 4000), (520, 5500), (3700, 2050)])
@pytest.mark.parametrize("n", [1, 13, 50, 64, 127, 128, 200, 450, 1090])
def test_numbers_of_tiles_and_slices(rq, ctx, T, m, n):
    """From a few tiles of outputs to many, over columns of less than a slice, one to seventeen and a rest."""
    g = gen(n + m)
    xq, wq = codes(T, n, g, -n % 16), codes(m, n, g, -n % 16)
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    check(rq, ctx, xq, sx, wq, sw, torch.randn(m, generator=g, device="cuda"))
    check(rq, ctx, xq, sx, wq, sw, None, F32)


@pytest.mark.parametrize("T", [3, 40, 400])
@pytest.mark.parametrize("off_x,off_w,pad", [(1, 0, 0), (0, 3, 5), (16, 16, 16), (8, 4, 4), (0, 0, 1)])
def test_strides_and_alignment(rq, ctx, T, off_x, off_w, pad):
    n, m = 333, 150
    g = gen(5)
    xq, wq = codes(T, n, g, pad, off_x), codes(m, n, g, pad, off_w)
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    for dtype in (BF16, F32):
        buf = torch.full((T, m + 9), 4.0, dtype=dtype, device="cuda")
        check(rq, ctx, xq, sx, wq, sw, out=buf[:, 4:4 + m])
        assert (buf[:, :4] == 4).all() and (buf[:, 4 + m:] == 4).all()


@pytest.mark.parametrize("T", [1, 20, 200])
def test_largest_sums(rq, ctx, T):
    """131071 columns of -128 times -128: 2147467264 of 2147483647; odd sums above 2^24 convert once."""
    n = 131071
    xq = torch.full((T, n + 1), -128, dtype=I8, device="cuda")[:, :n]
    wq = torch.full((3, n + 1), -128, dtype=I8, device="cuda")[:, :n]
    wq[1] = 127
    wq[2, ::2] = 1
    one = torch.ones(T, device="cuda"), torch.ones(3, device="cuda")
    check(rq, ctx, xq, one[0], wq, one[1], dtype=F32)


@pytest.mark.parametrize("T", [3, 70])
def test_weights_past_32_bits(rq, ctx, T):
    """Weights and outputs whose last rows lie past 2^31 elements; those rows are checked."""
    n, m = 65536, 33000
    g = gen(T)
    wq = torch.empty((m, n), dtype=I8, device="cuda").random_(-127, 128, generator=g)
    xq = codes(T, n, g)
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(m, generator=g, device="cuda")
    out = torch.empty((T, 1 << 30), dtype=BF16, device="cuda")[:, :m] if T == 3 else None
    y = rq.linear_i8(ctx, xq, sx, wq, sw, out=out)
    want, bound = ref.linear(xq, sx, wq[-100:], sw[-100:])
    ref.close(y[:, -100:], want, bound + ref.BF * (want.abs() + bound), "last rows")
    want, bound = ref.linear(xq, sx, wq[:100], sw[:100])
    ref.close(y[:, :100], want, bound + ref.BF * (want.abs() + bound), "first rows")


def test_a_per_row_quantized_module(rq, ctx):
    """The codes, zeros and scales of a module quantized per row (symmetric, the paper's main setting) as integer
    weights: the product is that of the dequantized weights with the dequantized tokens."""
    g = gen(3)
    m, n, T = 96, 256, 512
    W0 = torch.randn((m, n), generator=g, device="cuda").to(BF16).float() * 0.05
    X = torch.randn((T, n), generator=g, device="cuda").to(BF16)
    r = rq.quantize_layer(ctx, W0, X, X, qp=rq.qparams(bits=4, group=0, sym=True))
    w8 = (r.codes.to(torch.int16) - r.zeros.to(torch.int16)).to(I8)
    xq, sx = rq.quantize_rows_i8(ctx, X)
    y = check(rq, ctx, xq, sx, w8, r.scales[:, 0].contiguous(), dtype=F32)
    want = (xq.double() * sx.double()[:, None]) @ r.W_hat.double().t()
    ref.close(y, want, 1e-5 * ((xq.double() * sx.double()[:, None]).abs() @ r.W_hat.double().abs().t()), "module")


def test_no_tokens(rq, ctx):
    q, s = rq.quantize_rows_i8(ctx, torch.empty((0, 20), device="cuda"))
    y = rq.linear_i8(ctx, q, s, torch.ones((3, 20), dtype=I8, device="cuda"), torch.ones(3, device="cuda"))
    assert y.shape == (0, 3)


@pytest.mark.parametrize("T", [1, 30, 500])
def test_captured_and_replayed(rq, T):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = rq.Context(stream)
        g = gen(T)
        x = torch.randn((T, 2064), generator=g, device="cuda").to(BF16)
        w, sw = codes(272, 2064, g), torch.rand(272, generator=g, device="cuda")

        def run():
            return rq.linear_i8(c, *rq.quantize_rows_i8(c, x), w, sw)
        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = run()
        for i in range(4):
            x.normal_()
            graph.replay()
            stream.synchronize()
            torch.randn(1 << 16, device="cuda").sum().item()
            assert torch.equal(out, run()), i
        stream.synchronize()
        c.close()
