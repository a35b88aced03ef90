"""Contexts and calls of the operators that the binding has to refuse or prepare itself, without a GPU."""
import contextlib
import types

import pytest
import torch

from paper_2609_00049_amd import realq as rq

B = torch.bfloat16


@pytest.fixture
def ctx(monkeypatch):
    """A context whose tensors are on the host and whose calls into the C ABI fail the test."""
    def called(*args):
        raise AssertionError("the C ABI was called")

    monkeypatch.setattr(rq, "_current", lambda i: 0)
    monkeypatch.setattr(rq, "_lib", types.SimpleNamespace(**{n: called for n in rq.EXPORTS}))
    return types.SimpleNamespace(h=None, device=torch.device("cpu"), raw_stream=0, check=called)


def heads():
    return torch.zeros((6, 4, 64), dtype=B), torch.zeros((6, 2, 64), dtype=B), torch.tensor([0, 6], dtype=torch.int32)


@pytest.mark.parametrize("scale", [1e-50, 1e-46, -1e-50])
def test_a_scale_that_is_no_float32_above_zero(ctx, scale):
    """It would arrive as 0, which stands for the default."""
    q, k, cu = heads()
    lse = torch.zeros((4, 6))
    with pytest.raises(ValueError, match="scale"):
        rq.packed_attention(ctx, q, k, k, cu, scale=scale)
    with pytest.raises(ValueError, match="scale"):
        rq.packed_attention_backward(ctx, q, k, k, cu, q, lse, q, scale=scale)


def test_a_context_is_created_on_its_streams_device(monkeypatch):
    """The C ABI binds a context to the device that is current, which need not be the stream's."""
    current, seen = [torch.device("cuda:0")], []

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d)
        yield
        current[0] = before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(rq, "_lib", types.SimpleNamespace(
        realq_ctx_create=lambda h, stream: seen.append(current[0]) or 0, realq_ctx_destroy=lambda h: None))
    for name in ("cuda:1", "cuda:0"):
        c = rq.Context(types.SimpleNamespace(device=torch.device(name), cuda_stream=5))
        assert seen[-1] == c.device == torch.device(name)
        c.close()
    assert current[0] == torch.device("cuda:0")


def test_gradients_are_not_lost_silently(ctx):
    """The calls record no graph: tensors that require grad are refused while torch records one, and taken under
    no_grad and in an autograd.Function (where the call reaches the C ABI)."""
    q, k, cu = heads()
    z, y, one = torch.zeros((4, 50)), torch.zeros(4, dtype=torch.int64), torch.ones(4)
    i8, s = torch.zeros((4, 16), dtype=torch.int8), rq.TokenLogprobs(one, one, None, None, None)
    lse = torch.zeros((4, 6))

    def grad(t):
        return t.clone().requires_grad_()

    calls = [lambda g: rq.token_logprobs(ctx, g(z), y),
             lambda g: rq.token_logprobs_backward(ctx, z, y, s, dlogp=g(one)),
             lambda g: rq.packed_attention(ctx, g(q), k, k, cu),
             lambda g: rq.packed_attention(ctx, q, k, g(k), cu),
             lambda g: rq.packed_attention_backward(ctx, q, k, k, cu, g(q), lse, q),
             lambda g: rq.quantize_rows_i8(ctx, g(z)),
             lambda g: rq.linear_i8(ctx, i8, one, i8, g(one))]

    class Function(torch.autograd.Function):
        @staticmethod
        def forward(c, t, call):
            call(lambda x: t)

    for call in calls:
        with pytest.raises(ValueError, match="requires grad"):
            call(grad)
        with pytest.raises(AssertionError, match="the C ABI was called"), torch.no_grad():
            call(grad)
    with pytest.raises(AssertionError, match="the C ABI was called"):
        Function.apply(grad(z), calls[0])
