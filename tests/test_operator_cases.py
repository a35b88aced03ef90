"""The timed cases of perf/operators.py use a context of the stream that is current."""
import types

from perf import operators


def test_a_context_per_stream(monkeypatch):
    from paper_2609_00049_amd import realq
    made = []

    def stream(device, raw):
        return types.SimpleNamespace(device_index=device, cuda_stream=raw)

    current = [stream(0, 0)]
    monkeypatch.setattr(operators, "_KEPT", {})
    # (a build of torch without GPU support lacks these two)
    monkeypatch.setattr(operators.torch._C, "_cuda_getDevice", lambda: current[0].device_index, raising=False)
    monkeypatch.setattr(operators.torch._C, "_cuda_getCurrentRawStream", lambda device: current[0].cuda_stream,
                        raising=False)
    monkeypatch.setattr(operators.torch.cuda, "current_stream", lambda: current[0])
    monkeypatch.setattr(realq, "Context", lambda s: made.append(s) or s)
    got = []
    for s in (stream(0, 0), stream(0, 7), stream(1, 0), stream(0, 0), stream(0, 7)):
        current[0] = s
        binding, ctx = operators._lib()
        assert binding is realq and (ctx.device_index, ctx.cuda_stream) == (s.device_index, s.cuda_stream)
        got.append(ctx)
    assert len(made) == 3 and got[3] is got[0] and got[4] is got[1]
