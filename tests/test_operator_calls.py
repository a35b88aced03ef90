"""Refusals and launch limits of the scoring, attention and 8-bit product calls, without a GPU: the C ABI on a
runtime that only books launches, the binding on host tensors."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = os.path.join(ROOT, "tests", "host")
LIB = os.path.join(ROOT, "paper_2609_00049_amd", "librealq.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    so = tmp_path_factory.mktemp("fake_hip") / "libfake_hip.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror",
                    os.path.join(HOST, "fake_hip.cpp"), "-o", str(so)], check=True, capture_output=True, text=True)
    return str(so)


@pytest.mark.parametrize("check", ["logprobs", "attention", "linear"])
def test_calls_on_a_runtime_that_only_books(fake, check):
    res = subprocess.run([sys.executable, os.path.join(HOST, "operator_calls.py"), fake, LIB, check],
                         capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "passed" in res.stdout, res.stdout + res.stderr


def test_null_contexts():
    from paper_2609_00049_amd import realq
    lib = realq.lib()
    z = ctypes.c_void_p()
    assert lib.realq_token_logprobs_workspace(None, None, None) == -1
    assert lib.realq_token_logprobs(None, None, z, z, z, z, z, z, 0) == -1
    assert lib.realq_token_logprobs_backward(None, None, z, z, z, z, z, z, z, 0) == -1
    assert lib.realq_packed_attention(None, None, z, 0, z) == -1
    assert lib.realq_packed_attention_workspace(None, None, None) == -1
    assert lib.realq_packed_attention_backward(None, None, z, 0, z, z, 0, z, 0, z, 0, z, 0, z, 0) == -1
    assert lib.realq_quantize_rows_i8(None, z, 0, 0, 0, 0, z, 0, z) == -1
    assert lib.realq_linear_i8(None, z, 0, z, z, 0, z, z, 0, 0, 0, z, 0, 0) == -1


def test_binding_structs_match_the_c_layout(tmp_path):
    from paper_2609_00049_amd import realq
    structs = {"realq_logprobs_desc": realq.LogprobsDesc, "realq_attention_desc": realq.AttentionDesc}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "realq.h"', 'int main(void) {']
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ['return 0;', '}']) + "\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-Wall", "-Werror", f"-I{ROOT}/include", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out if x.strip()}
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py)
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


def test_binding_refuses_before_the_call(monkeypatch):
    import torch
    from paper_2609_00049_amd import realq as rq

    class NoCall:
        h = None
        device = torch.device("cuda:0")
        raw_stream = 0

        def check(self, rc):
            raise AssertionError("the C ABI was called")

    monkeypatch.setattr(rq, "_current", lambda i: 0)
    ctx = NoCall()
    z, y = torch.zeros((4, 50)), torch.zeros(4, dtype=torch.int64)
    s = rq.TokenLogprobs(torch.zeros(4), torch.zeros(4), None, None, None)
    B = torch.bfloat16
    q, k, cu = torch.zeros((6, 4, 64), dtype=B), torch.zeros((6, 2, 64), dtype=B), torch.zeros(2, dtype=torch.int32)
    i8 = torch.zeros((4, 16), dtype=torch.int8)
    one = torch.ones(4)
    calls = [
        lambda: rq.token_logprobs(ctx, z, y),                                   # on the host
        lambda: rq.token_logprobs(ctx, z.half(), y),
        lambda: rq.token_logprobs(ctx, z[0], y),
        lambda: rq.token_logprobs(ctx, z, y.int()),
        lambda: rq.token_logprobs(ctx, z, y[:3]),
        lambda: rq.token_logprobs(ctx, z, y, top=51),
        lambda: rq.token_logprobs(ctx, z, y, top=-1),
        lambda: rq.token_logprobs(ctx, z.t().contiguous().t(), y),
        lambda: rq.token_logprobs_backward(ctx, z, None, s, dlogp=one),
        lambda: rq.token_logprobs_backward(ctx, z, y, s, dentropy=one),
        lambda: rq.token_logprobs_backward(ctx, z, y, s, dtop=z),
        lambda: rq.packed_attention(ctx, q, k, k, cu),                          # on the host
        lambda: rq.packed_attention(ctx, q.float(), k, k, cu),
        lambda: rq.packed_attention(ctx, q, k[:5], k, cu),
        lambda: rq.packed_attention(ctx, q, k, k[:, :1], cu),
        lambda: rq.packed_attention(ctx, q, k, k, cu.long()),
        lambda: rq.packed_attention(ctx, q, k, k, cu[:0]),
        lambda: rq.packed_attention(ctx, q.transpose(0, 1).contiguous().transpose(0, 1), k, k, cu),
        lambda: rq.packed_attention(ctx, q[:1].expand(6, 4, 64), k, k, cu),
        lambda: rq.quantize_rows_i8(ctx, z),                                    # on the host
        lambda: rq.quantize_rows_i8(ctx, z.double()),
        lambda: rq.quantize_rows_i8(ctx, z[0]),
        lambda: rq.linear_i8(ctx, i8, one, i8[:, :8], one),
        lambda: rq.linear_i8(ctx, i8.float(), one, i8, one),
        lambda: rq.linear_i8(ctx, i8, one, i8, one),                            # on the host
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError, match="scale"):
            rq.packed_attention(ctx, q, k, k, cu, scale=scale)
