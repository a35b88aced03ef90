"""Workspace queries of the operators on the HIP runtime of fake_hip.cpp.  Run by tests/test_operator_workspaces.py
as a program of its own: operator_workspaces.py <fake runtime> <library>."""
import ctypes
import sys

from operator_calls import Library, LogprobsDesc

if __name__ == "__main__":
    L = Library(sys.argv[1], sys.argv[2])
    name = "realq_token_logprobs_workspace"

    def query(**kw):
        d = LogprobsDesc(7, 1000, 1000, None, None, 0, 5)
        for k, v in kw.items():
            setattr(d, k, v)
        n = ctypes.c_size_t(77)
        return *L.call(name, ctypes.byref(d), ctypes.byref(n)), n.value

    assert query()[::2] == (0, 0) and query(T=0, ld=0)[::2] == (0, 0)
    rc, _, n = query(T=3, V=(1 << 31) - 1, dtype=1, top=64)
    assert rc == 0 and 0 < n < 1 << 20
    # sizes that the calls themselves refuse, some of which wrap a product of 64 bits
    for kw, code in ((dict(V=1 << 31), -2), (dict(V=1 << 62), -2), (dict(T=1 << 62, V=1 << 30), -2), (dict(top=65), -2),
                     (dict(V=3, top=4), -2), (dict(dtype=2), -1), (dict(T=-1), -1), (dict(V=0), -1), (dict(top=-1), -1)):
        rc, message, n = query(**kw)
        assert rc == code and "workspace" in message and n == 77, (kw, rc, message, n)
    print("passed")
