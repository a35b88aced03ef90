"""Refusals and launch limits of the scoring, attention and 8-bit product calls on the HIP runtime of
fake_hip.cpp, which computes nothing.  Run by tests/test_operator_calls.py as a program of its own:
operator_calls.py <fake runtime> <library> <check>."""
import ctypes
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from host_logic import I64, VP, Library, buf  # noqa: E402

I32 = ctypes.c_int32


class LogprobsDesc(ctypes.Structure):
    _fields_ = [("T", I64), ("V", I64), ("ld", I64), ("logits", VP), ("targets", VP), ("dtype", I32), ("top", I32)]


class AttentionDesc(ctypes.Structure):
    _fields_ = [("T", I64), ("n_seqs", I64), ("n_heads", I32), ("n_kv", I32), ("head_dim", I32),
                ("scale", ctypes.c_float), ("cu_seqlens", VP), ("q", VP), ("k", VP), ("v", VP), ("ldq", I64),
                ("ldk", I64), ("ldv", I64)]


def at(p, off):
    return VP(p.value + off)


def refused(L, code, word, name, *args):
    L.fake.fake_reset()
    rc, msg = L.call(name, *args)
    assert rc == code and word in msg, (name, args, rc, msg)
    assert L.fake.fake_launches(b"") == 0


def launched(L, name, *args):
    L.fake.fake_reset()
    L.ok(name, *args)
    assert L.fake.fake_mallocs() == 0 and L.fake.fake_copies() == 0
    return L.fake.fake_launches(b"")


def work_for(L, d):
    n = ctypes.c_size_t()
    L.ok("realq_token_logprobs_workspace", ctypes.byref(d), ctypes.byref(n))
    return n.value


def logprobs(L):
    def desc(**kw):
        d = LogprobsDesc(7, 1000, 1000, buf(1), buf(2), 0, 5)
        for k, v in kw.items():
            setattr(d, k, v)
        return d

    def args(d, logp=buf(3), lse=buf(4), ent=buf(5), ids=buf(6), tl=buf(7), work=buf(8), size=1 << 40):
        return ctypes.byref(d), logp, lse, ent, ids, tl, work, ctypes.c_size_t(size)
    f = "realq_token_logprobs"
    assert launched(L, f, *args(desc())) >= 1
    assert launched(L, f, *args(desc(T=0))) == 0
    assert launched(L, f, *args(desc(targets=None, top=0), logp=None, ent=None, ids=None, tl=None)) >= 1
    refused(L, -1, "NULL", f, None, *args(desc())[1:])
    for kw, code in ((dict(dtype=2), -1), (dict(T=-1), -2), (dict(V=0), -2), (dict(V=1 << 31, ld=1 << 31), -2),
                     (dict(ld=999), -2), (dict(top=-1), -2), (dict(top=65), -2), (dict(V=3, ld=3, top=4), -2),
                     (dict(logits=None), -1), (dict(logits=at(buf(1), 1)), -1), (dict(targets=at(buf(2), 4)), -1),
                     (dict(targets=None), -1)):
        refused(L, code, "token_logprobs", f, *args(desc(**kw)))
    for kw in (dict(lse=None), dict(ids=None), dict(tl=None), dict(lse=at(buf(4), 2)), dict(ids=at(buf(6), 4)),
               dict(work=at(buf(8), 8))):
        refused(L, -1, "token_logprobs", f, *args(desc(), **kw))
    assert work_for(L, desc(T=0)) == 0
    few = desc(T=1, V=2000000, ld=2000000)
    need = work_for(L, few)
    assert need > 0
    refused(L, -1, str(need), f, *args(few, size=need - 1))
    refused(L, -1, str(need), f, *args(few, work=None))
    assert launched(L, f, *args(few, size=need)) >= 1
    # many rows: launch limits (a grid dimension times its block below 2^32)
    for T, V in ((1 << 24, 8), (1 << 33, 4), (1, (1 << 31) - 1), (40, (1 << 31) - 1)):
        d = desc(T=T, V=V, ld=V, top=2)
        work_for(L, d)
        assert launched(L, f, *args(d)) >= 1, (T, V)
    refused(L, -1, "workspace", "realq_token_logprobs_workspace", ctypes.byref(desc()), None)

    g = "realq_token_logprobs_backward"

    def back(d, lse=buf(4), ent=buf(5), ids=buf(6), dl=buf(9), de=buf(10), dt=buf(11), out=buf(12), ldd=None):
        return ctypes.byref(d), lse, ent, ids, dl, de, dt, out, d.ld if ldd is None else ldd
    assert launched(L, g, *back(desc())) >= 1
    assert launched(L, g, *back(desc(), out=buf(1))) >= 1
    assert launched(L, g, *back(desc(T=0))) == 0
    assert launched(L, g, *back(desc(targets=None, top=0), ent=None, ids=None, dl=None, de=None, dt=None)) >= 1
    for kw, code in ((dict(lse=None), -1), (dict(out=None), -1), (dict(ent=None), -1), (dict(ids=None), -1),
                     (dict(ldd=999), -2), (dict(out=buf(1), ldd=1001), -2), (dict(out=at(buf(12), 1)), -1)):
        refused(L, code, "token_logprobs_backward", g, *back(desc(), **kw))
    refused(L, -1, "targets", g, *back(desc(targets=None)))
    refused(L, -1, "dtop", g, *back(desc(top=0)))
    for T, V in ((1 << 24, 8), (1 << 33, 4), (3, (1 << 31) - 1)):
        assert launched(L, g, *back(desc(T=T, V=V, ld=V, top=2))) >= 1, (T, V)


def attention(L):
    def desc(**kw):
        d = AttentionDesc(100, 3, 8, 2, 64, 0.0, buf(1), buf(2), buf(3), buf(4), 512, 128, 128)
        for k, v in kw.items():
            setattr(d, k, v)
        return d
    f, g = "realq_packed_attention", "realq_packed_attention_backward"

    def fwd(d, o=buf(5), ldo=512, lse=buf(6)):
        return ctypes.byref(d), o, ldo, lse

    def bwd(d, **kw):
        a = dict(O=buf(5), ldo=512, lse=buf(6), dO=buf(7), lddo=512, work=buf(8), size=1 << 40, dQ=buf(9), lddq=512, dK=buf(10),
                 lddk=128, dV=buf(11), lddv=128)
        a.update(kw)
        a["size"] = ctypes.c_size_t(a["size"])
        return (ctypes.byref(d), *a.values())
    assert launched(L, f, *fwd(desc())) >= 1 and launched(L, f, *fwd(desc(), lse=None)) >= 1
    assert launched(L, g, *bwd(desc())) >= 1
    for kw in (dict(T=0), dict(n_seqs=0)):
        assert launched(L, f, *fwd(desc(**kw))) == 0 and launched(L, g, *bwd(desc(**kw))) == 0
    for kw, code in ((dict(T=-1), -2), (dict(T=1 << 31), -2), (dict(n_seqs=-1), -2), (dict(n_seqs=1 << 23), -2),
                     (dict(n_heads=0), -2), (dict(n_kv=0), -2), (dict(n_kv=3), -2), (dict(n_heads=65536), -2),
                     (dict(head_dim=0), -2), (dict(head_dim=12), -2), (dict(head_dim=264), -2),
                     (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
                     (dict(cu_seqlens=None), -1), (dict(cu_seqlens=at(buf(1), 2)), -1), (dict(q=None), -1),
                     (dict(k=None), -1), (dict(v=None), -1), (dict(q=at(buf(2), 8)), -1), (dict(ldq=504), -2),
                     (dict(ldk=124), -2), (dict(ldv=132), -2)):
        refused(L, code, "packed_attention", f, *fwd(desc(**kw)))
        refused(L, code, "packed_attention_backward", g, *bwd(desc(**kw)))
    for kw, code in ((dict(o=None), -1), (dict(o=at(buf(5), 8)), -1), (dict(ldo=504), -2), (dict(lse=at(buf(6), 2)), -1)):
        refused(L, code, "packed_attention", f, *fwd(desc(), **kw))
    for kw, code in ((dict(O=None), -1), (dict(lse=None), -1), (dict(work=None), -1), (dict(work=at(buf(8), 8)), -1), (dict(size=10), -1), (dict(dO=None), -1),
                     (dict(dQ=None), -1), (dict(dK=None), -1), (dict(dV=None), -1), (dict(lddq=508), -2),
                     (dict(lddk=120), -2), (dict(dV=at(buf(11), 2)), -1)):
        refused(L, code, "packed_attention_backward", g, *bwd(desc(), **kw))
    refused(L, -2, "2^23", f, *fwd(desc(T=1 << 28, n_seqs=1 << 10)))
    refused(L, -2, "2^24", f, *fwd(desc(ldq=(1 << 24) + 8)))
    h = "realq_packed_attention_workspace"
    n = ctypes.c_size_t()
    for kw in (dict(), dict(T=1), dict(T=4097, n_seqs=1), dict(T=100000), dict(n_heads=2, n_kv=1)):
        d = desc(**kw)
        L.ok(h, ctypes.byref(d), ctypes.byref(n))
        assert n.value >= 4 * d.T * d.n_heads
        assert launched(L, g, *bwd(d, size=n.value)) >= 1
        refused(L, -1, str(n.value), g, *bwd(d, size=n.value - 1))
    L.ok(h, ctypes.byref(desc(T=0, q=None, cu_seqlens=None)), ctypes.byref(n))
    assert n.value == 0
    refused(L, -1, "NULL", h, ctypes.byref(desc()), None)
    refused(L, -2, "head_dim", h, ctypes.byref(desc(head_dim=7)), ctypes.byref(n))
    for hd in (8, 64, 128, 256):
        for G in (2, 8):
            big = desc(T=(1 << 27) - 256, n_seqs=1, n_kv=G, head_dim=hd, ldq=8 * hd, ldk=G * hd, ldv=G * hd)
            assert launched(L, f, *fwd(big, ldo=8 * hd)) >= 1
            assert launched(L, g, *bwd(big, ldo=8 * hd, lddo=8 * hd, lddq=8 * hd, lddk=G * hd, lddv=G * hd)) >= 1
    refused(L, -2, "2^23", f, *fwd(desc(T=(1 << 27) - 128, n_seqs=1)))


def linear(L):
    q, f = "realq_quantize_rows_i8", "realq_linear_i8"

    def rows(X=buf(1), dtype=0, T=5, n=100, ldx=100, Q=buf(2), ldq=112, s=buf(3)):
        return X, I32(dtype), T, n, ldx, Q, ldq, s
    assert launched(L, q, *rows()) >= 1 and launched(L, q, *rows(T=0)) == 0
    for kw, code in ((dict(dtype=3), -1), (dict(T=-1), -2), (dict(n=0), -2), (dict(ldx=99), -2), (dict(ldq=99), -2),
                     (dict(X=None), -1), (dict(Q=None), -1), (dict(s=None), -1), (dict(X=at(buf(1), 1)), -1),
                     (dict(dtype=1, X=at(buf(1), 2)), -1)):
        refused(L, code, "quantize_rows_i8", q, *rows(**kw))
    for T, n in ((1 << 33, 4), (1, (1 << 31) - 1)):
        assert launched(L, q, *rows(T=T, n=n, ldx=n, ldq=n)) >= 1

    def lin(X=buf(1), ldx=112, sx=buf(2), W=buf(3), ldw=112, sw=buf(4), b=buf(5), T=5, n=100, m=70, Y=buf(6), dtype=0, ldy=70):
        return X, ldx, sx, W, ldw, sw, b, T, n, m, Y, I32(dtype), ldy
    assert launched(L, f, *lin()) >= 1 and launched(L, f, *lin(T=0)) == 0 and launched(L, f, *lin(b=None)) >= 1
    for kw, code in ((dict(dtype=2), -1), (dict(T=-1), -2), (dict(n=0), -2), (dict(n=131072, ldx=1 << 20, ldw=1 << 20), -2),
                     (dict(m=0), -2), (dict(ldx=99), -2), (dict(ldw=99), -2), (dict(ldy=69), -2), (dict(X=None), -1),
                     (dict(sx=None), -1), (dict(W=None), -1), (dict(sw=None), -1), (dict(Y=None), -1),
                     (dict(Y=at(buf(6), 1)), -1), (dict(b=at(buf(5), 2)), -1),
                     (dict(T=1 << 30, m=1 << 30, ldy=1 << 30), -2)):
        refused(L, code, "linear_i8", f, *lin(**kw))
    for T, m in ((1, 1 << 29), (64, 1 << 29), (1 << 29, 1), (1 << 20, 1 << 14)):
        assert launched(L, f, *lin(T=T, m=m, ldy=m)) >= 1, (T, m)


if __name__ == "__main__":
    L = Library(sys.argv[1], sys.argv[2])
    {"logprobs": logprobs, "attention": attention, "linear": linear}[sys.argv[3]](L)
    print("passed")
