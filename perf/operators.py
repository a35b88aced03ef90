"""Timed cases of the operators a quantized model is scored and differentiated with: log probabilities of
given tokens, causal attention over packed prompts, and the 8-bit integer product of quantized modules.

`run` computes a case with elementary torch operations in 32 bits, or, where `own` is set, through the
library's binding.  A program keeps one Context per stream and makes its outputs per call.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64

_KEPT = {}


def _lib():
    """The binding and the Context of the current stream (only where `own` is set)."""
    device = torch._C._cuda_getDevice()
    key = device, torch._C._cuda_getCurrentRawStream(device)  # without making a Stream object
    if key not in _KEPT:
        from paper_2609_00049_amd import realq
        _KEPT[key] = realq, realq.Context(torch.cuda.current_stream())
    return _KEPT[key]


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one token being generated: its 20 likeliest alternatives for a client, latency bound
        _logprobs("logprobs_decode", 1, 128256, "bf16", 20, False),
        # one calibration sample scored after quantization: perplexity, entropy and 5 alternatives a token
        _logprobs("logprobs_prompt", 2047, 151936, "bf16", 5, False),
        # float32 logits of an odd vocabulary over an odd batch, with the gradient Stage 0 starts from
        _logprobs("logprobs_train_odd", 777, 32003, "f32", 0, True),
        # two samples of 2048 tokens: scores and the gradient at the logits, alternatives distilled
        _logprobs("logprobs_train", 4096, 128256, "bf16", 8, True),
        # three short prompts in one batch, one of a single token: latency bound
        _attention("attention_short", "1,17,110", 16, 8, 64, False),
        # four calibration samples of 2048 tokens through the attention of the 8B-class decoder block
        _attention("attention_prompt", "2048,2048,2048,2048", 32, 8, 128, False),
        # a packed batch of unequal samples, one of them empty: forward and backward of Stage 0
        _attention("attention_train_ragged", "1500,3,0,2047,1,333,212", 16, 8, 128, True),
        # one long sample, forward and backward
        _attention("attention_train_long", "8192", 32, 8, 128, True),
        # one token through the gate projection of the 8B-class model: the weights are read once
        _linear("linear_decode", 1, 4096, 14336, "bf16", False),
        # a small batch of tokens through the down projection
        _linear("linear_few", 24, 14336, 4096, "bf16", False),
        # odd tokens, columns and rows, float32 output with a bias
        _linear("linear_ragged", 1999, 1352, 1000, "f32", True),
        # eight samples of 2048 tokens through the gate projection
        _linear("linear_prompt", 16384, 4096, 14336, "bf16", False),
    ]


def _logprobs(name, T, V, dtype, top, train):
    return dict(name=name, kind="logprobs", T=T, V=V, dtype=dtype, top=top, train=train)


def _attention(name, lens, heads, kv, hd, train):
    return dict(name=name, kind="attention", lens=lens, heads=heads, kv=kv, hd=hd, train=train)


def _linear(name, T, n, m, out, bias):
    return dict(name=name, kind="linear", T=T, n=n, m=m, out=out, bias=bias)


def _log(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprobs", "attention", "linear"])
    if kind == "logprobs":
        V = _log(rng, 1000, 160000)
        T = _log(rng, 1, min(4096, max(1, 262144000 // V)))
        c = _logprobs("", T, V, rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 1, 5, 8, 20]),
                      rng.random() < 0.5)
    elif kind == "attention":
        hd = rng.choice([64, 128, 128, 96])
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4])
        T = _log(rng, 1, 8192)
        cuts = sorted(rng.randint(0, T) for _ in range(rng.randint(0, 6)))
        lens = [b - a for a, b in zip([0] + cuts, cuts + [T])]
        c = _attention("", ",".join(str(x) for x in lens), heads, kv, hd, rng.random() < 0.5)
    else:
        T = _log(rng, 1, 16384)
        n = _log(rng, 64, 14336)
        m = _log(rng, 64, min(14336, max(64, 16384 * 4096 * 14336 // (T * n))))
        c = _linear("", T, n, m, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.3)
    del c["name"]
    return c


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def work(case):
    if case["kind"] == "logprobs":
        T, V = case["T"], case["V"]
        es = 2 if case["dtype"] == "bf16" else 4
        b = T * V * es + T * (8 + 3 * 4 + case["top"] * 12)
        if case["train"]:
            b += T * V * es + T * (2 + case["top"]) * 4
        return {"bytes": b, "flops": T * V * (6 if not case["train"] else 12)}
    if case["kind"] == "attention":
        H, G, hd = case["heads"], case["kv"], case["hd"]
        T = sum(_lens(case))
        pairs = sum(x * (x + 1) // 2 for x in _lens(case))
        b = 2 * T * hd * (2 * H + 2 * G) + 4 * T * H
        f = 4 * hd * H * pairs
        if case["train"]:
            b += 2 * T * hd * (2 * H + 2 * G)
            f += 10 * hd * H * pairs
        return {"bytes": b, "flops": f}
    T, n, m = case["T"], case["n"], case["m"]
    b = T * n * 2 + m * n + m * 4 + T * m * (2 if case["out"] == "bf16" else 4) + (m * 4 if case["bias"] else 0)
    return {"bytes": b, "flops": 2 * T * n * m}


# ----------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=F32)

    if own:
        _lib()
    return {"case": case, "in": {"logprobs": _prepare_logprobs, "attention": _prepare_attention,
                                 "linear": _prepare_linear}[case["kind"]](case, g, randn)}


def _prepare_logprobs(case, g, randn):
    """Logits of a trained head: a wide body, the target raised in most rows; incoming gradients per token."""
    T, V = case["T"], case["V"]
    z = randn(T, V).mul_(2.5)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    up = 4 + 6 * torch.rand((T,), generator=g, device=DEV)
    z[torch.arange(T, device=DEV), y] += up
    d = {"z": z.to(BF16 if case["dtype"] == "bf16" else F32), "y": y}
    if case["train"]:
        d["dlogp"] = randn(T) / T
        d["dent"] = randn(T) * 0.1 / T
        if case["top"]:
            d["dtop"] = randn(T, case["top"]) * 0.2 / T
    return d


def _prepare_attention(case, g, randn):
    """Queries and keys as a projection gives them (scores of a few units), the first token of each
    sequence a sink; the heads of a token in one row."""
    lens = _lens(case)
    T, H, G, hd = sum(lens), case["heads"], case["kv"], case["hd"]
    cu = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
    q = randn(T, H, hd) * 1.3
    k = randn(T, G, hd)
    k[cu[:-1].long().clamp(max=T - 1)] *= 2.0
    d = {"q": q.to(BF16), "k": k.to(BF16), "v": randn(T, G, hd).to(BF16), "cu": cu, "most": max(lens)}
    if case["train"]:
        d["do"] = (randn(T, H, hd) / math.sqrt(T)).to(BF16)
    return d


def _prepare_linear(case, g, randn):
    """Activations with outlier channels; weights as the quantizer leaves them, signed 8-bit codes with a
    scale per output channel, laid out once with rows on 16 bytes."""
    T, n, m = case["T"], case["n"], case["m"]
    x = randn(T, n) * torch.exp(0.5 * randn(n))
    buf = torch.zeros((m, -(-n // 16) * 16), dtype=torch.int8, device=DEV)
    w = buf[:, :n]
    w.copy_((randn(m, n) * 32).round_().clamp_(-127, 127))
    sw = torch.exp(0.3 * randn(m)) * (1 / (32 * math.sqrt(n)))
    return {"x": x.to(BF16), "w": w, "sw": sw, "bias": randn(m) if case["bias"] else None}


# ----------------------------------------------------------------------------- one pass

def run(state):
    case, d = state["case"], state["in"]
    if own:
        rq, ctx = _lib()
        return {"logprobs": _own_logprobs, "attention": _own_attention, "linear": _own_linear}[case["kind"]](
            rq, ctx, case, d)
    return {"logprobs": _plain_logprobs, "attention": _plain_attention, "linear": _plain_linear}[case["kind"]](case, d)


def _own_logprobs(rq, ctx, case, d):
    s = rq.token_logprobs(ctx, d["z"], d["y"], top=case["top"], entropy=True)
    r = {"logp": s.logp, "lse": s.lse, "entropy": s.entropy}
    if case["top"]:
        r["top_ids"], r["top_logp"] = s.top_ids, s.top_logp
    if case["train"]:
        r["dlogits"] = rq.token_logprobs_backward(ctx, d["z"], d["y"], s, dlogp=d["dlogp"], dentropy=d["dent"],
                                                  dtop=d.get("dtop"))
    return r


def _own_attention(rq, ctx, case, d):
    o, lse = rq.packed_attention(ctx, d["q"], d["k"], d["v"], d["cu"])
    r = {"o": o, "lse": lse}
    if case["train"]:
        r["dq"], r["dk"], r["dv"] = rq.packed_attention_backward(ctx, d["q"], d["k"], d["v"], d["cu"], o, lse, d["do"])
    return r


def _own_linear(rq, ctx, case, d):
    xq, sx = rq.quantize_rows_i8(ctx, d["x"])
    return rq.linear_i8(ctx, xq, sx, d["w"], d["sw"], bias=d["bias"], dtype=BF16 if case["out"] == "bf16" else F32)


def _order(z):
    """A whole number for each value that has its order."""
    b = z.view(torch.int32).to(torch.int64)
    return torch.where(b < 0, -(b & 0x7FFFFFFF), b)


def _plain_logprobs(case, d):
    z, y = d["z"].to(F32), d["y"]
    T, V = z.shape
    top = case["top"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    S = e.sum(1, keepdim=True)
    lse = m + torch.log(S)
    logp = z - lse
    p = e / S
    ent = -(p * logp).sum(1, keepdim=True)
    r = {"logp": logp.gather(1, y[:, None])[:, 0], "lse": lse[:, 0], "entropy": ent[:, 0]}
    if top:
        key = _order(z) * V + (V - 1 - torch.arange(V, device=z.device))
        r["top_ids"] = V - 1 - key.topk(top, 1).values.remainder(V)
        r["top_logp"] = logp.gather(1, r["top_ids"])
    if case["train"]:
        total = d["dlogp"][:, None] + (d["dtop"].sum(1, keepdim=True) if top else 0.0)
        dz = -p * (total + d["dent"][:, None] * (logp + ent))
        dz.scatter_add_(1, y[:, None], d["dlogp"][:, None])
        if top:
            dz.scatter_add_(1, r["top_ids"], d["dtop"])
        r["dlogits"] = dz.to(d["z"].dtype)
    return r


def _plain_attention(case, d):
    """Every sequence padded to the longest: [sequence, head, position, channel]."""
    q, k, v, cu = d["q"], d["k"], d["v"], d["cu"].long()
    T, H, hd = q.shape
    G, L, dev = k.shape[1], d["most"], q.device
    scale = 1.0 / math.sqrt(hd)
    at = torch.arange(L, device=dev)
    rows = (cu[:-1, None] + at).clamp(max=T - 1)
    there = at < (cu[1:] - cu[:-1])[:, None]
    seq = torch.searchsorted(cu, torch.arange(T, device=dev), right=True) - 1
    pos = torch.arange(T, device=dev) - cu[seq]

    def padded(x):
        x = (x[rows].to(F32) * there[:, :, None, None]).permute(0, 2, 1, 3)
        return x.repeat_interleave(H // x.shape[1], 1) if x.shape[1] < H else x.contiguous()

    def packed(x):
        return x.permute(0, 2, 1, 3)[seq, pos]

    def shared(x):
        return x.reshape(x.shape[0], G, H // G, L, hd).sum(2)

    qp, kp, vp = padded(q), padded(k), padded(v)
    s = torch.matmul(qp, kp.transpose(2, 3)).mul_(scale)
    s.masked_fill_(at[:, None] < at, -math.inf)
    m = s.amax(3, keepdim=True)
    p = s.sub_(m).exp_()
    z = p.sum(3, keepdim=True)
    p.div_(z)
    o = torch.matmul(p, vp)
    r = {"o": packed(o).to(BF16), "lse": packed(m + torch.log(z))[:, :, 0].t().contiguous()}
    if case["train"]:
        do = padded(d["do"])
        dv = torch.matmul(p.transpose(2, 3), do)
        dp = torch.matmul(do, vp.transpose(2, 3))
        ds = dp.sub_((p * dp).sum(3, keepdim=True)).mul_(p)
        r["dq"] = packed(torch.matmul(ds, kp).mul_(scale)).to(BF16)
        r["dk"] = packed(shared(torch.matmul(ds.transpose(2, 3), qp).mul_(scale))).to(BF16)
        r["dv"] = packed(shared(dv)).to(BF16)
    return r


def _plain_linear(case, d):
    x = d["x"].to(F32)
    s = (x.abs().amax(1, keepdim=True).to(F64) / 127).to(F32)
    # a quotient next to a half decides a code: in 64 bits
    q = torch.where(s > 0, x.to(F64) / s.to(F64), 0.0).round().clamp(-127, 127).to(F32)
    y = torch.matmul(q, d["w"].to(F32).t()) * s * d["sw"]
    if d["bias"] is not None:
        y = y + d["bias"]
    return y.to(BF16 if case["out"] == "bf16" else F32)


# ----------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    d = prepare(case, seed)["in"]
    return {"logprobs": _exact_logprobs, "attention": _exact_attention, "linear": _exact_linear}[case["kind"]](case, d)


def _exact_logprobs(case, d):
    T, V = d["z"].shape
    top, train = case["top"], case["train"]
    parts = []
    step = max(1, (1 << 27) // V)
    for a in range(0, T, step):
        part = {}
        y = d["y"][a:a + step, None]
        z = d["z"][a:a + step].to(F64).requires_grad_(train)
        logp = torch.log_softmax(z, 1)
        part["logp"] = logp.gather(1, y)[:, 0]
        part["lse"] = torch.logsumexp(z, 1)
        part["entropy"] = -torch.special.xlogy(logp.exp(), logp.exp()).sum(1)
        ids = []
        left = z.detach().clone()
        for _ in range(top):
            j = left.argmax(1, keepdim=True)
            left.scatter_(1, j, -math.inf)
            ids.append(j)
        if top:
            part["top_ids"] = torch.cat(ids, 1)
            part["top_logp"] = logp.gather(1, part["top_ids"])
        if train:
            loss = (part["logp"] * d["dlogp"][a:a + step]).sum() + (part["entropy"] * d["dent"][a:a + step]).sum()
            if top:
                loss = loss + (part["top_logp"] * d["dtop"][a:a + step]).sum()
            part["dlogits"], = torch.autograd.grad(loss, z)
        parts.append({n: t.detach() for n, t in part.items()})
    return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}


def _exact_attention(case, d):
    T, H, hd = d["q"].shape
    G = d["k"].shape[1]
    train = case["train"]
    names = ("q", "k", "v") + (("do",) if train else ())
    x = {n: d[n].to(F64) for n in names}
    o, lse = torch.zeros_like(x["q"]), torch.zeros((H, T), dtype=F64, device=x["q"].device)
    grads = {n: torch.zeros_like(x[n]) for n in ("q", "k", "v")} if train else {}
    begin = 0
    for length in _lens(case):
        rows = slice(begin, begin + length)
        begin += length
        if not length:
            continue
        keep = torch.ones((length, length), dtype=torch.bool, device=o.device).tril()
        for h in range(H):
            kv = h * G // H
            q, k, v = (t[rows, i].detach().requires_grad_(train) for t, i in ((x["q"], h), (x["k"], kv), (x["v"], kv)))
            s = (q @ k.t() / math.sqrt(hd)).masked_fill(~keep, -math.inf)
            lse[h, rows] = torch.logsumexp(s, 1).detach()
            out = torch.softmax(s, 1) @ v
            o[rows, h] = out.detach()
            if train:
                dq, dk, dv = torch.autograd.grad(out, (q, k, v), x["do"][rows, h])
                grads["q"][rows, h] = dq
                grads["k"][rows, kv] += dk
                grads["v"][rows, kv] += dv
    r = {"o": o, "lse": lse}
    r.update({"d" + n: t for n, t in grads.items()})
    return r


def _exact_linear(case, d):
    x = d["x"].to(F64)
    s = (x.abs().max(1).values / 127).to(F32).to(F64)
    q = torch.zeros_like(x)
    q[s > 0] = torch.round(x[s > 0] / s[s > 0, None]).clamp(-127, 127)
    y = (q @ d["w"].to(F64).t()) * torch.outer(s, d["sw"].to(F64))
    return y if d["bias"] is None else y + d["bias"].to(F64)
