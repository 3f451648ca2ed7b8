"""Timing cases of the token-model operators: what they run, their inputs, their work and their exact results.

A case is a dict of plain values.  ``kind`` names the operator and its direction:

* ``embed``, ``embed_grad``      rows of a table by token, scaled; the table's gradient
* ``norm``, ``norm_grad``        root-mean-square norm behind a residual addition, 8-bit output with block scales; its gradient
* ``fp8``, ``fp8_step``          product of 8-bit operands with a scale for each block of 128; a linear layer's training step:
                                 operands quantised, output, input gradient and weight gradient
* ``logprob``, ``logprob_grad``  log probabilities of given tokens, entropy and top alternatives; the logits' gradient

8-bit tensors are e4m3 codes with E8M0 scales (powers of two), one scale for 128 values of a row, or for 128 x 128 values
of a weight.  A row of codes is padded with zeros to a multiple of 16 bytes, a row of scales to a multiple of 4.

``prepare`` makes inputs and output buffers on the GPU, ``run`` is one pass, ``exact`` the same results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6
BLOCK = 128


def listed():
    return [
        # One decoding step of 16 sequences: sixteen rows of a table, all latency.
        dict(name="embed_16", kind="embed", dtype="bf16", n=1, tokens=16, vocab=32000, dim=1024),
        # Three replicas read a training batch of 3 x 8192 tokens, each from its own fp32 rows of parameters.
        dict(name="embed_batch", kind="embed", dtype="f32", n=3, tokens=8192, vocab=32000, dim=1024),
        # The gradient of such a batch: a table of odd length, frequent tokens, most rows untouched.
        dict(name="embed_grad_batch", kind="embed_grad", dtype="bf16", n=3, tokens=8192, vocab=50001, dim=512),
        # One decoding step of 8 sequences: the residual stream of 4096 columns, quantised for the product behind it.
        dict(name="norm_8", kind="norm", dtype="bf16", n=1, rows=8, dim=4096),
        # A prompt of 8192 tokens through the same norm.
        dict(name="norm_prompt", kind="norm", dtype="bf16", n=1, rows=8192, dim=4096),
        # The norm's gradient in the training of three replicas, 2048 columns, a ragged number of tokens.
        dict(name="norm_grad_batch", kind="norm_grad", dtype="bf16", n=3, rows=4099, dim=2048),
        # One decoding step of 4 sequences through a large layer: the weights are read once, nothing else matters.
        dict(name="fp8_4", kind="fp8", n=1, m=4, cols=8192, depth=4096),
        # A prompt through the same layer: all matrix instructions.
        dict(name="fp8_prompt", kind="fp8", n=1, m=8192, cols=8192, depth=4096),
        # A linear layer's training step of three replicas, odd numbers of tokens and outputs.
        dict(name="fp8_step", kind="fp8_step", n=3, m=2050, cols=4000, depth=1024),
        # The next token of 4 sequences with its 20 best alternatives.
        dict(name="logprob_4", kind="logprob", dtype="bf16", n=1, rows=4, classes=128000, top=20, ld=128000),
        # Scoring of a prompt: odd number of classes, rows that start at odd addresses, 5 alternatives.
        dict(name="logprob_prompt", kind="logprob", dtype="bf16", n=1, rows=4096, classes=50001, top=5, ld=50001),
        # The logits' gradient of a training batch of three replicas, with an entropy bonus.
        dict(name="logprob_grad_batch", kind="logprob_grad", dtype="bf16", n=3, rows=2048, classes=32000, top=0, ld=32000),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return min(hi, max(lo, v if rng.random() < 0.4 else v // 16 * 16))

    kind = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "fp8", "fp8_step", "logprob", "logprob_grad"])
    n, dtype = rng.choice([1, 1, 2, 3, 6]), rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("embed"):
        vocab, dim = size(256, 128000), size(64, 4096)
        n = max(1, min(n, (40 << 20) // (vocab * dim)))
        dim = min(dim, (40 << 20) // vocab)
        return dict(kind=kind, dtype=dtype, n=n, tokens=size(1, min(16384, (24 << 20) // (n * dim))), vocab=vocab, dim=dim)
    if kind.startswith("norm"):
        dim = size(64, 8192)
        return dict(kind=kind, dtype=dtype, n=n, rows=size(1, (12 << 20) // (n * dim)), dim=dim)
    if kind.startswith("fp8"):
        if kind == "fp8":
            return dict(kind=kind, n=n, m=size(1, 8192 // n), cols=size(128, 8192), depth=size(64, 4096))
        depth = size(64, 2048)
        cols = size(128, (12 << 20) // depth // n if depth * n > 2048 else 6144)
        return dict(kind=kind, n=n, m=size(32, 6144 // n), cols=cols, depth=depth)
    classes = size(1000, 128000)
    top = rng.choice([0, 1, 5, 20]) if kind == "logprob" else 0
    return dict(kind=kind, dtype=dtype, n=n, rows=size(1, (92 << 20) // (n * classes)), classes=classes, top=top,
                ld=classes + rng.choice([0, 0, 3, 16]))


def _up(v, to):
    return -(-v // to) * to


def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEVICE) * scale).to(dtype)


def _exponents(amax):
    """The smallest e with amax <= 448 * 2^e (0 where amax is 0), by comparison: frexp gives amax = f * 2^x, f in [0.5, 1)."""
    f, x = torch.frexp(amax)
    e = x - 9 + (f > 0.875)
    return torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127)


def _power(e):
    """2^e in fp32 from its bits, -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(v, block_rows):
    """v [..., R, C] fp32 -> codes [..., R, pitch] (float8_e4m3fn) and scale bytes [..., ceil(R/block_rows), pitch] (uint8)."""
    R, C = v.shape[-2:]
    Cb, Rb = _up(C, BLOCK) // BLOCK, _up(R, block_rows) // block_rows
    p = torch.nn.functional.pad(v, (0, Cb * BLOCK - C, 0, Rb * block_rows - R))
    p = p.reshape(*v.shape[:-2], Rb, block_rows, Cb, BLOCK)
    e = _exponents(p.abs().amax(dim=(-3, -1)))
    q = (p * _power(-e)[..., :, None, :, None]).to(torch.float8_e4m3fn)
    q = q.reshape(*v.shape[:-2], Rb * block_rows, Cb * BLOCK)[..., :R, :_up(C, 16)].contiguous()
    s = torch.nn.functional.pad(e + 127, (0, _up(Cb, 4) - Cb)).to(torch.uint8)
    return q, s


def _values(q, s, depth, block_rows):
    """The numbers that codes and scale bytes stand for, fp32 [..., R, depth]."""
    R, Cb = q.shape[-2], _up(depth, BLOCK) // BLOCK
    e = s[..., :Cb].to(torch.int32) - 127
    e = e.repeat_interleave(block_rows, dim=-2)[..., :R, :].repeat_interleave(BLOCK, dim=-1)[..., :depth]
    return q[..., :depth].float() * _power(e)


def _codes(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device=DEVICE)


def _empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEVICE)


def _tokens(g, n, count, vocab):
    """Token t with probability about 1/t, one in a hundred a padding token (-1)."""
    t = (torch.exp(torch.rand((n, count), generator=g, device=DEVICE, dtype=torch.float64) * math.log(vocab)) - 1).to(torch.int32)
    t = t.clamp(0, vocab - 1)
    return torch.where(torch.rand((n, count), generator=g, device=DEVICE) < 0.01, torch.full_like(t, -1), t)


def prepare(case, seed):
    g, c, kind = _gen(seed), case, case["kind"]
    s = {"case": dict(case)}
    if kind.startswith("embed"):
        n, T, V, D, dt = c["n"], c["tokens"], c["vocab"], c["dim"], DTYPES[c["dtype"]]
        s["rs"] = _up(V * D, 1024)
        s["tokens"] = _tokens(g, n, T, V)
        if kind == "embed":
            s["table"] = _normal(g, n, s["rs"], dtype=dt, scale=0.05)
            s["out"] = _empty(n, T, D, dtype=dt)
        else:
            s["dout"] = _normal(g, n, T, D, dtype=dt, scale=1e-3)
            s["dtable"] = _empty(n, s["rs"])
    elif kind.startswith("norm"):
        n, R, D, dt = c["n"], c["rows"], c["dim"], DTYPES[c["dtype"]]
        s["w"] = 1 + _normal(g, n, D, scale=0.1)
        spread = torch.exp(_normal(g, n, R, 1))     # rows of different sizes, some columns far larger than the rest
        columns = torch.where(torch.rand((1, 1, D), generator=g, device=DEVICE) < 0.01, 20.0, 1.0)
        if kind == "norm":
            s["x"] = (_normal(g, n, R, D) * spread).to(dt)
            s["resid"] = (_normal(g, n, R, D) * spread * columns).to(dt)
            s["h"], s["rstd"] = _empty(n, R, D, dtype=dt), _empty(n, R)
            s["q"], s["scales"] = _codes(n, R, _up(D, 16)), _codes(n, R, _up(_up(D, BLOCK) // BLOCK, 4))
        else:
            s["h"] = (_normal(g, n, R, D) * spread * columns).to(dt)
            s["rstd"] = torch.rsqrt(s["h"].double().square().mean(-1) + EPS).float()
            s["dout"], s["dresid"] = _normal(g, n, R, D, dtype=dt, scale=1e-3), _normal(g, n, R, D, dtype=dt, scale=1e-3)
            s["dx"], s["dw"] = _empty(n, R, D, dtype=dt), _empty(n, D)
    elif kind == "fp8":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        s["a"], s["a_scales"] = _quantise(_normal(g, n, M, K) * torch.exp(_normal(g, n, M, 1)), 1)
        s["b"], s["b_scales"] = _quantise(_normal(g, n, N, K, scale=K ** -0.5), BLOCK)
        s["out"] = _empty(n, M, N, dtype=torch.bfloat16)
    elif kind == "fp8_step":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        s["rs"] = _up(N * K, 1024)
        s["x"] = _normal(g, n, M, K, dtype=torch.bfloat16)
        s["w"] = _normal(g, n, s["rs"], scale=K ** -0.5)           # fp32 rows of parameters
        s["dy"] = _normal(g, n, M, N, dtype=torch.bfloat16, scale=1e-4)
        s["y"], s["dx"] = _empty(n, M, N, dtype=torch.bfloat16), _empty(n, M, K, dtype=torch.bfloat16)
        s["dw"] = _empty(n, s["rs"])
    else:
        n, R, C, ld, dt = c["n"], c["rows"], c["classes"], c["ld"], DTYPES[c["dtype"]]
        x = _normal(g, n, R, ld, scale=3.0)
        x[:, :, C - C // 50:] = -math.inf                          # classes that no token has
        if n * R > 8:
            x.view(n * R, ld)[n * R // 2, :] = -math.inf            # a row that its mask leaves empty
            if kind == "logprob_grad":
                x.view(n * R, ld)[3, 1:C] = torch.finfo(dt).min     # a row with one class left, masked by the lowest value
        s["logits"] = x.to(dt)
        s["labels"] = torch.randint(0, C - C // 50, (n, R), generator=g, device=DEVICE, dtype=torch.int32)
        s["labels"][:, ::37] = torch.where(torch.rand((n, R), generator=g, device=DEVICE)[:, ::37] < 0.5, s["labels"][:, ::37], torch.full_like(s["labels"][:, ::37], -1))
        if kind == "logprob":
            s["logp"], s["entropy"], s["lse"] = _empty(n, R), _empty(n, R), _empty(n, R)
            s["top_ids"], s["top_logp"] = _empty(n, R, c["top"], dtype=torch.int32), _empty(n, R, c["top"])
        else:
            _, s["entropy"], s["lse"] = (t.float() if t is not None else None for t in _stats64(s["logits"], C))
            s["dlogp"], s["dentropy"] = _normal(g, n, R, scale=1.0 / R), _normal(g, n, R, scale=0.01 / R)
            s["dlogits"] = torch.zeros((n, R, ld), dtype=dt, device=DEVICE)
    return s


def _stats64(logits, C):
    """Row by row in 64 bits: shifted sums, entropy and the logarithm of the sum of exponentials."""
    rows = logits.reshape(-1, logits.shape[-1])
    H, L = _empty(rows.shape[0], dtype=torch.float64), _empty(rows.shape[0], dtype=torch.float64)
    for i in range(0, rows.shape[0], 1024):
        x = rows[i:i + 1024, :C].double()
        m = x.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        e = torch.exp(x - m)
        z = e.sum(-1)
        x = torch.where(e > 0, x - m, torch.zeros_like(x))
        L[i:i + 1024] = torch.log(z) + m[:, 0]
        H[i:i + 1024] = torch.where(z > 0, torch.log(z) - (e * x).sum(-1) / torch.where(z > 0, z, torch.ones_like(z)), torch.zeros_like(z))
    return None, H.reshape(logits.shape[:-1]), L.reshape(logits.shape[:-1])


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    """The calls that a training or serving program makes; descriptors and scratch are made at a state's first pass."""
    from paper_1707_00424_amd import binding as pb
    c, kind = s["case"], s["case"]["kind"]

    def scratch(nbytes):
        return torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEVICE)

    if kind.startswith("embed"):
        if "desc" not in s:
            dt = int(c["dtype"] == "bf16")
            s["desc"] = pb.parle_embed_desc(dt, dt if kind == "embed" else 0, c["n"], c["tokens"], c["vocab"], c["dim"], s["rs"], math.sqrt(c["dim"]))
            s["scratch"] = scratch(pb.parle_k_embed_scratch_bytes(s["desc"])) if kind == "embed_grad" else None
        if kind == "embed":
            pb.parle_k_embed_forward(s["desc"], s["table"], s["tokens"], s["out"])
            return s["out"]
        pb.parle_k_embed_backward(s["desc"], s["tokens"], s["dout"], s["scratch"], s["dtable"])
        return s["dtable"][:, :c["vocab"] * c["dim"]]
    if kind.startswith("norm"):
        if "desc" not in s:
            s["desc"] = pb.parle_norm_desc(int(c["dtype"] == "bf16"), 0, c["n"], c["rows"], c["dim"], c["dim"], EPS)
            s["scratch"] = scratch(pb.parle_k_rmsnorm_scratch_bytes(s["desc"])) if kind == "norm_grad" else None
        if kind == "norm":
            pb.parle_k_rmsnorm_forward(s["desc"], s["x"], s["resid"], s["w"], s["h"], None, s["q"], s["scales"], s["rstd"])
            return {"h": s["h"], "q": s["q"].view(torch.float8_e4m3fn)[..., :c["dim"]],
                    "scales": s["scales"].view(torch.float8_e8m0fnu)[..., :_up(c["dim"], BLOCK) // BLOCK], "rstd": s["rstd"]}
        pb.parle_k_rmsnorm_backward(s["desc"], s["h"], s["w"], s["rstd"], s["dout"], s["dresid"], s["scratch"], s["dx"], s["dw"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if kind == "fp8":
        if "desc" not in s:
            s["desc"] = pb.parle_fp8_desc(1, BLOCK, 0, c["n"], c["m"], c["cols"], c["depth"], c["cols"], c["m"] * c["cols"])
            s["scratch"] = scratch(pb.parle_k_fp8_scratch_bytes(s["desc"]))
        pb.parle_k_fp8_matmul(s["desc"], s["a"], s["a_scales"], s["b"], s["b_scales"], None, s["scratch"], s["out"])
        return s["out"]
    if kind == "fp8_step":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        if "xd" not in s:
            def both(rows, cols, block):
                r = lambda v: _up(v, block) // block  # noqa: E731
                k = lambda v: _up(_up(v, BLOCK) // BLOCK, 4)  # noqa: E731
                return (_codes(n, rows, _up(cols, 16)), _codes(n, r(rows), k(cols)),
                        _codes(n, cols, _up(rows, 16)), _codes(n, r(cols), k(rows)))
            s["x8"], s["w8"], s["dy8"] = both(M, K, 1), both(N, K, BLOCK), both(M, N, 1)
            s["xd"] = pb.parle_quant_desc(1, 1, n, M, K, K, M * K)
            s["wd"] = pb.parle_quant_desc(0, BLOCK, n, N, K, K, s["rs"])
            s["dyd"] = pb.parle_quant_desc(1, 1, n, M, N, N, M * N)
            s["yd"] = pb.parle_fp8_desc(1, BLOCK, 0, n, M, N, K, N, M * N)
            s["dxd"] = pb.parle_fp8_desc(1, BLOCK, 0, n, M, K, N, K, M * K)
            s["dwd"] = pb.parle_fp8_desc(0, 1, 0, n, N, K, M, K, s["rs"])
            s["scratch"] = scratch(max(pb.parle_k_fp8_scratch_bytes(s[d]) for d in ("yd", "dxd", "dwd")))
        pb.parle_k_fp8_quantize(s["xd"], s["x"], *s["x8"])
        pb.parle_k_fp8_quantize(s["wd"], s["w"], *s["w8"])
        pb.parle_k_fp8_matmul(s["yd"], s["x8"][0], s["x8"][1], s["w8"][0], s["w8"][1], None, s["scratch"], s["y"])
        pb.parle_k_fp8_quantize(s["dyd"], s["dy"], *s["dy8"])
        pb.parle_k_fp8_matmul(s["dxd"], s["dy8"][0], s["dy8"][1], s["w8"][2], s["w8"][3], None, s["scratch"], s["dx"])
        pb.parle_k_fp8_matmul(s["dwd"], s["dy8"][2], s["dy8"][3], s["x8"][2], s["x8"][3], None, s["scratch"], s["dw"])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"][:, :N * K]}
    if "desc" not in s:
        s["desc"] = pb.parle_logprob_desc(int(c["dtype"] == "bf16"), c["n"], c["rows"], c["classes"], c["top"], c["ld"])
        s["scratch"] = scratch(pb.parle_k_logprob_scratch_bytes(s["desc"])) if kind == "logprob" else None
    if kind == "logprob":
        ids, alt = (s["top_ids"], s["top_logp"]) if c["top"] else (None, None)
        pb.parle_k_logprob_forward(s["desc"], s["logits"], s["labels"], s["scratch"], s["logp"], s["entropy"], s["lse"], ids, alt)
        return {"logp": s["logp"], "entropy": s["entropy"], "lse": s["lse"], "top_ids": s["top_ids"], "top_logp": s["top_logp"]}
    pb.parle_k_logprob_backward(s["desc"], s["logits"], s["labels"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["dlogits"])
    return s["dlogits"][..., :c["classes"]]


def _plain(s):
    """The same in elementary torch operations, in 32 bits, rounded once at the end."""
    c, kind = s["case"], s["case"]["kind"]
    if kind.startswith("embed"):
        n, T, V, D = c["n"], c["tokens"], c["vocab"], c["dim"]
        valid = s["tokens"] >= 0
        rows = (s["tokens"].clamp(min=0).long() + V * torch.arange(n, device=DEVICE)[:, None]).reshape(-1)
        if kind == "embed":
            table = s["table"][:, :V * D].reshape(n * V, D)
            out = table[rows].reshape(n, T, D).float() * math.sqrt(D)
            return (out * valid[..., None]).to(s["table"].dtype)
        d = s["dout"].float() * valid[..., None]
        sums = torch.zeros((n * V, D), device=DEVICE).index_add_(0, rows, d.reshape(n * T, D))
        return (sums * math.sqrt(D)).reshape(n, V * D)
    if kind == "norm":
        h = (s["x"].float() + s["resid"].float()).to(s["x"].dtype)
        f = h.float()
        rstd = 1.0 / torch.sqrt(f.square().mean(-1) + EPS)
        q, e = _quantise(f * rstd[..., None] * s["w"][:, None, :], 1)
        D = c["dim"]
        return {"h": h, "q": q[..., :D], "scales": e.view(torch.float8_e8m0fnu)[..., :_up(D, BLOCK) // BLOCK], "rstd": rstd}
    if kind == "norm_grad":
        h, d, r, w = s["h"].float(), s["dout"].float(), s["rstd"][..., None], s["w"][:, None, :]
        gr = d * w
        dx = r * (gr - h * ((gr * h).mean(-1, keepdim=True) * r * r)) + s["dresid"].float()
        return {"dx": dx.to(s["h"].dtype), "dw": (d * (h * r)).sum(1)}
    if kind == "fp8":
        K = c["depth"]
        a, b = _values(s["a"], s["a_scales"], K, 1), _values(s["b"], s["b_scales"], K, BLOCK)
        return torch.matmul(a, b.transpose(1, 2)).to(torch.bfloat16)
    if kind == "fp8_step":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        through = lambda v, block: _values(*_quantise(v, block), v.shape[-1], block)  # noqa: E731
        x, dy = s["x"].float(), s["dy"].float()
        w = through(s["w"][:, :N * K].reshape(n, N, K), BLOCK)
        y = torch.matmul(through(x, 1), w.transpose(1, 2))
        dx = torch.matmul(through(dy, 1), w)
        dyt, xt = through(dy.transpose(1, 2), 1), through(x.transpose(1, 2), 1)
        dw = torch.matmul(dyt, xt.transpose(1, 2).contiguous())
        return {"y": y.to(torch.bfloat16), "dx": dx.to(torch.bfloat16), "dw": dw.reshape(n, N * K)}
    C, labels = c["classes"], s["labels"]
    x = s["logits"][..., :C].float()
    inside = (labels >= 0) & (labels < C)
    at = torch.where(inside, labels, torch.zeros_like(labels)).long()[..., None]
    if kind == "logprob":
        m = x.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        d = x - m
        e = torch.exp(d)
        z = e.sum(-1)
        lse = torch.log(z) + m[..., 0]
        none = z == 0
        t = (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(-1)
        H = torch.where(none, torch.zeros_like(z), torch.log(z) - t / z)
        logp = torch.where(none, torch.full_like(z, -math.inf), torch.gather(x, -1, at)[..., 0] - lse)
        logp = torch.where(inside, logp, torch.zeros_like(logp))
        ids, alt = _best(x, lse, c["top"])
        return {"logp": logp, "entropy": H, "lse": lse, "top_ids": ids, "top_logp": alt}
    lse, H = s["lse"][..., None], s["entropy"][..., None]
    some = lse > -math.inf
    base = torch.where(some, lse, torch.zeros_like(lse))
    p = torch.exp(x - base) * some
    gl = (s["dlogp"] * inside)[..., None] * some
    d = -p * gl - s["dentropy"][..., None] * p * torch.where(p > 0, x - base + H, torch.zeros_like(x))
    return d.scatter_add_(-1, at, gl).to(s["logits"].dtype)


def _best(x, lse, top):
    """The `top` largest of every row, ties to the lowest index; -1 and -inf where a row has no more."""
    if top == 0:
        return torch.empty((*lse.shape, 0), dtype=torch.int32, device=DEVICE), torch.empty((*lse.shape, 0), device=DEVICE)
    C = x.shape[-1]
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 20) + (C - 1 - torch.arange(C, device=DEVICE))
    ids = C - 1 - (torch.topk(key, top, dim=-1).values & ((1 << 20) - 1))
    v = torch.gather(x, -1, ids)
    gone = v == -math.inf
    alt = torch.where(gone, v, v - lse[..., None])
    return torch.where(gone, torch.full_like(ids, -1), ids).to(torch.int32), alt


def work(case):
    c, kind = case, case["kind"]
    if kind.startswith("embed"):
        n, T, V, D, z = c["n"], c["tokens"], c["vocab"], c["dim"], SIZE[c["dtype"]]
        if kind == "embed":
            return {"bytes": n * (4 * T + (min(T, V) + T) * D * z), "flops": n * T * D}
        return {"bytes": n * (4 * T + T * D * z + V * D * 4), "flops": 2 * n * T * D}
    if kind.startswith("norm"):
        n, R, D, z = c["n"], c["rows"], c["dim"], SIZE[c["dtype"]]
        if kind == "norm":
            return {"bytes": n * (R * (D * (3 * z + 1) + _up(D, BLOCK) // BLOCK + 4) + 4 * D), "flops": 8 * n * R * D}
        return {"bytes": n * (R * (D * 4 * z + 4) + 8 * D), "flops": 10 * n * R * D}
    if kind.startswith("fp8"):
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        if kind == "fp8":
            return {"bytes": n * (M * K + N * K + M * _up(K, BLOCK) // BLOCK + 2 * M * N), "flops": 2 * n * M * N * K}
        return {"bytes": n * (2 * M * K + 4 * N * K + 2 * M * N + 2 * M * N + 2 * M * K + 4 * N * K), "flops": 6 * n * M * N * K}
    n, R, C, z = c["n"], c["rows"], c["classes"], SIZE[c["dtype"]]
    if kind == "logprob":
        return {"bytes": n * R * (C * z + 4 * 4 + 8 * c["top"]), "flops": 6 * n * R * C}
    return {"bytes": n * R * (2 * C * z + 5 * 4), "flops": 6 * n * R * C}


def _exact_codes(v, block_rows):
    """Codes and scales of v [n, R, C] from their definition, as 64-bit numbers: (code values, scales)."""
    n, R, C = v.shape
    pr, pc = _up(R, block_rows), _up(C, BLOCK)
    p = torch.zeros((n, pr, pc), dtype=torch.float64, device=v.device)
    p[:, :R, :C] = v
    most = p.abs().view(n, pr // block_rows, block_rows, pc // BLOCK, BLOCK).amax((2, 4))
    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -140) / 448.0))
    e = torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e)     # the logarithm's own rounding
    e = torch.where(most > 448.0 * torch.exp2(e), e + 1, e)
    scale = torch.exp2(torch.where(most == 0, torch.zeros_like(e), e.clamp(-127, 127)))
    u = p / scale.repeat_interleave(block_rows, 1).repeat_interleave(BLOCK, 2)
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(u / step) * step)[:, :R, :C], scale


def exact(case, seed):
    """What run() returns, in 64 bits, straight from the definitions."""
    s, c, kind = prepare(case, seed), case, case["kind"]
    if kind.startswith("embed"):
        n, T, V, D = c["n"], c["tokens"], c["vocab"], c["dim"]
        if kind == "embed":
            out = torch.zeros((n, T, D), dtype=torch.float64, device=DEVICE)
            for a in range(n):
                ok = s["tokens"][a] >= 0
                out[a, ok] = s["table"][a, :V * D].view(V, D)[s["tokens"][a, ok].long()].double() * math.sqrt(D)
            return out
        out = torch.zeros((n, V, D), dtype=torch.float64, device=DEVICE)
        for a in range(n):
            order = torch.argsort(s["tokens"][a], stable=True)
            tok, cnt = torch.unique_consecutive(s["tokens"][a][order], return_counts=True)
            run_sum = torch.cumsum(s["dout"][a][order].double(), 0)
            ends = torch.cumsum(cnt, 0) - 1
            upto = run_sum[ends]
            part = torch.cat([upto[:1], upto[1:] - upto[:-1]])
            out[a, tok[tok >= 0].long()] = part[tok >= 0] * math.sqrt(D)
        return out.view(n, V * D)
    if kind.startswith("norm"):
        if kind == "norm":
            h = (s["x"].double() + s["resid"].double()).to(s["x"].dtype).double()
            rstd = (h.square().sum(-1) / c["dim"] + EPS) ** -0.5
            q, scale = _exact_codes(h * rstd[..., None] * s["w"].double()[:, None], 1)
            return {"h": s["x"].double() + s["resid"].double(), "q": q, "scales": scale, "rstd": rstd}
        h, d, w = s["h"].double(), s["dout"].double(), s["w"].double()[:, None]
        r = s["rstd"].double()[..., None]
        unit = h * r
        g = d * w
        dx = r * (g - unit * (g * unit).sum(-1, keepdim=True) / c["dim"]) + s["dresid"].double()
        return {"dx": dx, "dw": torch.einsum("nrd,nrd->nd", d, unit)}
    if kind == "fp8":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]
        out = torch.empty((n, M, N), dtype=torch.float64, device=DEVICE)
        rows_a = torch.exp2(s["a_scales"].double() - 127)
        rows_b = torch.exp2(s["b_scales"].double() - 127)
        for a in range(n):
            left, right = s["a"][a].double(), s["b"][a].double()
            for k in range(0, K, BLOCK):
                left[:, k:k + BLOCK] *= rows_a[a, :, k // BLOCK, None]
                for j in range(0, N, BLOCK):
                    right[j:j + BLOCK, k:k + BLOCK] *= rows_b[a, j // BLOCK, k // BLOCK]
            out[a] = left[:, :K] @ right[:, :K].t()
        return out
    if kind == "fp8_step":
        n, M, N, K = c["n"], c["m"], c["cols"], c["depth"]

        def through(v, block):
            q, scale = _exact_codes(v.double(), block)
            return q * scale.repeat_interleave(block, 1).repeat_interleave(BLOCK, 2)[:, :v.shape[1], :v.shape[2]]

        w = through(s["w"][:, :N * K].view(n, N, K), BLOCK)
        y, dx, dw = through(s["x"], 1), through(s["dy"], 1), through(s["dy"].transpose(1, 2), 1)
        xt = through(s["x"].transpose(1, 2), 1)
        return {"y": torch.stack([y[a] @ w[a].t() for a in range(n)]), "dx": torch.stack([dx[a] @ w[a] for a in range(n)]),
                "dw": torch.stack([(dw[a] @ xt[a].t()).view(N * K) for a in range(n)])}
    n, R, C, top = c["n"], c["rows"], c["classes"], c["top"]
    if kind == "logprob":
        out = {"logp": _empty(n, R, dtype=torch.float64), "entropy": _empty(n, R, dtype=torch.float64), "lse": _empty(n, R, dtype=torch.float64),
               "top_ids": None, "top_logp": _empty(n, R, top, dtype=torch.float64)}
        for a in range(n):
            for i in range(0, R, 512):
                x, lab = s["logits"][a, i:i + 512, :C].double(), s["labels"][a, i:i + 512].long()
                lse = torch.logsumexp(x, -1)
                empty = lse == -math.inf
                logp = x - torch.where(empty, torch.zeros_like(lse), lse)[:, None]
                p = torch.exp(logp)
                out["lse"][a, i:i + 512] = lse
                out["entropy"][a, i:i + 512] = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(-1)
                out["logp"][a, i:i + 512] = torch.where(lab < 0, torch.zeros_like(lse), logp.gather(-1, lab.clamp(min=0)[:, None])[:, 0])
                out["top_logp"][a, i:i + 512] = torch.topk(logp, top, -1).values if top else torch.empty((len(lab), 0), device=DEVICE)
        return out
    out = torch.empty((n, R, C), dtype=torch.float64, device=DEVICE) if n * R * C < (1 << 28) else None
    for a in range(n if out is not None else 0):
        for i in range(0, R, 512):
            x, lab = s["logits"][a, i:i + 512, :C].double(), s["labels"][a, i:i + 512].long()
            lse, H = s["lse"][a, i:i + 512].double(), s["entropy"][a, i:i + 512].double()
            empty = (lse == -math.inf)[:, None]
            logp = torch.where(empty, torch.full_like(x, -math.inf), x - torch.where(empty[:, 0], torch.zeros_like(lse), lse)[:, None])
            p = torch.exp(logp)
            gl = s["dlogp"][a, i:i + 512].double() * (lab >= 0)
            d = -gl[:, None] * p - s["dentropy"][a, i:i + 512].double()[:, None] * torch.where(p > 0, p * (logp + H[:, None]), torch.zeros_like(p))
            d.scatter_add_(-1, lab.clamp(min=0)[:, None], torch.where(empty, torch.zeros_like(gl)[:, None], gl[:, None]))
            out[a, i:i + 512] = d
    return out
