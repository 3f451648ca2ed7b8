"""Timing cases of the attention operators and of the sampler: what they run, their inputs, their work and their exact results.

A case is a dict of plain values.  ``kind`` names the operator and its direction:

* ``rope``                           heads turned by the positions of one to four axes; ``inverse``: turned back, the gradient
* ``attention``, ``attention_grad``  attention over packed sequences with a sliding window and first tokens that stay visible
* ``store``, ``decode``              a prompt's keys and values into the caches; one new token of every sequence over its cache
* ``sample``                         a token of every row from given random numbers: temperature, top-k, top-p, min-p

Queries, keys and values lie side by side in one row per token, as a linear layer leaves them.  A cache is
[sequences, kv_heads, capacity, dim]: token p of a sequence lies in slot p where p < sinks, else in slot
sinks + (p - sinks) % (capacity - sinks), so that a cache of sinks + window slots serves sequences of any length.

``prepare`` makes inputs and output buffers on the GPU, ``run`` is one pass, ``exact`` the same results in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # One decoding step of 16 sequences: queries and keys of a token each, all latency.
        dict(name="rope_16", kind="rope", dtype="bf16", n=1, tokens=16, heads=40, dim=128, axes=1, turned=128, interleaved=False, inverse=False),
        # The gradient of a training batch of three replicas: time, height and width of an image's patches, a part of each head unturned.
        dict(name="rope_grad_images", kind="rope", dtype="f32", n=3, tokens=4099, heads=20, dim=80, axes=3, turned=64, interleaved=True, inverse=True),
        # A small fp32 training batch of three replicas: odd lengths, several documents, heads that share nothing.
        dict(name="attention_small", kind="attention", dtype="f32", n=3, tokens=515, sequences=5, heads=8, kv_heads=8, dim=64, window=100, sinks=1),
        # A prompt of 8192 tokens, each seeing all before it.
        dict(name="attention_prompt", kind="attention", dtype="bf16", n=1, tokens=8192, sequences=1, heads=32, kv_heads=8, dim=128, window=0, sinks=0),
        # Five documents in a row of 8192 tokens, a window of 1024 and four first tokens.
        dict(name="attention_window", kind="attention", dtype="bf16", n=1, tokens=8192, sequences=5, heads=16, kv_heads=2, dim=128, window=1024, sinks=4),
        # The gradient in the training of three replicas on packed documents with a window.
        dict(name="attention_grad_batch", kind="attention_grad", dtype="bf16", n=3, tokens=4096, sequences=3, heads=16, kv_heads=4, dim=64, window=1024, sinks=4),
        # The gradient of one long document, odd in length, without a window.
        dict(name="attention_grad_long", kind="attention_grad", dtype="bf16", n=1, tokens=4099, sequences=1, heads=16, kv_heads=16, dim=128, window=0, sinks=0),
        # A batch of prompts whose keys and values go to rolling caches, some longer than these.
        dict(name="store_prompts", kind="store", dtype="bf16", tokens=16384, sequences=16, kv_heads=8, dim=128, window=1024, sinks=4, capacity=1028),
        # One decoding step of 4 sequences over rolling caches that have come round.
        dict(name="decode_4", kind="decode", dtype="bf16", sequences=4, heads=32, kv_heads=8, dim=128, window=1024, sinks=4, capacity=1028, longest=5000),
        # One decoding step of 64 sequences of up to 8192 tokens: the caches are read once, nothing else matters.
        dict(name="decode_64", kind="decode", dtype="bf16", sequences=64, heads=32, kv_heads=8, dim=128, window=0, sinks=0, capacity=8192, longest=8192),
        # The next token of 4 sequences.
        dict(name="sample_4", kind="sample", dtype="bf16", n=1, rows=4, classes=128000, ld=128000, top_k=50, top_p=0.9, min_p=0.0),
        # Many answers to many prompts: odd number of classes, rows that start at odd addresses, no bound on their number.
        dict(name="sample_1024", kind="sample", dtype="bf16", n=1, rows=1024, classes=50001, ld=50001, top_k=0, top_p=0.95, min_p=0.02),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return min(hi, max(lo, v if rng.random() < 0.4 else v // 16 * 16))

    kind = rng.choice(["rope", "attention", "attention", "attention_grad", "attention_grad", "store", "decode", "decode", "sample", "sample"])
    n, dtype = rng.choice([1, 1, 2, 3, 6]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    window, sinks = (0, 0) if rng.random() < 0.4 else (size(16, 2048), rng.choice([0, 1, 4, 16]))
    if kind == "rope":
        heads, axes = size(1, 64), rng.choice([1, 1, 2, 3, 4])
        turned = rng.choice([dim, dim, dim // 16 * 8])
        return dict(kind=kind, dtype=dtype, n=n, tokens=size(1, (16 << 20) // (n * heads * dim)), heads=heads, dim=dim, axes=axes, turned=turned,
                    interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5)
    if kind.startswith("attention"):
        heads, kv_heads = min(heads, 24), min(heads, 24) // (heads // kv_heads) if heads <= 24 else 8
        heads = heads // kv_heads * kv_heads
        most = int(math.sqrt((1 << (29 if dtype == "bf16" else 27)) / (n * heads)))
        tokens = size(64, min(8192, most))
        return dict(kind=kind, dtype=dtype, n=n, tokens=tokens, sequences=rng.choice([1, 1, 2, 3, 7, 20]), heads=heads, kv_heads=kv_heads, dim=dim, window=window, sinks=sinks)
    longest = size(64, 16384)
    capacity = sinks + window if window and rng.random() < 0.7 else longest + sinks
    if kind == "store":
        sequences = size(1, 64)
        tokens = size(sequences, min(32768, sequences * longest))
        capacity = min(capacity, max((256 << 20) // (sequences * kv_heads * dim), sinks + 16))
        return dict(kind=kind, dtype=dtype, tokens=tokens, sequences=sequences, kv_heads=kv_heads, dim=dim, window=window, sinks=sinks, capacity=capacity)
    if kind == "decode":
        most = (512 << 20) // (capacity * kv_heads * dim)
        return dict(kind=kind, dtype=dtype, sequences=size(1, max(1, min(256, most))), heads=heads, kv_heads=kv_heads, dim=dim, window=window, sinks=sinks, capacity=capacity, longest=longest)
    classes = size(1000, 128000)
    return dict(kind=kind, dtype=dtype, n=n, rows=size(1, min(2048, (48 << 20) // classes) // n), classes=classes, ld=classes + rng.choice([0, 0, 3, 16]),
                top_k=rng.choice([0, 1, 40, 50, 500]), top_p=rng.choice([1.0, 0.95, 0.9, 0.5]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]))


def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, generator=g, device=DEVICE).mul_(scale).to(dtype)


def _empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEVICE)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _pairs(c):
    """Pairs of a head's elements that turn with each axis."""
    half, axes = c["turned"] // 2, c["axes"]
    each = half // axes
    return [half - each * (axes - 1)] + [each] * (axes - 1)


def _offsets(c):
    """Where the sequences of a row of tokens begin, replica by replica; one token in thirty is behind the last."""
    rng = random.Random("%d %d" % (c["tokens"], c["sequences"]))
    end = c["tokens"] if c["sequences"] == 1 else c["tokens"] - c["tokens"] // 30
    return [[0] + sorted(rng.randint(0, end) for _ in range(c["sequences"] - 1)) + [end] for _ in range(c.get("n", 1))]


def _seen(c, length):
    """Pairs of a query and a key it sees in a sequence of this length."""
    w, s = c["window"] or length, c["sinks"]
    return sum(min(i + 1, w) + max(0, min(s, i + 1 - w)) for i in range(length))


def _lengths(c):
    """Tokens of each sequence at a decoding step, the new one among them."""
    rng = random.Random("%d %d" % (c["sequences"], c["longest"]))
    return [c["longest"]] + [rng.randint(max(1, c["longest"] // 2), c["longest"]) for _ in range(c["sequences"] - 1)]


def _stored(c):
    """Tokens of each sequence behind a call of store: some have tokens of an earlier call."""
    o, rng = _offsets(c)[0], random.Random("%d %d" % (c["tokens"], c["capacity"]))
    return [o[b + 1] - o[b] + (0 if rng.random() < 0.7 else rng.randint(0, 100)) for b in range(c["sequences"])]


def prepare(case, seed):
    g, c, kind = _gen(seed), case, case["kind"]
    s = {"case": dict(case)}
    dt = DTYPES[c["dtype"]]
    if kind == "rope":
        n, T, H, D = c["n"], c["tokens"], c["heads"], c["dim"]
        # rows of the layer in front, which has values behind the turned heads too
        s["ld"] = (H + 4) * D
        s["x"] = _normal(g, n, T, s["ld"], dtype=dt)
        s["out"] = torch.zeros((n, T, s["ld"]), dtype=dt, device=DEVICE)
        s["freqs"] = 10000.0 ** (-torch.arange(c["turned"] // 2, device=DEVICE) / (c["turned"] / 2))
        far = 100000 if c["axes"] == 1 else 2000
        s["positions"] = torch.randint(0, far, (n, T, c["axes"]), generator=g, device=DEVICE, dtype=torch.int32)
    elif kind.startswith("attention"):
        n, T, H, K, D = c["n"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        s["ld"] = (H + 2 * K) * D
        s["qkv"] = _normal(g, n, T, s["ld"], dtype=dt)
        s["qkv"][..., :H * D] *= 2.0                       # scores of a standard deviation of two
        s["offsets"] = _ints(_offsets(c))
        s["out"], s["lse"] = _empty(n, T, H * D, dtype=dt), _empty(n, H, T)
        if kind == "attention_grad":
            s["out"], s["lse"] = _attention(c, s)
            s["dout"] = _normal(g, n, T, H * D, dtype=dt, scale=1e-3)
            s["dqkv"] = _empty(n, T, s["ld"], dtype=dt)
    elif kind == "store":
        T, K, D = c["tokens"], c["kv_heads"], c["dim"]
        s["ld"] = 2 * K * D
        s["kv"] = _normal(g, T, s["ld"], dtype=dt)
        s["offsets"], s["lengths"] = _ints(_offsets(c)[0]), _ints(_stored(c))
        s["k_cache"], s["v_cache"] = (torch.zeros((c["sequences"], K, c["capacity"], D), dtype=dt, device=DEVICE) for _ in range(2))
    elif kind == "decode":
        B, H, K, D = c["sequences"], c["heads"], c["kv_heads"], c["dim"]
        s["ld"] = (H + 2 * K) * D
        s["qkv"] = _normal(g, B, s["ld"], dtype=dt)
        s["qkv"][:, :H * D] *= 2.0
        s["k_cache"], s["v_cache"] = (_normal(g, B, K, c["capacity"], D, dtype=dt) for _ in range(2))
        s["lengths"] = _ints(_lengths(c))
        s["out"] = _empty(B, H * D, dtype=dt)
    else:
        n, R, C, ld = c["n"], c["rows"], c["classes"], c["ld"]
        x = _normal(g, n, R, ld, scale=3.0)
        x[:, :, C - C // 50:C] = -math.inf                 # classes that no token has
        s["logits"] = x.to(dt)
        s["uniform"] = torch.rand((n, R), generator=g, device=DEVICE)
        s["temperature"] = 0.5 + torch.rand((n, R), generator=g, device=DEVICE)
        s["temperature"][:, ::19] = 0.0                     # some requests want the most likely token
        s["top_k"] = torch.full((n, R), c["top_k"], dtype=torch.int32, device=DEVICE)
        s["top_p"], s["min_p"] = torch.full((n, R), c["top_p"], device=DEVICE), torch.full((n, R), c["min_p"], device=DEVICE)
        s["tokens"], s["kept"], s["logp"] = _empty(n, R, dtype=torch.int32), _empty(n, R, dtype=torch.int32), _empty(n, R)
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    """The calls that a training or serving program makes; descriptors and scratch are made at a state's first pass."""
    from paper_1707_00424_amd import binding as pb
    c, kind = s["case"], s["case"]["kind"]
    dt = int(c["dtype"] == "bf16")

    def scratch(nbytes):
        return torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEVICE)

    if kind == "rope":
        n, T, H, D, ld = c["n"], c["tokens"], c["heads"], c["dim"], s["ld"]
        if "desc" not in s:
            s["desc"] = pb.make_rope_desc(dt, n, T, H, D, _pairs(c), int(c["interleaved"]), int(c["inverse"]), ld, T * ld, ld, T * ld)
        pb.parle_k_rope(s["desc"], s["x"], s["positions"], s["freqs"], s["out"])
        return s["out"][..., :H * D]
    if kind.startswith("attention"):
        n, T, H, K, D, ld = c["n"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], s["ld"]
        if "desc" not in s:
            s["desc"] = pb.parle_attention_desc(dt, n, T, c["sequences"], H, K, D, c["window"], c["sinks"], D ** -0.5, ld, T * ld, ld, T * ld, H * D, T * H * D)
            s["scratch"] = scratch(pb.parle_k_attention_scratch_bytes(s["desc"])) if kind == "attention_grad" else None
        q, k, v = s["qkv"], s["qkv"][..., H * D:], s["qkv"][..., (H + K) * D:]
        if kind == "attention":
            pb.parle_k_attention_forward(s["desc"], q, k, v, s["offsets"], s["out"], s["lse"])
            return {"out": s["out"], "lse": s["lse"]}
        dq, dk, dv = s["dqkv"], s["dqkv"][..., H * D:], s["dqkv"][..., (H + K) * D:]
        pb.parle_k_attention_backward(s["desc"], q, k, v, s["offsets"], s["out"], s["lse"], s["dout"], s["scratch"], dq, dk, dv)
        return {"dq": dq[..., :H * D], "dk": dk[..., :K * D], "dv": dv}
    if kind in ("store", "decode"):
        B, K, D, ld = c["sequences"], c["kv_heads"], c["dim"], s["ld"]
        H = c.get("heads", K)
        if "desc" not in s:
            s["desc"] = pb.parle_cache_desc(dt, B, c["capacity"], H, K, D, c["window"], c["sinks"], D ** -0.5, ld, ld, H * D)
            s["scratch"] = scratch(pb.parle_k_decode_scratch_bytes(s["desc"])) if kind == "decode" else None
        if kind == "store":
            pb.parle_k_attention_store(s["desc"], c["tokens"], s["kv"], s["kv"][:, K * D:], s["offsets"], s["lengths"], s["k_cache"], s["v_cache"])
            return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        q, k, v = s["qkv"], s["qkv"][:, H * D:], s["qkv"][:, (H + K) * D:]
        pb.parle_k_attention_decode(s["desc"], q, k, v, s["lengths"], s["scratch"], s["k_cache"], s["v_cache"], s["out"])
        return {"out": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if "desc" not in s:
        s["desc"] = pb.parle_sample_desc(dt, c["n"], c["rows"], c["classes"], c["ld"])
        s["scratch"] = scratch(pb.parle_k_sample_scratch_bytes(s["desc"]))
    pb.parle_k_sample(s["desc"], s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["scratch"], s["tokens"], s["kept"], s["logp"])
    return {"tokens": s["tokens"], "kept": s["kept"], "logp": s["logp"]}


def _starts(T, offsets):
    """For every row the first row of its sequence, [n, T]; -1 for rows outside."""
    i = torch.arange(T, device=DEVICE)
    b = (i[None, :, None] >= offsets[:, None, :]).sum(-1)                       # 1 + the sequence, as offsets ascend
    inside = (b > 0) & (b < offsets.shape[1])
    return torch.where(inside, torch.gather(offsets.long(), 1, (b - 1).clamp(min=0)), torch.full_like(b, -1))


def _visible(c, offsets):
    """[n, 1, query, key]."""
    T = c["tokens"]
    start = _starts(T, offsets)
    i, j, a = torch.arange(T, device=DEVICE)[None, :, None], torch.arange(T, device=DEVICE)[None, None, :], start[:, :, None]
    see = (j <= i) & (j >= a) & (a >= 0)
    if c["window"]:
        see &= (j > i - c["window"]) | (j < a + c["sinks"])
    return see[:, None], start


def _heads(rows, first, count, dim, repeat=1):
    """Heads of rows [..., T, ld] as [n, count * repeat, T, dim] in 32 bits."""
    x = rows[..., first * dim:(first + count) * dim].float().unflatten(-1, (count, dim)).transpose(1, 2)
    return x.repeat_interleave(repeat, 1).contiguous()


def _attention(c, s):
    """The forward pass in elementary operations."""
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    see, start = _visible(c, s["offsets"])
    q, k, v = _heads(s["qkv"], 0, H, D), _heads(s["qkv"], H, K, D, H // K), _heads(s["qkv"], H + K, K, D, H // K)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = x.sub_(m).exp_()
    z = e.sum(-1, keepdim=True)
    out = torch.matmul(e, v) / torch.where(z > 0, z, torch.ones_like(z))
    return out.transpose(1, 2).flatten(2).to(s["qkv"].dtype), (torch.log(z) + m)[..., 0]


def _slots(c, lengths):
    """For every slot of a cache the token it holds, [sequences, capacity]; negative where it holds none."""
    s, ring = torch.arange(c["capacity"], device=DEVICE)[None], c["capacity"] - c["sinks"]
    last = (lengths.long() - 1)[:, None]
    newest = last - (last - s) % ring                      # the same residue, at most `last`
    return torch.where(s < c["sinks"], torch.where(s <= last, s, torch.full_like(s, -1)), torch.where(newest >= c["sinks"], newest, torch.full_like(newest, -1)))


def _slot(c, position):
    return torch.where(position < c["sinks"], position, c["sinks"] + (position - c["sinks"]) % (c["capacity"] - c["sinks"]))


def _plain(s):
    """The same in elementary torch operations, in 32 bits (64 for angles and for the sampler's sums), rounded once at the end."""
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rope":
        n, T, H, D, half = c["n"], c["tokens"], c["heads"], c["dim"], c["turned"] // 2
        axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEVICE), torch.tensor(_pairs(c), device=DEVICE))
        angle = s["positions"].double()[..., axis] * s["freqs"].double()
        cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None] * (-1.0 if c["inverse"] else 1.0)
        x = s["x"][..., :H * D].unflatten(-1, (H, D))
        a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if c["interleaved"] else (x[..., :half], x[..., half:2 * half])
        a, b = a.float(), b.float()
        u, v = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack((u, v), -1).flatten(-2) if c["interleaved"] else torch.cat((u, v), -1)
        return torch.cat((turned, x[..., 2 * half:].float()), -1).to(s["x"].dtype).flatten(2)
    if kind == "attention":
        out, lse = _attention(c, s)
        return {"out": out, "lse": lse}
    if kind == "attention_grad":
        n, T, H, K, D = c["n"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        see, _ = _visible(c, s["offsets"])
        q, k, v = _heads(s["qkv"], 0, H, D), _heads(s["qkv"], H, K, D, H // K), _heads(s["qkv"], H + K, K, D, H // K)
        o, do = _heads(s["out"], 0, H, D), _heads(s["dout"], 0, H, D)
        some = (s["lse"] > -math.inf)[..., None]
        base = torch.where(some, s["lse"][..., None], torch.zeros_like(s["lse"])[..., None])
        p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).sub_(base).masked_fill_(~see, -math.inf).exp_()
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
        ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((o * do).sum(-1, keepdim=True)).mul_(p).mul_(D ** -0.5)
        dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
        shared = lambda t: t.unflatten(1, (K, H // K)).sum(2)  # noqa: E731
        rows = lambda t: t.transpose(1, 2).flatten(2).to(s["qkv"].dtype)  # noqa: E731
        return {"dq": rows(dq), "dk": rows(shared(dk)), "dv": rows(shared(dv))}
    if kind == "store":
        K, D, T = c["kv_heads"], c["dim"], c["tokens"]
        i = torch.arange(T, device=DEVICE)
        b = (i[:, None] >= s["offsets"][None]).sum(-1) - 1
        inside = (b >= 0) & (b < c["sequences"])
        b = b.clamp(max=c["sequences"] - 1)
        length = s["lengths"].long()[b]
        position = length - (s["offsets"].long()[b + 1] - i)
        inside &= (position >= 0) & ((position < c["sinks"]) | (position >= length - (c["capacity"] - c["sinks"])))
        i, b, position = i[inside], b[inside], position[inside]
        for cache, first in ((s["k_cache"], 0), (s["v_cache"], K * D)):
            cache[b, :, _slot(c, position)] = s["kv"][i, first:first + K * D].unflatten(-1, (K, D))
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "decode":
        B, H, K, D = c["sequences"], c["heads"], c["kv_heads"], c["dim"]
        b, last = torch.arange(B, device=DEVICE), s["lengths"].long() - 1
        s["k_cache"][b, :, _slot(c, last)] = s["qkv"][:, H * D:(H + K) * D].unflatten(-1, (K, D))
        s["v_cache"][b, :, _slot(c, last)] = s["qkv"][:, (H + K) * D:].unflatten(-1, (K, D))
        position = _slots(c, s["lengths"])
        see = position >= 0
        if c["window"]:
            see &= (position > (last - c["window"])[:, None]) | (position < c["sinks"])
        q = s["qkv"][:, :H * D].float().reshape(B * K, H // K, D)
        x = torch.matmul(q, s["k_cache"].float().reshape(B * K, c["capacity"], D).transpose(1, 2).contiguous()).mul_(D ** -0.5)
        x = x.reshape(B, H, -1).masked_fill_(~see[:, None], -math.inf)
        e = torch.exp(x - x.amax(-1, keepdim=True))
        out = torch.matmul(e.reshape(B * K, H // K, -1), s["v_cache"].float().reshape(B * K, -1, D)).reshape(B, H, D) / e.sum(-1, keepdim=True)
        return {"out": out.reshape(B, H * D).to(s["qkv"].dtype), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    x, order = torch.sort(s["logits"][..., :c["classes"]], dim=-1, descending=True, stable=True)
    x = x.double()
    greedy = (s["temperature"] <= 0)[..., None]
    t = torch.where(greedy, torch.ones_like(s["temperature"])[..., None], s["temperature"][..., None]).double()
    w = torch.where(greedy, torch.arange(c["classes"], device=DEVICE) == 0, torch.exp((x - x[..., :1]) / t))
    rank = torch.arange(c["classes"], device=DEVICE)
    k = torch.where(greedy, torch.ones_like(s["top_k"])[..., None], s["top_k"][..., None])
    keep = (x > -math.inf) & ((rank < k) | (k <= 0))
    total = torch.cumsum(w * keep, -1)
    p = s["top_p"][..., None].double()
    before = total - w * keep
    keep &= (before < p * total[..., -1:]) | (p >= 1)
    keep &= w >= s["min_p"][..., None].double()
    kept = keep.sum(-1)
    total = torch.cumsum(w * keep, -1)
    target = s["uniform"].double()[..., None] * total[..., -1:]
    at = torch.minimum((total <= target).sum(-1), kept - 1)[..., None]
    logp = torch.log(torch.gather(w, -1, at) / total[..., -1:])[..., 0]
    return {"tokens": torch.gather(order, -1, at)[..., 0].to(torch.int32), "kept": kept.to(torch.int32), "logp": logp.float()}


def work(case):
    c, kind, z = case, case["kind"], SIZE[case["dtype"]]
    if kind == "rope":
        n, T, H, D = c["n"], c["tokens"], c["heads"], c["dim"]
        return {"bytes": n * T * (2 * H * D * z + 4 * c["axes"]), "flops": 3 * n * T * H * c["turned"]}
    if kind.startswith("attention"):
        n, T, H, K, D = c["n"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        pairs = sum(_seen(c, o[b + 1] - o[b]) for o in _offsets(c) for b in range(c["sequences"]))
        if kind == "attention":
            return {"bytes": n * T * ((2 * H + 2 * K) * D * z + 4 * H), "flops": 4 * pairs * H * D}
        return {"bytes": n * T * ((4 * H + 4 * K) * D * z + 4 * H), "flops": 10 * pairs * H * D}
    if kind == "store":
        o, ring = _offsets(c)[0], c["capacity"] - c["sinks"]
        rows = sum(min(o[b + 1] - o[b], ring + c["sinks"]) for b in range(c["sequences"]))
        return {"bytes": 4 * rows * c["kv_heads"] * c["dim"] * z, "flops": 0}
    if kind == "decode":
        ring = c["capacity"] - c["sinks"]
        window = min(c["window"] or ring, ring)
        seen = sum(min(t, window + c["sinks"]) for t in _lengths(c))
        B, H, K, D = c["sequences"], c["heads"], c["kv_heads"], c["dim"]
        return {"bytes": z * D * (2 * K * seen + 2 * B * H + 4 * B * K), "flops": 4 * seen * H * D}
    n, R, C = c["n"], c["rows"], c["classes"]
    return {"bytes": n * R * (C * z + 8 * 4), "flops": 6 * n * R * C}


def exact(case, seed):
    """What run() returns, in 64 bits, straight from the definitions."""
    s, c, kind = prepare(case, seed), case, case["kind"]
    if kind == "rope":
        H, D, half = c["heads"], c["dim"], c["turned"] // 2
        sizes = _pairs(c)
        out = s["x"][..., :H * D].double().unflatten(-1, (H, D)).clone()
        first = 0
        for axis, count in enumerate(sizes):
            angle = s["positions"][..., axis].double()[..., None] * s["freqs"][first:first + count].double()
            turn = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)[:, :, None]
            p = torch.arange(first, first + count, device=DEVICE)
            ia, ib = (2 * p, 2 * p + 1) if c["interleaved"] else (p, p + half)
            z = torch.complex(out[..., ia], out[..., ib]) * turn
            out[..., ia], out[..., ib] = z.real, z.imag
            first += count
        return out.flatten(2)
    if kind.startswith("attention"):
        n, T, H, K, D = c["n"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        x, group = s["qkv"], H // K
        qkv = lambda a, h: x[a, :, h * D:(h + 1) * D].double()  # noqa: E731
        out, lse = torch.zeros((n, T, H, D), dtype=torch.float64, device=DEVICE), torch.full((n, H, T), -math.inf, dtype=torch.float64, device=DEVICE)
        grad = torch.zeros((n, T, H + 2 * K, D), dtype=torch.float64, device=DEVICE)
        for a in range(n):
            o = s["offsets"][a].tolist()
            for first, end in zip(o[:-1], o[1:]):
                i = torch.arange(end - first, device=DEVICE)
                hidden = i[None, :] > i[:, None]
                if c["window"]:
                    hidden |= (i[None, :] <= i[:, None] - c["window"]) & (i[None, :] >= c["sinks"])
                for h in range(H if end > first else 0):
                    q, k, v = (qkv(a, m)[first:end] for m in (h, H + h // group, H + K + h // group))
                    score = (q @ k.t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
                    if kind == "attention":
                        lse[a, h, first:end] = torch.logsumexp(score, -1)
                        out[a, first:end, h] = torch.softmax(score, -1) @ v
                        continue
                    p = torch.exp(score - s["lse"][a, h, first:end].double()[:, None])
                    d = s["dout"][a, first:end, h * D:(h + 1) * D].double()
                    delta = (d * s["out"][a, first:end, h * D:(h + 1) * D].double()).sum(-1, keepdim=True)
                    ds = p * (d @ v.t() - delta) / math.sqrt(D)
                    grad[a, first:end, h] = ds @ k
                    grad[a, first:end, H + h // group] += ds.t() @ q
                    grad[a, first:end, H + K + h // group] += p.t() @ d
        if kind == "attention":
            return {"out": out.flatten(2), "lse": lse}
        return {"dq": grad[:, :, :H].flatten(2), "dk": grad[:, :, H:H + K].flatten(2), "dv": grad[:, :, H + K:].flatten(2)}
    if kind == "store":
        K, D, o, lengths = c["kv_heads"], c["dim"], s["offsets"].tolist(), s["lengths"].tolist()
        k, v = s["k_cache"].double(), s["v_cache"].double()
        ring = c["capacity"] - c["sinks"]
        for b in range(c["sequences"]):
            p = torch.arange(lengths[b] - (o[b + 1] - o[b]), lengths[b], device=DEVICE)
            live = (p < c["sinks"]) | (p >= lengths[b] - ring)
            at = torch.where(p < c["sinks"], p, (p - c["sinks"]) % ring + c["sinks"])[live]
            rows = s["kv"][o[b]:o[b + 1]][live].double().view(-1, 2, K, D)
            k[b, :, at], v[b, :, at] = rows[:, 0].transpose(0, 1), rows[:, 1].transpose(0, 1)
        return {"k_cache": k, "v_cache": v}
    if kind == "decode":
        B, H, K, D = c["sequences"], c["heads"], c["kv_heads"], c["dim"]
        ring, window = c["capacity"] - c["sinks"], c["window"] or c["longest"]
        out = torch.empty((B, H, D), dtype=torch.float64, device=DEVICE)
        for b, length in enumerate(s["lengths"].tolist()):
            new = length - 1 if length - 1 < c["sinks"] else (length - 1 - c["sinks"]) % ring + c["sinks"]
            s["k_cache"][b, :, new], s["v_cache"][b, :, new] = s["qkv"][b, H * D:].view(2, K, D)
            p = torch.arange(max(c["sinks"], length - min(window, ring)), length, device=DEVICE)
            at = torch.cat((torch.arange(min(c["sinks"], length), device=DEVICE), (p - c["sinks"]) % ring + c["sinks"]))
            q = s["qkv"][b, :H * D].double().view(K, H // K, D)
            score = torch.matmul(q, s["k_cache"][b, :, at].double().transpose(1, 2)) / math.sqrt(D)
            out[b] = torch.matmul(torch.softmax(score, -1), s["v_cache"][b, :, at].double()).view(H, D)
        return {"out": out.view(B, H * D), "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
    n, R, C = c["n"], c["rows"], c["classes"]
    tokens, kept, logp = (torch.zeros((n, R), dtype=d, device=DEVICE) for d in (torch.int32, torch.int32, torch.float64))
    for a in range(n):
        for r in range(R):
            x = s["logits"][a, r, :C].double()
            t = float(s["temperature"][a, r])
            if t <= 0:
                tokens[a, r], kept[a, r], logp[a, r] = x.argmax(), 1, 0.0
                continue
            ids = torch.argsort(x, descending=True, stable=True)
            ids = ids[:int((x > -math.inf).sum())]
            if c["top_k"] > 0:
                ids = ids[:c["top_k"]]
            q = torch.softmax(x[ids] / t, 0)
            if c["top_p"] < 1:
                ids = ids[:1 + int((torch.cumsum(q, 0) < float(s["top_p"][a, r])).sum())]
            q = q[:len(ids)]
            ids = ids[q / q[0] >= float(s["min_p"][a, r])]
            logq = torch.log_softmax(x[ids] / t, 0)
            at = min(int((torch.cumsum(torch.exp(logq), 0) <= float(s["uniform"][a, r])).sum()), len(ids) - 1)
            tokens[a, r], kept[a, r], logp[a, r] = ids[at], len(ids), logq[at]
    return {"tokens": tokens, "kept": kept, "logp": logp}
