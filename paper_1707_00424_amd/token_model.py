"""A small token model trained by Parle: the token-model operators and the update kernels together, as a program uses them.

n replicas predict the next token: embedding, ``layers`` residual blocks of an RMS norm and a linear layer, a last norm and the classes; where
``attention`` is given, each block begins with a norm, rotary positions and attention over its sequence, else the present token is all
that is seen.  Every linear layer runs in 8 bits, forward and backward.  Parameters are segments of the fp32 rows
[n, n_pad] of a flat :class:`binding.Parle` context; the operators read them there and write their gradients into the rows of
``grad``, so an inner step (8a), (8b) follows the backward pass without a copy.

    python -m paper_1707_00424_amd.token_model          # trains on a synthetic source, then prints alternatives for some tokens and how prompts go on
    python -m paper_1707_00424_amd.token_model --attention
"""
from __future__ import annotations

import dataclasses
import math
import sys

from . import binding as pb

EPS = 1e-6


def _up(v, to):
    return -(-v // to) * to


class _Codes:
    """8-bit codes and scales of a tensor [n, rows, cols] and of its transpose."""

    def __init__(self, torch, device, n, rows, cols, block):
        def make(*s):
            return torch.zeros(s, dtype=torch.uint8, device=device)
        self.q, self.s = make(n, rows, _up(cols, 16)), make(n, _up(rows, block) // block, _up(_up(cols, 128) // 128, 4))
        self.qt, self.st = make(n, cols, _up(rows, 16)), make(n, _up(cols, block) // block, _up(_up(rows, 128) // 128, 4))


class _Linear:
    """A linear layer [rows, depth] in 8 bits: its weights' codes and the descriptors of its calls for ``count`` rows of n replicas."""

    def __init__(self, torch, device, n, count, rows, depth, stride):
        self.rows, self.depth = rows, depth
        self.w8 = _Codes(torch, device, n, rows, depth, 128)
        self.quant_w = pb.parle_quant_desc(0, 128, n, rows, depth, depth, stride)
        self.quant_in = pb.parle_quant_desc(1, 1, n, count, depth, depth, count * depth)
        self.quant_out = pb.parle_quant_desc(1, 1, n, count, rows, rows, count * rows)
        self.forward = pb.parle_fp8_desc(1, 128, 0, n, count, rows, depth, rows, count * rows)
        self.input = pb.parle_fp8_desc(1, 128, 0, n, count, depth, rows, depth, count * depth)
        self.weight = pb.parle_fp8_desc(0, 1, 0, n, rows, depth, count, depth, stride)

    def scratch_bytes(self):
        return max(pb.parle_k_fp8_scratch_bytes(d) for d in (self.forward, self.input, self.weight))


@dataclasses.dataclass(frozen=True)
class Heads:
    """What attention in a :class:`TokenModel` is made of: ``heads`` query heads, ``kv_heads`` of keys and values, ``dim`` elements each; the last ``window``
    tokens (0: all) and the first ``sinks`` are seen; ``sequences`` of equal length lie one behind the other in a replica's tokens."""

    heads: int = 4
    kv_heads: int = 2
    dim: int = 32
    window: int = 0
    sinks: int = 0
    sequences: int = 1


class TokenModel:
    """``tokens``: positions per replica and step.  The context's rows hold, one behind the other and each at a multiple of 16 bytes:
    the table [vocab, dim], per block a norm's weights [dim] and a layer's [dim, dim], the last norm's, the classes' [vocab, dim].  With
    ``attention`` (:class:`Heads`) every block begins with a norm, queries, keys and values, and the layer behind them."""

    def __init__(self, n, tokens, vocab, dim, layers=2, device="cuda:0", seed=0, attention=None, **parle):
        import torch
        self.torch, self.n, self.T, self.V, self.D, self.L = torch, n, tokens, vocab, dim, layers
        self.A = A = attention
        self.at, end = {}, 0
        width = (A.heads + 2 * A.kv_heads) * A.dim if A else 0
        segments = [("table", vocab * dim)]
        for i in range(layers):
            if A:
                segments += [(f"norm_a{i}", dim), (f"qkv{i}", width * dim), (f"out{i}", dim * A.heads * A.dim)]
            segments += [(f"norm{i}", dim), (f"w{i}", dim * dim)]
        for name, size in segments + [("norm", dim), ("classes", vocab * dim)]:
            self.at[name] = (end, size)
            end += _up(size, 4)
        g = torch.Generator().manual_seed(seed)
        x0 = torch.zeros(n, end)
        for name, (at, size) in self.at.items():
            # all replicas begin at one point, as the reference of (8d) does
            scale = {"t": dim ** -0.5, "n": 0.0}.get(name[0], dim ** -0.5)
            x0[:, at:at + size] = torch.randn(size, generator=g) * scale + (1.0 if name.startswith("norm") else 0.0)
        cfg = dict(L=25, eta_inner=0.5, eta_outer=0.5, momentum=0.9, gamma0=0.01, rho0=0.1, scoping_B=100, xa_mode=1, fuse_outer=1)
        self.parle = pb.Parle(pb.make_config(model=pb.MODEL_FLAT, n_replicas=n, n_params=end, **(cfg | parle)), x0, device=device)
        self.parle.grad.zero_()
        self.rows = self.parle.sizes.n_pad

        def bf(*s):
            return torch.empty(s, dtype=torch.bfloat16, device=device)

        def f32(*s):
            return torch.empty(s, device=device)

        T, V, D, rs = tokens, vocab, dim, self.rows
        linear = lambda rows, depth: _Linear(torch, device, n, T, rows, depth, rs)  # noqa: E731
        self.x = bf(n, T, D)
        self.delta = [bf(n, T, D) for _ in range(layers)]
        self.h, self.y = [bf(n, T, D) for _ in range(layers + 1)], [bf(n, T, D) for _ in range(layers + 1)]
        self.rstd = [f32(n, T) for _ in range(layers + 1)]
        self.y8 = [_Codes(torch, device, n, T, D, 1) for _ in range(layers + 1)]
        self.linear = [linear(r, D) for r in [D] * layers + [V]]
        self.d8, self.g8 = _Codes(torch, device, n, T, D, 1), _Codes(torch, device, n, T, V, 1)
        self.logits = bf(n, T, V)
        self.logp, self.entropy, self.lse, self.dlogp = f32(n, T), f32(n, T), f32(n, T), f32(n, T)
        self.dy, self.dh, self.dh2 = bf(n, T, D), bf(n, T, D), bf(n, T, D)
        # descriptors: sizes are fixed, so that they and the scratch are made once
        self.embed = pb.parle_embed_desc(1, 0, n, T, V, D, rs, math.sqrt(D))
        self.norm = pb.parle_norm_desc(1, 0, n, T, D, rs, EPS)
        self.scores = pb.parle_logprob_desc(1, n, T, V, 0, V)
        need = [pb.parle_k_embed_scratch_bytes(self.embed), pb.parle_k_rmsnorm_scratch_bytes(self.norm), pb.parle_k_logprob_scratch_bytes(self.scores)]
        need += [lin.scratch_bytes() for lin in self.linear]
        if A:
            if T % A.sequences:
                raise ValueError(f"{T} tokens are not {A.sequences} sequences of equal length")
            W, H = width, A.heads * A.dim
            self.a = [dict(h=bf(n, T, D), y=bf(n, T, D), rstd=f32(n, T), y8=_Codes(torch, device, n, T, D, 1), qkv=bf(n, T, W), att=bf(n, T, H), lse=f32(n, A.heads, T),
                           delta=bf(n, T, D), to_qkv=linear(W, D), to_out=linear(D, H)) for _ in range(layers)]
            self.att8, self.qkv8 = _Codes(torch, device, n, T, H, 1), _Codes(torch, device, n, T, W, 1)
            self.datt, self.dqkv = bf(n, T, H), bf(n, T, W)
            length = T // A.sequences
            self.offsets = (torch.arange(A.sequences + 1, dtype=torch.int32, device=device) * length).expand(n, -1).contiguous()
            self.positions = (torch.arange(T, dtype=torch.int32, device=device) % length).reshape(1, T, 1).expand(n, -1, -1).contiguous()
            self.freqs = 10000.0 ** (-torch.arange(A.dim // 2, device=device) / (A.dim / 2))
            self.turn, self.turn_back = (self._rope(n, T, inverse) for inverse in (0, 1))
            self.attend = pb.parle_attention_desc(1, n, T, A.sequences, A.heads, A.kv_heads, A.dim, A.window, A.sinks, A.dim ** -0.5, W, T * W, W, T * W, H, T * H)
            need += [pb.parle_k_attention_scratch_bytes(self.attend)] + [x[k].scratch_bytes() for x in self.a[:1] for k in ("to_qkv", "to_out")]
        self.scratch = torch.empty(max(need + [16]), dtype=torch.uint8, device=device)

    def _rope(self, n, count, inverse=0):
        """Queries and keys, which lie side by side, turned in place by one axis."""
        A = self.A
        W = (A.heads + 2 * A.kv_heads) * A.dim
        return pb.make_rope_desc(1, n, count, A.heads + A.kv_heads, A.dim, [A.dim // 2], 0, inverse, W, count * W, W, count * W)

    def _parts(self, qkv):
        """Queries, keys and values of rows that hold all three."""
        A = self.A
        return qkv, qkv[..., A.heads * A.dim:], qkv[..., (A.heads + A.kv_heads) * A.dim:]

    def segment(self, rows, name):
        """A segment of parameter-like rows (``parle.y``, ``parle.grad``) as a view; an operator takes its stride separately."""
        at, size = self.at[name]
        return rows[:, at:at + size]

    def _names(self, i):
        return (f"norm{i}", f"w{i}") if i < self.L else ("norm", "classes")

    def _linear_forward(self, lin, w, codes, out):
        b = lin.w8
        pb.parle_k_fp8_quantize(lin.quant_w, w, b.q, b.s, b.qt, b.st)
        pb.parle_k_fp8_matmul(lin.forward, codes.q, codes.s, b.q, b.s, None, self.scratch, out)

    def _linear_backward(self, lin, codes, dcodes, x, dout, dx, dw):
        """From the input x, its codes' buffer and dout: dx and dw, through dcodes, a buffer for the codes of dout."""
        pb.parle_k_fp8_quantize(lin.quant_out, dout, dcodes.q, dcodes.s, dcodes.qt, dcodes.st)
        pb.parle_k_fp8_quantize(lin.quant_in, x, None, None, codes.qt, codes.st)
        pb.parle_k_fp8_matmul(lin.input, dcodes.q, dcodes.s, lin.w8.qt, lin.w8.st, None, self.scratch, dx)
        pb.parle_k_fp8_matmul(lin.weight, dcodes.qt, dcodes.st, codes.qt, codes.st, None, self.scratch, dw)

    def forward(self, tokens, labels):
        """Fills ``logp`` and ``entropy`` for tokens, labels int32 [n, tokens]; -1 is padding in both."""
        y = self.parle.y
        pb.parle_k_embed_forward(self.embed, self.segment(y, "table"), tokens, self.x)
        x, resid = self.x, None
        for i in range(self.L + 1):
            if self.A and i < self.L:
                a = self.a[i]
                c = a["y8"]
                pb.parle_k_rmsnorm_forward(self.norm, x, resid, self.segment(y, f"norm_a{i}"), a["h"], a["y"], c.q, c.s, a["rstd"])
                self._linear_forward(a["to_qkv"], self.segment(y, f"qkv{i}"), c, a["qkv"])
                pb.parle_k_rope(self.turn, a["qkv"], self.positions, self.freqs, a["qkv"])
                pb.parle_k_attention_forward(self.attend, *self._parts(a["qkv"]), self.offsets, a["att"], a["lse"])
                pb.parle_k_fp8_quantize(a["to_out"].quant_in, a["att"], self.att8.q, self.att8.s, None, None)
                self._linear_forward(a["to_out"], self.segment(y, f"out{i}"), self.att8, a["delta"])
                x, resid = a["delta"], a["h"]
            norm, w = self._names(i)
            c = self.y8[i]
            pb.parle_k_rmsnorm_forward(self.norm, x, resid, self.segment(y, norm), self.h[i], self.y[i], c.q, c.s, self.rstd[i])
            out = self.delta[i] if i < self.L else self.logits
            self._linear_forward(self.linear[i], self.segment(y, w), c, out)
            x, resid = out, self.h[i]
        pb.parle_k_logprob_forward(self.scores, self.logits, labels, self.scratch, self.logp, self.entropy, self.lse, None, None)

    def backward(self, tokens, labels):
        """Gradient of the mean of -logp over the labels that are given, into ``parle.grad``."""
        grad, y = self.parle.grad, self.parle.y
        given = (labels >= 0).sum(1, keepdim=True).clamp(min=1)
        self.dlogp.copy_((-1.0 / given).expand_as(self.dlogp))
        # over the logits: nobody needs them any more
        pb.parle_k_logprob_backward(self.scores, self.logits, labels, self.lse, None, self.dlogp, None, self.logits)
        out, dresid = self.logits, None
        for i in range(self.L, -1, -1):
            norm, w = self._names(i)
            self._linear_backward(self.linear[i], self.y8[i], self.d8 if i < self.L else self.g8, self.y[i], out, self.dy, self.segment(grad, w))
            dx = self.dh if dresid is not self.dh else self.dh2
            pb.parle_k_rmsnorm_backward(self.norm, self.h[i], self.segment(y, norm), self.rstd[i], self.dy, dresid, self.scratch, dx, self.segment(grad, norm))
            out = dresid = dx
            if self.A and i < self.L:
                a = self.a[i]
                self._linear_backward(a["to_out"], self.att8, self.d8, a["att"], out, self.datt, self.segment(grad, f"out{i}"))
                pb.parle_k_attention_backward(self.attend, *self._parts(a["qkv"]), self.offsets, a["att"], a["lse"], self.datt, self.scratch, *self._parts(self.dqkv))
                pb.parle_k_rope(self.turn_back, self.dqkv, self.positions, self.freqs, self.dqkv)
                self._linear_backward(a["to_qkv"], a["y8"], self.qkv8, a["y"], self.dqkv, self.dy, self.segment(grad, f"qkv{i}"))
                dx = self.dh if dresid is not self.dh else self.dh2
                pb.parle_k_rmsnorm_backward(self.norm, a["h"], self.segment(y, f"norm_a{i}"), a["rstd"], self.dy, dresid, self.scratch, dx, self.segment(grad, f"norm_a{i}"))
                out = dresid = dx
        pb.parle_k_embed_backward(self.embed, tokens, out, self.scratch, self.segment(grad, "table"))

    def step(self, tokens, labels):
        """One inner step of every replica on its own tokens."""
        self.forward(tokens, labels)
        self.backward(tokens, labels)
        self.parle.parle_inner_step()

    def _reference_logits(self, tokens, positions=None, attend=None):
        """Logits bf16 [1, count, vocab] behind ``tokens`` (int32 [count]), by the reference x_ref: single rows through the same operators.
        ``attend(i, qkv, out)`` is block i's attention."""
        torch, count, D, V, A = self.torch, tokens.numel(), self.D, self.V, self.A
        y, dev = self.parle.x_ref[None], tokens.device
        stride = self.rows

        def bf(cols):
            return torch.empty((1, count, cols), dtype=torch.bfloat16, device=dev)

        def linear(name, rows, depth, codes):
            b = _Codes(torch, dev, 1, rows, depth, 128)
            pb.parle_k_fp8_quantize(pb.parle_quant_desc(0, 128, 1, rows, depth, depth, stride), self.segment(y, name), b.q, b.s, None, None)
            desc = pb.parle_fp8_desc(1, 128, 0, 1, count, rows, depth, rows, count * rows)
            scratch = torch.empty(max(16, pb.parle_k_fp8_scratch_bytes(desc)), dtype=torch.uint8, device=dev)
            out = bf(rows)
            pb.parle_k_fp8_matmul(desc, codes.q, codes.s, b.q, b.s, None, scratch, out)
            return out

        def norm(name, x, resid):
            h, a = bf(D), _Codes(torch, dev, 1, count, D, 1)
            pb.parle_k_rmsnorm_forward(pb.parle_norm_desc(1, 0, 1, count, D, stride, EPS), x, resid, self.segment(y, name), h, None, a.q, a.s, None)
            return h, a

        x, resid = bf(D), None
        pb.parle_k_embed_forward(pb.parle_embed_desc(1, 0, 1, count, V, D, stride, math.sqrt(D)), self.segment(y, "table"), tokens.reshape(1, -1), x)
        for i in range(self.L + 1):
            if A and i < self.L:
                h, a = norm(f"norm_a{i}", x, resid)
                qkv = linear(f"qkv{i}", (A.heads + 2 * A.kv_heads) * A.dim, D, a)
                pb.parle_k_rope(self._rope(1, count), qkv, positions, self.freqs, qkv)
                att, c = bf(A.heads * A.dim), _Codes(torch, dev, 1, count, A.heads * A.dim, 1)
                attend(i, qkv, att)
                pb.parle_k_fp8_quantize(pb.parle_quant_desc(1, 1, 1, count, A.heads * A.dim, A.heads * A.dim, count * A.heads * A.dim), att, c.q, c.s, None, None)
                x, resid = linear(f"out{i}", D, A.heads * A.dim, c), h
            name, w = self._names(i)
            h, a = norm(name, x, resid)
            x, resid = linear(w, D if i < self.L else V, D, a), h
        return x

    def alternatives(self, tokens, top=5):
        """The ``top`` most likely next tokens after each of ``tokens`` (int32 [count]), each the first of its sequence, and their log probabilities, by
        the reference x_ref."""
        torch, count, V, dev = self.torch, tokens.numel(), self.V, tokens.device
        A = self.A

        def alone(i, qkv, out):
            W, H = qkv.shape[-1], out.shape[-1]
            desc = pb.parle_attention_desc(1, 1, count, count, A.heads, A.kv_heads, A.dim, A.window, A.sinks, A.dim ** -0.5, W, count * W, W, count * W, H, count * H)
            pb.parle_k_attention_forward(desc, *self._parts(qkv), torch.arange(count + 1, dtype=torch.int32, device=dev), out, None)

        logits = self._reference_logits(tokens, torch.zeros((1, count, 1), dtype=torch.int32, device=dev), alone)
        ids = torch.empty((1, count, top), dtype=torch.int32, device=dev)
        logp, lse = torch.empty((1, count, top), device=dev), torch.empty((1, count), device=dev)
        desc = pb.parle_logprob_desc(1, 1, count, V, top, V)
        scratch = torch.empty(max(16, pb.parle_k_logprob_scratch_bytes(desc)), dtype=torch.uint8, device=dev)
        pb.parle_k_logprob_forward(desc, logits, None, scratch, None, None, lse, ids, logp)
        return ids[0], logp[0]

    def answer(self, prompts, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
        """Tokens behind ``prompts``, a list of int32 tensors: one for each of the numbers ``uniform`` [prompts, count] out of [0, 1), by
        the reference x_ref: int32 [prompts, count].  temperature, top_k, top_p, min_p: [prompts] each, or None.  All may be of any type and on any
        device.  A model with attention keeps rolling caches of sinks + window tokens (all of them without a window); one without sees the last token only."""
        torch, A, V = self.torch, self.A, self.V
        count, B, dev = uniform.shape[1], len(prompts), self.x.device
        if not B or B != uniform.shape[0] or not all(len(p) for p in prompts):
            raise ValueError("answer needs a row of numbers for each prompt, and prompts of one token at least")

        def rule(name, value, dtype):
            if value is None:
                return None
            value = torch.as_tensor(value)
            if value.numel() != B:
                raise ValueError(f"answer needs one {name} for each prompt")
            return value.reshape(B).to(device=dev, dtype=dtype, copy=True).contiguous()  # a tensor of its own is aligned

        temperature, top_p, min_p = (rule(k, v, torch.float32) for k, v in (("temperature", temperature), ("top_p", top_p), ("min_p", min_p)))
        top_k = rule("top_k", top_k if top_k is None else torch.as_tensor(top_k).clamp(-1, V), torch.int32)
        lengths = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=dev)
        offsets = torch.nn.functional.pad(torch.cumsum(lengths, 0, dtype=torch.int32), (1, 0))
        packed = torch.cat(list(prompts)).to(device=dev, dtype=torch.int32)
        total = packed.numel()
        positions = (torch.arange(total, dtype=torch.int32, device=dev) - offsets[:-1].repeat_interleave(lengths)).reshape(1, -1, 1)
        if A:
            W, H = (A.heads + 2 * A.kv_heads) * A.dim, A.heads * A.dim
            # (a cache has a slot behind its sinks, also where a whole answer is no longer than they are)
            capacity = A.sinks + A.window if A.window else max(max(len(p) for p in prompts) + count, A.sinks + 1)
            caches = [[torch.zeros((B, A.kv_heads, capacity, A.dim), dtype=torch.bfloat16, device=dev) for _ in range(2)] for _ in range(self.L)]
            cache = pb.parle_cache_desc(1, B, capacity, A.heads, A.kv_heads, A.dim, A.window, A.sinks, A.dim ** -0.5, W, W, H)
            attention = pb.parle_attention_desc(1, 1, total, B, A.heads, A.kv_heads, A.dim, A.window, A.sinks, A.dim ** -0.5, W, total * W, W, total * W, H, total * H)
            scratch = torch.empty(max(16, pb.parle_k_decode_scratch_bytes(cache)), dtype=torch.uint8, device=dev)

        def prompt(i, qkv, out):
            q, k, v = self._parts(qkv)
            pb.parle_k_attention_forward(attention, q, k, v, offsets, out, None)
            pb.parle_k_attention_store(cache, total, k, v, offsets, lengths, *caches[i])

        def token(i, qkv, out):
            pb.parle_k_attention_decode(cache, *self._parts(qkv), lengths, scratch, *caches[i], out)

        desc = pb.parle_sample_desc(1, 1, B, V, V)
        sampling = torch.empty(max(16, pb.parle_k_sample_scratch_bytes(desc)), dtype=torch.uint8, device=dev)
        chosen = torch.empty((count, B), dtype=torch.int32, device=dev)
        numbers = uniform.to(device=dev, dtype=torch.float32).t().contiguous()
        logits = self._reference_logits(packed, positions, prompt)[:, (offsets[1:] - 1).long()].contiguous()
        for step in range(count):
            # each step's row of numbers and tokens is copied: rows of B begin anywhere, and a tensor of its own is aligned
            into, u = torch.empty(B, dtype=torch.int32, device=dev), numbers[step].clone()
            pb.parle_k_sample(desc, logits, u, temperature, top_k, top_p, min_p, sampling, into, None, None)
            chosen[step] = into
            if step + 1 < count:
                lengths += 1
                logits = self._reference_logits(into, (lengths - 1).reshape(1, B, 1), token)
        return chosen.t().contiguous()


def source(torch, vocab, seed=0, device="cuda:0"):
    """A synthetic source: after token t comes (7 t + 3) mod vocab with probability 3/4, any token otherwise.  batch(n, tokens)."""
    g = torch.Generator(device=device).manual_seed(seed)

    def batch(n, tokens):
        t = torch.randint(0, vocab, (n, tokens), generator=g, device=device, dtype=torch.int32)
        other = torch.randint(0, vocab, (n, tokens), generator=g, device=device, dtype=torch.int32)
        follow = torch.rand((n, tokens), generator=g, device=device) < 0.75
        return t, torch.where(follow, (7 * t + 3) % vocab, other)

    return batch


def main(steps=200, n=3, tokens=2048, vocab=512, dim=256, attention=None):
    import time

    import torch
    model = TokenModel(n, tokens, vocab, dim, attention=attention)
    batch = source(torch, vocab)
    start = time.perf_counter()
    for k in range(steps):
        model.step(*batch(n, tokens))
        if (k + 1) % model.parle.cfg.L == 0:
            model.parle.parle_outer_step()
            print(f"step {k + 1}: mean loss {-model.logp.mean().item():.3f} nats, {(time.perf_counter() - start) / (k + 1) * 1e3:.2f} ms a step", flush=True)
    ids, logp = model.alternatives(torch.arange(5, dtype=torch.int32, device="cuda:0"), top=3)
    for t in range(5):
        print(f"after {t}: " + ", ".join(f"{int(i)} (p = {math.exp(float(p)):.2f})" for i, p in zip(ids[t], logp[t])))
    prompts = [torch.tensor([1, 10], dtype=torch.int32), torch.tensor([7], dtype=torch.int32)]
    uniform = torch.rand((2, 8), generator=torch.Generator().manual_seed(1)).cuda()
    for p, a in zip(prompts, model.answer(prompts, uniform, top_p=torch.full((2,), 0.6, device="cuda:0")).tolist()):
        print(f"{p.tolist()} goes on {a}")


if __name__ == "__main__":
    main(attention=Heads(heads=4, kv_heads=2, dim=64, window=64, sinks=2, sequences=8) if "--attention" in sys.argv[1:] else None)
