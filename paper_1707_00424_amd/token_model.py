"""A small token model trained by Parle: the token-model operators and the update kernels together, as a program uses them.

n replicas predict the next token from the present one: embedding, ``layers`` residual blocks of an RMS norm and a linear layer, a
last norm and the classes.  Every linear layer runs in 8 bits, forward and backward.  Parameters are segments of the fp32 rows
[n, n_pad] of a flat :class:`binding.Parle` context; the operators read them there and write their gradients into the rows of
``grad``, so an inner step (8a), (8b) follows the backward pass without a copy.

    python -m paper_1707_00424_amd.token_model          # trains on a synthetic source, then prints alternatives for some tokens
"""
from __future__ import annotations

import math

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


class TokenModel:
    """``tokens``: positions per replica and step.  The context's rows hold, one behind the other and each at a multiple of 16 bytes:
    the table [vocab, dim], per block a norm's weights [dim] and a layer's [dim, dim], the last norm's, the classes' [vocab, dim]."""

    def __init__(self, n, tokens, vocab, dim, layers=2, device="cuda:0", seed=0, **parle):
        import torch
        self.torch, self.n, self.T, self.V, self.D, self.L = torch, n, tokens, vocab, dim, layers
        self.at, end = {}, 0
        segments = [("table", vocab * dim)] + [s for i in range(layers) for s in ((f"norm{i}", dim), (f"w{i}", dim * dim))]
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
        self.x = bf(n, T, D)
        self.delta = [bf(n, T, D) for _ in range(layers)]
        self.h, self.y = [bf(n, T, D) for _ in range(layers + 1)], [bf(n, T, D) for _ in range(layers + 1)]
        self.rstd = [f32(n, T) for _ in range(layers + 1)]
        self.y8 = [_Codes(torch, device, n, T, D, 1) for _ in range(layers + 1)]
        self.w8 = [_Codes(torch, device, n, D, D, 128) for _ in range(layers)] + [_Codes(torch, device, n, V, D, 128)]
        self.d8, self.g8 = _Codes(torch, device, n, T, D, 1), _Codes(torch, device, n, T, V, 1)
        self.logits = bf(n, T, V)
        self.logp, self.entropy, self.lse, self.dlogp = f32(n, T), f32(n, T), f32(n, T), f32(n, T)
        self.dy, self.dh, self.dh2 = bf(n, T, D), bf(n, T, D), bf(n, T, D)
        # descriptors: sizes are fixed, so that they and the scratch are made once
        self.embed = pb.parle_embed_desc(1, 0, n, T, V, D, rs, math.sqrt(D))
        self.norm = pb.parle_norm_desc(1, 0, n, T, D, rs, EPS)
        self.scores = pb.parle_logprob_desc(1, n, T, V, 0, V)
        self.quant_y, self.quant_g = pb.parle_quant_desc(1, 1, n, T, D, D, T * D), pb.parle_quant_desc(1, 1, n, T, V, V, T * V)
        self.quant_w = [pb.parle_quant_desc(0, 128, n, r, D, D, rs) for r in [D] * layers + [V]]
        self.forward_of = [pb.parle_fp8_desc(1, 128, 0, n, T, r, D, r, T * r) for r in [D] * layers + [V]]
        self.input_of = [pb.parle_fp8_desc(1, 128, 0, n, T, D, r, D, T * D) for r in [D] * layers + [V]]
        self.weight_of = [pb.parle_fp8_desc(0, 1, 0, n, r, D, T, D, rs) for r in [D] * layers + [V]]
        need = [pb.parle_k_embed_scratch_bytes(self.embed), pb.parle_k_rmsnorm_scratch_bytes(self.norm), pb.parle_k_logprob_scratch_bytes(self.scores)]
        need += [pb.parle_k_fp8_scratch_bytes(d) for d in self.forward_of + self.input_of + self.weight_of]
        self.scratch = torch.empty(max(need + [16]), dtype=torch.uint8, device=device)

    def segment(self, rows, name):
        """A segment of parameter-like rows (``parle.y``, ``parle.grad``) as a view; an operator takes its stride separately."""
        at, size = self.at[name]
        return rows[:, at:at + size]

    def _names(self, i):
        return (f"norm{i}", f"w{i}") if i < self.L else ("norm", "classes")

    def forward(self, tokens, labels):
        """Fills ``logp`` and ``entropy`` for tokens, labels int32 [n, tokens]; -1 is padding in both."""
        y = self.parle.y
        pb.parle_k_embed_forward(self.embed, self.segment(y, "table"), tokens, self.x)
        x, resid = self.x, None
        for i in range(self.L + 1):
            norm, w = self._names(i)
            a, b = self.y8[i], self.w8[i]
            pb.parle_k_rmsnorm_forward(self.norm, x, resid, self.segment(y, norm), self.h[i], self.y[i], a.q, a.s, self.rstd[i])
            pb.parle_k_fp8_quantize(self.quant_w[i], self.segment(y, w), b.q, b.s, b.qt, b.st)
            out = self.delta[i] if i < self.L else self.logits
            pb.parle_k_fp8_matmul(self.forward_of[i], a.q, a.s, b.q, b.s, None, self.scratch, out)
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
            a, b, d = self.y8[i], self.w8[i], self.d8 if i < self.L else self.g8
            pb.parle_k_fp8_quantize(self.quant_y if i < self.L else self.quant_g, out, d.q, d.s, d.qt, d.st)
            pb.parle_k_fp8_quantize(self.quant_y, self.y[i], None, None, a.qt, a.st)
            pb.parle_k_fp8_matmul(self.input_of[i], d.q, d.s, b.qt, b.st, None, self.scratch, self.dy)
            pb.parle_k_fp8_matmul(self.weight_of[i], d.qt, d.st, a.qt, a.st, None, self.scratch, self.segment(grad, w))
            dx = self.dh if i % 2 == 0 else self.dh2
            pb.parle_k_rmsnorm_backward(self.norm, self.h[i], self.segment(y, norm), self.rstd[i], self.dy, dresid, self.scratch, dx, self.segment(grad, norm))
            out = dresid = dx
        pb.parle_k_embed_backward(self.embed, tokens, out, self.scratch, self.segment(grad, "table"))

    def step(self, tokens, labels):
        """One inner step of every replica on its own tokens."""
        self.forward(tokens, labels)
        self.backward(tokens, labels)
        self.parle.parle_inner_step()

    def alternatives(self, tokens, top=5):
        """The ``top`` most likely next tokens after each of ``tokens`` (int32 [count]) and their log probabilities, by the reference
        x_ref: single rows through the same operators."""
        torch, count, D, V = self.torch, tokens.numel(), self.D, self.V
        y, dev = self.parle.x_ref[None], tokens.device
        stride = self.rows
        x, h = torch.empty((1, count, D), dtype=torch.bfloat16, device=dev), torch.empty((1, count, D), dtype=torch.bfloat16, device=dev)
        delta, logits = torch.empty_like(x), torch.empty((1, count, V), dtype=torch.bfloat16, device=dev)
        a = _Codes(torch, dev, 1, count, D, 1)
        pb.parle_k_embed_forward(pb.parle_embed_desc(1, 0, 1, count, V, D, stride, math.sqrt(D)), self.segment(y, "table"), tokens.reshape(1, -1), x)
        resid = None
        for i in range(self.L + 1):
            norm, w = self._names(i)
            rows = D if i < self.L else V
            b = _Codes(torch, dev, 1, rows, D, 128)
            into = torch.empty_like(h)
            pb.parle_k_rmsnorm_forward(pb.parle_norm_desc(1, 0, 1, count, D, stride, EPS), x, resid, self.segment(y, norm), into, None, a.q, a.s, None)
            pb.parle_k_fp8_quantize(pb.parle_quant_desc(0, 128, 1, rows, D, D, stride), self.segment(y, w), b.q, b.s, None, None)
            desc = pb.parle_fp8_desc(1, 128, 0, 1, count, rows, D, rows, count * rows)
            scratch = torch.empty(max(16, pb.parle_k_fp8_scratch_bytes(desc)), dtype=torch.uint8, device=dev)
            out = delta if i < self.L else logits
            pb.parle_k_fp8_matmul(desc, a.q, a.s, b.q, b.s, None, scratch, out)
            x, resid, delta = out, into, torch.empty_like(delta)
        ids = torch.empty((1, count, top), dtype=torch.int32, device=dev)
        logp, lse = torch.empty((1, count, top), device=dev), torch.empty((1, count), device=dev)
        desc = pb.parle_logprob_desc(1, 1, count, V, top, V)
        scratch = torch.empty(max(16, pb.parle_k_logprob_scratch_bytes(desc)), dtype=torch.uint8, device=dev)
        pb.parle_k_logprob_forward(desc, logits, None, scratch, None, None, lse, ids, logp)
        return ids[0], logp[0]


def source(torch, vocab, seed=0, device="cuda:0"):
    """A synthetic source: after token t comes (7 t + 3) mod vocab with probability 3/4, any token otherwise.  batch(n, tokens)."""
    g = torch.Generator(device=device).manual_seed(seed)

    def batch(n, tokens):
        t = torch.randint(0, vocab, (n, tokens), generator=g, device=device, dtype=torch.int32)
        other = torch.randint(0, vocab, (n, tokens), generator=g, device=device, dtype=torch.int32)
        follow = torch.rand((n, tokens), generator=g, device=device) < 0.75
        return t, torch.where(follow, (7 * t + 3) % vocab, other)

    return batch


def main(steps=200, n=3, tokens=2048, vocab=512, dim=256):
    import time

    import torch
    model = TokenModel(n, tokens, vocab, dim)
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


if __name__ == "__main__":
    main()
