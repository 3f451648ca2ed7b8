"""Attention, its gradient and its cache in 64 bits on the CPU, with bounds for what the kernels may be off by; used by the GPU tests.

u = 2^-24 is half a step of fp32, H half a step of the tensors' type (2^-8 for bf16).  Scores are sums of D products: off by D u A, where A is
the largest scale * sum |q k| of a row; the exponent's multiply-add and the exponential add 4 u (1 + |t|), |t| <= 1.45 (A + |lse|).  What is
then rounded to the tensors' type on its way into the next product adds H of itself."""
import torch

U = 2.0 ** -24


def half(dtype):
    return 2.0 ** -8 if dtype else U


def visible(tokens, offsets, window, sinks):
    """[query, key] of one replica from the definition, key by key."""
    see = torch.zeros(tokens, tokens, dtype=torch.bool)
    for first, end in zip(offsets[:-1], offsets[1:]):
        for i in range(end - first):
            for_i = torch.arange(i + 1)
            ok = torch.ones(i + 1, dtype=torch.bool)
            if window:
                ok = (for_i > i - window) | (for_i < sinks)
            see[first + i, first:first + i + 1] = ok
    return see


class Head:
    """One query head: q, k, v [T, D] float64 on the CPU."""

    def __init__(self, q, k, v, see, scale, dtype):
        self.q, self.k, self.v, self.see, self.scale, self.h = q, k, v, see, scale, half(dtype)
        T, D = q.shape
        s = (q @ k.t()) * scale
        s = s.masked_fill(~see, -torch.inf)
        self.lse = torch.logsumexp(s, -1)
        some = self.lse > -torch.inf
        self.p = torch.where(see, torch.exp(s - torch.where(some, self.lse, torch.zeros_like(self.lse))[:, None]), torch.zeros_like(s))
        self.out = self.p @ v
        mass = (q.abs() @ k.abs().t()) * scale
        self.a = mass.masked_fill(~see, 0).amax(-1, keepdim=True)
        self.size = torch.where(some, self.lse, torch.zeros_like(self.lse)).abs()[:, None]
        # relative error of a probability before its rounding
        self.eps = (D + 4) * U * self.a + 4 * U * (1 + 1.45 * (self.a + self.size))
        self.n = see.sum(-1, keepdim=True)

    def forward_bounds(self):
        most = self.p @ self.v.abs()
        out = most * (2 * self.eps + self.h + 2 * self.n * U) + self.out.abs() * self.h
        lse = (self.eps + (self.n + 4) * U + 4 * U * self.size)[:, 0]
        return out, lse

    def backward(self, out, lse, dout):
        """dq, dk, dv and their bounds, from out and lse of a forward pass (as stored) and dout."""
        D = self.q.shape[1]
        some = lse > -torch.inf
        s = (self.q @ self.k.t()) * self.scale
        p = torch.where(self.see & some[:, None], torch.exp(s - torch.where(some, lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(s))
        delta = (dout * out).sum(-1, keepdim=True)
        dp = dout @ self.v.t()
        ds = p * (dp - delta)
        # dP and delta are sums of D products, their difference one more rounding
        e_ds = ds.abs() * (self.eps + 2 * U) + p * ((D + 2) * U * (dout.abs() @ self.v.abs().t() + (dout * out).abs().sum(-1, keepdim=True)))
        e_ds = e_ds + self.h * (ds.abs() + e_ds)
        e_p = p * (self.eps + self.h + U)
        n = float(self.see.sum(0).max()) + 4
        m_ds = ds.abs() * n * U
        dq, dk, dv = (ds @ self.k) * self.scale, (ds.t() @ self.q) * self.scale, p.t() @ dout
        bq = ((e_ds + ds.abs() * (self.n + 4) * U) @ self.k.abs()) * self.scale
        bk = ((e_ds + m_ds).t() @ self.q.abs()) * self.scale
        bv = (e_p + p * n * U).t() @ dout.abs()
        return (dq, dk, dv), (bq, bk, bv)


def slot(p, sinks, capacity):
    return p if p < sinks else sinks + (p - sinks) % (capacity - sinks)


def seen(length, window, sinks, capacity):
    """Tokens that a sequence's newest one sees through a cache."""
    reach = min(window or capacity - sinks, capacity - sinks)
    return [p for p in range(length) if p < sinks or p >= length - reach]
