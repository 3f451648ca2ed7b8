"""Attention over packed sequences on the GPU, forward and backward, against 64 bits, through the C ABI's binding."""
import math

import pytest

from attention_reference import Head, half, visible

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1707_00424_amd import binding as pb
    pb.lib()
    return torch, pb


def dt(torch, code):
    return torch.bfloat16 if code else torch.float32


class Problem:
    """q, k, v side by side in rows with `pad` elements behind, n replicas with `gap` elements between, outside filled with NaN."""

    def __init__(self, torch, pb, dtype, n, tokens, offsets, heads, kv, dim, window, sinks, pad=0, gap=0, seed=0, scale=None, sharp=2.0):
        self.torch, self.pb = torch, pb
        self.dtype, self.n, self.T, self.H, self.K, self.D, self.window, self.sinks = dtype, n, tokens, heads, kv, dim, window, sinks
        self.offsets = offsets if offsets is not None else [[0, tokens]] * n
        self.ld = (heads + 2 * kv) * dim + pad
        self.stride, self.ld_out = tokens * self.ld + gap, heads * dim + pad
        self.out_stride = tokens * self.ld_out + gap
        self.scale = scale or dim ** -0.5
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(n, tokens, heads + 2 * kv, dim, generator=g)
        x[:, :, :heads] *= sharp
        self.x = x.to(dt(torch, dtype))
        self.rows = torch.full((n * self.stride + 16,), math.nan, dtype=dt(torch, dtype), device="cuda")
        self.view(self.rows, self.stride, self.ld, heads + 2 * kv).copy_(self.x)
        self.desc = pb.parle_attention_desc(dtype, n, tokens, len(self.offsets[0]) - 1, heads, kv, dim, window, sinks, self.scale, self.ld, self.stride,
                                            self.ld, self.stride, self.ld_out, self.out_stride)
        self.off = torch.tensor(self.offsets, dtype=torch.int32, device="cuda") if offsets is not None else None

    def view(self, flat, stride, ld, heads):
        return self.torch.as_strided(flat, (self.n, self.T, heads, self.D), (stride, ld, self.D, 1))

    def empty(self, stride, fill=7.0):
        return self.torch.full((self.n * stride + 16,), fill, dtype=dt(self.torch, self.dtype), device="cuda")

    def parts(self, flat):
        return flat, flat[self.H * self.D:], flat[(self.H + self.K) * self.D:]

    def forward(self, stream=None):
        out = self.empty(self.out_stride)
        lse = self.torch.full((self.n, self.H, self.T), 5.0, device="cuda")
        self.pb.parle_k_attention_forward(self.desc, *self.parts(self.rows), self.off, out, lse, stream=stream)
        return out, lse

    def scratch(self):
        return self.torch.full((max(16, self.pb.parle_k_attention_scratch_bytes(self.desc)),), 0xA5, dtype=self.torch.uint8, device="cuda")

    def backward(self, out, lse, dout, scratch=None, stream=None):
        d = self.empty(self.stride)
        sc = self.scratch() if scratch is None else scratch
        self.pb.parle_k_attention_backward(self.desc, *self.parts(self.rows), self.off, out, lse, dout, sc, *self.parts(d), stream=stream)
        return d

    def heads(self, rep, head):
        x = self.x[rep].double()
        kv = head // (self.H // self.K)
        return x[:, head], x[:, self.H + kv], x[:, self.H + self.K + kv]


def within(got, want, tol, what):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= tol) & ~(got == want)
    if bad.any():
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i} of {tuple(bad.shape)}: {got.reshape(-1)[i]} for {want.reshape(-1)[i]}, "
                             f"tolerance {tol.expand_as(want).reshape(-1)[i]}")


def outside_untouched(torch, P, flat, stride, ld, heads, fill=7.0):
    mask = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
    P.view(mask, stride, ld, heads).fill_(False)
    left = flat[mask]
    assert (left == fill).all(), "what lies between rows was written"


# dtype, n, tokens, offsets, heads, kv_heads, dim, window, sinks, pad, gap
CASES = [
    (1, 1, 1, None, 1, 1, 8, 0, 0, 0, 0),
    (0, 1, 1, [[0, 1]], 2, 1, 64, 1, 0, 0, 0),
    (1, 2, 3, [[0, 2, 3], [0, 0, 3]], 2, 2, 16, 0, 0, 3, 5),
    (1, 1, 32, None, 3, 1, 72, 5, 0, 0, 0),
    (0, 2, 33, [[1, 7, 7, 30], [0, 33, 33, 33]], 4, 2, 40, 4, 2, 1, 3),
    (1, 1, 64, None, 1, 1, 128, 0, 0, 0, 0),
    (1, 1, 127, None, 5, 5, 64, 1, 0, 0, 0),
    (1, 1, 128, [[0, 128]], 4, 1, 96, 1, 3, 8, 8),
    (0, 1, 129, None, 2, 2, 128, 0, 0, 0, 0),
    (1, 2, 129, [[0, 64, 129], [3, 60, 125]], 6, 2, 80, 50, 1, 0, 0),
    (1, 1, 200, [[0, 1, 2, 3, 100, 131, 199]], 8, 1, 32, 16, 4, 0, 0),
    (1, 1, 257, [[10, 10, 11, 240]], 3, 3, 104, 33, 7, 5, 1),
    (0, 1, 300, [[0, 150, 300]], 2, 1, 96, 64, 16, 0, 0),
    (1, 1, 300, None, 2, 1, 64, 100000, 5, 0, 0),
    (1, 1, 513, None, 2, 1, 64, 385, 4, 0, 0),          # one token beyond the first chunk that sinks leave to others
    (1, 1, 1000, None, 2, 2, 64, 20, 128, 0, 0),        # sinks of a tile's size
    (1, 1, 1100, [[5, 1097]], 4, 2, 128, 100, 3, 0, 0),  # sinks that begin inside a tile, far chunks
    (0, 1, 1300, [[0, 30, 1290]], 2, 1, 64, 128, 33, 0, 0),
    (1, 1, 1600, [[0, 500, 1600]], 3, 1, 48, 64, 100, 0, 0),  # sinks over two tiles
    (1, 2, 700, [[0, 699], [100, 600]], 2, 1, 112, 0, 0, 0, 0),
]
# so many workgroups that wavefronts share no queries, and two share keys
MANY = [
    (1, 4, 200, [[0, 90, 200]] * 4, 40, 40, 64, 30, 3, 0, 0),
    (1, 4, 200, None, 40, 8, 40, 0, 0, 3, 5),
    (1, 4, 140, [[0, 50, 139]] * 4, 24, 24, 128, 33, 5, 0, 0),
    (1, 4, 140, None, 24, 24, 96, 0, 0, 1, 1),
    (1, 4, 140, [[3, 70, 140]] * 4, 24, 6, 88, 20, 2, 0, 0),
    (1, 4, 140, None, 24, 24, 104, 0, 0, 1, 0),
    (0, 4, 140, [[0, 50, 139]] * 4, 40, 40, 64, 33, 5, 0, 0),
    (0, 4, 140, None, 40, 10, 48, 0, 0, 1, 1),
    (0, 4, 140, [[0, 50, 139]] * 4, 40, 20, 128, 33, 5, 0, 0),
    (0, 4, 140, None, 40, 8, 72, 0, 0, 1, 0),
    (1, 1, 700, [[0, 300, 690]], 48, 48, 64, 64, 4, 0, 0),      # the same with sinks that leave queries to chunks
]


@pytest.mark.parametrize("case", CASES + MANY, ids=lambda c: "-".join(str(v) for i, v in enumerate(c) if i != 3))
def test_forward_and_backward(gpu, case):
    torch, pb = gpu
    P = Problem(torch, pb, *case)
    out, lse = P.forward()
    got_out = P.view(out, P.out_stride, P.ld_out, P.H)
    outside_untouched(torch, P, out, P.out_stride, P.ld_out, P.H)
    g = torch.Generator().manual_seed(11)
    dout = torch.randn(P.n, P.T, P.H, P.D, generator=g).to(dt(torch, P.dtype))
    dflat = torch.full_like(out, math.nan)
    P.view(dflat, P.out_stride, P.ld_out, P.H).copy_(dout)
    d = P.backward(out, lse, dflat)
    outside_untouched(torch, P, d, P.stride, P.ld, P.H + 2 * P.K)
    assert torch.equal(d, P.backward(out, lse, dflat)), "two calls differ"
    grads = P.view(d, P.stride, P.ld, P.H + 2 * P.K).cpu().double()
    h = half(P.dtype)
    for a in range(P.n):
        see = visible(P.T, P.offsets[a], P.window, P.sinks)
        want_kv, tol_kv = torch.zeros(P.T, 2 * P.K, P.D).double(), torch.zeros(P.T, 2 * P.K, P.D).double()
        for head in range(P.H):
            R = Head(*P.heads(a, head), see, P.scale, P.dtype)
            tol, tol_lse = R.forward_bounds()
            within(got_out[a, :, head], R.out, tol, f"out of head {head}")
            within(lse[a, head], R.lse, tol_lse, f"lse of head {head}")
            (dq, dk, dv), (bq, bk, bv) = R.backward(got_out[a, :, head].cpu().double(), lse[a, head].cpu().double(), dout[a, :, head].double())
            within(grads[a, :, head], dq, bq + h * (dq.abs() + bq), f"dq of head {head}")
            kv = head // (P.H // P.K)
            want_kv[:, kv] += dk
            tol_kv[:, kv] += bk
            want_kv[:, P.K + kv] += dv
            tol_kv[:, P.K + kv] += bv
        within(grads[a, :, P.H:], want_kv, tol_kv + h * (want_kv.abs() + tol_kv), "dk, dv")


def test_scores_far_from_zero(gpu):
    """Scores of thousands, and a row whose largest comes last: nothing overflows, sums stay relative to the largest."""
    torch, pb = gpu
    P = Problem(torch, pb, 1, 1, 300, None, 2, 1, 64, 0, 0, sharp=1.0)
    ramp = torch.linspace(-30, 30, 300)[:, None]
    P.x[0, :, 2] = (ramp * torch.ones(64)).to(P.x.dtype)
    P.x[0, :, 0] = 40.0
    P.x[0, :, 1] = -40.0
    P.view(P.rows, P.stride, P.ld, 4).copy_(P.x)
    out, lse = P.forward()
    see = visible(300, [0, 300], 0, 0)
    for head in range(2):
        R = Head(*P.heads(0, head), see, P.scale, 1)
        tol, tol_lse = R.forward_bounds()
        within(P.view(out, P.out_stride, P.ld_out, 2)[0, :, head], R.out, tol, "out")
        within(lse[0, head], R.lse, tol_lse, "lse")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_has_no_influence(gpu, dtype, bad):
    """NaN and infinities in k, v, q and dout of single tokens: only tokens that see them, or that they see, change."""
    torch, pb = gpu
    case = (dtype, 1, 200, [[3, 90, 195]], 2, 1, 64, 40, 2)
    clean, dirty = Problem(torch, pb, *case), Problem(torch, pb, *case)
    H, K = 2, 1
    at = 120                                     # token 30 of the second sequence
    view = dirty.view(dirty.rows, dirty.stride, dirty.ld, H + 2 * K)
    view[0, :3], view[0, 195:] = math.nan, math.nan   # rows outside
    view[0, at, H + K, 5] = bad                  # one element of v
    out, lse = clean.forward()
    out2, lse2 = dirty.forward()
    a, b = (P.view(o, P.out_stride, P.ld_out, H)[0].cpu() for P, o in ((clean, out), (dirty, out2)))
    see = visible(200, [3, 90, 195], 40, 2)[:, at]
    assert torch.equal(a[~see], b[~see]) and torch.equal(lse, lse2)
    assert torch.isnan(b[see][:, :, 5]).logical_or(torch.isinf(b[see][:, :, 5])).all()
    rest = [i for i in range(64) if i != 5]
    assert torch.equal(a[see][:, :, rest], b[see][:, :, rest])
    # k: rows that see it are NaN, the others as they were
    view[0, at, H + K, 5] = clean.x[0, at, H + K, 5].to(view.dtype)
    view[0, at, H, 7] = math.nan
    out3, lse3 = dirty.forward()
    c = dirty.view(out3, dirty.out_stride, dirty.ld_out, H)[0].cpu()
    assert torch.equal(a[~see], c[~see]) and torch.isnan(c[see]).all()
    # backward: a NaN key reaches dq of rows that see it only; its own dk, dv; rows that those rows see
    g = torch.Generator().manual_seed(1)
    dout = torch.randn(out.numel(), generator=g).to(out.dtype).cuda()
    d0 = clean.view(clean.backward(out, lse, dout), clean.stride, clean.ld, H + 2 * K)[0].cpu()
    d1 = dirty.view(dirty.backward(out, lse, dout), dirty.stride, dirty.ld, H + 2 * K)[0].cpu()
    assert torch.equal(d0[~see][:, :H], d1[~see][:, :H])
    assert torch.isnan(d1[see][:, :H, 7]).all()
    # q and dout of token `at`: keys that it does not see keep their gradients
    keys = visible(200, [3, 90, 195], 40, 2)[at]
    view[0, at, H, 7] = clean.x[0, at, H, 7].to(view.dtype)
    view[0, at, 0, 9] = bad
    dirty_dout = dout.clone()
    dirty.view(dirty_dout, dirty.out_stride, dirty.ld_out, H)[0, at, 0, 11] = bad
    d2 = dirty.view(dirty.backward(out, lse, dirty_dout), dirty.stride, dirty.ld, H + 2 * K)[0].cpu()
    rows = torch.arange(200) != at
    assert torch.equal(d0[rows][:, :H], d2[rows][:, :H])
    assert torch.equal(d0[~keys][:, H:], d2[~keys][:, H:])
    assert not torch.isfinite(d2[keys][:, H:].float()).all()


@pytest.mark.parametrize("dtype,H,K,D", [(1, 40, 20, 64), (1, 24, 24, 128), (0, 40, 20, 64), (0, 40, 40, 128)])
def test_what_is_not_seen_among_many_heads(gpu, dtype, H, K, D):
    """The same where wavefronts share no queries: a NaN or an infinity in a replica's head changes nothing but what sees it."""
    torch, pb = gpu
    n, T, at, offsets = 4, 140, 100, [[0, 50, 139]] * 4
    clean, dirty = (Problem(torch, pb, dtype, n, T, offsets, H, K, D, 33, 5) for _ in range(2))
    heads = H + 2 * K
    view = dirty.view(dirty.rows, dirty.stride, dirty.ld, heads)
    see, keys, group = visible(T, offsets[0], 33, 5)[:, at], visible(T, offsets[0], 33, 5)[at], slice(0, H // K)
    out, lse = clean.forward()
    dout = torch.randn(out.numel(), generator=torch.Generator().manual_seed(1)).to(out.dtype).cuda()
    a, grad = clean.view(out, clean.out_stride, clean.ld_out, H).cpu(), clean.view(clean.backward(out, lse, dout), clean.stride, clean.ld, heads).cpu()

    def others(x, rows, first, count):
        """x [n, T, heads, D] without the given rows of the heads first .. first + count - 1 of replica 0."""
        x = x.clone()
        x[0, rows, first:first + count] = 0
        return x

    for part, bad in ((H + K, math.inf), (H + K, math.nan), (H, math.nan)):
        view[0, at, part, 5] = bad
        got, _ = dirty.forward()
        b = dirty.view(got, dirty.out_stride, dirty.ld_out, H).cpu()
        assert torch.equal(others(a, see, 0, H // K), others(b, see, 0, H // K)) and not torch.isfinite(b[0, see][:, group, 5].float()).any()
        d = dirty.view(dirty.backward(out, lse, dout), dirty.stride, dirty.ld, heads).cpu()
        assert torch.equal(others(grad, see, 0, H // K)[:, :, :H], others(d, see, 0, H // K)[:, :, :H])
        view[0, at, part, 5] = clean.x[0, at, part, 5].to(view.dtype)
    view[0, at, 0, 9] = math.inf
    bad_dout = dout.clone()
    dirty.view(bad_dout, dirty.out_stride, dirty.ld_out, H)[0, at, 0, 3] = math.nan
    d = dirty.view(dirty.backward(out, lse, bad_dout), dirty.stride, dirty.ld, heads).cpu()
    one = torch.arange(T) == at
    x, y = others(grad, one, 0, 1), others(d, one, 0, 1)
    for first in (H, H + K):
        x, y = others(x, keys, first, 1), others(y, keys, first, 1)
    assert torch.equal(x, y) and not torch.isfinite(d[0, keys, H].float()).all()


@pytest.mark.parametrize("dtype,n,H,K,D", [(0, 1, 2, 1, 64), (1, 1, 2, 1, 64), (1, 1, 4, 2, 96), (0, 4, 40, 40, 64), (1, 4, 40, 20, 64), (1, 4, 24, 24, 128)])
def test_scores_of_minus_infinity(gpu, dtype, n, H, K, D):
    """A softmax over scores of -inf only is NaN, here as for a token over its cache; where a row sees another score as well, such a key counts for nothing."""
    torch, pb = gpu
    T = 140
    P = Problem(torch, pb, dtype, n, T, [[3, 60, T - 1]] * n, H, K, D, 0, 0)
    P.x[:, :, :H, 0] = 1.0
    P.x[:, 3, H:H + K, 0] = -math.inf                          # the first sequence's first two tokens
    P.x[:, 4, H:H + K, 0] = -math.inf
    P.view(P.rows, P.stride, P.ld, H + 2 * K).copy_(P.x)
    out, lse = P.forward()
    o, lse = P.view(out, P.out_stride, P.ld_out, H).cpu().double(), lse.cpu()
    assert o[:, 3:5].isnan().all() and (lse[:, :, 3:5] == -math.inf).all()
    assert (o[:, :3] == 0).all() and (o[:, T - 1:] == 0).all() and (lse[:, :, :3] == -math.inf).all()
    assert o[:, 5:T - 1].isfinite().all() and lse[:, :, 5:T - 1].isfinite().all()
    see = visible(T, [0, T], 0, 0)
    for head in range(H):
        q, k, v = P.heads(0, head)
        # without those two, from token 5 on
        R = Head(q[5:60], k[5:60], v[5:60], see[:55, :55], P.scale, dtype)
        tol, tol_lse = R.forward_bounds()
        within(o[0, 5:60, head], R.out, tol, f"out of head {head}")
        within(lse[0, head, 5:60], R.lse, tol_lse, f"lse of head {head}")
    # the same of caches
    rows = P.x[:, :, :].to(dt(torch, dtype))
    caches = [rows[:, 3:6, H + i * K:H + (i + 1) * K].transpose(1, 2).contiguous().cuda() for i in (0, 1)]
    desc = pb.parle_cache_desc(dtype, n, 3, H, K, D, 0, 0, P.scale, H * D, K * D, H * D)
    got = torch.empty(n, H * D, dtype=dt(torch, dtype), device="cuda")
    sc = torch.empty(max(16, pb.parle_k_decode_scratch_bytes(desc)), dtype=torch.uint8, device="cuda")
    for length in (2, 3):
        q = rows[:, 2 + length, :H].reshape(n, H * D).contiguous().cuda()
        pb.parle_k_attention_decode(desc, q, None, None, torch.full((n,), length, dtype=torch.int32, device="cuda"), sc, *caches, got)
        assert got.isnan().all() if length == 2 else torch.isfinite(got).all()


def test_gradient_by_differences(gpu):
    """fp32: the derivative of <out, dout> along a direction of q, k and v, by central differences at two widths."""
    torch, pb = gpu
    P = Problem(torch, pb, 0, 1, 150, [[0, 60, 148]], 4, 2, 64, 30, 2, sharp=1.0)
    out, lse = P.forward()
    g = torch.Generator().manual_seed(5)
    dout = torch.randn(out.numel(), generator=g).cuda()
    d = P.backward(out, lse, dout)
    inside = torch.zeros(P.rows.numel(), dtype=torch.bool, device="cuda")
    P.view(inside, P.stride, P.ld, 8).fill_(True)
    valid = torch.zeros(out.numel(), dtype=torch.bool, device="cuda")
    P.view(valid, P.out_stride, P.ld_out, 4).fill_(True)
    base = P.rows.clone()
    for part in range(3):
        direction = torch.zeros_like(base)
        v = P.view(direction, P.stride, P.ld, 8)[:, :, (0, 4, 6)[part]:(4, 6, 8)[part]]
        v.copy_(torch.randn(v.shape, generator=g))

        def value(step):
            P.rows = torch.where(inside, base + step * direction, base)
            o, _ = P.forward()
            return float((o[valid].double() * dout[valid].double()).sum()), float((o[valid].double() * dout[valid].double()).abs().sum())

        def slope(step):
            (x, mass), (y, _) = value(step), value(-step)
            return (x - y) / (2 * step), mass

        e = 2.0 ** -6
        (one, mass), (two, _) = slope(e), slope(2 * e)
        want = float((d[inside].double() * direction[inside].double()).sum())
        # the error of a central difference falls with the square of its width: that of `one` is a third of two - one; the values' own
        # rounding: 2e-5 is (D + 4) u A with A of 5, at random signs over the sum
        tol = abs(two - one) + 2e-5 * mass / e / math.sqrt(P.T)
        assert abs(want - one) <= tol, (part, want, one, two, tol)
        P.rows = base


def test_offsets_beyond_32_bits(gpu):
    torch, pb = gpu
    T, H, D = 2100, 1, 64
    ld = 1 << 20                                              # 2100 * 2^20 elements from the first row to the last
    rows = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(T, 3, D, generator=torch.Generator().manual_seed(3)).bfloat16()
    torch.as_strided(rows, (T, 3, D), (ld, D, 1)).copy_(x)
    desc = pb.parle_attention_desc(1, 1, T, 1, H, 1, D, 0, 0, D ** -0.5, ld, 0, ld, 0, D, 0)
    near = pb.parle_attention_desc(1, 1, T, 1, H, 1, D, 0, 0, D ** -0.5, 3 * D, 0, 3 * D, 0, D, 0)
    close = x.reshape(-1).cuda()
    results = []
    for de, r in ((desc, rows), (near, close)):
        out, lse = torch.empty(T, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 1, T, device="cuda")
        pb.parle_k_attention_forward(de, r, r[D:], r[2 * D:], None, out, lse)
        results.append((out, lse))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    out, lse = results[0]
    sc = torch.empty(pb.parle_k_attention_scratch_bytes(desc), dtype=torch.uint8, device="cuda")
    d = torch.empty_like(close)
    pb.parle_k_attention_backward(near, close, close[D:], close[2 * D:], None, out, lse, out, sc, d, d[D:], d[2 * D:])
    far = torch.empty_like(rows)
    pb.parle_k_attention_backward(desc, rows, rows[D:], rows[2 * D:], None, out, lse, out, sc, far, far[D:], far[2 * D:])
    assert torch.equal(torch.as_strided(far, (T, 3, D), (ld, D, 1)), d.reshape(T, 3, D))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,row_bytes", [(1, 805306368), (1, (1 << 31) - 16), (3, 1 << 29), (16, 100663296), (16, (1 << 31) // 143 // 16 * 16), (16, (1 << 31) // 144 // 16 * 16)])
def test_few_rows_far_apart(gpu, dtype, T, row_bytes):
    """Tensors that end with their last row's heads: the tiles' rows behind the last lie far beyond, and beyond 2^32 bytes."""
    torch, pb = gpu
    t, D = dt(torch, dtype), 64
    ld = row_bytes // (2 if dtype else 4)
    x = torch.randn(T, 3 * D, generator=torch.Generator().manual_seed(6)).to(t).cuda()
    far = torch.empty((T - 1) * ld + 3 * D, dtype=t, device="cuda")
    rows = torch.as_strided(far, (T, 3 * D), (ld, 1))
    rows.copy_(x)
    results = []
    for r, step in ((far, ld), (x, 3 * D)):
        flat = r.reshape(-1)
        desc = pb.parle_attention_desc(dtype, 1, T, 1, 1, 1, D, 0, 0, D ** -0.5, step, 0, step, 0, step, 0)
        out, d = torch.empty_like(flat), torch.empty_like(flat)
        lse = torch.empty(1, 1, T, device="cuda")
        pb.parle_k_attention_forward(desc, flat, flat[D:], flat[2 * D:], None, out, lse)
        sc = torch.empty(pb.parle_k_attention_scratch_bytes(desc), dtype=torch.uint8, device="cuda")
        pb.parle_k_attention_backward(desc, flat, flat[D:], flat[2 * D:], None, out, lse, flat[2 * D:], sc, d, d[D:], d[2 * D:])
        view = lambda v, c: torch.as_strided(v, (T, c), (step, 1)).clone()  # noqa: E731
        results.append((view(out, D), lse, view(d, 3 * D)))
    for a, b in zip(*results):
        assert torch.equal(a, b) and torch.isfinite(a.float()).all()


def test_graph_and_stream(gpu):
    """Captured once and replayed between eager runs on other data, and run on a stream of its own: every result is the eager one."""
    torch, pb = gpu
    P = Problem(torch, pb, 1, 2, 700, [[0, 300, 690], [0, 50, 700]], 4, 2, 64, 64, 4)
    scratch = P.scratch()
    side = torch.cuda.Stream()
    out, lse = P.forward()
    dout = torch.randn(out.numel(), generator=torch.Generator().manual_seed(1)).to(out.dtype).cuda()
    want = P.backward(out, lse, dout, scratch)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        o2, l2 = P.forward(stream=side)
        d2 = P.backward(o2, l2, dout, P.scratch(), stream=side)
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2) and torch.equal(want, d2)
    go, gl, gd = torch.empty_like(out), torch.empty_like(lse), torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pb.parle_k_attention_forward(P.desc, *P.parts(P.rows), P.off, go, gl)
        pb.parle_k_attention_backward(P.desc, *P.parts(P.rows), P.off, go, gl, dout, scratch, *P.parts(gd))
    view = P.view(P.rows, P.stride, P.ld, 8)
    for step in range(3):
        view.copy_(torch.randn(view.shape, generator=torch.Generator().manual_seed(step)))
        out, lse = P.forward()
        want = P.view(P.backward(out, lse, dout, P.scratch()), P.stride, P.ld, 8).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(P.view(go, P.out_stride, P.ld_out, 4), P.view(out, P.out_stride, P.ld_out, 4)) and torch.equal(gl, lse)
        assert torch.equal(P.view(gd, P.stride, P.ld, 8), want)


def test_lse_may_be_left_out(gpu):
    torch, pb = gpu
    P = Problem(torch, pb, 1, 1, 70, None, 2, 1, 64, 0, 0)
    out, _ = P.forward()
    got = P.empty(P.out_stride)
    pb.parle_k_attention_forward(P.desc, *P.parts(P.rows), P.off, got, None)
    assert torch.equal(out, got)
