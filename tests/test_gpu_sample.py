"""The sampler on the GPU against its definition in 64 bits, row by row: tokens and counts exactly, logarithms within fp32's rounding."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1707_00424_amd import binding as pb
    pb.lib()
    return torch, pb


def reference(torch, x, u, t, k, p, m):
    """x float64 [classes]; token, how many stayed, logarithm of the token's share."""
    if x.isnan().any():
        return -1, 0, math.nan
    most = float(x.max())
    if most == -math.inf:
        return -1, 0, -math.inf
    if not t > 0:
        return int((x == most).nonzero()[0]), 1, 0.0
    # stable: the lower class first where two are equal
    v, ids = torch.sort(x, descending=True, stable=True)
    count = int((v > -math.inf).sum())
    v, ids = v[:count], ids[:count]
    log = torch.where(v == most, torch.zeros_like(v), (v - most) / t)
    log = torch.where(log.isnan(), torch.full_like(log, -math.inf), log)
    w = torch.exp(log)
    if 0 < k < count:
        w, ids, log = w[:k], ids[:k], log[:k]
    if p < 1:
        c = torch.cumsum(w, 0)
        stay = 1 + int((c < p * float(c[-1])).sum())
        w, ids, log = w[:stay], ids[:stay], log[:stay]
    if m > 0:
        stay = max(1, int((w >= m).sum()))
        w, ids, log = w[:stay], ids[:stay], log[:stay]
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    c = torch.cumsum(w, 0)
    at = int((c <= u * float(c[-1])).sum())
    return int(ids[at]), len(ids), float(log[at]) - math.log(float(c[-1]))


def check(torch, pb, logits, u, t=None, k=None, p=None, m=None, classes=None):
    """logits [n, rows, ld] of their type on the CPU, the others lists or None, for every row."""
    n, rows, ld = logits.shape
    classes = classes or ld
    f32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.float32).reshape(n, rows).cuda()  # noqa: E731
    uu, tt, pp, mm = f32(u), f32(t), f32(p), f32(m)
    kk = None if k is None else torch.tensor(k, dtype=torch.int32).reshape(n, rows).cuda()
    tokens, kept = (torch.full((n, rows), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    logp = torch.full((n, rows), 9.0, device="cuda")
    desc = pb.parle_sample_desc(int(logits.dtype == torch.bfloat16), n, rows, classes, ld)
    sc = torch.full((max(16, pb.parle_k_sample_scratch_bytes(desc)),), 0xA5, dtype=torch.uint8, device="cuda")
    dev = logits.cuda()
    pb.parle_k_sample(desc, dev, uu, tt, kk, pp, mm, sc, tokens, kept, logp)
    at = lambda v, i, other: other if v is None else v.reshape(-1)[i].item()  # noqa: E731
    for i, x in enumerate(logits.reshape(n * rows, ld)):
        want = reference(torch, x[:classes].double(), at(uu, i, 0), at(tt, i, 1.0), at(kk, i, 0), at(pp, i, 1.0), at(mm, i, 0.0))
        got = (int(tokens.reshape(-1)[i]), int(kept.reshape(-1)[i]), float(logp.reshape(-1)[i]))
        assert got[:2] == want[:2], (i, got, want)
        # rounded once from 64 bits; its terms are held to 2^-40 of the largest weight, a token is never drawn far below that
        assert got[2] == want[2] or abs(got[2] - want[2]) <= 2.0 ** -23 * max(1.0, abs(want[2])) or (got[2] != got[2] and want[2] != want[2]), (i, got, want)
    again = torch.full_like(tokens, -7)
    pb.parle_k_sample(desc, dev, uu, tt, kk, pp, mm, sc, again, None, None)
    assert torch.equal(tokens, again)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,rows,classes,pad", [(1, 1, 1, 0), (2, 3, 2, 1), (1, 40, 7, 0), (1, 33, 1000, 5), (3, 5, 1025, 0), (1, 16, 8193, 3), (1, 12, 50001, 0), (1, 4, 130000, 7), (1, 300, 300, 0)])
def test_random_rows(gpu, dtype, n, rows, classes, pad):
    torch, pb = gpu
    g = torch.Generator().manual_seed(classes)
    x = (3 * torch.randn(n, rows, classes + pad, generator=g)).to(torch.bfloat16 if dtype else torch.float32)
    x[:, :, classes:] = math.nan
    x[:, ::3, : classes // 3] = -math.inf
    R = n * rows
    rand = lambda: torch.rand(R, generator=g).tolist()  # noqa: E731
    pick = lambda v: [v[int(i)] for i in torch.randint(0, len(v), (R,), generator=g)]  # noqa: E731
    for _ in range(3):
        check(torch, pb, x, rand(), pick([1.0, 0.7, 1.3, 0.1, 3.0, 0.0]), pick([0, 1, 2, 50, 1000, classes, classes + 1]), pick([1.0, 0.9, 0.5, 0.99, 0.0]),
              pick([0.0, 0.0, 0.05, 0.5, 1.0, 2.0]), classes)
    check(torch, pb, x, rand(), classes=classes)
    check(torch, pb, x, rand(), t=pick([1.0, 0.5]), classes=classes)
    check(torch, pb, x, rand(), p=pick([0.3, 0.95]), classes=classes)
    check(torch, pb, x, rand(), k=pick([3, 40]), classes=classes)
    check(torch, pb, x, rand(), m=pick([0.1, 1e-3, 1e-25]), classes=classes)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("classes", [5, 1024, 1025, 5000, 40000])
def test_many_equal(gpu, dtype, classes):
    """Rows of one value or of few, more of them than are sorted at once: ties go to the lower class."""
    torch, pb = gpu
    t = torch.bfloat16 if dtype else torch.float32
    one = torch.full((classes,), -2.5)
    two = torch.where(torch.arange(classes) % 3 == 0, 1.0, 0.0)
    near = torch.arange(classes) % 7 * 2.0 ** -7                             # values within one step of the weight's logarithm
    signs = torch.where(torch.arange(classes) % 2 == 0, 0.0, -0.0)
    x = torch.stack([one, two, near, signs] * 6)[None].to(t)
    u = [0.0] * 4 + [0.25] * 4 + [0.5] * 4 + [0.999] * 4 + [0.625] * 4 + [0.125] * 4
    check(torch, pb, x, u)
    check(torch, pb, x, u, k=[0, 3, classes - 1, classes // 2] * 6)
    check(torch, pb, x, u, p=[0.5, 0.25, 0.75, 0.125] * 6)
    check(torch, pb, x, u, k=[classes // 2 + 1] * 24, p=[0.5] * 24, m=[0.9] * 24, t=[2.0, 0.25, 1.0, 1.0] * 6)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("classes", [40, 513, 1500, 9000])
def test_more_rows_than_compute_units(gpu, dtype, classes):
    """They go through smaller workgroups."""
    torch, pb = gpu
    R = 260
    g = torch.Generator().manual_seed(classes + 1)
    x = (3 * torch.randn(1, R, classes, generator=g)).to(torch.bfloat16 if dtype else torch.float32)
    x[:, ::3, : classes // 3] = -math.inf
    x[:, 1::7] = (x[:, 1::7] > 1).to(x.dtype)                                 # two values, one of them zero
    x[:, 2::7] = 0.5
    rand = lambda: torch.rand(R, generator=g).tolist()  # noqa: E731
    pick = lambda v: [v[int(i)] for i in torch.randint(0, len(v), (R,), generator=g)]  # noqa: E731
    check(torch, pb, x, rand(), pick([1.0, 0.7, 0.1, 3.0, 0.0]), pick([0, 1, 50, 299, 300, 301, 600, classes]), pick([1.0, 0.9, 0.5]), pick([0.0, 0.05, 0.5]))
    check(torch, pb, x, rand())
    check(torch, pb, x, rand(), k=pick([3, 400]))
    check(torch, pb, x, rand(), p=pick([0.3, 0.95]))
    check(torch, pb, x, rand(), m=pick([0.1, 1e-3, 1e-25]))


@pytest.mark.parametrize("dtype", [0, 1])
def test_zeros_of_both_signs_among_tiny_logits(gpu, dtype):
    """A temperature as small as the logits: weights of all classes near zero differ, those of 0 and -0 do not."""
    torch, pb = gpu
    C = 2000
    g = torch.Generator().manual_seed(8)
    x = (torch.randn(8, C, generator=g) * 1e-37).to(torch.bfloat16 if dtype else torch.float32)
    zero = torch.rand(8, C, generator=g) < 0.2
    x = torch.where(zero, torch.where(torch.rand(8, C, generator=g) < 0.5, 0.0, -0.0).to(x.dtype), x)
    x[4:] = x[4:].abs() * -1.0                                               # nothing above zero
    for u in (0.0, 0.2, 0.5, 0.8, 0.99):
        check(torch, pb, x[None], [u] * 8, t=[1e-37] * 8)
        check(torch, pb, x[None], [u] * 8, t=[3e-37] * 8, p=[0.7] * 8, k=[1500] * 8)


@pytest.mark.parametrize("rows", [4, 260])
def test_more_zeros_than_are_listed(gpu, rows):
    """bf16 rows of zeros of both signs below a few larger logits, with every rule."""
    torch, pb = gpu
    C = 6000
    g = torch.Generator().manual_seed(9)
    x = torch.where(torch.rand(1, rows, C, generator=g) < 0.5, 0.0, -0.0)
    x[:, :, ::40] = 4 * torch.rand(1, rows, C // 40, generator=g)
    x = x.bfloat16()
    rand = lambda: torch.rand(rows, generator=g).tolist()  # noqa: E731
    check(torch, pb, x, rand())
    check(torch, pb, x, rand(), m=[0.5] * rows)
    check(torch, pb, x, rand(), m=[0.01] * rows, p=[0.9] * rows)
    check(torch, pb, x, rand(), k=[2000] * rows, p=[0.5] * rows, t=[0.5] * rows)


@pytest.mark.parametrize("rows", [5, 260])
def test_a_largest_logit_just_above_zero(gpu, rows):
    """bf16 rows whose largest logit is tiny and whose others are not: far more octaves lie below zero than above."""
    torch, pb = gpu
    C = 5000
    g = torch.Generator().manual_seed(10)
    x = -3 * torch.randn(1, rows, C, generator=g).abs()
    x[:, :, ::7] *= 1e-3
    x[:, ::2, 3::5] = -math.inf
    x[:, 1::4, 500:] = -2.0                                                   # thousands of one value
    tiny = torch.tensor([1e-9, 1e-12, 1e-20, 1e-30, 1e-40])[torch.arange(rows) % 5]
    x[0, torch.arange(rows), torch.randint(0, C, (rows,), generator=g)] = tiny
    x = x.bfloat16()
    rand = lambda: torch.rand(rows, generator=g).tolist()  # noqa: E731
    check(torch, pb, x, rand())
    check(torch, pb, x, rand(), t=[1.0, 0.1, 5.0, 0.01] * (rows // 4) + [1.0] * (rows % 4))
    check(torch, pb, x, rand(), p=[0.9] * rows)
    check(torch, pb, x, rand(), m=[0.2] * rows)
    check(torch, pb, x, rand(), p=[0.5] * rows, m=[0.05] * rows, k=[2000] * rows)


@pytest.mark.parametrize("C,most,t", [(20000, 7.15625, 0.21069972217082977), (10000, 7.90625, 0.2281261533498764)])
def test_weights_that_end_just_below_zero(gpu, C, most, t):
    """bf16 rows whose last weight is that of a logit just below zero: far more octaves lie above zero than below."""
    torch, pb = gpu
    g = torch.Generator().manual_seed(11)
    x = most * torch.rand(4, C, generator=g)
    x[1] = most * 2.0 ** (-34 * torch.rand(C, generator=g))                   # all octaves alike
    x[2, ::3] *= -1.0
    x[3, ::2] = -math.inf
    x[:, 17] = most
    x = x.bfloat16()[None]
    for u in (0.0, 0.3, 0.999999):
        check(torch, pb, x, [u] * 4, t=[t] * 4)
        check(torch, pb, x, [u] * 4, t=[t] * 4, p=[0.9, 0.999999, 0.5, 0.99] * 1)
        check(torch, pb, x, [u] * 4, t=[t] * 4, m=[1e-3] * 4, k=[1500] * 4)


@pytest.mark.parametrize("rows,C", [(257, 2200000), (257, 1 << 22), (3, 1 << 22)])
def test_millions_of_equal_logits(gpu, rows, C):
    """bf16: each row's classes are equal or -inf, so the token is known: weights are one, and u times their number has 46 bits at most."""
    torch, pb = gpu
    ids = torch.arange(C, device="cuda")
    patterns = [ids >= 0, ids % 3 == 1, (ids >= C // 2) | (ids == 5), ids < 700]
    x = torch.empty(1, rows, C, dtype=torch.bfloat16, device="cuda")
    left = [p.nonzero()[:, 0] for p in patterns]
    for i, p in enumerate(patterns):
        x[0, i::4] = torch.where(p, 1.5, -math.inf).to(x.dtype)
    u = torch.rand(1, rows, generator=torch.Generator().manual_seed(12))
    u[0, :8] = torch.tensor([0.0, 0.5, 0.25, 0.75, 0.99999994, 0.99999994, 0.0, 0.99999994][:rows])
    tokens, kept = (torch.full((1, rows), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    desc = pb.parle_sample_desc(1, 1, rows, C, C)
    sc = torch.empty(max(16, pb.parle_k_sample_scratch_bytes(desc)), dtype=torch.uint8, device="cuda")
    pb.parle_k_sample(desc, x, u.cuda(), None, None, None, None, sc, tokens, kept, None)
    for i in range(rows):
        of = left[i % 4]
        assert int(kept[0, i]) == len(of)
        assert int(tokens[0, i]) == int(of[math.floor(float(u[0, i]) * len(of))]), i


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,C", [(6, 300), (6, 5000), (300, 2000)])
def test_a_min_p_below_what_is_counted(gpu, dtype, rows, C):
    """Weights under 2^-52 of the largest are nothing to a sum, but min-p still says which of their classes stay."""
    torch, pb = gpu
    g = torch.Generator().manual_seed(13)
    x = (3 * torch.randn(1, rows, C, generator=g)).to(torch.bfloat16 if dtype else torch.float32)
    x[:, 1::3, ::2] = -math.inf
    x[:, 2::3, 7:9] = math.inf
    u = torch.rand(rows, generator=g).tolist()
    for t in (0.05, 0.2):
        for m in (1e-15, 1e-17, 1e-25, 1e-38, 1e-44):
            check(torch, pb, x, u, t=[t] * rows, m=[m] * rows)
        check(torch, pb, x, u, t=[t] * rows, m=[1e-25] * rows, k=[C - 100] * rows, p=[0.99] * rows)
        check(torch, pb, x, u, t=[t] * rows, m=[1e-30] * rows, k=[C - 100] * rows)


def test_special_rows(gpu):
    torch, pb = gpu
    inf, nan = math.inf, math.nan
    base = torch.randn(100, generator=torch.Generator().manual_seed(1)).tolist()
    rows = [[-inf] * 100, base[:50] + [nan] + base[51:], [inf] + base[1:], [inf, -inf, inf] + base[3:], [-inf] * 99 + [2.0], [3e38] * 2 + [-3e38] * 98, [v * 1e30 for v in base],
            [v * 1e-30 for v in base], [nan] * 100, [-1e9] * 100, [-1e9] * 50 + base[50:]]
    x = torch.tensor(rows)[None]
    R = len(rows)
    for u in (0.0, 0.3, 0.99999994, 1.0, 2.0, -1.0, nan):
        for t in (1.0, 0.0, -1.0, nan, 1e-30, 1e30, inf):
            check(torch, pb, x, [u] * R, t=[t] * R)
    check(torch, pb, x, [0.5] * R, k=[2] * R, p=[nan] * R, m=[nan] * R)
    check(torch, pb, x, [0.5] * R, k=[-3] * R, p=[-1.0] * R)
    check(torch, pb, x, [0.5] * R, p=[1e-30] * R, m=[3.0] * R)
    check(torch, pb, x, [0.7] * R, t=[1e-4] * R, k=[20] * R)                 # weights that are zero among the first twenty


def test_shares_of_many_draws(gpu):
    """A row drawn with 4096 evenly spread numbers: each class as often as its share says, to one."""
    torch, pb = gpu
    R, C = 4096, 50
    x = torch.randn(C, generator=torch.Generator().manual_seed(2))
    logits = x.expand(1, R, C).contiguous().cuda()
    u = ((torch.arange(R) + 0.5) / R)[None].cuda()
    tokens = torch.empty(1, R, dtype=torch.int32, device="cuda")
    desc = pb.parle_sample_desc(0, 1, R, C, C)
    sc = torch.empty(max(16, pb.parle_k_sample_scratch_bytes(desc)), dtype=torch.uint8, device="cuda")
    pb.parle_k_sample(desc, logits, u, None, None, None, None, sc, tokens, None, None)
    counts = torch.bincount(tokens[0].long().cpu(), minlength=C).double()
    assert ((counts - R * torch.softmax(x.double(), 0)).abs() <= 1 + 1e-9).all()


def test_graph_and_stream(gpu):
    torch, pb = gpu
    n, R, C = 1, 8, 20000
    g = torch.Generator().manual_seed(3)
    x, u = torch.randn(n, R, C, generator=g).cuda(), torch.rand(n, R, generator=g).cuda()
    t, p = torch.full((n, R), 0.8, device="cuda"), torch.full((n, R), 0.9, device="cuda")
    desc = pb.parle_sample_desc(0, n, R, C, C)
    make = lambda: (torch.empty(max(16, pb.parle_k_sample_scratch_bytes(desc)), dtype=torch.uint8, device="cuda"), torch.empty(n, R, dtype=torch.int32, device="cuda"),  # noqa: E731
                    torch.empty(n, R, dtype=torch.int32, device="cuda"), torch.empty(n, R, device="cuda"))
    a, b, c = make(), make(), make()
    pb.parle_k_sample(desc, x, u, t, None, p, None, *a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pb.parle_k_sample(desc, x, u, t, None, p, None, *a)
    side = torch.cuda.Stream()
    for step in range(4):
        x.copy_(3 * torch.randn(x.shape, generator=g))
        u.copy_(torch.rand(u.shape, generator=g))
        pb.parle_k_sample(desc, x, u, t, None, p, None, *b)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            pb.parle_k_sample(desc, x, u, t, None, p, None, *c, stream=side)
        side.synchronize()
        for i in (1, 2, 3):
            assert torch.equal(a[i], b[i]) and torch.equal(a[i], c[i])


def test_far_offsets(gpu):
    torch, pb = gpu
    ld, R = (1 << 30) + 8, 3
    x = torch.empty(R * ld, dtype=torch.bfloat16, device="cuda")
    rows = torch.randn(R, 500, generator=torch.Generator().manual_seed(4)).bfloat16()
    torch.as_strided(x, (R, 500), (ld, 1)).copy_(rows)
    u = torch.tensor([[0.1, 0.5, 0.9]], device="cuda")
    tokens = torch.empty(1, R, dtype=torch.int32, device="cuda")
    desc = pb.parle_sample_desc(1, 1, R, 500, ld)
    sc = torch.empty(max(16, pb.parle_k_sample_scratch_bytes(desc)), dtype=torch.uint8, device="cuda")
    pb.parle_k_sample(desc, x, u, None, None, None, None, sc, tokens, None, None)
    for i in range(R):
        assert int(tokens[0, i]) == reference(torch, rows[i].double(), float(u[0, i]), 1.0, 0, 1.0, 0.0)[0]
