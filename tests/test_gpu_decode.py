"""The rolling caches on the GPU: a prompt stored, single tokens decoded, against 64 bits and against the attention of whole sequences."""
import math

import pytest

from attention_reference import U, half, seen, slot

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


def scratch(torch, nbytes):
    return torch.full((max(nbytes, 16),), 0xA5, dtype=torch.uint8, device="cuda")


# dtype, lengths, heads, kv_heads, dim, window, sinks, capacity
CASES = [
    (1, [1], 1, 1, 8, 0, 0, 1),
    (0, [1, 0, 2, -3], 2, 1, 64, 0, 0, 3),
    (1, [5, 31, 32, 33], 4, 2, 128, 0, 0, 40),
    (1, [100, 7, 1000, 3], 8, 2, 64, 16, 4, 20),             # rolled over, and still in the sinks
    (0, [50, 130, 129], 6, 3, 72, 64, 1, 65),
    (1, [300, 299], 3, 1, 96, 100, 0, 300),                  # a window smaller than the cache
    (1, [260], 40, 2, 128, 0, 0, 100),                       # a cache smaller than the sequence; twenty heads share keys
    (0, [700, 1], 16, 1, 40, 0, 3, 1024),
    (1, [3000, 1500, 2048], 4, 1, 128, 0, 0, 4096),          # many shares of a cache
    (1, [12], 2, 2, 80, 5, 128, 140),                        # sinks that the sequence has not left
    (1, [129, 257, 0, 513], 33, 1, 56, 512, 128, 640),
]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[2:]) + f"-{c[0]}-{len(c[1])}")
def test_decode(gpu, case, fused):
    torch, pb = gpu
    dtype, lengths, H, K, D, window, sinks, capacity = case
    B = len(lengths)
    g = torch.Generator().manual_seed(1)
    pad = 5
    q = (2 * torch.randn(B, H * D + pad, generator=g)).to(dt(torch, dtype))
    kn, vn = (torch.randn(B, K * D + pad, generator=g).to(dt(torch, dtype)) for _ in range(2))
    # slots that hold no token of the sequence are NaN
    caches = [torch.full((B, K, capacity, D), math.nan, dtype=dt(torch, dtype)) for _ in range(2)]
    for b, n in enumerate(lengths):
        for p in seen(n, 0, sinks, capacity):
            for c in caches:
                c[b, :, slot(p, sinks, capacity)] = torch.randn(K, D, generator=g).to(dt(torch, dtype))
        if n > 0:
            s = slot(n - 1, sinks, capacity)
            for c, new in zip(caches, (kn, vn)):
                c[b, :, s] = math.nan if fused else new[b, :K * D].reshape(K, D)
    dev = [c.cuda() for c in caches]
    out = torch.full((B, H * D + pad), 7.0, dtype=dt(torch, dtype), device="cuda")
    desc = pb.parle_cache_desc(dtype, B, capacity, H, K, D, window, sinks, D ** -0.5, H * D + pad, K * D + pad, H * D + pad)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    new = (kn.cuda(), vn.cuda()) if fused else (None, None)
    pb.parle_k_attention_decode(desc, q.cuda(), *new, ln, scratch(torch, pb.parle_k_decode_scratch_bytes(desc)), *dev, out)
    assert (out[:, H * D:] == 7.0).all()
    h = half(dtype)
    for b, n in enumerate(lengths):
        got = out[b, :H * D].reshape(H, D).cpu().double()
        if n > 0:
            s = slot(n - 1, sinks, capacity)
            for c, new_rows in zip(caches, (kn, vn)):
                c[b, :, s] = new_rows[b, :K * D].reshape(K, D)
        else:
            assert (got == 0).all()
            continue
        at = [slot(p, sinks, capacity) for p in seen(n, window, sinks, capacity)]
        for head in range(H):
            kv = head // (H // K)
            x = q[b, head * D:(head + 1) * D].double()
            k, v = caches[0][b, kv, at].double(), caches[1][b, kv, at].double()
            s = (k @ x) * D ** -0.5
            p = torch.softmax(s, 0)
            a = float((k.abs() @ x.abs()).max()) * D ** -0.5
            # as in attention_reference; joining shares adds a factor and a sum more
            eps = (D + 4) * U * a + 4 * U * (1 + 3 * a) + 8 * U
            tol = (p @ v.abs()) * (2 * eps + h + 2 * len(at) * U) + h * (p @ v).abs()
            assert ((got[head] - p @ v).abs() <= tol).all(), (b, head, float(((got[head] - p @ v).abs() - tol).max()))
    for c, dev_c in zip(caches, dev):
        same = (c == dev_c.cpu()) | (c.isnan() & dev_c.cpu().isnan())
        assert same.all(), "the caches hold something else"


SPREAD = [1, 0, 31, 513, 600, 1024, 1099, 700]
# 128 workgroups of sequences, key heads and sixteens of query heads, or more: up to 1536 visible tokens go through one workgroup, more are shared
MANY = [
    (1, SPREAD + [1100] * 8, 16, 8, 64, 0, 0, 1100),
    (0, SPREAD * 4, 4, 4, 64, 700, 3, 703),
    (0, SPREAD + [1536] * 8, 8, 8, 128, 0, 0, 1536),
    (1, SPREAD + [2000, 513, 514], 160, 4, 128, 0, 100, 613),
    (1, SPREAD + [1537] * 8, 8, 8, 72, 0, 0, 1537),
]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(str(v) for v in c[2:]) + f"-{c[0]}-{len(c[1])}")
def test_decode_of_many_sequences(gpu, case, fused):
    test_decode(gpu, case, fused)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("sinks,capacity", [(0, 7), (3, 10), (0, 64), (5, 300), (128, 129)])
def test_store(gpu, dtype, sinks, capacity):
    torch, pb = gpu
    K, D, pad = 3, 24, 4
    offsets, T = [2, 2, 3, 40, 47, 247, 250], 255
    lengths = [0, 1, 37, 20, 200, 2]                          # one with tokens in front, one with fewer tokens than rows
    B = len(lengths)
    g = torch.Generator().manual_seed(2)
    rows = [torch.randn(T, K * D + pad, generator=g).to(dt(torch, dtype)) for _ in range(2)]
    want = [torch.full((B, K, capacity, D), 7.0, dtype=dt(torch, dtype)) for _ in range(2)]
    for b in range(B):
        count = offsets[b + 1] - offsets[b]
        for i in range(count):
            p = lengths[b] - count + i
            if p >= 0 and (p < sinks or p >= lengths[b] - (capacity - sinks)):
                for w, r in zip(want, rows):
                    w[b, :, slot(p, sinks, capacity)] = r[offsets[b] + i, :K * D].reshape(K, D)
    got = [torch.full((B, K, capacity, D), 7.0, dtype=dt(torch, dtype), device="cuda") for _ in range(2)]
    desc = pb.parle_cache_desc(dtype, B, capacity, K, K, D, 0, sinks, 1.0, K * D, K * D + pad, K * D)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pb.parle_k_attention_store(desc, T, rows[0].cuda(), rows[1].cuda(), i32(offsets), i32(lengths), *got)
    for w, c in zip(want, got):
        assert torch.equal(w, c.cpu())


@pytest.mark.parametrize("window,sinks,capacity", [(0, 0, 64), (12, 3, 15), (12, 3, 40)])
def test_answers_follow_whole_sequences(gpu, window, sinks, capacity):
    """Prompts stored, then tokens one by one: each sees what it would in attention over the whole sequence."""
    torch, pb = gpu
    H, K, D, prompts, total = 4, 2, 64, [20, 1, 9], 50
    B = len(prompts)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(B, total, H + 2 * K, D, generator=g).bfloat16().cuda()
    W = (H + 2 * K) * D
    flat = x.reshape(B, total, W)
    desc = pb.parle_attention_desc(1, B, total, 1, H, K, D, window, sinks, D ** -0.5, W, total * W, W, total * W, H * D, total * H * D)
    whole, lse = torch.empty(B, total, H * D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, total, device="cuda")
    pb.parle_k_attention_forward(desc, flat, flat[..., H * D:], flat[..., (H + K) * D:], None, whole, lse)
    cd = pb.parle_cache_desc(1, B, capacity, H, K, D, window, sinks, D ** -0.5, W, W, H * D)
    caches = [torch.full((B, K, capacity, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    packed = torch.cat([flat[b, :n] for b, n in enumerate(prompts)])
    offsets = torch.tensor([0] + [sum(prompts[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
    lengths = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    pb.parle_k_attention_store(cd, sum(prompts), packed[:, H * D:], packed[:, (H + K) * D:], offsets, lengths, *caches)
    sc = scratch(torch, pb.parle_k_decode_scratch_bytes(cd))
    out = torch.empty(B, H * D, dtype=torch.bfloat16, device="cuda")
    for step in range(total - max(prompts)):
        lengths += 1
        row = torch.stack([flat[b, int(n) - 1] for b, n in enumerate(lengths.tolist())])
        pb.parle_k_attention_decode(cd, row, row[:, H * D:], row[:, (H + K) * D:], lengths, sc, *caches, out)
        want = torch.stack([whole[b, int(n) - 1] for b, n in enumerate(lengths.tolist())])
        # both are off by one rounding of the probabilities and one of the result, of values up to about 4
        assert (out.float() - want.float()).abs().max() <= 4 * 4 * 2.0 ** -8


def test_graph_steps_through_a_sequence(gpu):
    """One captured step, lengths counted up on the device: each replay is the eager step."""
    torch, pb = gpu
    B, H, K, D, capacity = 3, 4, 2, 64, 300
    desc = pb.parle_cache_desc(1, B, capacity, H, K, D, 0, 0, D ** -0.5, H * D, K * D, H * D)
    g = torch.Generator().manual_seed(4)
    make = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    q, k, v = make(B, H * D), make(B, K * D), make(B, K * D)
    kc, vc = make(B, K, capacity, D), make(B, K, capacity, D)
    lengths = torch.tensor([150, 200, 1], dtype=torch.int32, device="cuda")
    out, sc = torch.empty(B, H * D, dtype=torch.bfloat16, device="cuda"), scratch(torch, pb.parle_k_decode_scratch_bytes(desc))
    ekc, evc, eout, esc = kc.clone(), vc.clone(), out.clone(), sc.clone()
    el = lengths.clone()
    pb.parle_k_attention_decode(desc, q, k, v, lengths, sc, kc, vc, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lengths.add_(1)
        pb.parle_k_attention_decode(desc, q, k, v, lengths, sc, kc, vc, out)
    pb.parle_k_attention_decode(desc, q, k, v, el, esc, ekc, evc, eout)
    for step in range(4):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g))
        graph.replay()
        el += 1
        pb.parle_k_attention_decode(desc, q, k, v, el, esc, ekc, evc, eout)
        torch.cuda.synchronize()
        assert torch.equal(out, eout) and torch.equal(kc, ekc) and torch.equal(vc, evc)


def test_caches_beyond_32_bits(gpu):
    torch, pb = gpu
    B, K, D, capacity = 2, 1, 128, 9 << 20                    # 1.2e9 elements a sequence: the second begins beyond 2^31 bytes, ends beyond 2^31 elements
    kc, vc = (torch.zeros((B, K, capacity, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    desc = pb.parle_cache_desc(1, B, capacity, 1, K, D, 8, 1, 1.0, D, D, D)
    q, k, v = (torch.full((B, D), x, dtype=torch.bfloat16, device="cuda") for x in (1.0, 1.0, 3.0))
    lengths = torch.tensor([capacity, capacity - 1], dtype=torch.int32, device="cuda")
    out = torch.empty(B, D, dtype=torch.bfloat16, device="cuda")
    pb.parle_k_attention_decode(desc, q, k, v, lengths, scratch(torch, pb.parle_k_decode_scratch_bytes(desc)), kc, vc, out)
    assert (out == 3.0).all()                                 # its own key scores 128 above the others
    assert (vc[0, 0, -1] == 3).all() and (vc[1, 0, -2] == 3).all() and int((vc != 0).sum()) == 2 * D
