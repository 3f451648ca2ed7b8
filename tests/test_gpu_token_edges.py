"""Token-model operators at the edges of their dispatch rules: sizes on both sides of each limit, against 64 bits."""
import math

import pytest

from test_gpu_token_ops import HALF, U, _embed_grad_reference, _largest_of_eight, _random_codes, d64, gpu, randn, scratch, up, within  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,tokens,vocab,dim,same", [
    (1, 512, 40, 24, False), (2, 513, 40, 24, False), (1, 512, 3, 2051, True), (3, 300, 5000, 17, False), (1, 256, 9000, 8, False), (2, 257, 1, 5, True),
    (1, 1024, 33, 40, False), (1, 4096, 33, 8, False), (1, 8192, 70, 8, False), (1, 8193, 70, 9, False), (1, 32769, 40, 8, True)])
def test_embed_backward_limits(gpu, dtype, n, tokens, vocab, dim, same):
    torch, pb = gpu
    g = torch.Generator().manual_seed(tokens)
    t = torch.full((n, tokens), vocab - 1, dtype=torch.int32) if same else torch.randint(-1, vocab + 1, (n, tokens), generator=g, dtype=torch.int32)
    dout = randn(torch, 4, n, tokens, dim, dtype=dtype)
    rs = vocab * dim + 1
    desc = pb.parle_embed_desc(dtype, 0, n, tokens, vocab, dim, rs, 1.5)
    got = torch.full((n, rs), 9.0, device="cuda")
    pb.parle_k_embed_backward(desc, t.cuda(), dout, scratch(torch, pb.parle_k_embed_scratch_bytes(desc)), got)
    want, mass, count = _embed_grad_reference(torch, t, d64(dout), vocab, 1.5)
    within(got[:, :vocab * dim].reshape(n, vocab, dim), want, mass * (count[..., None] + 1) * U, "dtable")
    assert (got[:, vocab * dim:] == 9.0).all()


@pytest.mark.parametrize("kind", ["uniform", "tail", "same", "none"])
@pytest.mark.parametrize("dtype,n,tokens,vocab,dim,gap", [
    (1, 2, 600, 24001, 515, 1), (0, 1, 600, 3000000, 7, 0), (1, 2, 700, 6000, 2050, 2), (0, 2, 520, 1500, 9001, 3), (1, 1, 4100, 50001, 1024, 0), (1, 2, 1000, 3 << 20, 5, 3),
    (0, 1, 17000, 60000, 1028, 0), (1, 2, 600, 1 << 22, 4, 1), (1, 1, 600, 1 << 22, 3, 0),
    # few tokens: on both sides of the rule for one launch, by tokens (16, 17) and by tokens times bytes
    (1, 1, 16, 100000, 1024, 0), (0, 1, 17, 100000, 1024, 0), (0, 2, 100, 24001, 515, 1), (1, 2, 60, 24001, 515, 1), (1, 2, 64, 24001, 515, 2), (1, 2, 512, 700, 1023, 3),
    (0, 2, 511, 400, 2, 1), (1, 2, 300, 401, 1, 2), (0, 2, 90, 1000, 3, 3), (1, 3, 200, 3001, 5, 2), (1, 1, 300, 20, 9001, 0)])
def test_embed_backward_long_tables(gpu, dtype, n, tokens, vocab, dim, gap, kind):
    """Tables that are cleared beside the sums as well: the tokens' rows by the formula, zeros in all others, nothing behind a table."""
    torch, pb = gpu
    g = torch.Generator().manual_seed(11)
    low = {"uniform": -1, "tail": max(0, vocab - 300), "same": vocab - 1, "none": vocab}[kind]
    t = torch.randint(low, vocab + 1, (n, tokens), generator=g, dtype=torch.int32) if kind in ("uniform", "tail") else torch.full((n, tokens), low, dtype=torch.int32)
    dout = randn(torch, 12, n, tokens, dim, dtype=dtype)
    rs = vocab * dim + gap
    desc = pb.parle_embed_desc(dtype, 0, n, tokens, vocab, dim, rs, 1.25)
    got = torch.full((n, rs), 9.0, device="cuda")
    pb.parle_k_embed_backward(desc, t.cuda(), dout, scratch(torch, pb.parle_k_embed_scratch_bytes(desc)), got)
    assert (got[:, vocab * dim:] == 9.0).all(), "what lies behind the table was written"
    for a in range(n):
        rows, at = torch.unique(t[a].clamp(min=-1), return_inverse=True)
        at = torch.where((t[a] >= 0) & (t[a] < vocab), at, -1)
        want, mass, count = _embed_grad_reference(torch, at[None].int(), d64(dout[a:a + 1]), len(rows), 1.25)
        kept = (rows >= 0) & (rows < vocab)
        table = got[a, :vocab * dim].view(vocab, dim)
        of = rows[kept].long().cuda()
        # a sum of c terms in any order: c - 1 roundings at most on the way of each term, one more for the scale
        within(table[of][None], want[:, kept], mass[:, kept] * (count[:, kept, None] + 1) * U, "dtable")
        table[of] = 0.0
        assert not table.any(), "a row without tokens is not zero"



@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("n,rows,cols,depth,b_block", [
    (1, 16, 40, 1024, 1), (1, 17, 40, 1024, 128), (1, 17, 130, 1025, 1), (2, 40, 70, 4224, 128), (1, 100, 520, 2048, 128), (3, 500, 260, 130, 1), (1, 16, 33, 2048, 128),
    (1, 5, 100, 1000, 1), (2, 400, 1100, 260, 128), (1, 700, 2100, 520, 128), (6, 130, 515, 1024, 1), (1, 2600, 300, 140, 1)])
def test_fp8_matmul_limits(gpu, out_dtype, n, rows, cols, depth, b_block):
    torch, pb = gpu
    a, sa, av = _random_codes(torch, 16, n, rows, depth, 1)
    b, sb, bv = _random_codes(torch, 17, n, cols, depth, b_block)
    out = torch.full((n, rows, cols), 3.0, device="cuda").to(torch.bfloat16 if out_dtype else torch.float32)
    old, bias = out.clone(), randn(torch, 18, n, cols)
    desc = pb.parle_fp8_desc(out_dtype, b_block, 1, n, rows, cols, depth, cols, rows * cols)
    sc = scratch(torch, pb.parle_k_fp8_scratch_bytes(desc), fill=0xFF)
    pb.parle_k_fp8_matmul(desc, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), bias, sc, out)
    c = d64(bias)[:, None, :]
    want = torch.matmul(av, bv.transpose(1, 2)) + c + 3.0
    mass = torch.matmul(av.abs(), bv.abs().transpose(1, 2)) + c.abs() + 3.0
    cut = torch.stack([_largest_of_eight(torch, av[i], bv[i]) for i in range(n)]) * 7 * 2.0 ** -13 if out_dtype else 0.0
    within(out, want, mass * (depth + 2) * U + cut + want.abs() * (HALF[1] + U if out_dtype else 0), "out")
    again = old.clone()
    pb.parle_k_fp8_matmul(desc, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), bias, sc, again)
    assert torch.equal(again, out), "two calls differ"


@pytest.mark.parametrize("dim", [3, 8, 16, 63, 127, 128, 129, 200, 256, 257, 512, 513, 1024, 1536, 2047, 4096, 16384, 16385])
def test_rmsnorm_scales_and_padding(gpu, dim):
    """Codes, scales and their padding at every row length's kernel; nothing behind them is written."""
    torch, pb = gpu
    n, rows = 2, 5
    x = randn(torch, 1, n, rows, dim, dtype=1)
    w = torch.ones((n, dim), device="cuda")
    pitch, s_pitch = up(dim, 16), up(up(dim, 128) // 128, 4)
    q = torch.full((n * rows * pitch + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    s = torch.full((n * rows * s_pitch + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    desc = pb.parle_norm_desc(1, 0, n, rows, dim, dim, 1e-6)
    y = torch.empty_like(x, dtype=torch.bfloat16)
    pb.parle_k_rmsnorm_forward(desc, x, None, w, None, y, q, s, None)
    assert (q[n * rows * pitch:] == 0xEE).all() and (s[n * rows * s_pitch:] == 0xEE).all()
    codes, scales = q[:n * rows * pitch].reshape(n, rows, pitch).cpu(), s[:n * rows * s_pitch].reshape(n, rows, s_pitch).cpu()
    kb = up(dim, 128) // 128
    assert (codes[..., dim:] == 0).all() and (scales[..., kb:] == 0).all()
    wide = (2.0 ** (scales[..., :kb].double() - 127)).repeat_interleave(128, -1)[..., :dim]
    f = d64(x)
    want = f * (f.square().mean(-1, keepdim=True) + float(torch.tensor(1e-6))) ** -0.5
    t = ((dim + 3) / 2 + 6) * U
    within(codes.view(torch.float8_e4m3fn).double()[..., :dim] * wide, want, torch.maximum(want.abs() * 2.0 ** -4, wide * 2.0 ** -10) * (1 + t) + want.abs() * t, "codes")


def test_logits_at_every_alignment(gpu):
    """Rows that begin at every offset from 16 bytes; what lies next to them does not count, even where it is NaN."""
    torch, pb = gpu
    for dtype, size in ((0, 4), (1, 2)):
        for C in (1, 3, 8, 2050):
            ld = C + 1 + (C % 2)
            rows = 16 // size + 1
            x = torch.full((1, rows, ld), math.nan)
            x[..., :C] = torch.randn(1, rows, C, generator=torch.Generator().manual_seed(C))
            x = x.to(torch.bfloat16 if dtype else torch.float32)
            desc = pb.parle_logprob_desc(dtype, 1, rows, C, 1, ld)
            lse, ids, alt = torch.empty((1, rows), device="cuda"), torch.empty((1, rows, 1), dtype=torch.int32, device="cuda"), torch.empty((1, rows, 1), device="cuda")
            pb.parle_k_logprob_forward(desc, x.cuda(), None, scratch(torch, pb.parle_k_logprob_scratch_bytes(desc)), None, None, lse, ids, alt)
            v = x[0, :, :C].double()
            want = torch.logsumexp(v, -1)
            within(lse[0], want, want.abs() * 2 * U + (C / 256 + 48) * U, "lse")
            assert torch.equal(ids[0, :, 0].cpu(), v.argmax(-1).int())
            dl = torch.ones((1, rows), device="cuda")
            label = torch.zeros((1, rows), dtype=torch.int32, device="cuda")
            out = torch.full_like(x, 7.0).cuda()
            pb.parle_k_logprob_backward(desc, x.cuda(), label, lse, None, dl, None, out)
            assert out[..., :C].isfinite().all() and (out[..., C:] == 7).all()
