"""Sums of the 8-bit product: what large products that cancel leave of a small one beside them."""
import pytest

from test_gpu_token_ops import gpu, scratch, up  # noqa: F401

pytestmark = pytest.mark.gpu


def _code(torch, v):
    return int(torch.tensor([v]).to(torch.float8_e4m3fn).view(torch.uint8))


def _cancelling(torch, n, rows, cols, depth, small):
    """Products 2^16, -2^16 and `small` among each eight neighbours of the contraction, in places that move on with the row."""
    a = torch.zeros(n, rows, depth, dtype=torch.uint8)
    b = torch.zeros(n, cols, depth, dtype=torch.uint8)
    k = torch.arange(depth)
    b[:] = torch.where(k % 8 < 6, _code(torch, 256.0), _code(torch, 1.0)).to(torch.uint8)
    for r in range(rows):
        for place, v in (((r % 6), 256.0), ((r + 1 + r // 6 % 5) % 6, -256.0), (6 + r % 2, small)):
            a[:, r, place::8] = _code(torch, v)
    scales = lambda count: torch.nn.functional.pad(torch.full((n, count, up(depth, 128) // 128), 127, dtype=torch.uint8), (0, up(up(depth, 128) // 128, 4) - up(depth, 128) // 128))  # noqa: E731
    return a.cuda(), scales(rows).cuda(), b.cuda(), scales(cols).cuda()


# a bf16 result of up to 16 rows and any fp32 result have fp32 sums: 2^16, -2^16 and what is beside them are exact in 24 bits, in any order
@pytest.mark.parametrize("out_dtype,rows", [(1, 1), (1, 4), (1, 16), (0, 1), (0, 16), (0, 17), (0, 100), (0, 300)])
@pytest.mark.parametrize("cols,depth", [(40, 16), (130, 128), (300, 1024), (70, 4096)])
@pytest.mark.parametrize("small", [0.25, 1.0, 4.0])
def test_fp8_sums_are_fp32(gpu, out_dtype, rows, cols, depth, small):
    torch, pb = gpu
    n = 2
    a, sa, b, sb = _cancelling(torch, n, rows, cols, depth, small)
    desc = pb.parle_fp8_desc(out_dtype, 1, 0, n, rows, cols, depth, cols, rows * cols)
    out = torch.zeros((n, rows, cols), dtype=torch.bfloat16 if out_dtype else torch.float32, device="cuda")
    pb.parle_k_fp8_matmul(desc, a, sa, b, sb, None, scratch(torch, pb.parle_k_fp8_scratch_bytes(desc)), out)
    assert (out.double() == small * depth / 8).all()      # powers of two: exact in either type
