"""NaN codes and NaN scales through every kernel of the 8-bit product: they stay in their row and column."""
import pytest

from test_gpu_token_ops import _random_codes, gpu, scratch  # noqa: F401

pytestmark = pytest.mark.gpu


# few rows with one to eight shares of the contraction, tiles of every size, a contraction in shares
@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("n,rows,cols,depth,b_block", [
    (1, 4, 200, 300, 1), (2, 16, 40, 1024, 128), (1, 5, 70, 2100, 1), (1, 16, 33, 4100, 1), (1, 17, 40, 4224, 1), (2, 64, 130, 1030, 128), (1, 200, 200, 300, 1), (1, 600, 600, 256, 128),
    (1, 700, 2100, 520, 1), (3, 500, 1100, 260, 128), (1, 2600, 300, 140, 1), (2, 1500, 2000, 1024, 1), (1, 4100, 4000, 300, 128), (1, 2100, 8192, 1024, 1)])
def test_fp8_nan_stays(gpu, out_dtype, n, rows, cols, depth, b_block):
    torch, pb = gpu
    a, sa, _ = _random_codes(torch, 1, n, rows, depth, 1)
    b, sb, _ = _random_codes(torch, 2, n, cols, depth, b_block)
    a, b = a | 1, b | 1                                   # no zeros: every product with a NaN scale is a NaN by any reading
    a[(a & 0x7F) == 0x7F], b[(b & 0x7F) == 0x7F] = 0x31, 0x31
    a[..., depth:], b[..., depth:] = 0, 0
    want = torch.zeros(n, rows, cols, dtype=torch.bool)
    a[0, rows - 1, depth - 1] = 0x7F
    want[0, rows - 1] = True
    b[n - 1, cols // 2, 0] = 0xFF
    want[n - 1, :, cols // 2] = True
    sa[n - 1, 0, (depth - 1) // 128] = 0xFF
    want[n - 1, 0] = True
    sb[0, -1, 0] = 0xFF                                   # the last row of b, or its last block of rows
    want[0, :, (cols - 1) // b_block * b_block:] = True
    desc = pb.parle_fp8_desc(out_dtype, b_block, 0, n, rows, cols, depth, cols, rows * cols)
    out = torch.zeros((n, rows, cols), dtype=torch.bfloat16 if out_dtype else torch.float32, device="cuda")
    pb.parle_k_fp8_matmul(desc, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, scratch(torch, pb.parle_k_fp8_scratch_bytes(desc)), out)
    assert torch.equal(out.isnan().cpu(), want)
