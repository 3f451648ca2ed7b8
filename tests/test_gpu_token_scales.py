"""The 8-bit product at the ends of the scales' range: blocks whose scale is next to 2^-127."""
import pytest

from test_gpu_token_ops import HALF, gpu, scratch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("rows", [4, 64, 300])
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 9, 10])
def test_fp8_smallest_scales(gpu, out_dtype, rows, byte):
    """A block of a under 2^(byte - 127), b under the scale that brings products back to the codes': no scale counts as 0.  fp32 sums
    take operands as bf16 numbers, whose smallest step is 2^-133: half of that may be missing from each."""
    torch, pb = gpu
    cols, depth, other = 130, 128, 227 - byte
    codes = [0x01, 0x07, 0x0F, 0x38, 0x7E, 0xB9]
    for c in codes:
        a, b = torch.full((1, rows, depth), c, dtype=torch.uint8, device="cuda"), torch.full((1, cols, depth), 0x38, dtype=torch.uint8, device="cuda")
        sa, sb = torch.full((1, rows, 4), byte, dtype=torch.uint8, device="cuda"), torch.full((1, cols, 4), other, dtype=torch.uint8, device="cuda")
        desc = pb.parle_fp8_desc(out_dtype, 1, 0, 1, rows, cols, depth, cols, rows * cols)
        out = torch.zeros((1, rows, cols), dtype=torch.bfloat16 if out_dtype else torch.float32, device="cuda")
        pb.parle_k_fp8_matmul(desc, a, sa, b, sb, None, scratch(torch, pb.parle_k_fp8_scratch_bytes(desc)), out)
        value = float(torch.tensor([c], dtype=torch.uint8).view(torch.float8_e4m3fn).double())
        want = value * 2.0 ** (byte - 127) * 2.0 ** (other - 127) * depth
        step = 2.0 ** -134 * 2.0 ** (other - 127) * depth if not out_dtype or rows <= 16 else 0.0
        assert ((out.double() - want).abs() <= step + abs(want) * HALF[out_dtype]).all(), hex(c)
