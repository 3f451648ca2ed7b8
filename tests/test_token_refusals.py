"""CPU-only: calls of the token-model operators that are refused for their buffers or the last of their sizes, and scratch by the row."""
from test_token_api import P, _call, norm, pb

OTHER = P + 0x1000


def test_norm_refuses_h_and_y_in_one_buffer():
    status, text = _call("parle_k_rmsnorm_forward", norm(), P, None, P, OTHER, OTHER, None, None, None)
    assert status == pb.PARLE_EINVAL and "one buffer" in text


def test_norm_gradient_has_a_row_for_every_thread():
    """Scratch holds a part of dw for each workgroup: no more of them than rows divided by what one takes at a time."""
    for dim, at_once in ((3, 16), (8, 32), (64, 32), (65, 16), (128, 16), (129, 8), (256, 8), (257, 4), (1024, 4)):
        for rows in (1, 31, 500, 8000, 20000, 33000, 100001):
            parts = pb.parle_k_rmsnorm_scratch_bytes(norm(n=1, rows=rows, dim=dim, w_stride=dim)) // (4 * (-(-dim // 8) * 8))
            strip = next(k for k in range(1, rows + at_once + 1) if -(-rows // k) <= parts)        # the fewest rows that a part may have
            assert parts <= -(-rows // at_once) and (parts == 1 or -(-rows // (-(-strip // at_once) * at_once)) == parts), (dim, rows, parts)
