"""CPU-only: calls of the token-model operators that are refused for their buffers or the last of their sizes, and scratch by the row."""
from test_token_api import P, _call, embed, norm, pb

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


def test_embed_refuses_rows_that_its_loops_do_not_count():
    for dim in (2 ** 31 - 1, 2 ** 31 - 2048, (1 << 22) + 1):
        d = embed(n=1, tokens=1, vocab=1, dim=dim, table_stride=dim)
        assert pb.parle_k_embed_scratch_bytes(d) == -1, dim
        for name, ptrs in (("parle_k_embed_forward", (P, P, P)), ("parle_k_embed_backward", (P, P, None, 0, P))):
            status, text = _call(name, d, *ptrs)
            assert status == pb.PARLE_ESIZE and "2^22" in text
    assert pb.parle_k_embed_scratch_bytes(embed(n=1, tokens=1, vocab=1, dim=1 << 22, table_stride=1 << 22)) == 0


def test_norm_refuses_a_grid_beyond_a_launch():
    """A launch takes less than 2^32 threads; rows of more than 4096 elements have 1024 each."""
    for dim, rows, ok in ((4096, 1 << 22, True), (4097, 1 << 22, False), (4097, (1 << 22) - 1, True), (20000, 1 << 22, False)):
        d = norm(n=1, rows=rows, dim=dim, w_stride=dim)
        assert (pb.parle_k_rmsnorm_scratch_bytes(d) >= 0) == ok, (dim, rows)
        if not ok:
            status, text = _call("parle_k_rmsnorm_forward", d, P, None, P, OTHER, None, P, P, None)
            assert status == pb.PARLE_ESIZE and "2^22 - 1" in text
