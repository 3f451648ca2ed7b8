"""CPU-only: calls of the token-model operators that are refused for their buffers or the last of their sizes."""
from test_token_api import P, _call, norm, pb

OTHER = P + 0x1000


def test_norm_refuses_h_and_y_in_one_buffer():
    status, text = _call("parle_k_rmsnorm_forward", norm(), P, None, P, OTHER, OTHER, None, None, None)
    assert status == pb.PARLE_EINVAL and "one buffer" in text
