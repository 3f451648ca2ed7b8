"""RMS norm with results written over what they come from, at every row length's kernel: the bits of calls with buffers of their own."""
import itertools

import pytest

from test_gpu_token_ops import gpu, randn, scratch, up  # noqa: F401

pytestmark = pytest.mark.gpu

# widths of every kernel, most of them odd: threads at a row's end then share elements with neighbours, of other wavefronts from 1025 on
DIMS = [5, 57, 125, 250, 511, 1001, 1025, 1531, 2047, 2049, 4095, 4097, 8191, 8193, 16383, 16384, 16385, 20001]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_over_its_inputs(gpu, dtype, dim):
    torch, pb = gpu
    n, rows = 2, 150
    x, resid, w = randn(torch, 1, n, rows, dim, dtype=dtype), randn(torch, 2, n, rows, dim, dtype=dtype), randn(torch, 3, n, dim)
    desc = pb.parle_norm_desc(dtype, 0, n, rows, dim, dim, 1e-6)
    codes = lambda: (torch.zeros((n, rows, up(dim, 16)), dtype=torch.uint8, device="cuda"), torch.zeros((n, rows, up(up(dim, 128) // 128, 4)), dtype=torch.uint8, device="cuda"))  # noqa: E731
    for r in (resid, None):
        h, y, rstd, q = torch.empty_like(x), torch.empty_like(x), torch.empty((n, rows), device="cuda"), codes()
        pb.parle_k_rmsnorm_forward(desc, x, r, w, h, y, *q, rstd)
        places = [None, "x", "own"] + (["resid"] if r is not None else [])
        for at_h, at_y in itertools.product(places, places):
            if at_h == at_y and at_h in ("x", "resid"):
                continue
            bufs = {"x": x.clone(), "resid": None if r is None else r.clone()}
            out_h, out_y = (None if at is None else bufs[at] if at in bufs else torch.empty_like(x) for at in (at_h, at_y))
            q2, rstd2 = codes(), torch.empty_like(rstd)
            pb.parle_k_rmsnorm_forward(desc, bufs["x"], bufs["resid"], w, out_h, out_y, *q2, rstd2)
            for got, want in ((out_h, h), (out_y, y), (rstd2, rstd), (q2[0], q[0]), (q2[1], q[1])):
                assert got is None or torch.equal(got, want), (at_h, at_y, r is not None)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_gradient_over_its_inputs(gpu, dtype, dim):
    torch, pb = gpu
    n, rows = 2, 150
    h, dout, dresid = (randn(torch, i, n, rows, dim, dtype=dtype) for i in (1, 2, 3))
    w, rstd = randn(torch, 4, n, dim), randn(torch, 5, n, rows).abs() + 0.5
    desc = pb.parle_norm_desc(dtype, 0, n, rows, dim, dim, 1e-6)
    sc = scratch(torch, pb.parle_k_rmsnorm_scratch_bytes(desc))
    for e in (dresid, None):
        dx, dw = torch.empty_like(h), torch.empty_like(w)
        pb.parle_k_rmsnorm_backward(desc, h, w, rstd, dout, e, sc, dx, dw)
        for at in range(3 if e is not None else 2):
            bufs, dw2 = [h.clone(), dout.clone(), None if e is None else e.clone()], torch.empty_like(w)
            pb.parle_k_rmsnorm_backward(desc, bufs[0], w, rstd, bufs[1], bufs[2], sc, bufs[at], dw2)
            assert torch.equal(bufs[at], dx) and torch.equal(dw2, dw), (at, e is not None)
