"""Log probabilities of rows whose logits lie far from zero: finite masks of any magnitude, whole rows of them, and forced classes, against 64 bits."""
import math

import pytest

from test_gpu_token_ops import U, _logprob_reference, dt, gpu, randn, scratch, within  # noqa: F401

pytestmark = pytest.mark.gpu

PATTERNS = 6


def _far_logits(torch, rows, classes, dtype, value):
    """Row i by i % 6: normal logits with `value` in every third class, from class 20 on, in the second half, everywhere, everywhere with
    normal differences (where the type keeps them), and in one class."""
    x = randn(torch, 21, 1, rows, classes, scale=3.0).cpu()
    at = torch.arange(classes)
    for kind, where in enumerate((at % 3 == 0, at >= 20, at >= classes // 2, at >= 0, at < 0, at == classes * 2 // 3)):
        x[:, kind::PATTERNS] = torch.where(where, torch.full((), value), x[:, kind::PATTERNS])
    x[:, 4::PATTERNS] += value
    return x.to(dt(torch, dtype))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes,top", [(6, 129, 3), (6, 40000, 5), (516, 3001, 4)])
@pytest.mark.parametrize("value", [-9e5, -1e6, -1.1e6, -1e9, -3e9, -5e9, -1e10, -1e11, -1e18, -1e20, -1e30, -3e38, 9e5, 1e6, 1.1e6, 1e10, 1e12, 1e30, 2.4e38, 3.3e38])
def test_logprob_far_values(gpu, dtype, rows, classes, top, value):
    torch, pb = gpu
    x = _far_logits(torch, rows, classes, dtype, value)
    label = torch.randint(0, classes, (1, rows), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    label[:, 1::PATTERNS] %= 20
    desc = pb.parle_logprob_desc(dtype, 1, rows, classes, top, classes)
    logp, ent, lse, alt = (torch.full(s, 3.0, device="cuda") for s in ((1, rows), (1, rows), (1, rows), (1, rows, top)))
    ids = torch.full((1, rows, top), 3, dtype=torch.int32, device="cuda")
    pb.parle_k_logprob_forward(desc, x.cuda(), label.cuda(), scratch(torch, pb.parle_k_logprob_scratch_bytes(desc)), logp, ent, lse, ids, alt)
    pick = torch.cat([torch.arange(PATTERNS), torch.arange(max(PATTERNS, rows - PATTERNS), rows)])
    some = lambda t: t[0, pick.to(t.device)]  # noqa: E731
    wl, wh, wp, wi, wa = _logprob_reference(torch, some(x).double(), some(label), top)
    # a thread adds classes / 256 terms (a vector's eight at least), and some forty roundings join lanes, wavefronts and parts, an
    # exponential's own among them
    chain = (classes / 256 + 48) * U
    within(some(lse), wl, wl.abs() * 2 * U + chain, "lse")
    # (x - m) - log z: the difference, log z and their difference are rounded once each
    tp = lambda w: chain + 3 * U * (w.abs() + math.log(classes))  # noqa: E731
    within(some(logp), wp, tp(wp), "logp")
    within(some(ent), wh, (2 * (wh.abs() + math.log(classes)) + 2) * chain, "entropy")
    assert torch.equal(some(ids).cpu(), wi), "alternatives"
    within(some(alt), wa, tp(wa), "top_logp")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(4, 40000), (516, 3001)])
def test_logprob_nan_beside_far_values(gpu, dtype, rows, classes):
    """A NaN makes its row NaN whatever lies beside it, and no other row."""
    torch, pb = gpu
    x = torch.full((1, rows, classes), -1e10)
    x[0, 1] = -math.inf
    x[0, 2] = 1e10
    x[0, 0, 77] = x[0, 1, 77] = x[0, 2, classes - 1] = math.nan
    desc = pb.parle_logprob_desc(dtype, 1, rows, classes, 0, classes)
    out = [torch.zeros((1, rows), device="cuda") for _ in range(3)]
    label = torch.zeros((1, rows), dtype=torch.int32, device="cuda")
    pb.parle_k_logprob_forward(desc, x.to(dt(torch, dtype)).cuda(), label, scratch(torch, pb.parle_k_logprob_scratch_bytes(desc)), *out, None, None)
    for t in out:
        assert t.isnan().nonzero().tolist() == [[0, 0], [0, 1], [0, 2]]
