"""The token model on the GPU: its gradient against the same model in 64 bits, its training by Parle, its answers."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1707_00424_amd import token_model
    return torch, token_model


def _reference(torch, model, rep, tokens, labels):
    """Loss and gradient of one replica's parameters, in 64 bits without any 8-bit operand."""
    y = model.parle.y[rep].detach().cpu().double().requires_grad_(True)
    seg = lambda name, *shape: y[model.at[name][0]:model.at[name][0] + model.at[name][1]].reshape(shape)  # noqa: E731
    V, D = model.V, model.D
    t = tokens[rep].cpu().long()
    h = seg("table", V, D)[t.clamp(min=0)] * math.sqrt(D) * (t >= 0)[:, None]
    for i in range(model.L + 1):
        norm, w = model._names(i)
        n = h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * seg(norm, D)
        out = n @ seg(w, D if i < model.L else V, D).t()
        h = h + out if i < model.L else out
    lab = labels[rep].cpu().long()
    logp = torch.log_softmax(h, -1).gather(-1, lab.clamp(min=0)[:, None])[:, 0]
    loss = -(logp * (lab >= 0)).sum() / (lab >= 0).sum()
    loss.backward()
    return float(loss.detach()), y.grad


def test_gradient_follows_the_model(gpu):
    torch, tm = gpu
    n, T, V, D = 2, 190, 300, 72
    model = tm.TokenModel(n, T, V, D, layers=2, seed=3)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(-1, V, (n, T), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(-1, V, (n, T), generator=g, device="cuda", dtype=torch.int32)
    model.parle.y.mul_(1.0 + 0.1 * torch.arange(n, device="cuda")[:, None])     # replicas that differ
    model.forward(tokens, labels)
    given = (labels >= 0).sum(1)
    loss = -(model.logp * (labels >= 0)).sum(1) / given
    model.backward(tokens, labels)
    torch.cuda.synchronize()
    for rep in range(n):
        want, grad = _reference(torch, model, rep, tokens, labels)
        # e4m3 is off by 2^-4 at most of a value, about a third of that on average; an 8-bit product of D such terms with random signs is
        # off by 2^-4 * sqrt(2) / 3 of its own size, three layers of them
        assert abs(float(loss[rep]) - want) <= 0.1 * want
        for name, (at, size) in model.at.items():
            a, b = model.parle.grad[rep, at:at + size].cpu().double(), grad[at:at + size]
            cos = float((a * b).sum() / (a.norm() * b.norm()))
            # errors of 3 % of each of the six to eight products on the way are at right angles to the gradient: cos > 1 - 8 * 0.05^2
            assert cos > 0.98 and abs(float(a.norm() / b.norm()) - 1) < 0.1, (name, cos, float(a.norm() / b.norm()))
        untouched = torch.ones(V, dtype=torch.bool)
        untouched[tokens[rep][tokens[rep] >= 0].cpu().long()] = False
        table = model.parle.grad[rep, :V * D].reshape(V, D).cpu()
        assert (table[untouched] == 0).all() and (table[~untouched] != 0).any(1).all()


def test_training_learns_the_source(gpu):
    torch, tm = gpu
    n, T, V, D = 3, 512, 64, 64
    model = tm.TokenModel(n, T, V, D, layers=1)
    batch = tm.source(torch, V)
    for k in range(100):
        model.step(*batch(n, T))
        if (k + 1) % model.parle.cfg.L == 0:
            model.parle.parle_outer_step()
    loss = -model.logp.mean().item()
    # the source's entropy: p = 3/4 + 1/256 for one token, 1/256 for each other
    p = 0.75 + 0.25 / V
    entropy = -p * math.log(p) - (V - 1) * (0.25 / V) * math.log(0.25 / V)
    assert entropy - 0.1 < loss < entropy + 0.35, (loss, entropy)
    ids, logp = model.alternatives(torch.arange(V, dtype=torch.int32, device="cuda"), top=2)
    want = (7 * torch.arange(V) + 3) % V
    assert (ids[:, 0].cpu() == want).float().mean() > 0.9
    assert logp[:, 0].exp().mean() > 0.4
