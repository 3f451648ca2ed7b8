"""The token model with attention on the GPU: its gradient against the same model in 64 bits, and its answers token by token."""
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


def _logits(torch, model, y, tokens, length):
    """Logits of one replica's parameters y (float64) for tokens [T], sequences of ``length``, without any 8-bit operand."""
    V, D, A = model.V, model.D, model.A
    seg = lambda name, *shape: y[model.at[name][0]:model.at[name][0] + model.at[name][1]].reshape(shape)  # noqa: E731
    t = tokens.long()
    T = len(t)
    pos = torch.arange(T) % length
    i = torch.arange(T)
    see = (i[:, None] // length == i[None, :] // length) & (i[None, :] <= i[:, None])
    if A.window:
        see &= (i[None, :] > i[:, None] - A.window) | (pos[None, :] < A.sinks)
    angle = pos.double()[:, None] * (10000.0 ** (-torch.arange(A.dim // 2) / (A.dim / 2))).double()

    def turn(x):
        a, b = x[..., :A.dim // 2], x[..., A.dim // 2:]
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        return torch.cat((a * c - b * s, a * s + b * c), -1)

    def norm(h, name):
        return h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * seg(name, D)

    h = seg("table", V, D)[t.clamp(min=0)] * math.sqrt(D) * (t >= 0)[:, None]
    for layer in range(model.L):
        qkv = norm(h, f"norm_a{layer}") @ seg(f"qkv{layer}", (A.heads + 2 * A.kv_heads) * A.dim, D).t()
        q, k, v = qkv.reshape(T, -1, A.dim).split((A.heads, A.kv_heads, A.kv_heads), 1)
        q, k = turn(q), turn(k).repeat_interleave(A.heads // A.kv_heads, 1)
        v = v.repeat_interleave(A.heads // A.kv_heads, 1)
        p = torch.softmax((torch.einsum("ihd,jhd->hij", q, k) * A.dim ** -0.5).masked_fill(~see, -math.inf), -1)
        h = h + torch.einsum("hij,jhd->ihd", p, v).reshape(T, -1) @ seg(f"out{layer}", D, A.heads * A.dim).t()
        h = h + norm(h, f"norm{layer}") @ seg(f"w{layer}", D, D).t()
    return norm(h, "norm") @ seg("classes", V, D).t()


@pytest.mark.parametrize("window,sinks", [(0, 0), (17, 2)])
def test_gradient_follows_the_model(gpu, window, sinks):
    torch, tm = gpu
    n, T, V, D, sequences = 2, 192, 300, 72, 3
    A = tm.Heads(heads=6, kv_heads=2, dim=24, window=window, sinks=sinks, sequences=sequences)
    model = tm.TokenModel(n, T, V, D, layers=2, seed=3, attention=A)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(-1, V, (n, T), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(-1, V, (n, T), generator=g, device="cuda", dtype=torch.int32)
    model.parle.y.mul_(1.0 + 0.1 * torch.arange(n, device="cuda")[:, None])     # replicas that differ
    model.forward(tokens, labels)
    given = (labels >= 0).sum(1)
    loss = -(model.logp * (labels >= 0)).sum(1) / given
    model.backward(tokens, labels)
    first = model.parle.grad.clone()
    model.forward(tokens, labels)
    model.backward(tokens, labels)
    assert torch.equal(first, model.parle.grad), "two passes differ"
    for rep in range(n):
        y = model.parle.y[rep].detach().cpu().double().requires_grad_(True)
        lab = labels[rep].cpu().long()
        logp = torch.log_softmax(_logits(torch, model, y, tokens[rep].cpu(), T // sequences), -1).gather(-1, lab.clamp(min=0)[:, None])[:, 0]
        want = -(logp * (lab >= 0)).sum() / (lab >= 0).sum()
        want.backward()
        # an 8-bit product is off by 2^-4 * sqrt(2) / 3 of its own size, 3 %; seven of them lie on the way of the loss
        assert abs(float(loss[rep]) - want.item()) <= 0.15 * want.item()
        for name, (at, size) in model.at.items():
            a, b = model.parle.grad[rep, at:at + size].cpu().double(), y.grad[at:at + size]
            cos = float((a * b).sum() / (a.norm() * b.norm()))
            # errors of 3 % of each of up to fourteen products at right angles to the gradient: cos > 1 - 14 * 0.05^2
            assert cos > 0.96 and abs(float(a.norm() / b.norm()) - 1) < 0.15, (name, cos, float(a.norm() / b.norm()))


@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 1)])
def test_answers_are_those_of_whole_sequences(gpu, window, sinks):
    """The most likely token after each answered one, from caches, is near the most likely of the model on the whole sequence in 64 bits."""
    torch, tm = gpu
    V, D = 200, 64
    A = tm.Heads(heads=4, kv_heads=2, dim=32, window=window, sinks=sinks)
    model = tm.TokenModel(1, 64, V, D, layers=2, seed=5, attention=A)
    g = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, V, (k,), generator=g, dtype=torch.int32) for k in (9, 1, 4)]
    count = 12
    uniform = torch.rand((3, count), generator=g).cuda()
    got = model.answer(prompts, uniform, temperature=torch.zeros(3, device="cuda")).cpu()
    assert torch.equal(got, model.answer(prompts, uniform * 0.5, temperature=torch.zeros(3, device="cuda")).cpu()), "greedy answers depend on the numbers"
    y = model.parle.x_ref.cpu().double()
    for p, a in zip(prompts, got):
        whole = torch.cat((p, a))
        logits = _logits(torch, model, y, whole, len(whole))[len(p) - 1:-1]
        spread = logits.std(-1)
        # each product is off by 3 % of its size, seven of them by 8 %; two logits of 200 that are that near may change places, by three of those at most
        assert ((logits.amax(-1) - logits.gather(-1, a.long()[:, None])[:, 0]) <= 3 * 2 * 0.08 * spread).all()
    drawn = model.answer(prompts, uniform, top_k=torch.full((3,), 20, dtype=torch.int32, device="cuda"), top_p=torch.full((3,), 0.9, device="cuda"))
    assert ((drawn >= 0) & (drawn < V)).all() and drawn.shape == (3, count)


@pytest.mark.parametrize("sinks", [4, 5, 128])
def test_answers_no_longer_than_the_sinks(gpu, sinks):
    """Without a window all tokens are seen, sinks or not: the answers are those of the same model without sinks."""
    torch, tm = gpu
    prompts = [torch.tensor([3], dtype=torch.int32), torch.tensor([5, 6], dtype=torch.int32)]
    uniform = torch.rand((2, 3), generator=torch.Generator().manual_seed(1)).cuda()
    make = lambda s: tm.TokenModel(1, 32, 100, 32, layers=1, seed=4, attention=tm.Heads(heads=2, kv_heads=1, dim=16, sinks=s))  # noqa: E731
    assert torch.equal(make(sinks).answer(prompts, uniform), make(0).answer(prompts, uniform))


def test_rules_of_any_type_and_place(gpu):
    """Numbers and rules are converted, not read as what they are not; every second row of a 64-bit top_k had none."""
    torch, tm = gpu
    model = tm.TokenModel(1, 32, 100, 32, layers=1, seed=4, attention=tm.Heads(heads=2, kv_heads=1, dim=16))
    B = 4
    prompts = [torch.tensor([3 + i], dtype=torch.int32) for i in range(B)]
    uniform = torch.rand((B, 6), generator=torch.Generator().manual_seed(1))
    rules = dict(temperature=torch.tensor([2.0, 1.0, 3.0, 0.5]), top_k=torch.tensor([1, 2, 1, 3]), top_p=torch.tensor([0.9, 0.8, 1.0, 0.7]), min_p=torch.tensor([0.0, 0.1, 0.0, 0.2]))
    want = model.answer(prompts, uniform.cuda(), **{k: v.to(torch.int32 if k == "top_k" else torch.float32).cuda() for k, v in rules.items()})
    assert torch.equal(want, model.answer(prompts, uniform, **rules))
    assert torch.equal(want, model.answer([p.cuda().long() for p in prompts], uniform.double().cuda(), **{k: (v if k == "top_k" else v.double()).cuda() for k, v in rules.items()}))
    assert torch.equal(want, model.answer(prompts, uniform, **{k: torch.stack((v, v), 1)[:, 0] for k, v in rules.items()}))
    # more classes than 32 bits count are all of them
    assert torch.equal(model.answer(prompts, uniform), model.answer(prompts, uniform, top_k=torch.full((B,), 1 << 40)))
    for k, v in rules.items():
        for bad in (v[:3], v[0]):
            with pytest.raises(ValueError, match=k):
                model.answer(prompts, uniform, **{k: bad})
    with pytest.raises(ValueError, match="answer needs"):
        model.answer([], uniform[:0])


def test_a_model_without_attention_answers_too(gpu):
    torch, tm = gpu
    model = tm.TokenModel(1, 32, 100, 32, layers=1)
    prompts = [torch.tensor([3, 4], dtype=torch.int32), torch.tensor([5], dtype=torch.int32)]
    uniform = torch.rand((2, 4), generator=torch.Generator().manual_seed(1)).cuda()
    got = model.answer(prompts, uniform, temperature=torch.zeros(2, device="cuda"))
    ids, _ = model.alternatives(torch.tensor([4, 5], dtype=torch.int32, device="cuda"), top=1)
    assert torch.equal(got[:, 0], ids[:, 0])


def test_refusals(gpu):
    torch, tm = gpu
    with pytest.raises(ValueError, match="equal length"):
        tm.TokenModel(1, 10, 50, 32, attention=tm.Heads(sequences=3))
    model = tm.TokenModel(1, 32, 100, 32, layers=1, attention=tm.Heads(heads=2, kv_heads=1, dim=16))
    one, uniform = torch.tensor([3], dtype=torch.int32), torch.zeros((2, 3), device="cuda")
    for prompts in ([one], [one, one[:0]], [one] * 3):
        with pytest.raises(ValueError, match="answer needs"):
            model.answer(prompts, uniform)


def test_training_runs(gpu):
    torch, tm = gpu
    n, T, V = 2, 256, 64
    model = tm.TokenModel(n, T, V, 64, layers=1, attention=tm.Heads(heads=4, kv_heads=1, dim=16, window=20, sinks=1, sequences=2))
    batch = tm.source(torch, V)
    for k in range(6):
        model.step(*batch(n, T))
    model.parle.parle_outer_step()
    assert torch.isfinite(model.parle.x).all() and torch.isfinite(model.logp).all()
