"""CPU-only checks of the token-model operators' entry points: descriptors, scratch sizes and every refusal.

Pointers here are numbers that nothing reads: each call is refused on the host before a launch."""
import ctypes as C

import pytest

from paper_1707_00424_amd import binding as pb

P, ODD = 0x10000, 0x10004        # 16-byte aligned; not


def _call(name, desc, *ptrs):
    fn = getattr(pb.lib(), name)
    status = fn(None, None if desc is None else C.byref(desc), *ptrs)
    return status, pb.lib().parle_last_error(None).decode()


def embed(**kw):
    d = dict(dtype=1, table_dtype=0, n=2, tokens=5, vocab=10, dim=3, table_stride=32, scale=1.0) | kw
    return pb.parle_embed_desc(**d)


def norm(**kw):
    return pb.parle_norm_desc(**(dict(dtype=1, w_dtype=0, n=2, rows=5, dim=3, w_stride=8, eps=1e-6) | kw))


def quant(**kw):
    return pb.parle_quant_desc(**(dict(dtype=1, block=1, n=2, rows=5, cols=3, ld=3, stride=15) | kw))


def fp8(**kw):
    return pb.parle_fp8_desc(**(dict(out_dtype=1, b_block=128, accumulate=0, n=2, rows=5, cols=3, depth=7, ld_out=3, out_stride=15) | kw))


def logprob(**kw):
    return pb.parle_logprob_desc(**(dict(dtype=1, n=2, rows=5, classes=7, top=2, ld=8) | kw))


BIG = 1 << 40
CALLS = {
    "parle_k_embed_forward": (embed, (P, P, P)),
    "parle_k_embed_backward": (embed, (P, P, P, BIG, P)),
    "parle_k_rmsnorm_forward": (norm, (P, P, P, P, P, P, P, P)),
    "parle_k_rmsnorm_backward": (norm, (P, P, P, P, P, P, BIG, P, P)),
    "parle_k_fp8_quantize": (quant, (P, P, P, P, P)),
    "parle_k_fp8_matmul": (fp8, (P, P, P, P, P, P, BIG, P)),
    "parle_k_logprob_forward": (logprob, (P, P, P, BIG, P, P, P, P, P)),
    "parle_k_logprob_backward": (logprob, (P, P, P, P, P, P, P)),
}
# fields that each family refuses, and how
BAD = {
    embed: [(dict(dtype=2), pb.PARLE_EINVAL), (dict(dtype=-1), pb.PARLE_EINVAL), (dict(table_dtype=3), pb.PARLE_EINVAL),
            (dict(n=0), pb.PARLE_EINVAL), (dict(n=65536), pb.PARLE_EINVAL), (dict(tokens=-1), pb.PARLE_EINVAL),
            (dict(vocab=0), pb.PARLE_EINVAL), (dict(dim=0), pb.PARLE_EINVAL), (dict(table_stride=29), pb.PARLE_EINVAL),
            (dict(tokens=(1 << 22) + 1), pb.PARLE_ESIZE), (dict(vocab=(1 << 22) + 1, table_stride=1 << 26), pb.PARLE_ESIZE),
            (dict(table_stride=(1 << 40)), pb.PARLE_ESIZE), (dict(tokens=1 << 22, dim=1 << 20, vocab=1, table_stride=1 << 20), pb.PARLE_ESIZE)],
    norm: [(dict(dtype=2), pb.PARLE_EINVAL), (dict(w_dtype=2), pb.PARLE_EINVAL), (dict(n=0), pb.PARLE_EINVAL), (dict(rows=-1), pb.PARLE_EINVAL),
           (dict(dim=0), pb.PARLE_EINVAL), (dict(w_stride=2), pb.PARLE_EINVAL), (dict(eps=-1e-6), pb.PARLE_EINVAL),
           (dict(eps=float("nan")), pb.PARLE_EINVAL), (dict(eps=float("inf")), pb.PARLE_EINVAL),
           (dict(rows=(1 << 22) + 1), pb.PARLE_ESIZE), (dict(dim=(1 << 22) + 1, w_stride=1 << 23), pb.PARLE_ESIZE),
           (dict(rows=1 << 22, dim=1 << 20, w_stride=1 << 20), pb.PARLE_ESIZE)],
    quant: [(dict(dtype=2), pb.PARLE_EINVAL), (dict(block=64), pb.PARLE_EINVAL), (dict(n=0), pb.PARLE_EINVAL), (dict(rows=-1), pb.PARLE_EINVAL),
            (dict(cols=0), pb.PARLE_EINVAL), (dict(ld=2), pb.PARLE_EINVAL), (dict(stride=14), pb.PARLE_EINVAL),
            (dict(rows=(1 << 22) + 1), pb.PARLE_ESIZE), (dict(ld=1 << 39), pb.PARLE_ESIZE), (dict(stride=1 << 40), pb.PARLE_ESIZE)],
    fp8: [(dict(out_dtype=2), pb.PARLE_EINVAL), (dict(b_block=2), pb.PARLE_EINVAL), (dict(accumulate=2), pb.PARLE_EINVAL), (dict(n=0), pb.PARLE_EINVAL),
          (dict(rows=-1), pb.PARLE_EINVAL), (dict(cols=0), pb.PARLE_EINVAL), (dict(depth=-1), pb.PARLE_EINVAL), (dict(ld_out=2), pb.PARLE_EINVAL),
          (dict(out_stride=14), pb.PARLE_EINVAL), (dict(depth=(1 << 22) + 1), pb.PARLE_ESIZE), (dict(out_stride=1 << 40), pb.PARLE_ESIZE)],
    logprob: [(dict(dtype=2), pb.PARLE_EINVAL), (dict(n=0), pb.PARLE_EINVAL), (dict(rows=-1), pb.PARLE_EINVAL), (dict(classes=0), pb.PARLE_EINVAL),
              (dict(top=-1), pb.PARLE_EINVAL), (dict(top=65), pb.PARLE_EINVAL), (dict(ld=6), pb.PARLE_EINVAL),
              (dict(classes=(1 << 22) + 1, ld=1 << 23), pb.PARLE_ESIZE), (dict(rows=(1 << 21) + 1), pb.PARLE_ESIZE), (dict(ld=1 << 39), pb.PARLE_ESIZE)],
}
# positions of pointers that may be NULL (scratch where these small sizes want none, y where q is given)
# scratch among them where a call of these sizes needs none
MAY_BE_NULL = {"parle_k_embed_backward": {2}, "parle_k_rmsnorm_forward": {1, 3, 4, 7}, "parle_k_rmsnorm_backward": {4}, "parle_k_fp8_matmul": {4, 5}, "parle_k_logprob_forward": {2, 4, 5, 6},
               "parle_k_logprob_backward": {5}}


@pytest.mark.parametrize("name", CALLS)
def test_bad_fields_are_refused(name):
    make, ptrs = CALLS[name]
    for kw, want in BAD[make]:
        status, text = _call(name, make(**kw), *ptrs)
        assert status == want and text.startswith(name + ": "), (name, kw, status, text)
    status, text = _call(name, None, *ptrs)
    assert status == pb.PARLE_EINVAL and "desc" in text


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers_are_refused(name):
    make, ptrs = CALLS[name]
    for i, p in enumerate(ptrs):
        if p == BIG:
            continue
        status, text = _call(name, make(), *ptrs[:i], ODD, *ptrs[i + 1:])
        assert status == pb.PARLE_EALIGN and text.startswith(name), (name, i, status, text)
        if i not in MAY_BE_NULL.get(name, ()):
            status, text = _call(name, make(), *ptrs[:i], None, *ptrs[i + 1:])
            assert status == pb.PARLE_EINVAL and text.startswith(name), (name, i, status, text)


def test_outputs_that_come_together():
    assert _call("parle_k_rmsnorm_forward", norm(), P, P, P, P, None, None, None, P)[0] == pb.PARLE_EINVAL
    assert _call("parle_k_rmsnorm_forward", norm(), P, P, P, P, P, P, None, P)[0] == pb.PARLE_EINVAL
    assert _call("parle_k_fp8_quantize", quant(), P, None, None, None, None)[0] == pb.PARLE_EINVAL
    assert _call("parle_k_fp8_quantize", quant(), P, P, P, P, None)[0] == pb.PARLE_EINVAL
    assert _call("parle_k_logprob_forward", logprob(top=0), P, P, P, BIG, P, P, P, P, P)[0] == pb.PARLE_EINVAL
    assert _call("parle_k_logprob_backward", logprob(), P, P, P, None, P, P, P)[0] == pb.PARLE_EINVAL


def test_scratch():
    for make, name, call, at in [(embed, "parle_k_embed_scratch_bytes", "parle_k_embed_backward", 3), (norm, "parle_k_rmsnorm_scratch_bytes", "parle_k_rmsnorm_backward", 6),
                                 (logprob, "parle_k_logprob_scratch_bytes", "parle_k_logprob_forward", 3), (fp8, "parle_k_fp8_scratch_bytes", "parle_k_fp8_matmul", 6)]:
        size = getattr(pb, name)(make())
        assert 0 <= size < 1 << 30
        bad = BAD[make][0][0]
        assert getattr(pb, name)(make(**bad)) == -1
        if size:
            ptrs = CALLS[call][1]
            status, text = _call(call, make(), *ptrs[:at], size - 1, *ptrs[at + 1:])
            assert status == pb.PARLE_ESIZE and "scratch" in text
    # a call that needs scratch refuses NULL, one that needs none is asked for none
    many = embed(tokens=600)
    assert pb.parle_k_embed_scratch_bytes(many) > 0 and pb.parle_k_embed_scratch_bytes(embed()) == 0
    status, text = _call("parle_k_embed_backward", many, P, P, None, BIG, P)
    assert status == pb.PARLE_EINVAL and "scratch" in text
    # more tokens, rows or classes never want less than a part of them
    assert pb.parle_k_embed_scratch_bytes(embed(tokens=1 << 20)) > pb.parle_k_embed_scratch_bytes(embed(tokens=1 << 14)) > 0
    assert pb.parle_k_logprob_scratch_bytes(logprob(n=1, rows=4, classes=128000, ld=128000, top=20)) > 0


def test_nothing_to_do_needs_no_pointers():
    none = (None,) * 9
    assert _call("parle_k_embed_forward", embed(tokens=0), *none[:3])[0] == pb.PARLE_OK
    assert _call("parle_k_rmsnorm_forward", norm(rows=0), *none[:8])[0] == pb.PARLE_OK
    assert _call("parle_k_fp8_quantize", quant(rows=0), *none[:5])[0] == pb.PARLE_OK
    assert _call("parle_k_fp8_matmul", fp8(rows=0), None, None, None, None, None, None, 0, None)[0] == pb.PARLE_OK
    assert _call("parle_k_logprob_forward", logprob(rows=0), None, None, None, 0, None, None, None, None, None)[0] == pb.PARLE_OK
    assert _call("parle_k_logprob_backward", logprob(rows=0), *none[:7])[0] == pb.PARLE_OK
