"""CPU-only checks of the entry points of rotary positions, attention, its caches and the sampler: descriptors, scratch and every refusal.

Pointers here are numbers that nothing reads: each call is refused on the host before a launch."""
import ctypes as C

import pytest

from paper_1707_00424_amd import binding as pb

P, ODD = 0x10000, 0x10004        # 16-byte aligned; not
BIG = 1 << 40
Q, K, V, O, DQ, DK, DV = (P + 0x1000 * i for i in range(7))


def _call(name, desc, *args):
    status = getattr(pb.lib(), name)(None, None if desc is None else C.byref(desc), *args)
    return status, pb.lib().parle_last_error(None).decode()


def rope(**kw):
    d = dict(dtype=1, n=2, tokens=5, heads=3, dim=16, pairs=[2, 3], interleaved=0, inverse=0, ld=48, stride=240, ld_out=50, out_stride=250) | kw
    axes = d.pop("axes", None)
    r = pb.make_rope_desc(**d)
    if axes is not None:
        r.axes = axes
    return r


def attention(**kw):
    return pb.parle_attention_desc(**(dict(dtype=1, n=2, tokens=5, sequences=2, heads=4, kv_heads=2, dim=16, window=0, sinks=0, scale=0.25, ld_q=64, q_stride=320,
                                           ld_kv=32, kv_stride=160, ld_out=64, out_stride=320) | kw))


def cache(**kw):
    return pb.parle_cache_desc(**(dict(dtype=1, sequences=3, capacity=20, heads=4, kv_heads=2, dim=16, window=16, sinks=4, scale=0.25, ld_q=64, ld_kv=32, ld_out=64) | kw))


def sample(**kw):
    return pb.parle_sample_desc(**(dict(dtype=1, n=2, rows=5, classes=7, ld=8) | kw))


CALLS = {
    "parle_k_rope": (rope, (Q, K, V, O)),
    "parle_k_attention_forward": (attention, (Q, K, V, P + 0x10000, O, DQ)),
    "parle_k_attention_backward": (attention, (Q, K, V, P + 0x10000, O, P + 0x20000, P + 0x30000, P + 0x40000, BIG, DQ, DK, DV)),
    "parle_k_attention_store": (cache, (6, K, V, P + 0x10000, P + 0x20000, DK, DV)),
    "parle_k_attention_decode": (cache, (Q, K, V, P + 0x20000, P + 0x40000, BIG, DK, DV, O)),
    "parle_k_sample": (sample, (P,) * 6 + (P, BIG, P, P, P)),
}
E, S = pb.PARLE_EINVAL, pb.PARLE_ESIZE
HEADS = [(dict(dtype=2), E), (dict(heads=3), E), (dict(heads=0), E), (dict(kv_heads=0), E), (dict(kv_heads=-2), E), (dict(dim=0), E), (dict(dim=12), E), (dict(window=-1), E),
         (dict(sinks=-1), E), (dict(scale=0.0), E), (dict(scale=-1.0), E), (dict(scale=float("nan")), E), (dict(scale=float("inf")), E)]
BAD = {
    rope: [(dict(dtype=2), E), (dict(interleaved=2), E), (dict(inverse=-1), E), (dict(n=0), E), (dict(n=65536), E), (dict(tokens=-1), E), (dict(heads=0), E), (dict(dim=0), E),
           (dict(axes=0), E), (dict(axes=5), E), (dict(pairs=[-1, 3]), E), (dict(pairs=[4, 5]), E), (dict(ld=47), E), (dict(ld_out=47), E), (dict(stride=239), E), (dict(out_stride=247), E),
           (dict(dim=4098, ld=1 << 20, stride=1 << 30, ld_out=1 << 20, out_stride=1 << 30), S), (dict(tokens=(1 << 22) + 1), S), (dict(ld=1 << 39), S), (dict(out_stride=1 << 40), S)],
    attention: HEADS + [(dict(n=0), E), (dict(tokens=-1), E), (dict(sequences=0), E), (dict(ld_q=63), E), (dict(ld_kv=31), E), (dict(ld_out=63), E), (dict(q_stride=319), E),
                        (dict(kv_stride=159), E), (dict(out_stride=319), E), (dict(dim=136, ld_q=1000, ld_kv=1000, ld_out=1000, q_stride=5000, kv_stride=5000, out_stride=5000), S),
                        (dict(sinks=129), S), (dict(tokens=(1 << 22) + 1), S), (dict(sequences=(1 << 22) + 1), S), (dict(ld_q=1 << 39), S), (dict(kv_stride=1 << 40), S),
                        (dict(n=1, tokens=1 << 22, heads=256, kv_heads=256, dim=8, ld_q=2048, ld_kv=2048, ld_out=2048), S)],
    cache: HEADS + [(dict(sequences=-1), E), (dict(capacity=4), E), (dict(ld_q=63), E), (dict(ld_kv=31), E), (dict(ld_out=63), E), (dict(sinks=129, capacity=200), S),
                    (dict(dim=136, ld_q=1000, ld_kv=1000, ld_out=1000), S), (dict(sequences=65536), S), (dict(sequences=65535, capacity=1 << 30), S), (dict(ld_q=1 << 39), S),
                    (dict(ld_kv=1 << 30), S)],
    sample: [(dict(dtype=2), E), (dict(n=0), E), (dict(rows=-1), E), (dict(classes=0), E), (dict(ld=6), E), (dict(classes=(1 << 22) + 1, ld=1 << 23), S), (dict(rows=1 << 21), S),
             (dict(ld=1 << 39), S)],
}
# positions of pointers that may be NULL by themselves
MAY_BE_NULL = {"parle_k_attention_forward": {5}, "parle_k_sample": {2, 3, 4, 5, 9, 10}}


@pytest.mark.parametrize("name", CALLS)
def test_bad_fields_are_refused(name):
    make, args = CALLS[name]
    for kw, want in BAD[make]:
        status, text = _call(name, make(**kw), *args)
        assert status == want and text.startswith(name + ": "), (name, kw, status, text)
    status, text = _call(name, None, *args)
    assert status == E and "desc" in text


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers_are_refused(name):
    make, args = CALLS[name]
    needs = {"parle_k_attention_backward": 7, "parle_k_attention_decode": 4, "parle_k_sample": 6}.get(name)
    wanted = getattr(pb, {"parle_k_attention_backward": "parle_k_attention_scratch_bytes", "parle_k_attention_decode": "parle_k_decode_scratch_bytes",
                          "parle_k_sample": "parle_k_sample_scratch_bytes"}.get(name, "_nbytes"))(make() if needs else None)
    for i, p in enumerate(args):
        if p == BIG or (name == "parle_k_attention_store" and i == 0):
            continue
        status, text = _call(name, make(), *args[:i], ODD, *args[i + 1:])
        assert status == pb.PARLE_EALIGN and text.startswith(name), (name, i, status, text)
        if i in MAY_BE_NULL.get(name, ()) or (i == needs and wanted == 0):
            continue
        status, text = _call(name, make(), *args[:i], None, *args[i + 1:])
        assert status == E and text.startswith(name), (name, i, status, text)


def test_buffers_that_meet():
    assert _call("parle_k_rope", rope(), Q, K, V, Q)[0] == E                       # in place in another layout
    d = list(CALLS["parle_k_attention_forward"][1])
    for i in range(3):
        assert _call("parle_k_attention_forward", attention(), *d[:4], d[i], d[5])[0] == E
    a = list(CALLS["parle_k_attention_backward"][1])
    for g in (9, 10, 11):
        for i in (0, 1, 2, 4, 6, 9, 10, 11):
            if i != g:
                b = list(a)
                b[g] = a[i]
                assert _call("parle_k_attention_backward", attention(), *b)[0] == E, (g, i)
    assert _call("parle_k_attention_store", cache(), 6, K, V, P, P, DK, DK)[0] == E
    s = list(CALLS["parle_k_attention_decode"][1])
    assert _call("parle_k_attention_decode", cache(), *s[:7], s[6], s[8])[0] == E
    for i in range(3):
        assert _call("parle_k_attention_decode", cache(), *s[:8], s[i])[0] == E
    assert _call("parle_k_attention_decode", cache(), s[0], None, *s[2:])[0] == E     # k without v


def test_a_gradient_of_more_threads_than_a_launch_has():
    """Refused in front of its first launch; the forward pass of the same descriptor has half as many and asks for its pointers."""
    most = dict(n=1, tokens=16384, sequences=1, heads=65535, kv_heads=65535, dim=8, q_stride=0, kv_stride=0, out_stride=0, ld_q=65535 * 8, ld_kv=65535 * 8, ld_out=65535 * 8)
    others = most | dict(tokens=26843, heads=40000, kv_heads=40000)               # 420 workgroups for each of 40000 heads
    fits = most | dict(heads=65534, kv_heads=32767)
    for kw, ok in ((most | dict(window=1, sinks=128), False), (others, False), (most, True), (fits | dict(window=1, sinks=128), True)):
        d = attention(**kw)
        assert (pb.parle_k_attention_scratch_bytes(d) > 0) == ok
        status, text = _call("parle_k_attention_backward", d, None, *CALLS["parle_k_attention_backward"][1][1:])
        assert (status, "threads" in text) == ((E, False) if ok else (S, True)), (kw, status, text)
        status, text = _call("parle_k_attention_forward", d, None, *CALLS["parle_k_attention_forward"][1][1:])
        assert status == E and "q is NULL" in text


def test_scratch():
    for make, query, name, at in [(attention, "parle_k_attention_scratch_bytes", "parle_k_attention_backward", 8), (cache, "parle_k_decode_scratch_bytes", "parle_k_attention_decode", 5),
                                  (sample, "parle_k_sample_scratch_bytes", "parle_k_sample", 7)]:
        assert getattr(pb, query)(make(dtype=2)) == -1
        size = getattr(pb, query)(make())
        assert size >= 0
        if size:
            args = CALLS[name][1]
            status, text = _call(name, make(), *args[:at], size - 1, *args[at + 1:])
            assert status == pb.PARLE_ESIZE and "scratch" in text
    assert pb.parle_k_attention_scratch_bytes(attention()) >= 2 * 4 * 5 * 4
    far = dict(n=1, tokens=2000, window=100, q_stride=0, kv_stride=0, out_stride=0)
    assert pb.parle_k_attention_scratch_bytes(attention(sinks=4, **far)) > pb.parle_k_attention_scratch_bytes(attention(sinks=0, **far))
    assert pb.parle_k_decode_scratch_bytes(cache(capacity=10000, window=0)) > 0


def test_nothing_to_do_needs_no_pointers():
    assert _call("parle_k_rope", rope(tokens=0), *(None,) * 4)[0] == pb.PARLE_OK
    assert _call("parle_k_attention_forward", attention(tokens=0), *(None,) * 6)[0] == pb.PARLE_OK
    assert _call("parle_k_attention_backward", attention(tokens=0), *(None,) * 8, 0, None, None, None)[0] == pb.PARLE_OK
    assert pb.parle_k_attention_scratch_bytes(attention(tokens=0)) == 0
    assert _call("parle_k_attention_store", cache(), 0, *(None,) * 6)[0] == pb.PARLE_OK
    assert _call("parle_k_attention_store", cache(sequences=0), 6, *(None,) * 6)[0] == pb.PARLE_OK
    assert _call("parle_k_attention_decode", cache(sequences=0), *(None,) * 5, 0, None, None, None)[0] == pb.PARLE_OK
    assert _call("parle_k_sample", sample(rows=0), *(None,) * 7, 0, None, None, None)[0] == pb.PARLE_OK
    # offsets say where sequences begin; one sequence needs none
    assert _call("parle_k_attention_store", cache(), -1, K, V, P, P, DK, DV)[0] == E
    assert _call("parle_k_attention_store", cache(), (1 << 22) + 1, K, V, P, P, DK, DV)[0] == S


def test_struct_layouts_match_the_header(tmp_path):
    """The ctypes mirrors have the size and field offsets that a C compiler gives the header."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {n: getattr(pb, n) for n in ("parle_rope_desc", "parle_attention_desc", "parle_cache_desc", "parle_sample_desc")}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "parle.h"', 'int main(void) {']
    for name, st in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split() for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, st in structs.items():
        assert int(out[name]) == C.sizeof(st)
        for f in st._fields_:
            assert int(out[f"{name}.{f[0]}"]) == getattr(st, f[0]).offset, (name, f[0])
