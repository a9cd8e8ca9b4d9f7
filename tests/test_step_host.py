"""Host-side checks of attention behind shared prefixes, norms and sampling: sizes and refusals of the C-ABI and the binding.  No GPU: every refusal comes
before the first HIP call."""
import ctypes

import pytest
import torch

from paper_2402_10517_amd import binding as B
from test_decode_host import INVALID, P, SHAPE, SMALL, Cached, cache, cached, of, rows

vp, i64, ci, cf = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float


class Shared(ctypes.Structure):
    _fields_ = [("own", Cached), ("prefixes", ci), ("prefix_starts", vp), ("prefix_lengths", vp), ("prefix_tables", vp), ("prefix_width", i64), ("max_prefix", i64)]


class Rows(ctypes.Structure):
    _fields_ = [("data", vp), ("stride", i64)]


class Normed(ctypes.Structure):
    _fields_ = [(n, Rows) for n in ("x", "residual", "gate", "residual_out", "out")] + [("tokens", i64), ("columns", i64), ("half", ci), ("post", ci), ("centred", ci)] + [
        (n, vp) for n in ("weight", "bias", "post_weight", "post_bias")] + [("scale", cf), ("eps", cf)]


class Sampling(ctypes.Structure):
    _fields_ = [("logits", vp), ("stride", i64), ("half", ci), ("half_probabilities", ci), ("rows", i64), ("vocabulary", i64)] + [
        (n, vp) for n in ("uniform", "temperature", "top_p", "min_p", "top_k", "tokens", "probabilities", "work")] + [("work_bytes", ctypes.c_size_t)]


def shared(own=None, **kw):
    return Shared(**dict(dict(own=cached(**(own or {})), prefixes=2, prefix_starts=P, prefix_lengths=P, prefix_tables=P, prefix_width=4, max_prefix=200), **kw))


def normed(**kw):
    r = lambda: Rows(P, 64)  # noqa: E731
    return Normed(**dict(dict(x=r(), residual=r(), gate=r(), residual_out=r(), out=r(), tokens=3, columns=64, half=0, post=1, centred=0, weight=P, bias=P, post_weight=P,
                              post_bias=P, scale=1.0, eps=1e-6), **kw))


def sampling(**kw):
    return Sampling(**dict(dict(logits=P, stride=100, half=0, half_probabilities=0, rows=2, vocabulary=100, uniform=P, temperature=P, top_p=P, min_p=P, top_k=P, tokens=P,
                                probabilities=P + (1 << 20), work=P, work_bytes=1 << 40), **kw))


def test_shared_refusals():
    ask = lambda c, a: of(B.lib.ap_attention_shared, c, a)  # noqa: E731
    assert ask(None, shared()) == INVALID and ask(cache(), None) == INVALID and ask(None, None) == INVALID and ask(cache(data=None), shared()) == INVALID
    for bad in (dict(q=rows(data=None)), dict(q=rows(head_stride=12)), dict(lengths=None), dict(lengths=P + 2), dict(q_starts=P + 1), dict(tables=None),
                dict(tables=P + 2), dict(out=None), dict(out=P + 8), dict(scale=float("nan")), dict(work=None), dict(work=P + 4)):
        assert ask(cache(), shared(bad)) == INVALID, bad
    for bad in (dict(prefix_lengths=None), dict(prefix_lengths=P + 2), dict(prefix_starts=P + 2), dict(prefix_tables=None), dict(prefix_tables=P + 3)):
        assert ask(cache(), shared(**bad)) == INVALID, bad
    for bad in (dict(heads=0), dict(heads=7), dict(tokens=-1), dict(sequences=0), dict(sequences=2, q_starts=None), dict(max_length=257), dict(table_width=1 << 40),
                dict(tokens=1 << 21, heads=8)):                                    # 2^24 rows to join
        assert ask(cache(), shared(bad)) == SHAPE, bad
    for bad in (dict(prefixes=-1), dict(prefixes=(1 << 20) + 1), dict(prefixes=2, prefix_starts=None), dict(prefix_width=-1), dict(prefix_width=1 << 31), dict(max_prefix=-1),
                dict(max_prefix=257), dict(prefix_width=1 << 30, max_prefix=(1 << 30) + 1)):
        assert ask(cache(), shared(**bad)) == SHAPE, bad
    assert ask(cache(kv_heads=1024), shared(dict(heads=1024, sequences=1 << 13), prefixes=1 << 13)) == SHAPE                        # more workgroups than a launch has
    assert ask(cache(), shared(dict(work_bytes=100))) == SMALL
    assert ask(cache(), shared(dict(tokens=0, q=rows(data=None)))) == 0
    size = ctypes.c_size_t(7)
    ask_size = lambda a: B.lib.ap_attention_shared_size(ctypes.byref(cache()), ctypes.byref(a), ctypes.byref(size))  # noqa: E731
    assert ask_size(shared(dict(tokens=0))) == 0 and size.value == 0
    assert B.lib.ap_attention_shared_size(ctypes.byref(cache()), ctypes.byref(shared()), None) == INVALID and ask_size(shared(max_prefix=-1)) == SHAPE
    assert ask_size(shared(prefixes=0)) == 0 and size.value > 0


def plan_sizes(own, kv=8, D=128, **kw):
    size = ctypes.c_size_t(0)
    a = shared(own, **kw)
    status = B.lib.ap_attention_shared_size(ctypes.byref(cache(kv_heads=kv, head_dim=D)), ctypes.byref(a), ctypes.byref(size))
    return status, size.value


def test_workspace_of_shared_attention_is_bounded():
    # every row's sums of its own keys and of its prefix are kept once at least; ranges beyond that only as far as they fill the card
    for sequences in (1, 3, 64, 1000, 1 << 14):
        for queries in (1, 5):
            for prefixes in (1, 2, 60):
                for own in (1, 300, 1 << 15, 1 << 30):
                    for prefix in (1, 1000, 1 << 17, 1 << 30):
                        for D in (64, 128):
                            tokens = sequences * queries
                            status, size = plan_sizes(dict(tokens=tokens, heads=64, sequences=sequences, table_width=1 << 26, max_length=own), prefixes=prefixes,
                                                      prefix_width=1 << 26, max_prefix=prefix, D=D)
                            assert status == 0
                            row = (D + 2) * 4
                            few = queries * 8 <= 16 and sequences * queries * 8 <= 16 * prefixes        # ranges of 4096 keys at most
                            assert size <= 2 * tokens * 64 * row + (300 << 20) + few * tokens * 64 * (own + prefix) // 4096 * row, (sequences, queries, prefixes, own, prefix, size)


def test_norm_refusals():
    ask = lambda a: of(B.lib.ap_norm, a)  # noqa: E731
    assert ask(None) == INVALID
    none = Rows(None, 0)
    for bad in (dict(x=none, residual=none), dict(x=Rows(P + 1, 64)), dict(residual=Rows(P + 2, 64)), dict(residual_out=Rows(P + 2, 64)), dict(gate=Rows(P + 1, 0)),
                dict(out=Rows(P + 1, 64)), dict(weight=P + 1), dict(bias=P + 1), dict(post_weight=P + 1), dict(post_bias=P + 1), dict(x=Rows(P, 1 << 40)),
                dict(out=Rows(P, -(1 << 40))), dict(out=Rows(P, 63)), dict(out=Rows(P, 0)), dict(residual_out=Rows(P, -63)), dict(scale=float("nan")), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(half=1, residual=Rows(P + 1, 64))):
        assert ask(normed(**bad)) == INVALID, bad
    for bad in (dict(tokens=-1), dict(tokens=1 << 31), dict(columns=0), dict(columns=32769), dict(columns=-64)):
        assert ask(normed(**bad)) == SHAPE, bad
    assert ask(normed(tokens=0, x=none, residual=none)) == 0
    assert ask(normed(out=none, residual_out=none)) == 0                       # nothing is wanted


def test_sample_refusals():
    ask = lambda a: of(B.lib.ap_sample, a)  # noqa: E731
    assert ask(None) == INVALID
    for bad in (dict(logits=None), dict(logits=P + 2), dict(half=1, logits=P + 1), dict(uniform=None), dict(uniform=P + 2), dict(temperature=P + 1), dict(top_k=P + 2),
                dict(top_p=P + 3), dict(min_p=P + 1), dict(tokens=None), dict(tokens=P + 4), dict(probabilities=P + 2), dict(half_probabilities=1, probabilities=P + 1)):
        assert ask(sampling(**bad)) == INVALID, bad
    for bad in (dict(rows=-1), dict(rows=(1 << 21) + 1), dict(vocabulary=0), dict(vocabulary=(1 << 20) + 1), dict(stride=1 << 40), dict(stride=-(1 << 40))):
        assert ask(sampling(**bad)) == SHAPE, bad
    assert ask(sampling(rows=0, logits=None)) == 0
    size = ctypes.c_size_t(7)
    assert B.lib.ap_sample_size(ctypes.byref(sampling(rows=0)), ctypes.byref(size)) == 0 and size.value == 0
    assert B.lib.ap_sample_size(ctypes.byref(sampling()), None) == INVALID
    for rows_, vocabulary in ((1, 1 << 20), (1, 131071), (64, 131071), (1 << 21, 1 << 20)):
        assert B.lib.ap_sample_size(ctypes.byref(sampling(rows=rows_, vocabulary=vocabulary)), ctypes.byref(size)) == 0
        assert size.value <= 64 << 20
        if size.value:
            assert ask(sampling(rows=rows_, vocabulary=vocabulary, work_bytes=size.value - 1)) == SMALL
            assert ask(sampling(rows=rows_, vocabulary=vocabulary, work=None, work_bytes=size.value)) == INVALID


def test_probabilities_in_the_logits_memory_are_refused():
    def ask(first, stride, at, rows=3, half=0, half_probabilities=0, V=8):
        return of(B.lib.ap_sample, sampling(logits=P + first, stride=stride, rows=rows, vocabulary=V, half=half, half_probabilities=half_probabilities, probabilities=P + at))
    size = 8 * 4
    for first, stride, at in ((0, 8, 0), (0, 8, 3 * size - 4), (3 * size - 4, 8, 0), (0, 8, size), (0, 0, 0), (size, 0, 0), (4 * size, -8, 0), (4 * size, -8, 4 * size), (0, 1000, 4000),
                              (0, 1000, 4000 + size - 4), (0, 1000, 8000), (0, 1000, 4004 - 3 * size), ((1 << 39) * 8, -(1 << 40) + 1, (1 << 39) * 8)):
        assert ask(first, stride, at) == INVALID, (first, stride, at)
    if not torch.cuda.is_available():                            # (asked for in earnest these addresses would be written)
        for first, stride, at in ((0, 8, 3 * size), (3 * size, 8, 0), (0, 0, size), (3 * size, 0, 0), (0, 1000, size), (0, 1000, 4000 - 3 * size), (4 * size, -8, 5 * size), (0, 1000, 8000 + size)):
            assert ask(first, stride, at) not in (0, INVALID, SHAPE), (first, stride, at)
    assert ask(0, 8, 3 * 16 - 2, half=1, half_probabilities=1) == INVALID


def test_binding_refuses_tensors_that_do_not_fit():
    x, u = torch.zeros((2, 8), dtype=torch.float16), torch.zeros(2)
    with pytest.raises(AssertionError):
        B.ap_norm(x, x)                                          # not on the GPU
    with pytest.raises(AssertionError):
        B.ap_sample(x, u)
    with pytest.raises(AssertionError):
        B.ap_sample(x, u, probabilities=torch.int64)
    with pytest.raises(TypeError):
        B.ap_norm(3.0, x)
    with pytest.raises(TypeError):
        B.ap_sample(None, u)


def test_sampling_needs_no_workspace():
    size = ctypes.c_size_t(7)
    for rows_, vocabulary in ((0, 1), (1, 1), (1, 1 << 20), (64, 131071), (1 << 21, 1 << 20)):
        size.value = 7
        assert B.lib.ap_sample_size(ctypes.byref(sampling(rows=rows_, vocabulary=vocabulary)), ctypes.byref(size)) == 0 and size.value == 0
    if not torch.cuda.is_available():                            # (asked for in earnest the addresses would be written)
        assert of(B.lib.ap_sample, sampling(work=None, work_bytes=0)) not in (0, INVALID, SHAPE, SMALL)
