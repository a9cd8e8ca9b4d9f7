"""Host-side checks of the decoder operators: exports, sizes and refusals of the C-ABI.  No GPU: every refusal comes before the first HIP call."""
import ctypes
import os
import re

import pytest

from paper_2402_10517_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE, SMALL = 1, 2, 5
vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int


class Heads(ctypes.Structure):
    _fields_ = [("data", vp), ("token_stride", i64), ("head_stride", i64)]


class Append(ctypes.Structure):
    _fields_ = [(n, Heads) for n in ("q", "k", "v", "q_out", "k_out")] + [("heads", ci), ("tokens", i64), ("slots", vp), ("positions", vp), ("rotary", vp),
                                                                         ("rotary_rows", i64), ("rot_dim", ci), ("interleaved", ci)]


class Cached(ctypes.Structure):
    _fields_ = [("q", Heads), ("heads", ci), ("tokens", i64), ("sequences", ci), ("q_starts", vp), ("lengths", vp), ("tables", vp), ("table_width", i64),
                ("max_length", i64), ("scale", ctypes.c_float), ("out", vp), ("work", vp), ("work_bytes", ctypes.c_size_t)]


class Prompt(ctypes.Structure):
    _fields_ = [("q", Heads), ("k", Heads), ("v", Heads), ("heads", ci), ("kv_heads", ci), ("head_dim", ci), ("tokens", i64), ("keys", i64), ("sequences", ci),
                ("q_starts", vp), ("k_starts", vp), ("scale", ctypes.c_float), ("out", vp), ("work", vp), ("work_bytes", ctypes.c_size_t)]


class Verification(ctypes.Structure):
    _fields_ = [("target", vp), ("draft", vp), ("half", ci), ("sequences", ci), ("drafts", ci), ("vocabulary", i64), ("drafted", vp), ("uniform", vp), ("noise", vp),
                ("counts", vp), ("tokens", vp), ("accepted", vp), ("work", vp), ("work_bytes", ctypes.c_size_t)]


P = 4096          # an address that is aligned and never followed: every call here is refused before it would be


def cache(data=P, pages=10, page_tokens=64, kv_heads=2, head_dim=128):
    return B._Cache(data, pages, page_tokens, kv_heads, head_dim)


def rows(**kw):
    return Heads(**dict(dict(data=P, token_stride=1024, head_stride=128), **kw))


def append(**kw):
    return Append(**dict(dict(q=rows(), k=rows(), v=rows(), q_out=rows(), k_out=rows(), heads=8, tokens=3, slots=P, positions=P, rotary=P, rotary_rows=9,
                              rot_dim=128, interleaved=0), **kw))


def cached(**kw):
    return Cached(**dict(dict(q=rows(), heads=8, tokens=3, sequences=3, q_starts=P, lengths=P, tables=P, table_width=4, max_length=200, scale=0.1, out=P, work=P,
                              work_bytes=1 << 40), **kw))


def prompt(**kw):
    return Prompt(**dict(dict(q=rows(), k=rows(), v=rows(), heads=8, kv_heads=2, head_dim=128, tokens=3, keys=3, sequences=2, q_starts=P, k_starts=P, scale=0.1,
                              out=P, work=P, work_bytes=1 << 40), **kw))


def verification(**kw):
    return Verification(**dict(dict(target=P, draft=P, half=0, sequences=2, drafts=3, vocabulary=100, drafted=P, uniform=P, noise=P, counts=P, tokens=P, accepted=P,
                                    work=P, work_bytes=1 << 40), **kw))


def test_library_exports_every_declared_decoder_symbol():
    header = open(os.path.join(ROOT, "include", "apdecode.h")).read()
    declared = set(re.findall(r"^ap_status (ap_[a-z_]+)\(", header, re.M))
    assert declared == set(B.DECODE_EXPORTS)
    for name in declared:
        assert hasattr(ctypes.CDLL(B.LIB_PATH), name), name


def test_attention_kernels_keep_their_registers():
    # waves per SIMD that the division of the work counts on, and nothing spilled
    from test_kernel_resources import _kernels
    waves = {r"attention_cached_kernelILi64ELi1E": 4, r"attention_cached_kernelILi128ELi1E": 3, r"attention_cached_kernelILi(64|128)ELi2E": 2,
             r"attention_prompt_kernelILi64E": 4, r"attention_prompt_kernelILi128E": 2}
    seen = set()
    for name, k in _kernels().items():
        for pattern, least in waves.items():
            if re.search(pattern, name):
                seen.add(pattern)
                assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
                assert 512 // ((k[".vgpr_count"] + 7) // 8 * 8) >= least, "%s: %d registers" % (name, k[".vgpr_count"])
    assert seen == set(waves)


def test_cache_size():
    assert B.ap_cache_size(10, 2, 128, 64) == 10 * 64 * 2 * 136            # 4 bits a value and 4 bytes a row, keys and values
    assert B.ap_cache_size(1, 1, 64, 16) == 16 * 72
    for bad in (dict(pages=0), dict(pages=-1), dict(pages=1 << 40), dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=8), dict(page_tokens=512),
                dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=96), dict(head_dim=0), dict(head_dim=256)):
        args = dict(dict(pages=4, kv_heads=2, head_dim=64, page_tokens=16), **bad)
        with pytest.raises(B.ApError) as e:
            B.ap_cache_size(**args)
        assert e.value.status == SHAPE
    assert B.lib.ap_cache_size(None, None) == INVALID and B.lib.ap_cache_size(ctypes.byref(cache()), None) == INVALID


@pytest.mark.parametrize("bad", [dict(page_tokens=2 ** 32 + 64), dict(kv_heads=2 ** 32 + 2), dict(head_dim=2 ** 32 + 64), dict(pages=2 ** 64 + 4), dict(page_tokens=-2 ** 32 + 16)])
def test_cache_sizes_are_not_taken_modulo(bad):
    with pytest.raises(B.ApError) as e:
        B.ap_cache_size(**dict(dict(pages=4, kv_heads=2, head_dim=64, page_tokens=16), **bad))
    assert e.value.status == SHAPE


def of(function, *structs):
    return function(*[None if s is None else ctypes.byref(s) for s in structs], None)


def test_append_refusals():
    ask = lambda c, a: of(B.lib.ap_cache_append, c, a)
    assert ask(None, append()) == INVALID and ask(cache(), None) == INVALID and ask(cache(data=None), append()) == INVALID
    assert ask(cache(data=P + 128), append()) == INVALID and ask(cache(head_dim=80), append()) == SHAPE
    for bad in (dict(k=rows(data=None)), dict(v=rows(data=P + 2)), dict(k=rows(token_stride=100)), dict(v=rows(head_stride=-4)), dict(q_out=rows(data=None)),
                dict(q=rows(data=P + 8)), dict(k_out=rows(head_stride=1)), dict(slots=None), dict(slots=P + 4), dict(positions=None), dict(positions=P + 1),
                dict(rotary=P + 4), dict(k=rows(token_stride=1 << 41))):
        assert ask(cache(), append(**bad)) == INVALID, bad
    for bad in (dict(tokens=-1), dict(tokens=1 << 40), dict(heads=0), dict(heads=5000), dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=144), dict(rotary_rows=-1)):
        assert ask(cache(), append(**bad)) == SHAPE, bad
    assert ask(cache(), append(tokens=0, slots=None)) == 0
    read = lambda c, slots, n, k, v: B.lib.ap_cache_read(ctypes.byref(c), slots, n, k, v, None)
    assert read(cache(), P, -1, P, P) == SHAPE and read(cache(), None, 1, P, P) == INVALID and read(cache(), P, 1, P + 2, P) == INVALID
    assert read(cache(), P, 1, P, None) == INVALID and read(cache(), None, 0, None, None) == 0 and read(cache(data=None), P, 1, P, P) == INVALID


def test_cached_refusals():
    ask = lambda c, a: of(B.lib.ap_attention_cached, c, a)
    assert ask(None, cached()) == INVALID and ask(cache(), None) == INVALID and ask(cache(data=None), cached()) == INVALID
    for bad in (dict(q=rows(data=None)), dict(q=rows(head_stride=12)), dict(lengths=None), dict(lengths=P + 2), dict(q_starts=P + 1), dict(tables=None),
                dict(tables=P + 2), dict(out=None), dict(out=P + 8), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert ask(cache(), cached(**bad)) == INVALID, bad
    for bad in (dict(heads=0), dict(heads=7), dict(heads=-2), dict(tokens=-1), dict(sequences=0), dict(sequences=-1), dict(sequences=2, q_starts=None),
                dict(table_width=-1), dict(max_length=-1), dict(max_length=257), dict(table_width=1 << 40)):
        assert ask(cache(), cached(**bad)) == SHAPE, bad
    assert ask(cache(kv_heads=3), cached()) == SHAPE
    size = ctypes.c_size_t(7)
    ask_size = lambda a, out: B.lib.ap_attention_cached_size(ctypes.byref(cache()), ctypes.byref(a), out)
    assert ask_size(cached(tokens=0), ctypes.byref(size)) == 0 and size.value == 0
    assert ask_size(cached(), None) == INVALID and ask_size(cached(heads=3), ctypes.byref(size)) == SHAPE
    long = cached(table_width=1 << 12, max_length=1 << 18)
    assert ask_size(long, ctypes.byref(size)) == 0
    if size.value:
        long.work_bytes = size.value - 1
        assert ask(cache(), long) == SMALL
        long.work, long.work_bytes = None, size.value
        assert ask(cache(), long) == INVALID
    assert ask(cache(), cached(tokens=0, q=rows(data=None))) == 0


def test_prompt_refusals():
    ask = lambda a: of(B.lib.ap_attention_prompt, a)
    assert ask(None) == INVALID
    for bad in (dict(q=rows(data=None)), dict(k=rows(data=None)), dict(v=rows(data=P + 2)), dict(k=rows(token_stride=4)), dict(q_starts=None), dict(k_starts=None),
                dict(q_starts=P + 2), dict(out=None), dict(out=P + 4), dict(scale=float("-inf"))):
        assert ask(prompt(**bad)) == INVALID, bad
    for bad in (dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(head_dim=96), dict(tokens=-1), dict(keys=-1), dict(sequences=0), dict(keys=1 << 40)):
        assert ask(prompt(**bad)) == SHAPE, bad
    assert ask(prompt(tokens=0, q=rows(data=None))) == 0
    for bad in (dict(k=rows(token_stride=-128)), dict(v=rows(token_stride=(1 << 24) + 8))):
        assert ask(prompt(**bad)) == SHAPE, bad
    size = ctypes.c_size_t(7)
    long = prompt(keys=1 << 18)
    assert B.lib.ap_attention_prompt_size(ctypes.byref(long), ctypes.byref(size)) == 0 and size.value > 0
    long.work_bytes = size.value - 1
    assert ask(long) == SMALL
    long.work, long.work_bytes = None, size.value
    assert ask(long) == INVALID
    assert B.lib.ap_attention_prompt_size(ctypes.byref(prompt(tokens=0)), ctypes.byref(size)) == 0 and size.value == 0
    assert B.lib.ap_attention_prompt_size(ctypes.byref(prompt()), None) == INVALID


@pytest.mark.parametrize("head_dim", [64, 128])
def test_prompt_ranges_grow_with_the_keys_up_to_a_bound(head_dim):
    # the workspace holds head_dim + 2 floats per row and range: 64 ranges at most, however many would fit
    size = ctypes.c_size_t(0)
    ranges = []
    for keys in (1 << 14, 1 << 15, 100000, 131000, (1 << 17) - 1, 1 << 17, 1 << 20, 1 << 25):
        a = prompt(tokens=1, heads=8, kv_heads=1, keys=keys, sequences=1, head_dim=head_dim)
        assert B.lib.ap_attention_prompt_size(ctypes.byref(a), ctypes.byref(size)) == 0
        ranges.append(size.value // (8 * (head_dim + 2) * 4))
    assert ranges == sorted(ranges) and ranges[-1] == 64, ranges


def test_sizes_that_no_launch_can_have_are_refused():
    # a grid has fewer than 2^32 threads; workgroups have 256
    size = ctypes.c_size_t(7)
    cached_size = lambda kv, **kw: B.lib.ap_attention_cached_size(ctypes.byref(cache(kv_heads=kv)), ctypes.byref(cached(**kw)), ctypes.byref(size))
    prompt_size = lambda **kw: B.lib.ap_attention_prompt_size(ctypes.byref(prompt(**kw)), ctypes.byref(size))
    for kv, bad in ((2, dict(tokens=1 << 24, heads=16)), (8, dict(tokens=1 << 22, heads=64, sequences=1, q_starts=None)), (16, dict(tokens=3, heads=16, sequences=1 << 20)),
                    (1024, dict(tokens=1 << 14, heads=1024, sequences=1 << 14))):
        assert cached_size(kv, **bad) == SHAPE, (kv, bad)
        assert of(B.lib.ap_attention_cached, cache(kv_heads=kv), cached(**bad)) == SHAPE, (kv, bad)
    for bad in (dict(heads=16, kv_heads=16, sequences=1 << 20), dict(heads=1024, kv_heads=1024, sequences=1 << 14), dict(tokens=1 << 21, heads=1000, kv_heads=1000, sequences=1 << 10)):
        assert prompt_size(**bad) == SHAPE, bad
        assert of(B.lib.ap_attention_prompt, prompt(**bad)) == SHAPE, bad
    # and what is just within them is not
    assert cached_size(2, tokens=(1 << 24) - 64, heads=16, sequences=1) == 0 and cached_size(15, tokens=3, heads=15, sequences=1 << 20) == 0
    assert prompt_size(heads=15, kv_heads=15, sequences=1 << 20) == 0 and prompt_size(tokens=(1 << 25) - (1 << 12), heads=63, kv_heads=9) == 0


def test_prompt_keys_whose_ranges_would_end_beyond_32_bits_are_refused():
    # the last of 64 ranges of 2^31 - 256 keys would end at 2^31: with token strides of 0 they need no memory
    size = ctypes.c_size_t(7)
    for keys, status in ((1 << 30, 0), ((1 << 30) + 1, SHAPE), (0x7fffff00, SHAPE)):
        a = prompt(keys=keys, k=rows(token_stride=0), v=rows(token_stride=0))
        assert B.lib.ap_attention_prompt_size(ctypes.byref(a), ctypes.byref(size)) == status


def test_rows_that_are_joined_have_a_workgroup_each():
    # the join has a workgroup of 256 threads per row: fewer than 2^24 of them
    size = ctypes.c_size_t(0)
    for heads, kv_heads, sequences in ((16, 1, 1 << 20), (16, 1, (1 << 20) - 1), (32, 2, 1 << 19), (64, 8, 1 << 17), (64, 8, 1 << 18), (128, 8, 1 << 17)):
        for length in (4000, 4096, 5000, 8192, 1 << 16):
            a = cached(tokens=sequences, heads=heads, sequences=sequences, q_starts=None, table_width=1 << 10, max_length=length)
            assert B.lib.ap_attention_cached_size(ctypes.byref(cache(kv_heads=kv_heads)), ctypes.byref(a), ctypes.byref(size)) == 0
            assert size.value == 0 or sequences * heads < 1 << 24, (heads, sequences, length)


def test_workspace_of_cached_attention_is_bounded():
    # Sums of ranges are kept where row tiles are too few for the card; many rows over long caches need no more.  Few rows (16 of a key head at most, 2080 bytes per
    # range of 4096 keys of 272 bytes, twice for row tiles that are not full) need a small part of what the cache holds.
    size = ctypes.c_size_t(0)
    for tokens in (1, 64, 511, 512, 1000, 2048, 4096, 1 << 14, 1 << 18, 1 << 20):
        for length in (300, 4096, 5000, 32768, 131072, 1 << 20, 1 << 30):
            for sequences in (1, 8, 64):
                for head_dim in (64, 128):
                    if tokens % sequences == 0:
                        a = cached(tokens=tokens, heads=64, sequences=sequences, q_starts=None, table_width=1 << 24, max_length=length)
                        assert B.lib.ap_attention_cached_size(ctypes.byref(cache(kv_heads=8, head_dim=head_dim)), ctypes.byref(a), ctypes.byref(size)) == 0
                        few = tokens // sequences * 8 <= 16
                        assert size.value <= (300 << 20) + few * sequences * length * 8 * (head_dim + 8) // 32, (tokens, length, sequences, size.value)


def test_verify_refusals():
    ask = lambda a: of(B.lib.ap_verify, a)
    assert ask(None) == INVALID
    for bad in (dict(target=None), dict(draft=None), dict(target=P + 2), dict(drafted=None), dict(drafted=P + 4), dict(uniform=None), dict(noise=None),
                dict(noise=P + 2), dict(counts=P + 1), dict(tokens=None), dict(tokens=P + 4), dict(accepted=None), dict(half=1, target=P + 1)):
        assert ask(verification(**bad)) == INVALID, bad
    for bad in (dict(sequences=-1), dict(drafts=-1), dict(drafts=2000), dict(vocabulary=0), dict(vocabulary=1 << 31)):
        assert ask(verification(**bad)) == SHAPE, bad
    assert ask(verification(sequences=0, target=None)) == 0
    size = ctypes.c_size_t(0)
    assert B.lib.ap_verify_size(ctypes.byref(verification(vocabulary=1 << 20)), ctypes.byref(size)) == 0
    if size.value:
        assert ask(verification(vocabulary=1 << 20, work_bytes=size.value - 1)) == SMALL
        assert ask(verification(vocabulary=1 << 20, work=None, work_bytes=size.value)) == INVALID
    assert B.lib.ap_verify_size(ctypes.byref(verification()), None) == INVALID


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    x = torch.zeros((2, 4, 64), dtype=torch.float16)
    starts = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError):
        B.ap_attention_prompt(x, x, x, starts)                 # not on the GPU
    with pytest.raises(AssertionError):
        B.ap_verify(torch.zeros((1, 3, 8)), torch.zeros((1, 2, 8)), starts, starts, starts)
    with pytest.raises(TypeError):
        B.ap_attention_prompt(None, x, x, starts)
