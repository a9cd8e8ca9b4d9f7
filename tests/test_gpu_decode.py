"""GPU tests of the decoder operators against plain 64-bit forms: sizes, layouts, masks and values at which they can go wrong."""
import numpy as np
import pytest
import torch

import decode_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2402_10517_amd import binding
    return binding


def normal(seed, *shape, outlier=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)
    if outlier:
        x[..., shape[-1] // 3] *= 8
    return x


# ------------------------------------------------------------------------------------------------ append


def full_cache(B, pages, G, D, page):
    """A cache whose memory holds the bytes that hurt most: NaN scales, full codes."""
    cache = B.KVCache(pages, G, D, page_tokens=page)
    cache.buf.fill_(255)
    return cache


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tokens,H,G,rot,inter,page", [(1, 1, 1, 0, False, 16), (1, 32, 32, 1.0, False, 64), (17, 3, 1, 1.0, True, 16), (5, 40, 8, 0.5, False, 32),
                                                       (33, 7, 7, 0.25, True, 128), (130, 64, 8, 1.0, False, 256), (3, 0, 5, 1.0, True, 16)])
def test_append_rotates_and_rounds(B, D, tokens, H, G, rot, inter, page):
    table, pages = U.page_table([tokens + 5], page, seed=tokens)
    slots = U.slots_of(table, page, 0, 5, tokens + 5)
    slots[tokens // 2] = -1                                     # a token that is not kept
    q = normal(1, tokens, H, D) if H else None
    k, v = normal(2, tokens, G, D, outlier=True), normal(3, tokens, G, D)
    v[0, 0] = 1.5                                               # a row of one value: its step is 0
    k[-1, -1] *= 2.0 ** -14                                     # subnormal values and steps
    rotary = B.rotary_table(300, int(rot * D)) if rot else None
    positions = torch.randint(0, 300, (tokens,), generator=torch.Generator().manual_seed(4))
    cache = full_cache(B, pages, G, D, page)
    before = cache.buf.clone()
    q_out, k_out = B.ap_cache_append(cache, k, v, slots.cuda(), q=q, positions=positions.cuda() if rot else None, rotary=rotary, interleaved=inter)
    for x, got in ((q, q_out), (k, k_out)):
        if x is None:
            assert got is None
            continue
        want = U.rotate(x, rotary, positions.cuda(), inter)
        # two products and a sum in binary32 of values up to the larger of the pair, then one rounding
        U.check(got, want, U.HALF_EPS16 * want.abs() + 4 * U.EPS32 * x.double().abs().amax(-1, keepdim=True) + U.SUBNORMAL16, "rotated")
    k_got, v_got = B.ap_cache_read(cache, slots.cuda())
    kept = (slots >= 0).cuda()[:, None, None]
    for x, got in ((k_out, k_got), (v, v_got)):
        codes, low, step = U.codes_of(x)
        assert torch.equal(got, torch.where(kept, low + step * codes, torch.zeros_like(low)).half())
    # only the bytes of the tokens that were kept have changed
    changed = int((cache.buf != before).sum())
    assert changed <= int(kept.sum()) * G * (D + 8)
    assert changed >= int(kept.sum()) * G * (D + 8) // 2


def test_append_strided_in_place_and_in_any_order(B):
    T, H, G, D, page = 29, 6, 2, 128, 16
    x = normal(5, T, H + 2 * G, D)
    q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    rotary = B.rotary_table(64, D)
    positions = torch.arange(T).cuda()
    slots = torch.randperm(4 * page, generator=torch.Generator().manual_seed(1))[:T].cuda()
    one, two = full_cache(B, 4, G, D, page), full_cache(B, 4, G, D, page)
    q1, k1 = B.ap_cache_append(one, k.contiguous(), v.contiguous(), slots, q=q.contiguous(), positions=positions, rotary=rotary)
    heads_first = q.transpose(0, 1).contiguous().transpose(0, 1)        # (heads, tokens, head_dim) in memory
    back = torch.arange(T - 1, -1, -1).cuda()
    q2, k2 = B.ap_cache_append(two, k[back], v[back], slots[back], q=heads_first[back], positions=positions[back], rotary=rotary)
    assert torch.equal(q1, q2[back]) and torch.equal(k1, k2[back]) and torch.equal(one.buf, two.buf)
    q3, k3 = B.ap_cache_append(two, k, v, slots, q=q, positions=positions, rotary=rotary, q_out=q, k_out=k)
    assert q3 is not None and torch.equal(x[:, :H], q1) and torch.equal(x[:, H:H + G], k1) and torch.equal(one.buf, two.buf)


def test_append_values_out_of_range(B):
    G, D, page = 2, 64, 16
    cache = full_cache(B, 2, G, D, page)
    before = cache.buf.clone()
    k, v = normal(1, 5, G, D), normal(2, 5, G, D)
    far = torch.tensor([-1, 2 * page, -2 ** 63, 2 ** 62, 2 ** 40], device="cuda")
    B.ap_cache_append(cache, k, v, far)
    assert torch.equal(cache.buf, before)
    kz, vz = B.ap_cache_read(cache, far)
    assert not kz.any() and not vz.any()
    # a position outside the table: its rotated channels are NaN, the others stay
    rotary = B.rotary_table(8, 32)
    _, k_out = B.ap_cache_append(cache, k, v, far, positions=torch.tensor([7, 8, -1, 2 ** 62, 0], device="cuda"), rotary=rotary)
    lost = torch.tensor([False, True, True, True, False], device="cuda")
    assert torch.equal(torch.isnan(k_out[..., :32]).all(-1).all(-1), lost) and not torch.isnan(k_out[~lost]).any()
    assert torch.equal(k_out[..., 32:], k[..., 32:])
    # rows with an infinity or NaN read back as NaN, and only they; extreme finite values do not overflow
    k[1, 0, 5], v[2, 1, 63], v[3, 0, 0] = float("inf"), float("nan"), float("-inf")
    k[4, 0, :2] = torch.tensor([65504.0, -65504.0])
    slots = torch.arange(5, device="cuda") + 11                 # across the end of the first page
    B.ap_cache_append(cache, k, v, slots)
    kz, vz = B.ap_cache_read(cache, slots)
    for x, got in ((k, kz), (v, vz)):
        assert torch.equal(torch.isnan(got).all(-1), ~torch.isfinite(x).all(-1)) and torch.equal(torch.isnan(got).any(-1), torch.isnan(got).all(-1))
    assert torch.isfinite(kz[4]).all()
    empty = k[:0]
    assert B.ap_cache_append(cache, empty, empty, slots[:0])[1].shape == (0, G, D) and B.ap_cache_read(cache, slots[:0])[0].shape == (0, G, D)


def test_tensors_that_do_not_fit_are_refused(B):
    G, D, page, T = 2, 64, 16, 4
    cache = full_cache(B, 3, G, D, page)
    k, v, q, slots = normal(1, T, G, D), normal(2, T, G, D), normal(3, T, 4, D), torch.arange(T).cuda()
    rotary, positions = B.rotary_table(8, 32), torch.arange(T).cuda()
    table, lens, starts = torch.zeros((T, 3), dtype=torch.int32).cuda(), torch.ones(T, dtype=torch.int32).cuda(), torch.arange(T + 1, dtype=torch.int32).cuda()
    append = lambda **kw: B.ap_cache_append(cache, **dict(dict(k=k, v=v, slots=slots, q=q, positions=positions, rotary=rotary), **kw))
    for bad in (dict(k=k[:3]), dict(v=v.float()), dict(k=k.cpu()), dict(v=normal(1, T, G + 1, D)), dict(k=normal(1, T, G, 2 * D)[..., ::2]), dict(slots=slots.int()),
                dict(slots=slots[:2]), dict(positions=None), dict(positions=positions.cpu()), dict(rotary=rotary.half()), dict(rotary=rotary[:0]), dict(q=q[0]),
                dict(q_out=torch.empty_like(k)), dict(k_out=k.float())):
        with pytest.raises(AssertionError):
            append(**bad)
    for bad in (dict(rotary=B.rotary_table(8, 8)), dict(k=normal(1, T * G * D + 4)[4:].as_strided((T, G, D), (G * D, D, 1), 4))):
        with pytest.raises(B.ApError):
            append(**bad)
    attend = lambda **kw: B.ap_attention_cached(cache, **dict(dict(q=q, tables=table, lengths=lens), **kw))
    for bad in (dict(q=q.float()), dict(tables=table.long()), dict(tables=table[:, :2]), dict(lengths=lens[:2]), dict(q_starts=starts[:-1]), dict(out=q[:2]),
                dict(out=q.float()), dict(work=torch.zeros(8)), dict(tables=table[0])):
        with pytest.raises(AssertionError):
            attend(**bad)
    for bad in (dict(max_length=49), dict(max_length=-1), dict(scale=float("nan")), dict(q=normal(3, T, 3, D)), dict(q=normal(3, T + 1, 4, D))):
        with pytest.raises(B.ApError):
            attend(**bad)
    prompt = lambda **kw: B.ap_attention_prompt(**dict(dict(q=q, k=k, v=v, q_starts=starts), **kw))
    for bad in (dict(k=k.float()), dict(v=v[:2]), dict(q_starts=starts.long()), dict(k_starts=starts[:3]), dict(q=q[:, 0])):
        with pytest.raises(AssertionError):
            prompt(**bad)
    for bad in (dict(q=normal(3, T, 3, D)), dict(scale=float("inf"))):
        with pytest.raises(B.ApError):
            prompt(**bad)
    with pytest.raises(B.ApError):                              # a workspace that is too small
        B.ap_attention_prompt(normal(1, 1, 4, D), normal(2, 5000, 4, D), normal(3, 5000, 4, D), U.starts([1]).cuda(), U.starts([5000]).cuda(),
                              work=torch.empty(16, dtype=torch.uint8, device="cuda"))
    p = [torch.from_numpy(x).cuda() for x in verify_inputs(2, 3, 50, False, 1)]
    for i, bad in ((0, p[0].double()), (0, p[0][:, :3].contiguous()), (1, p[1].half()), (2, p[2].int()), (3, p[3][:1]), (4, p[4].cpu())):
        with pytest.raises(AssertionError):
            B.ap_verify(*[bad if j == i else x for j, x in enumerate(p)])
    with pytest.raises(AssertionError):
        B.ap_verify(*p, counts=torch.zeros(3, dtype=torch.int32).cuda())


@pytest.mark.parametrize("D,rot", [(64, 32), (128, 64), (128, 16), (128, 112), (128, 128)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("tokens", [5, 300])
def test_channels_beyond_the_rotation_stay(B, D, rot, inter, tokens):
    H, G = 6, 2
    q, k, v = normal(1, tokens, H, D), normal(2, tokens, G, D), normal(3, tokens, G, D)
    if rot < D:
        for x in (q, k):
            x[..., rot], x[1::3, :, rot + 5], x[2::3, :, D - 2], x[::2, :, D - 3] = -0.0, float("inf"), float("nan"), float("-inf")
    rotary = B.rotary_table(tokens + 3, rot)
    positions = torch.arange(tokens).cuda() + 3
    positions[tokens // 2] = 2 ** 40                            # no row of the table
    cache = full_cache(B, -(-tokens // 16), G, D, 16)
    q_out, k_out = B.ap_cache_append(cache, k, v, torch.arange(tokens).cuda(), q=q, positions=positions, rotary=rotary, interleaved=inter)
    positions[tokens // 2] = 0
    for x, got in ((q, q_out), (k, k_out)):
        assert torch.equal(got[..., rot:].view(torch.int16), x[..., rot:].view(torch.int16))
        want = U.rotate(x, rotary, positions, inter)[..., :rot]
        want[tokens // 2] = float("nan")
        U.check(got[..., :rot], want, U.HALF_EPS16 * want.abs() + 4 * U.EPS32 * x[..., :rot].double().abs().amax(-1, keepdim=True) + U.SUBNORMAL16)
    k_got, _ = B.ap_cache_read(cache, torch.arange(tokens).cuda())
    assert torch.equal(torch.isnan(k_got).all(-1), ~torch.isfinite(k_out).all(-1))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rot,inter", [(0, False), (1.0, False), (0.5, False), (1.0, True), (0.25, True)])
@pytest.mark.parametrize("tokens,H,G,fused", [(255, 32, 4, True), (256, 5, 1, False), (257, 32, 8, True), (1003, 64, 8, True), (2000, 40, 40, False), (8201, 28, 4, True)])
def test_append_many_tokens(B, D, rot, inter, tokens, H, G, fused):
    # from 256 tokens on 16 adjacent ones are taken together, and from some thousand rows on several rows by the same lanes
    page = 64
    table, pages = U.page_table([tokens + 5], page, seed=tokens)
    slots = U.slots_of(table, page, 0, 5, tokens + 5)
    slots[-tokens // 9:] = -1
    x = normal(tokens, tokens, H + 2 * G, D)
    q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    if not fused:
        q, k, v = q.contiguous(), k.transpose(0, 1).contiguous().transpose(0, 1), v.contiguous()
    rotary = B.rotary_table(9000, int(rot * D)) if rot else None
    positions = torch.randint(0, 9000, (tokens,), generator=torch.Generator().manual_seed(4)).cuda()
    cache = full_cache(B, pages, G, D, page)
    before = cache.buf.clone()
    q_out, k_out = B.ap_cache_append(cache, k, v, slots.cuda(), q=q, positions=positions if rot else None, rotary=rotary, interleaved=inter)
    for y, got in ((q, q_out), (k, k_out)):
        want = U.rotate(y, rotary, positions, inter)
        U.check(got, want, U.HALF_EPS16 * want.abs() + 4 * U.EPS32 * y.double().abs().amax(-1, keepdim=True) + U.SUBNORMAL16, "rotated")
    k_got, v_got = B.ap_cache_read(cache, slots.cuda())
    kept = (slots >= 0).cuda()[:, None, None]
    for y, got in ((k_out, k_got), (v, v_got)):
        codes, low, step = U.codes_of(y)
        assert torch.equal(got, torch.where(kept, low + step * codes, torch.zeros_like(low)).half())
    changed = int((cache.buf != before).sum())
    assert int(kept.sum()) * G * (D + 8) // 2 <= changed <= int(kept.sum()) * G * (D + 8)
    # one token at a time, which takes the other kernel: the same bits
    few = torch.arange(tokens - tokens // 9 - 40, tokens - tokens // 9 + 3).cuda()
    again = full_cache(B, pages, G, D, page)
    q_few, k_few = B.ap_cache_append(again, k[few], v[few], slots.cuda()[few], q=q[few], positions=positions[few] if rot else None, rotary=rotary, interleaved=inter)
    assert torch.equal(q_few, q_out[few]) and torch.equal(k_few, k_out[few])
    assert all(torch.equal(a, b[few]) for a, b in zip(B.ap_cache_read(again, slots.cuda()[few]), (k_got, v_got)))
    q_in, k_in = q.clone(), k.clone()
    B.ap_cache_append(again, k_in, v, slots.cuda(), q=q_in, positions=positions if rot else None, rotary=rotary, interleaved=inter, q_out=q_in, k_out=k_in)
    assert torch.equal(q_in, q_out) and torch.equal(k_in, k_out) and torch.equal(again.buf, cache.buf)


def test_interleaved_without_a_truth_value(B):
    k = normal(1, 2, 1, 64)
    cache = full_cache(B, 1, 1, 64, 16)
    with pytest.raises(ValueError):                             # numpy's own error, and not one of a call that has succeeded
        B.ap_cache_append(cache, k, k, torch.arange(2).cuda(), positions=torch.arange(2).cuda(), rotary=B.rotary_table(4, 64), interleaved=np.zeros(2))


# ------------------------------------------------------------------------------------------------ attention over the cache


def cached_case(B, lengths, queries, H, G, D, page, seed=0, scale=None, uniform=False, max_length=None, spoil=None, view=False, width=None, base=0):
    """Runs one call and checks every row.  base: pages in front of the case's own, for addresses far into the cache."""
    table, pages = U.page_table(lengths, page, seed=seed, width=width)
    table = torch.where(table >= 0, table + base, table)
    cache = B.KVCache(pages + base, G, D, page_tokens=page)
    first = base * (cache.buf.numel() // (pages + base))
    cache.buf[first:].fill_(255)
    slots = torch.cat([U.slots_of(table, page, i, 0, n) for i, n in enumerate(lengths)])
    total = len(slots)
    k, v = normal(seed + 1, total, G, D, outlier=True), normal(seed + 2, total, G, D)
    if spoil:
        spoil(k, v)
    B.ap_cache_append(cache, k, v, slots.cuda())
    T = sum(queries)
    q = normal(seed + 3, T, H + 2, D)[:, 1:H + 1] if view else normal(seed + 3, T, H, D)
    st = U.starts(queries)
    scale = D ** -0.5 if scale is None else scale
    args = dict(q_starts=None if uniform else st.cuda(), scale=scale, max_length=max_length)
    lens = torch.tensor(lengths, dtype=torch.int32).cuda()
    out = B.ap_attention_cached(cache, q, table.cuda(), lens, **args)
    again = B.ap_attention_cached(cache, q, table.cuda(), lens, **args)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    at, worst = 0, 0.0
    for i, (n, m) in enumerate(zip(queries, lengths)):
        m = m if max_length is None else min(m, max_length)
        rows = slice(int(st[i]), int(st[i]) + n)
        kk, vv = k[at:at + m], v[at:at + m]
        _, kl, ks = U.codes_of(kk)
        _, vl, vs = U.codes_of(vv)
        sees = m - n + 1 + torch.arange(n)
        # values enter the sums as low + step (offset + code) with an offset up to 128: the magnitudes that bound the rounding of the sums
        want, bound = U.attention(q[rows].double(), U.cache_values(kk), U.cache_values(vv), scale, sees,
                                  (kl.abs() + 143 * ks).double().expand(-1, -1, D), (vl.abs() + vs * 15).double().expand(-1, -1, D))
        worst = max(worst, U.check(out[rows], want, bound, "sequence %d of %d keys" % (i, m)))
        at += lengths[i]
    return out, worst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (8, 1), (14, 2), (20, 1), (33, 1), (32, 32)])
def test_cached_head_layouts(B, H, G, D):
    cached_case(B, [1, 2, 15, 16, 17, 31, 32, 33, 130, 0, 257], [1] * 11, H, G, D, 16, seed=H, uniform=True)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_cached_pages_and_lengths(B, page, D):
    cached_case(B, [page - 1, page, page + 1, 511, 512, 513, 1023, 1025, 2049, 1], [1, 2, 1, 5, 1, 3, 1, 0, 4, 1], 8, 2, D, page, seed=page)


@pytest.mark.parametrize("queries", [2, 5, 8, 17, 40])
def test_cached_many_queries(B, queries):
    # some sequences are shorter than their queries: the first ones see nothing
    cached_case(B, [3, 100, 0, 700, queries, 1, 1500], [queries] * 7, 16, 4, 128, 64, seed=queries, uniform=True, view=True)
    cached_case(B, [3, 100, 0, 700, queries, 1], [queries, 1, 2, 0, queries, 3], 6, 2, 64, 16, seed=queries)


def test_cached_long(B):
    cached_case(B, [70001, 3], [1, 1], 8, 1, 128, 64, uniform=True)
    cached_case(B, [33000], [3], 4, 2, 64, 16, uniform=True)


@pytest.mark.parametrize("D,H,G,S,longest,queries", [(128, 32, 32, 64, 20001, 1), (128, 32, 16, 256, 70000, 10), (128, 16, 16, 128, 30000, 17),
                                                       (64, 16, 16, 256, 40001, 20)])
def test_cached_ranges_longer_than_the_pages_that_a_wave_holds(B, D, H, G, S, longest, queries):
    # with 32 rows a tile, and tiles enough for the card: ranges of more than 4096 keys; and calls of one query beside them
    lengths = [longest, 1, 5003, 40] + [(i * 13) % 70 for i in range(S - 6)] + [longest - 3000, longest]
    cached_case(B, lengths, [queries] * S, H, G, D, 64, uniform=True)


def test_cached_few_rows_and_a_bound_far_above_the_lengths(B):
    # as many ranges of 4096 keys as no launch can have
    cached_case(B, [300], [1], 1024, 1024, 64, 16, max_length=2 ** 30, width=2 ** 26)


def test_cached_pages_outside_the_cache_in_long_ranges(B):
    S, n, G, D, page, longest, kept = 128, 17, 32, 64, 16, 70000, 5008
    cache = full_cache(B, kept // page, G, D, page)
    B.ap_cache_append(cache, normal(1, kept, G, D), normal(2, kept, G, D), torch.arange(kept).cuda())
    q = normal(3, S * n, G, D)
    table = torch.full((S, longest // page), 2 ** 30, dtype=torch.int32)
    table[1::2] = -1
    table[:, :kept // page] = torch.arange(kept // page)
    at = lambda length: torch.full((S,), length, dtype=torch.int32).cuda()
    # the last query alone: the others see fewer keys of the shorter length
    outs = [B.ap_attention_cached(cache, q, table.cuda(), at(length)).view(S, n, G, D)[:, -1] for length in (longest, kept)]
    assert torch.equal(*outs)


def test_cached_scales_and_bounds(B):
    for scale in (0.0, -0.3, 1.0, 1e-6):
        cached_case(B, [100, 40], [1, 2], 4, 2, 128, 32, scale=scale)
    cached_case(B, [300, 40, 128], [1, 2, 1], 4, 2, 128, 32, max_length=128)     # longer sequences are cut at max_length
    cached_case(B, [300, 40], [1, 2], 4, 2, 64, 16, width=400)                   # a table much wider than what it holds
    cached_case(B, [0, 0], [1, 2], 4, 2, 64, 16)


def test_cached_nan_reaches_only_rows_that_see_it(B):
    def spoil(k, v):
        v[90, 0, 3] = float("inf")        # token 90 of 96: of 8 queries the last 6 see it
        k[95, 1, 0] = float("nan")        # the last token: only the last query sees it
    out, _ = cached_case(B, [96], [8], 4, 2, 128, 32, spoil=spoil)
    bad = torch.isnan(out).all(-1)
    assert bad[:, :2].any(1).tolist() == [False] * 2 + [True] * 6 and bad[:, 2:].any(1).tolist() == [False] * 7 + [True]


def test_cached_pages_outside_the_cache_hold_nothing(B):
    G, D, page = 2, 128, 16
    cache = full_cache(B, 4, G, D, page)
    k, v = normal(1, 32, G, D), normal(2, 32, G, D)
    B.ap_cache_append(cache, k, v, torch.arange(32).cuda())
    q = normal(3, 1, 4, D)
    table = torch.tensor([[0, -1, 1, 4, 2 ** 31 - 1]], dtype=torch.int32).cuda()
    out = B.ap_attention_cached(cache, q, table, torch.tensor([80], dtype=torch.int32).cuda())
    want = B.ap_attention_cached(cache, q, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), torch.tensor([32], dtype=torch.int32).cuda())
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -9 * want.float().abs().max()
    gone = B.ap_attention_cached(cache, q, torch.full_like(table, -7), torch.tensor([80], dtype=torch.int32).cuda())
    assert not gone.any()
    # lengths and starts that make no sense: no fault, and rows of no sequence stay as they were
    q = normal(4, 6, 4, D)
    out = torch.full_like(q, 7.0)
    bad = torch.tensor([0, 2, 2, -5, 4], dtype=torch.int32).cuda()
    B.ap_attention_cached(cache, q, table.expand(4, -1).contiguous(), torch.tensor([-3, 2 ** 31 - 1, 1, 16], dtype=torch.int32).cuda(), q_starts=bad, out=out)
    assert not out[:2].any() and (out[4:] == 7).all()


def test_cached_offsets_beyond_32_bits(B):
    # 2.2 million tokens in front: the case's pages lie beyond 4 GiB
    cached_case(B, [200, 77], [1, 2], 32, 16, 128, 64, base=35000)


def test_cached_on_a_named_stream(B):
    table, pages = U.page_table([600], 64)
    cache = full_cache(B, pages, 2, 128, 64)
    k, v = normal(1, 600, 2, 128), normal(2, 600, 2, 128)
    slots = U.slots_of(table, 64, 0, 0, 600).cuda()
    q, tables, lens = normal(3, 1, 8, 128), table.cuda(), torch.tensor([600], dtype=torch.int32).cuda()
    B.ap_cache_append(cache, k, v, slots)
    want = B.ap_attention_cached(cache, q, tables, lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        cache.buf.fill_(255)
        side.wait_stream(torch.cuda.current_stream())
        B.ap_cache_append(cache, k, v, slots, stream=side)
        out = B.ap_attention_cached(cache, q, tables, lens, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------------ attention over prompts


def prompt_case(B, q_counts, k_counts, H, G, D, seed=0, scale=None, fused=False, spoil=None, tensors=None):
    T, M = sum(q_counts), sum(k_counts)
    if tensors:
        q, k, v = tensors
    elif fused:
        x = normal(seed, T, H + 2 * G, D)
        q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    else:
        q, k, v = normal(seed, T, H, D), normal(seed + 1, M, G, D), normal(seed + 2, M, G, D)
    if spoil:
        spoil(k, v)
    qs, ks = U.starts(q_counts), U.starts(k_counts)
    scale = D ** -0.5 if scale is None else scale
    out = B.ap_attention_prompt(q, k, v, qs.cuda(), ks.cuda(), scale=scale)
    again = B.ap_attention_prompt(q, k, v, qs.cuda(), ks.cuda(), scale=scale)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    worst = 0.0
    for i, (n, m) in enumerate(zip(q_counts, k_counts)):
        rows, keys = slice(int(qs[i]), int(qs[i]) + n), slice(int(ks[i]), int(ks[i]) + m)
        want, bound = U.attention(q[rows].double(), k[keys].double(), v[keys].double(), scale, m - n + 1 + torch.arange(n))
        worst = max(worst, U.check(out[rows], want, bound, "sequence %d, %d of %d" % (i, n, m)))
    return out, worst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (4, 4), (8, 1), (14, 2), (20, 1)])
def test_prompt_lengths(B, H, G, D):
    n = [1, 2, 15, 16, 17, 0, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
    prompt_case(B, n, n, H, G, D, seed=H, fused=True)


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_pieces(B, D):
    prompt_case(B, [1, 5, 64, 130, 1, 0, 33], [300, 77, 1000, 131, 1, 40, 2000], 6, 2, D)
    # more queries than keys: the first ones see nothing; none at all
    prompt_case(B, [70, 200, 3, 1], [64, 3, 0, 0], 6, 2, D)


@pytest.mark.parametrize("S", [63, 64, 65, 130])
def test_prompt_many_sequences(B, S):
    # every sequence and tile is some workgroup's, whatever order they go in
    n = [(i * 37) % 290 if i % 5 else 0 for i in range(S)]
    prompt_case(B, n, [x + i % 3 for i, x in enumerate(n)], 4, 2, 64, seed=S)


def test_prompt_long(B):
    prompt_case(B, [2500], [2500], 2, 1, 128)
    prompt_case(B, [1100, 900], [5000, 901], 5, 1, 64)


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_keys_divided_among_workgroups(B, D):
    # few rows and many keys; with sequences whose keys are one range, several, none, and queries that see only some of the ranges
    prompt_case(B, [1], [5000], 8, 8, D)
    prompt_case(B, [3, 40, 1, 5, 2], [6000, 41, 0, 9000, 1], 8, 2, D)
    def spoil(k, v):
        v[4100, 0, 3] = float("nan")
        v[4201, 1, 5] = float("inf")                            # seen by the last query only
    out, _ = prompt_case(B, [200], [4202], 2, 2, D, spoil=spoil)
    bad = ~torch.isfinite(out).all(-1)
    assert bad[:, 0].tolist() == [4002 + i >= 4100 for i in range(200)] and bad[:, 1].tolist() == [False] * 199 + [True]


def test_weights_far_below_the_greatest(B):
    # one key far above 8191 equal ones, whose weights are small numbers of binary16: they count by their sum
    for low in (2.0 ** -14, 2.0 ** -18, 2.0 ** -21):
        q, k, v = torch.zeros((1, 1, 128)), torch.zeros((8192, 1, 128)), torch.ones((8192, 1, 128))
        q[0, 0, 0], k[0, 0, 0], v[0] = 1.0, 64.0, 0.0
        q, k, v = q.half().cuda(), k.half().cuda(), v.half().cuda()
        scale = -np.log(low) / 64
        out = B.ap_attention_prompt(q, k, v, U.starts([1]).cuda(), U.starts([8192]).cuda(), scale=scale)
        want = 8191 * low / (1 + 8191 * low)
        # half a step of binary16 in the result, and the same in the weights down to 2^-21
        assert (out.double() - want).abs().max().item() <= want * 2 * U.HALF_EPS16 + U.SUBNORMAL16, low


@pytest.mark.parametrize("size", [8.0, 300.0, 20000.0])
def test_large_scores(B, size):
    # scores up to 10^10: their own binary32 rounding decides which key wins, but the weights stay weights
    q, k, v = normal(1, 70, 2, 128) * size, normal(2, 300, 2, 128) * size, normal(3, 300, 2, 128)
    prompt_case(B, [70], [300], 2, 2, 128, tensors=(q, k, v))
    q, k = q.clamp(-60000, 60000), k.clamp(-60000, 60000)
    k[1::2] = k[0::2]                                           # pairs of equal keys: the weights of a pair are equal whatever they are
    v[1::2] = -v[0::2]
    out = B.ap_attention_prompt(q[:2], k, v, U.starts([2]).cuda(), U.starts([299]).cuda())
    assert out[1].abs().max().item() <= 2.0 and torch.isfinite(out).all()
    cached_case(B, [300], [4], 2, 2, 128, 32, scale=size * size / 11)


def test_prompt_scales(B):
    for scale in (0.0, -0.2, 1.0, 30.0):
        prompt_case(B, [100, 40], [100, 40], 2, 1, 128, scale=scale)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [0, 5, 63, 64, 70, 149])
def test_prompt_values_that_are_not_seen_do_not_matter(B, D, at):
    def spoil(k, v):
        v[at, 0, 3], v[at, 0, 9], v[at, 0, 17] = float("inf"), float("-inf"), float("nan")
        k[150 + 20, 1, 5] = float("nan")                        # the second sequence's token 20
        v[150 + 30, 1] = 65504.0
    out, _ = prompt_case(B, [150, 60, 1], [150, 60, 1], 4, 2, D, spoil=spoil)
    bad = ~torch.isfinite(out[:, :2]).all(-1).all(-1)
    assert bad.tolist() == [at <= i < 150 for i in range(211)]
    assert (~torch.isfinite(out[:, 2:]).all(-1).all(-1)).tolist() == [170 <= i < 210 for i in range(211)]


def test_prompt_strides_and_offsets(B):
    T, H, G, D = 90, 4, 2, 128
    q, k, v = normal(1, H, T, D).transpose(0, 1), normal(2, G, T, D).transpose(0, 1), normal(3, T, G, D)
    prompt_case(B, [50, 40], [50, 40], H, G, D, tensors=(q, k, v.flip(0).contiguous()))
    # rows of the keys 2^24 elements apart: offsets beyond 2^32 bytes
    far = torch.zeros(T << 24, dtype=torch.float16, device="cuda").as_strided((T, G, D), (1 << 24, D, 1))
    far.copy_(k)
    prompt_case(B, [50, 40], [50, 40], H, G, D, tensors=(q, far, v))


def test_prompt_starts_that_make_no_sense(B):
    q, k, v = normal(1, 40, 2, 64), normal(2, 40, 2, 64), normal(3, 40, 2, 64)
    out = torch.full_like(q, 7.0)
    B.ap_attention_prompt(q, k, v, torch.tensor([0, 10, 5, 2 ** 31 - 1, -4], dtype=torch.int32).cuda(),
                          torch.tensor([-9, 10, 2 ** 31 - 1, 3, 50], dtype=torch.int32).cuda(), out=out)
    torch.cuda.synchronize()
    empty = q[:0]
    assert B.ap_attention_prompt(empty, k, v, torch.zeros(2, dtype=torch.int32).cuda(), torch.tensor([0, 40], dtype=torch.int32).cuda()).shape == (0, 2, 64)


def test_prompt_rows_of_senseless_starts(B):
    q, k, v = normal(1, 40, 2, 64), normal(2, 40, 2, 64), normal(3, 40, 2, 64)
    out = torch.full_like(q, 7.0)
    B.ap_attention_prompt(q, k, v, torch.tensor([0, 10, 5, 2 ** 31 - 1, -4], dtype=torch.int32).cuda(),
                          torch.tensor([-9, 10, 2 ** 31 - 1, 3, 50], dtype=torch.int32).cuda(), out=out)
    assert not out[:10].any() and (out[10:] == 7).all()


# ------------------------------------------------------------------------------------------------ scores of any size


def attend(B, kernel, q, k, v, scale=None):
    """One sequence whose queries are its last tokens, by either kernel: (out, keys, values, bound): what stands for k and v there, and the error of
    a weighted mean of values with exact weights."""
    if kernel == "prompt":
        out = B.ap_attention_prompt(q, k, v, U.starts([len(q)]).cuda(), U.starts([len(k)]).cuda(), scale=scale)
        return out, k.double(), v.double(), 64 * U.EPS32 * v.double().abs().amax()
    page = 32
    table, pages = U.page_table([len(k)], page)
    cache = full_cache(B, pages, k.shape[1], k.shape[2], page)
    B.ap_cache_append(cache, k, v, U.slots_of(table, page, 0, 0, len(k)).cuda())
    out = B.ap_attention_cached(cache, q, table.cuda(), torch.tensor([len(k)], dtype=torch.int32).cuda(), scale=scale)
    _, low, step = U.codes_of(v)
    # values enter the sums as low + step (offset + code), weights times steps as two bfloat16 numbers
    return out, U.cache_values(k), U.cache_values(v), (64 * U.EPS32 * (low.abs() + 143 * step) + 2.0 ** -16 * 15 * step).double().amax()


@pytest.mark.parametrize("kernel", ["cached", "prompt"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1.0, 300.0, 20000.0, 30000.0, 40000.0, 65504.0])
def test_equal_keys_of_any_size_are_averaged(B, kernel, D, size):
    # equal keys have equal scores, however these and their product with the scale round: in a tile, across waves and across ranges
    for n, m in ((3, 20), (2, 130), (5, 700), (1, 5000)):
        q, k, v = torch.full((n, 4, D), size, dtype=torch.float16, device="cuda"), torch.full((m, 2, D), size, dtype=torch.float16, device="cuda"), normal(m, m, 2, D)
        for scale in (None, -0.2):
            out, _, values, err = attend(B, kernel, q, k, v, scale)
            for i in range(n):
                want = values[:m - n + 1 + i].mean(0).repeat_interleave(2, 0)
                U.check(out[i], want, U.HALF_EPS16 * want.abs() + err + U.SUBNORMAL16, "query %d of %d keys" % (i, m))


@pytest.mark.parametrize("kernel", ["cached", "prompt"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size,scale", [(30.0, None), (300.0, None), (20000.0, None), (20000.0, -1.0), (1.0, 3e4), (1.0, 1e30), (20000.0, 1e30), (1.0, 3e38), (300.0, -3e38)])
def test_the_greatest_score_of_any_size_takes_all(B, kernel, D, size, scale):
    n, m = 8, 700
    k, v = (normal(1, m, 2, D).float() * size).clamp(-60000, 60000).half(), normal(2, m, 2, D)
    of = torch.tensor([(i * 97 + 40) % (m - n) for i in range(n)]).cuda()
    q = k[of].repeat_interleave(2, 1) * (-1 if scale and scale < 0 else 1)
    out, keys, values, err = attend(B, kernel, q, k, v, scale)
    s = torch.matmul(q.double().transpose(0, 1), keys.repeat_interleave(2, 1).permute(1, 2, 0).contiguous()) * (scale or D ** -0.5)   # (heads, n, m)
    first, second = s.topk(2, dim=2).values.unbind(2)
    assert (first - second > 60 + s.abs().amax() * 2.0 ** -16).all() and (s.argmax(2) == of).all()
    want = values[of].repeat_interleave(2, 1)
    U.check(out, want, U.HALF_EPS16 * want.abs() + err + U.SUBNORMAL16)


@pytest.mark.parametrize("D", [64, 128])
def test_cached_scores_keep_their_bits(B, D):
    # Two keys of close scores far below the sum of the magnitudes that enter them.  The products of queries and codes are whole multiples of one quantum,
    # all sums of them below 2^24 quanta: binary32 holds them exactly, and only the score's own roundings are left.
    S, g = 64, torch.Generator().manual_seed(D)
    quantum = 1 / 8 if D == 128 else 1 / 16
    q = torch.empty((S, 1, D))
    q[..., :D // 2] = torch.randint(1024, 2048, (S, 1, D // 2), generator=g).float()
    q[..., D // 2:] = torch.randint(1024, 2048, (S, 1, D // 2), generator=g).float() * quantum
    q[..., 2] = 65 * quantum if D == 128 else 129 * quantum
    codes = torch.randint(0, 16, (S, 2, 1, D), generator=g)
    codes[:, 1] = codes[:, 0]
    codes[..., 0], codes[..., 1] = 0, 15                        # least and greatest of the row
    codes[:, 0, :, 2], codes[:, 1, :, 2] = 7, 8
    k, v = codes / 8 - 1, torch.tensor([0.0, 1.0]).view(1, 2, 1, 1).expand(S, 2, 1, D)
    sums = (q.double() * codes[:, 0].double()).sum(-1).amax().item()
    assert 2.0 ** 22 < sums / quantum < 2.0 ** 24
    cache = full_cache(B, S, 1, D, 16)
    slots = torch.arange(S)[:, None] * 16 + torch.arange(2)
    B.ap_cache_append(cache, k.half().flatten(0, 1).cuda(), v.half().flatten(0, 1).contiguous().cuda(), slots.flatten().cuda())
    out = B.ap_attention_cached(cache, q.half().cuda(), torch.arange(S).int()[:, None].cuda(), torch.full((S,), 2, dtype=torch.int32).cuda(), scale=1.0)
    s = torch.matmul(k.double()[:, :, 0], q.double()[:, 0, :, None])[..., 0]
    want = torch.sigmoid(s[:, 1] - s[:, 0])
    # low * sum and step * sum are exact too; a score is rounded once, at its own size, and the weight's slope is at most 1 / 4
    off = 2 * U.EPS32 * s.abs().amax().item() / 4 + 16 * U.EPS32
    U.check(out, want[:, None, None].expand(S, 1, D).cuda(), torch.full((S, 1, D), U.HALF_EPS16 + off, dtype=torch.float64).cuda())


@pytest.mark.parametrize("D", [64, 128])
def test_cached_sums_of_values_keep_their_bits(B, D):
    # Equal weights, and values that cancel in pairs: what is left is the rounding of the sums.  A wave of four has 512 of 2048 keys, 16 products of 32 in two
    # parts, each a rounding or two of sums up to 512 * step * 31 in binary32 (codes with an offset of 16), of the values and of what takes the offset
    # out again; the roundings are independent and uniform, of variance ulp^2 / 12 with ulp <= 2^-23 of the sum.
    S, G, m = 32, 8, 2048
    g = torch.Generator(device="cuda").manual_seed(D)
    step = (torch.randint(512, 1024, (m // 2, G, 1), generator=g, device="cuda") * 2 + 1).float() / 1024       # 11 bits, 1 to 2
    codes = torch.randint(1, 16, (m // 2, G, D), generator=g, device="cuda").float()
    codes = torch.stack([codes, 16 - codes], dim=1).flatten(0, 1)
    codes[..., 0], codes[..., 1] = 0, 15
    mixed = torch.randperm(m, generator=g, device="cuda")       # a pair's keys are far apart
    codes, step = codes[mixed], step.repeat_interleave(2, 0)[mixed]
    v = ((codes - 8) * step).half()
    got, low, scale = U.codes_of(v)
    assert torch.equal(got, codes) and torch.equal(scale, step) and torch.equal(low, -8 * scale)
    cache = full_cache(B, m // 64, G, D, 64)
    B.ap_cache_append(cache, normal(1, m, G, D), v, torch.arange(m).cuda())
    q = torch.zeros((S, G, D), dtype=torch.float16, device="cuda")
    out = B.ap_attention_cached(cache, q, torch.arange(m // 64).int().expand(S, -1).contiguous().cuda(), torch.full((S,), m, dtype=torch.int32).cuda())
    rms = out[..., 2:].double().square().mean().sqrt().item()
    most = 512 * 31 * step.mean().item()
    bound = (2 * 4 * (2 * 2 * 16 + 8) / 12) ** 0.5 * 2.0 ** -23 * most / m
    assert rms <= bound


# ------------------------------------------------------------------------------------------------ verification


def verify_plain(target, draft, drafted, uniform, noise, counts):
    """Token by token, on the host."""
    S, N, V = draft.shape
    tokens, accepted = np.full((S, N + 1), -1, dtype=np.int64), np.zeros(S, dtype=np.int32)
    target, draft = target.astype(np.float32), draft.astype(np.float32)
    for s in range(S):
        count = min(max(int(counts[s]), 0), N)
        n = 0
        while n < count and 0 <= drafted[s, n] < V and uniform[s, n] * draft[s, n, drafted[s, n]] < target[s, n, drafted[s, n]]:
            n += 1
        def race(w):
            with np.errstate(all="ignore"):
                ratio = w / noise[s]
            ok = (w > 0) & (ratio >= 0)
            return int(np.argmax(np.where(ok, ratio, -1))) if ok.any() else -1
        won = race(target[s, n] - draft[s, n]) if n < count else -1
        if won < 0:
            won = race(target[s, n])
        tokens[s, :n], tokens[s, n], accepted[s] = drafted[s, :n], won, n
    return tokens, accepted


def verify_inputs(S, N, V, half, seed):
    rng = np.random.default_rng(seed)
    logits = rng.normal(size=(S, N + 1, V)) * 2
    def softmax(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return e / e.sum(-1, keepdims=True)
    target = softmax(logits).astype(np.float16 if half else np.float32)
    draft = softmax(logits[:, :N] + rng.normal(size=(S, N, V)) * 0.5).astype(target.dtype)
    drafted = rng.integers(0, V, size=(S, N))
    for s in range(S):
        for i in range(N):
            if rng.random() < 0.8:
                drafted[s, i] = draft[s, i].argmax()
    return target, draft, drafted, rng.random((S, N)).astype(np.float32), rng.exponential(size=(S, V)).astype(np.float32)


def check_verify(B, target, draft, drafted, uniform, noise, counts=None):
    S, N, _ = draft.shape
    d = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (target, draft, drafted, uniform, noise)]
    tokens, accepted = B.ap_verify(*d, counts=None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda())
    want = verify_plain(target, draft, drafted, uniform, noise, [N] * S if counts is None else counts)
    assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
    return want


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("S,N,V", [(1, 1, 1), (1, 4, 32000), (3, 2, 7), (5, 7, 255), (7, 3, 257), (64, 4, 1001), (2, 8, 50257), (300, 1, 33), (1, 1, 131071), (2, 3, 8191), (2, 3, 16384), (2, 3, 16385),
                                   (1030, 2, 2049)])
def test_verify(B, half, S, N, V):
    inputs = verify_inputs(S, N, V, half, seed=S * 1000 + V)
    check_verify(B, *inputs)
    counts = np.random.default_rng(V).integers(-1, N + 2, size=S)
    check_verify(B, *inputs, counts=counts)


@pytest.mark.parametrize("half", [False, True])
def test_verify_edges(B, half):
    target, draft, drafted, uniform, noise = verify_inputs(8, 3, 1003, half, seed=5)
    uniform[0] = 0.0                                            # accepts whatever the target can produce
    drafted[1, 0], drafted[2, 1] = -1, 1003                     # tokens outside the vocabulary
    draft[3] = target[3, :3]
    uniform[3] = 0.999                                          # equal probabilities: all are accepted
    draft[4, 0] = target[4, 0]
    uniform[4, 0] = 1.0                                         # refused where no token has more than its draft: from the target itself
    target[5] = 0
    target[5, :, 77] = 1                                        # one token only, refused until it comes
    noise[6, 10:20] = 0.0                                       # infinite ratios: the lowest of equals
    noise[6, 20] = float("nan")
    target[7], draft[7] = 0, 0                                  # nothing to choose from
    want = check_verify(B, target, draft, drafted, uniform, noise)
    assert want[0][7, 0] == -1 and (want[0][5][want[1][5]] == 77)
    target[:] = np.float32(1 / 1003)
    noise[:] = 1.0                                              # all equal: the lowest index
    draft[:] = 0
    want = check_verify(B, target, draft, drafted, uniform, noise)
    assert want[0][0, want[1][0]] == 0
    check_verify(B, target, draft, drafted, uniform, noise, counts=[0] * 8)
    check_verify(B, target[:, :1], draft[:, :0], drafted[:, :0], uniform[:, :0], noise)      # no drafts: a plain sample


def test_verify_tokens_follow_the_target(B):
    # a small vocabulary many times over: the first token's frequencies are the target's
    S, V = 20000, 5
    rng = np.random.default_rng(3)
    p, q = np.array([0.5, 0.2, 0.2, 0.1, 0.0], np.float32), np.array([0.1, 0.4, 0.2, 0.1, 0.2], np.float32)
    drafted = rng.choice(V, size=(S, 1), p=q / q.sum())
    d = [np.broadcast_to(p, (S, 2, V)), np.broadcast_to(q, (S, 1, V)), drafted, rng.random((S, 1)).astype(np.float32),
         rng.exponential(size=(S, V)).astype(np.float32)]
    tokens, _ = B.ap_verify(*[torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in d])
    share = np.bincount(tokens[:, 0].cpu().numpy(), minlength=V) / S
    assert np.abs(share - p).max() < 5 * 0.5 / S ** 0.5         # five standard deviations of a share


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_verify_where_no_noise_of_the_rest_counts(B, half, V):
    # refused drafts, and tokens with more than their draft: the token after them is one of these, or none where none of their noise is a number from 0 on
    target, draft, drafted, uniform, noise = verify_inputs(6, 2, V, half, seed=V)
    drafted[:, 0] = 3
    draft[:, 0], target[:, 0] = 2.0 / V, 1.0 / V                # more in the draft, but for two tokens
    target[:, 0, 3] = 0                                         # refused
    for at in (7, V - 2):
        target[:, 0, at] = 4.0 / V
    noise[0, [7, V - 2]] = np.nan
    noise[1, [7, V - 2]] = -1.0
    noise[2, [7, V - 2]] = np.nan, 5.0
    noise[3, [7, V - 2]] = 0.5, -np.inf
    noise[4, [7, V - 2]] = np.inf, -1.0                         # a ratio of 0 counts
    d = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (target, draft, drafted, uniform, noise)]
    tokens, accepted = B.ap_verify(*d)
    assert not accepted.any() and (tokens[:, 1:] == -1).all()
    assert tokens[:5, 0].tolist() == [-1, -1, V - 2, 7, 7] and tokens[5, 0].item() == (7 if noise[5, 7] <= noise[5, V - 2] else V - 2)


# ------------------------------------------------------------------------------------------------ all of them


def test_calls_in_a_graph(B):
    G, D, page, H = 2, 128, 16, 8
    table, pages = U.page_table([400, 300], page)
    cache = full_cache(B, pages, G, D, page)
    k, v = normal(1, 700, G, D), normal(2, 700, G, D)
    old = torch.cat([U.slots_of(table, page, 0, 0, 400), U.slots_of(table, page, 1, 0, 300)]).cuda()
    new = torch.cat([U.slots_of(table, page, 0, 399, 400), U.slots_of(table, page, 1, 299, 300)]).cuda()
    rotary, positions = B.rotary_table(512, D), torch.tensor([399, 299]).cuda()
    x = normal(3, 2, H + 2 * G, D)
    lens, tables, starts = torch.tensor([400, 300], dtype=torch.int32).cuda(), table.cuda(), torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    p = [torch.from_numpy(a).cuda() for a in verify_inputs(2, 3, 5000, False, 1)]

    def step():
        q, kk = B.ap_cache_append(cache, x[:, H:H + G], x[:, H + G:], new, q=x[:, :H], positions=positions, rotary=rotary)
        return (q, kk, B.ap_attention_cached(cache, q, tables, lens), B.ap_attention_prompt(q, kk, x[:, H + G:], starts)) + B.ap_verify(*p)

    B.ap_cache_append(cache, k, v, old)
    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (7, 8, 9):
        x.copy_(normal(seed, 2, H + 2 * G, D))
        p[3].copy_(torch.rand_like(p[3]))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        cache.buf.fill_(255)
        B.ap_cache_append(cache, k, v, old)
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ sequences that begin in an earlier one


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("width", [3, 40])                       # one launch, and ranges that are joined
@pytest.mark.parametrize("seed", range(8))
def test_cached_tokens_have_one_sequence(B, width, seed):
    S, T, H, G, D, page = (70, 6)[seed % 2], 90, 8, 2, 64, 16
    cache = full_cache(B, 64, G, D, page)
    B.ap_cache_append(cache, normal(1, 1024, G, D), normal(2, 1024, G, D), torch.arange(1024).cuda())
    g = torch.Generator().manual_seed(seed)
    tables = torch.randint(0, 64, (S, width), generator=g).int().cuda()
    lengths = torch.randint(0, width * page + 1, (S,), generator=g).int().cuda()
    q, starts = normal(3, T, H, D), U.senseless_starts(seed, S, T)
    work = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")      # sums that nobody has written are NaN
    out = B.ap_attention_cached(cache, q, tables, lengths, q_starts=int32(starts), out=torch.full_like(q, 7.0), work=work)
    live = U.live_sequences(starts, T)
    rows = [i for _, a, b in live for i in range(a, b)]
    rest = [i for i in range(T) if i not in rows]
    assert (out[rest] == 7).all()
    if live:
        of = [s for s, _, _ in live]
        want = B.ap_attention_cached(cache, q[rows].contiguous(), tables[of].contiguous(), lengths[of].contiguous(), q_starts=U.starts([b - a for _, a, b in live]).cuda())
        assert torch.isfinite(out).all() and (out[rows].float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()


@pytest.mark.parametrize("starts,same", [([0, 40, 0, 60], [0, 40, 40, 40]), ([0, 40, 10, 60], [0, 40, 40, 40]), ([70, 5, 40, 60], [5, 5, 40, 60])])
def test_cached_sequences_in_an_earlier_one_have_no_tokens(B, starts, same):
    cache = full_cache(B, 64, 2, 128, 16)
    B.ap_cache_append(cache, normal(1, 1024, 2, 128), normal(2, 1024, 2, 128), torch.arange(1024).cuda())
    q, tables = normal(3, 60, 4, 128), torch.arange(64, dtype=torch.int32).cuda().expand(3, -1).contiguous()
    for lengths in ([64, 64, 64], [1000, 900, 800]):
        call = lambda st: B.ap_attention_cached(cache, q, tables, int32(lengths), q_starts=int32(st), max_length=max(lengths), out=torch.full_like(q, 7.0),  # noqa: E731
                                                work=torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda"))
        assert torch.equal(call(starts), call(same))


@pytest.mark.parametrize("keys", [60, 4000])
@pytest.mark.parametrize("seed", range(8))
def test_prompt_tokens_have_one_sequence(B, keys, seed):
    S, T, H, G, D = (70, 6)[seed % 2], 90, 4, 2, 64
    q, k, v = normal(3, T, H, D), normal(1, keys, G, D), normal(2, keys, G, D)
    starts = U.senseless_starts(seed, S, T)
    cuts = sorted(torch.randint(0, keys + 1, (S + 1,), generator=torch.Generator().manual_seed(seed)).tolist())
    work = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    out = B.ap_attention_prompt(q, k, v, int32(starts), int32(cuts), out=torch.full_like(q, 7.0), work=work)
    live = U.live_sequences(starts, T)
    rows = [i for _, a, b in live for i in range(a, b)]
    rest = [i for i in range(T) if i not in rows]
    assert (out[rest] == 7).all()
    for s, a, b in live:
        mine = slice(cuts[s], cuts[s + 1])
        want = B.ap_attention_prompt(q[a:b].contiguous(), k[mine].contiguous(), v[mine].contiguous(), int32([0, b - a]), int32([0, cuts[s + 1] - cuts[s]]))
        assert (out[a:b].float() - want.float()).abs().max() <= 2.0 ** -9 * max(float(want.abs().max()), 2.0 ** -9), s
