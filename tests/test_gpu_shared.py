"""GPU tests of attention behind shared prefixes against a plain 64-bit form."""
import pytest
import torch

import decode_util as U
import step_util as S

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


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(B, prefixes, lengths, G, D, page, seed, spoil=None, base=0):
    """A cache with prefixes' and sequences' keys and values: (cache, prefix tables, tables, values of each)."""
    table, pages = U.page_table(list(prefixes) + list(lengths), page, seed=seed)
    table = torch.where(table >= 0, table + base, table)
    cache = B.KVCache(pages + base, G, D, page_tokens=page)
    cache.buf[base * (cache.buf.numel() // (pages + base)):].fill_(255)
    k = [normal(seed + 10 * i + 1, n, G, D, outlier=True) for i, n in enumerate(list(prefixes) + list(lengths))]
    v = [normal(seed + 10 * i + 2, n, G, D) for i, n in enumerate(list(prefixes) + list(lengths))]
    if spoil:
        spoil(k, v)
    slots = torch.cat([U.slots_of(table, page, i, 0, len(x)) for i, x in enumerate(k)]).cuda()
    B.ap_cache_append(cache, torch.cat(k), torch.cat(v), slots)
    table = table.cuda()
    return cache, table[:len(prefixes)].contiguous(), table[len(prefixes):].contiguous(), k, v


def shared_case(B, prefixes, sizes, lengths, queries, H, G, D, page, seed=0, scale=None, spoil=None, view=False, base=0, starts=True, bounds=True, **kw):
    """One call, every row checked.  sizes: sequences of each prefix; sequences behind the last have none.  Returns (out, worst share of the bound)."""
    cache, prefix_table, table, k, v = filled(B, prefixes, lengths, G, D, page, seed, spoil, base)
    T, P = sum(queries), len(prefixes)
    q = normal(seed + 3, T, H + 2, D)[:, 1:H + 1] if view else normal(seed + 3, T, H, D)
    st = U.starts(queries)
    args = dict(prefix_starts=int32([0] + list(torch.tensor(sizes).cumsum(0))) if starts else None, q_starts=st.cuda() if starts else None, scale=scale, **kw)
    if bounds:
        args = dict(dict(max_prefix=max(prefixes), max_length=max(lengths)), **args)
    call = lambda: B.ap_attention_shared(cache, q, prefix_table, int32(prefixes), table, int32(lengths), **args)  # noqa: E731
    out = call()
    assert torch.equal(out.view(torch.int16), call().view(torch.int16))
    scale = D ** -0.5 if scale is None else scale
    worst, owner = 0.0, [p for p, n in enumerate(sizes) for _ in range(n)]
    for i, (n, m) in enumerate(zip(queries, lengths)):
        parts = ([owner[i]] if i < len(owner) else []) + [P + i]
        kk, vv = torch.cat([k[j] for j in parts]), torch.cat([v[j] for j in parts])
        before = len(kk) - m
        # a token of a sequence with fewer keys of its own than queries sees the prefix, and none of the sequence's keys
        sees = before + (m - n + 1 + torch.arange(n)).clamp(min=0)
        (_, kl, ks), (_, vl, vs) = U.codes_of(kk), U.codes_of(vv)
        want, bound = S.shared_attention(q[int(st[i]):int(st[i]) + n].double(), U.cache_values(kk), U.cache_values(vv), scale, sees,
                                         (kl.abs() + 143 * ks).double().expand(-1, -1, D), (vl.abs() + vs * 15).double().expand(-1, -1, D))
        worst = max(worst, U.check(out[int(st[i]):int(st[i]) + n], want, bound, "sequence %d: %d + %d keys" % (i, before, m)))
    return out, worst


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (8, 1), (14, 2), (20, 1), (33, 1), (32, 32)])
def test_head_layouts(B, H, G, D):
    shared_case(B, [130, 17], [5, 3], [1, 2, 15, 16, 17, 33, 130, 300], [1] * 8, H, G, D, 16, seed=H)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_pages_and_lengths(B, page, D):
    shared_case(B, [page - 1, page, page + 1, 1, 515], [3, 1, 2, 1, 3], [page, 1, 511, 3, 513, 1023, 1, page + 1, 2, 700], [1, 2, 1, 3, 1, 1, 0, 4, 1, 1], 8, 2, D, page,
                seed=page)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 127, 128, 129, 200, 255, 256, 257, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_a_prefix(B, rows, D):
    # rows of one key head, from one token to several tiles
    shared_case(B, [777], [rows], [1 + i % 5 for i in range(rows)], [1] * rows, 2, 2, D, 64, seed=rows)


@pytest.mark.parametrize("prefix", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 4095, 4097, 9001])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths_of_a_prefix(B, prefix, D):
    shared_case(B, [prefix], [7], [3, 1, 8, 60, 2, 1, 129], [1, 1, 5, 2, 1, 1, 3], 24, 3, D, 16, seed=prefix)          # 112 rows of a key head
    shared_case(B, [prefix], [2], [3, 1], [2, 1], 4, 4, D, 16, seed=prefix)                                             # 3 rows


@pytest.mark.parametrize("queries", [2, 5, 17, 40])
def test_many_queries(B, queries):
    # some sequences have fewer keys of their own than queries: the first ones see the prefix alone
    shared_case(B, [900, 33], [4, 3], [3, 100, 1, 700, queries, 1, 1500], [queries] * 7, 16, 4, 128, 64, seed=queries, view=True)
    shared_case(B, [900, 33], [4, 2], [3, 100, 1, 7, queries, 1], [queries, 1, 2, 0, queries, 3], 6, 2, 64, 16, seed=queries)


def test_equal_numbers_without_starts(B):
    shared_case(B, [100, 3, 260], [2, 2, 2], [5, 9, 70, 1, 2, 300], [2] * 6, 8, 2, 128, 32, starts=False)
    shared_case(B, [100], [4], [5, 9, 70, 1], [1] * 4, 8, 8, 64, 32, starts=False, bounds=False)


def test_sequences_without_a_prefix(B):
    shared_case(B, [100], [2], [5, 9, 70, 1], [1, 1, 2, 1], 8, 2, 128, 32)                     # behind the last
    cache, prefix_table, table, k, v = filled(B, [50], [5, 40, 9], 2, 128, 16, 5)
    q = normal(1, 3, 8, 128)
    out = B.ap_attention_shared(cache, q, prefix_table, int32([50]), table, int32([5, 40, 9]), prefix_starts=int32([1, 2]))
    own = B.ap_attention_cached(cache, q, table, int32([5, 40, 9]))
    for i in (0, 2):                                                                           # before the first and behind the last
        assert (out[i].float() - own[i].float()).abs().max() <= 2.0 ** -9 * own[i].abs().max()
    assert (out[1].float() - own[1].float()).abs().max() > 0.05
    # no prefix at all, and one without keys
    none = torch.empty((0, 1), dtype=torch.int32, device="cuda")
    for tables, lengths in ((none, int32([])), (prefix_table, int32([0])), (prefix_table, int32([-4])), (torch.full_like(prefix_table, -1), int32([50]))):
        out = B.ap_attention_shared(cache, q, tables, lengths, table, int32([5, 40, 9]))
        assert (out.float() - own.float()).abs().max() <= 2.0 ** -9 * own.abs().max()


def test_no_keys_of_their_own(B):
    cache, prefix_table, table, k, v = filled(B, [300], [1, 1, 1], 2, 64, 16, 5)
    q = normal(1, 3, 8, 64)
    for tables, most in ((table, None), (table, 0), (torch.empty((3, 0), dtype=torch.int32, device="cuda"), None)):
        out = B.ap_attention_shared(cache, q, prefix_table, int32([300]), tables, int32([0, 0, -1]), max_length=most)
        want = B.ap_attention_cached(cache, q, prefix_table.expand(3, -1).contiguous(), int32([300] * 3))
        assert (out.float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()
    out = B.ap_attention_shared(cache, q, prefix_table, int32([0]), table, int32([0] * 3), out=torch.full_like(q, 9))
    assert not out.any()


def test_many_prefixes(B):
    P = 70                                                       # more than a wave looks at at once
    sizes = [i % 3 for i in range(P)]
    n = sum(sizes)
    shared_case(B, [1 + (i * 37) % 90 for i in range(P)], sizes, [1 + (i * 13) % 40 for i in range(n)], [i % 3 for i in range(n)], 4, 2, 64, 16)


def test_many_prefixes_of_many_rows(B):
    sizes = [i % 5 for i in range(70)]
    n = sum(sizes)
    shared_case(B, [(i * 37) % 290 for i in range(70)], sizes, [1 + (i * 13) % 40 for i in range(n)], [1 + i % 2 for i in range(n)], 40, 1, 64, 16)
    shared_case(B, [2000 + i for i in range(17)], [3] * 17, [1 + (i * 13) % 40 for i in range(51)], [1] * 51, 66, 3, 64, 32)


def test_large_batches(B):
    shared_case(B, [1500, 2600], [70, 61], [1 + (i * 31) % 200 for i in range(131)], [1] * 131, 16, 2, 128, 64)
    shared_case(B, [1500, 2600], [70, 61], [1 + (i * 31) % 200 for i in range(131)], [1 + i % 3 for i in range(131)], 8, 2, 64, 32)


def test_joins_of_many_rows(B):
    # rows from which on a wave joins each, with few and with many ranges, some of them empty, and tokens of no sequence
    shared_case(B, [5000], [33], [1 + (i * 97) % 900 for i in range(33)], [1] * 33, 32, 4, 128, 64)
    shared_case(B, [20000, 0, 700], [3, 2, 6], [5 + (i * 517) % 3000 for i in range(13)], [1 + i % 5 for i in range(13)], 40, 40, 64, 16)
    cache, prefix_table, table, k, v = filled(B, [300], [9] * 40, 2, 64, 16, 5)
    q, out = normal(1, 80, 16, 64), torch.full((80, 16, 64), 7.0, dtype=torch.float16, device="cuda")
    starts = int32([3 + i for i in range(41)])
    B.ap_attention_shared(cache, q, prefix_table, int32([300]), table, int32([9] * 40), q_starts=starts, out=out)
    want = B.ap_attention_shared(cache, q[3:43].contiguous(), prefix_table, int32([300]), table, int32([9] * 40))
    assert (out[:3] == 7).all() and (out[43:] == 7).all() and (out[3:43].float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()


def test_long_prefixes(B):
    shared_case(B, [70001], [20], [3] * 20, [1] * 20, 8, 1, 128, 64)
    shared_case(B, [33000, 5], [1, 1], [3, 700], [1, 1], 8, 2, 64, 16)


@pytest.mark.parametrize("sequences", [2, 40])
def test_scales_and_bounds(B, sequences):
    for scale in (0.0, -0.3, 1.0, 1e-6):
        shared_case(B, [100], [sequences], [40] * sequences, [1] * sequences, 4, 2, 128, 32, scale=scale)
    cache, prefix_table, table, k, v = filled(B, [300], [50] * sequences, 2, 128, 32, 7)
    q, own = normal(1, sequences, 8, 128), int32([50] * sequences)
    cut = B.ap_attention_shared(cache, q, prefix_table, int32([300]), table, own, max_prefix=70)           # longer ones are cut at max_prefix
    want = B.ap_attention_shared(cache, q, prefix_table, int32([70]), table, own, max_prefix=70)
    assert torch.equal(cut, want)


@pytest.mark.parametrize("sequences", [2, 40])
@pytest.mark.parametrize("size,scale", [(30.0, None), (300.0, None), (20000.0, None), (20000.0, -1.0), (1.0, 3e4), (1.0, 1e30), (300.0, -3e38)])
def test_the_greatest_score_of_any_size_takes_all(B, sequences, size, scale):
    # keys of one value each: the scores are exact, and far apart
    G, D, page, m = 1, 128, 16, 200
    cache = B.KVCache(40, G, D, page_tokens=page)
    cache.buf.fill_(255)
    order = torch.randperm(m, generator=torch.Generator().manual_seed(3)).cuda()
    k = ((order.float() + 1) * (size / 256)).half()[:, None, None].expand(m, G, D).contiguous()
    v = normal(1, m, G, D)
    B.ap_cache_append(cache, k, v, torch.arange(m).cuda())
    q = torch.full((sequences, 4, D), 0.5, dtype=torch.float16, device="cuda")
    table = torch.arange(13, dtype=torch.int32).cuda()
    out = B.ap_attention_shared(cache, q, table[None, :9].contiguous(), int32([144]), table[9:].expand(sequences, -1).contiguous(), int32([56] * sequences), scale=scale)
    s = q[0].double() @ k[:, 0].double().t() * (D ** -0.5 if scale is None else max(min(scale, 1e30), -1e30))
    p = torch.softmax(s, dim=1)
    want = p @ U.cache_values(v)[:, 0]
    assert torch.isfinite(out).all()
    # scores of 16 EPS32 of their size, and the roundings of weights, values and result
    rel = torch.minimum(2 * 20 * U.EPS32 * s.abs().amax(1, keepdim=True), torch.ones(4, 1, dtype=torch.float64, device="cuda"))
    gap = (s.amax(1) - s.topk(2, dim=1).values[:, 1])
    rel = torch.where((gap > 80)[:, None], torch.zeros_like(rel), rel)
    bound = (3 * U.HALF_EPS16 + 64 * U.EPS32 + rel) * (p @ U.cache_values(v)[:, 0].abs()) + 2.0 ** -20
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("sequences", [3, 50])
def test_nan_and_infinities_reach_who_sees_them(B, sequences):
    def own(k, v):
        v[1][4, 0, 3] = float("inf")              # the first sequence's last key
        k[2][0, 1, 0] = float("nan")              # the second's first
    out, _ = shared_case(B, [96], [sequences], [5] * sequences, [2] * sequences, 4, 2, 128, 32, spoil=own)
    bad = torch.isnan(out).all(-1)
    assert bad[:, :2].any(1).tolist() == [False, True] + [False] * (2 * sequences - 2)
    assert bad[:, 2:].any(1).tolist() == [False, False, True, True] + [False] * (2 * sequences - 4)

    def prefix(k, v):
        v[0][90, 0, 3] = float("inf")
    out, _ = shared_case(B, [96, 50], [sequences, 2], [5] * (sequences + 2), [1] * (sequences + 2), 4, 2, 128, 32, spoil=prefix)
    bad = torch.isnan(out).all(-1)
    assert bad[:sequences, :2].all() and not bad[:, 2:].any() and not bad[sequences:].any()


@pytest.mark.parametrize("sequences", [2, 60])
def test_values_at_the_end_of_the_range(B, sequences):
    def spoil(k, v):
        v[0][::3] *= 2.0 ** -14                     # rows of subnormal steps
        v[0][1, :, :2] = torch.tensor([65504.0, -65504.0])
        v[0][2] = 65504.0
        v[0][4, :, 5] = 60000.0
    shared_case(B, [40], [sequences], [2] * sequences, [1] * sequences, 4, 2, 64, 16, spoil=spoil)
    def small(k, v):
        v[0] *= 2.0 ** -14
    shared_case(B, [400], [sequences], [2] * sequences, [1] * sequences, 4, 2, 128, 16, spoil=small)


@pytest.mark.parametrize("sequences", [1, 30, 70])
def test_pages_outside_the_cache_hold_nothing(B, sequences):
    G, D, page = 2, 128, 16
    cache = B.KVCache(4, G, D, page_tokens=page)
    cache.buf.fill_(255)
    B.ap_cache_append(cache, normal(1, 48, G, D), normal(2, 48, G, D), torch.arange(48).cuda())
    q = normal(3, sequences, 4, D)
    tables, own = int32([[2]] * sequences), int32([16] * sequences)
    out = B.ap_attention_shared(cache, q, int32([[0, -1, 1, 4, 2 ** 31 - 1]]), int32([80]), tables, own)
    want = B.ap_attention_shared(cache, q, int32([[0, 1]]), int32([32]), tables, own)
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -9 * want.float().abs().max()


def test_starts_that_make_no_sense(B):
    cache, prefix_table, table, k, v = filled(B, [100, 60], [20] * 6, 2, 64, 16, 5)
    q, own = normal(1, 6, 8, 64), int32([20] * 6)
    call = lambda prefix_starts, **kw: B.ap_attention_shared(cache, q, prefix_table, int32([100, 60]), table, own, prefix_starts=int32(prefix_starts), **kw)  # noqa: E731
    alone = B.ap_attention_cached(cache, q, table, own)
    close = lambda a, b: (a.float() - b.float()).abs().max() <= 2.0 ** -9 * b.abs().max()  # noqa: E731
    for starts in ([0, -1, 2 ** 31 - 1], [7, 7, 9], [-5, -3, -1], [3, 3, 3]):
        assert close(call(starts), alone), starts
    good = call([0, 3, 6])
    bad = call([0, 3, 7])                                       # the second prefix leaves the sequences: they have none
    assert close(bad[:3], good[:3]) and close(bad[3:], alone[3:])
    # tokens of no sequence stay as they were; a prefix whose sequences' tokens descend or leave the tokens is not seen
    out = torch.full_like(q, 7.0)
    call([0, 3, 6], q_starts=int32([0, 1, 2, 3, 3, 4, 4]), out=out)
    assert close(out[:3], good[:3]) and (out[4:] == 7).all()
    out = torch.full_like(q, 7.0)
    call([0, 3, 6], q_starts=int32([0, 1, 2, 3, 4, 5, 70]), out=out)
    assert close(out[:3], good[:3]) and close(out[3:5], alone[3:5]) and (out[5:] == 7).all()
    call([0, 3, 6], q_starts=int32([-9, 5, 2, 2 ** 31 - 1, -2 ** 31, 6, 6]), out=out)


def test_starts_that_make_no_sense_with_many_rows(B):
    n = 40
    cache, prefix_table, table, k, v = filled(B, [300, 700, 90], [20] * n, 2, 64, 16, 5)
    q, own = normal(1, n, 16, 64), int32([20] * n)
    call = lambda starts, **kw: B.ap_attention_shared(cache, q, prefix_table, int32([300, 700, 90]), table, own, prefix_starts=int32(starts), **kw)  # noqa: E731
    alone = B.ap_attention_cached(cache, q, table, own)
    close = lambda a, b: (a.float() - b.float()).abs().max() <= 2.0 ** -9 * b.abs().max()  # noqa: E731
    for starts in ([0, -1, 2 ** 31 - 1, 0], [70, 70, 90, 90], [-5, -3, -1, -1], [3, 3, 3, 3]):
        assert close(call(starts), alone), starts
    good = call([0, 10, 30, 40])
    assert not close(good, alone)
    assert close(call([0, 10, 30, 41])[:30], good[:30])
    assert torch.isfinite(call([0, 40, 0, 40])).all()           # prefixes that overlap
    out = torch.full_like(q, 7.0)
    call([0, 10, 30, 40], q_starts=int32(list(range(n)) + [70]), out=out)
    assert close(out[:30], good[:30]) and close(out[30:-1], alone[30:-1]) and (out[-1] == 7).all()
    # more of overlapping prefixes than there are workgroups for
    many = 300
    tables, lengths = prefix_table[:1].expand(many, -1).contiguous(), int32([300] * many)
    q, own, table = normal(2, many * 3, 44, 64), int32([20] * many * 3), table[:1].expand(many * 3, -1).contiguous()
    starts = [0] + [many * 3 if i % 2 else 0 for i in range(1, many)] + [many * 3]
    out = B.ap_attention_shared(cache, q, tables, lengths, table, own, prefix_starts=int32(starts))
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("D", [64, 128])
def test_many_row_tiles_and_prefixes(B, D):
    # more tiles than workgroups, and prefixes of every share of them: none, one range, several
    shared_case(B, [0, 64, 2000, 1, 129, 3000], [3, 30, 4, 90, 1, 60], [1 + i % 7 for i in range(188)], [1 + i % 3 for i in range(188)], 24, 2, D, 16)
    shared_case(B, [70] * 20, [9] * 20, [1 + i % 7 for i in range(180)], [1] * 180, 32, 4, D, 32)


def test_offsets_beyond_32_bits(B):
    shared_case(B, [500], [40], [9] * 40, [1] * 40, 32, 16, 128, 64, base=35000)


def test_a_prefix_is_read_as_the_own_keys_of_each(B):
    # the same keys as one sequence each, through the cached attention
    P, n, G, D, page = 256, 48, 2, 128, 64
    cache, prefix_table, table, k, v = filled(B, [P], [64] * n, G, D, page, 11)
    q = normal(1, n, 8, D)
    out = B.ap_attention_shared(cache, q, prefix_table, int32([P]), table, int32([64] * n))
    joined = torch.cat([prefix_table[:, :P // page].expand(n, -1), table[:, :1]], dim=1).contiguous()
    want = B.ap_attention_cached(cache, q, joined, int32([P + 64] * n))
    # both are within their bounds of the exact result: some roundings of binary16 apart
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()


def test_named_streams_and_workspaces(B):
    cache, prefix_table, table, k, v = filled(B, [600], [30] * 33, 2, 128, 64, 3)
    q, own = normal(3, 33, 8, 128), int32([30] * 33)
    args = (prefix_table, int32([600]), table, own)
    want = B.ap_attention_shared(cache, q, *args)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for i in range(6):                                          # two calls at once
        outs.append(B.ap_attention_shared(cache, q, *args, stream=(side, other)[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    assert B.ap_attention_shared(cache, q, *args, work=work, out=out) is not None and torch.equal(out, want)
    with pytest.raises(B.ApError):
        B.ap_attention_shared(cache, q, *args, work=work[:64])


def test_tensors_that_do_not_fit_are_refused(B):
    cache, prefix_table, table, k, v = filled(B, [60], [20] * 4, 2, 64, 16, 5)
    q, own, lens = normal(1, 4, 8, 64), int32([20] * 4), int32([60])
    call = lambda **kw: B.ap_attention_shared(cache, **dict(dict(q=q, prefix_tables=prefix_table, prefix_lengths=lens, tables=table, lengths=own), **kw))  # noqa: E731
    call()
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(prefix_tables=prefix_table.long()), dict(prefix_tables=prefix_table[0]), dict(prefix_lengths=own),
                dict(prefix_lengths=lens.cpu()), dict(tables=table[:, ::2]), dict(lengths=own[:3]), dict(prefix_starts=int32([0, 1, 2])),
                dict(q_starts=int32([0, 4])), dict(out=q.float()), dict(out=q[:2])):
        with pytest.raises(AssertionError):
            call(**bad)
    two = prefix_table.expand(2, -1).contiguous()
    for bad in (dict(max_prefix=10 ** 6), dict(max_prefix=-1), dict(max_length=10 ** 6), dict(scale=float("nan")), dict(q=normal(1, 4, 7, 64)), dict(q=normal(1, 5, 8, 64)),
                dict(prefix_tables=torch.cat([two, two, two]), prefix_lengths=int32([1] * 6)),
                dict(prefix_tables=torch.cat([two, prefix_table]), prefix_lengths=int32([1] * 3))):
        with pytest.raises(B.ApError):
            call(**bad)
    with pytest.raises(TypeError):
        call(prefix_tables=None)
    assert call(q=q[:0], tables=table[:0], lengths=own[:0], prefix_tables=prefix_table[:0], prefix_lengths=lens[:0]).shape == (0, 8, 64)


@pytest.mark.parametrize("heads,group", [(8, 4), (32, 16)])       # prefixes of few rows on average, and of many
def test_overlapping_prefixes_go_to_the_first(B, heads, group):
    # a prefix that begins before the end of an earlier one has no sequences: the same bits as with starts that say so
    n = 20
    cache, prefix_table, table, k, v = filled(B, [300, 700, 90, 400], [20 + i for i in range(n)], heads // group, 64, 16, 5)
    q, own, lengths = normal(1, n, heads, 64), int32([20 + i for i in range(n)]), int32([300, 700, 90, 400])
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def call(starts, lengths=lengths, **kw):
        work.fill_(255)                                          # sums that nobody has written are NaN
        return B.ap_attention_shared(cache, q, prefix_table, lengths, table, own, prefix_starts=int32(starts), work=work, out=torch.full_like(q, 7.0), **kw)
    for starts, same in (([0, 8, 0, 12, 12], [0, 8, 8, 8, 8]), ([0, n, 0, n, n], [0, n, n, n, n]), ([0, n, 0, n, 0], [0, n, n, n, n]),
                         ([3, 8, 2, 8, n], [3, 8, 8, 8, n]), ([99, 0, 5, 5, 9], [0, 0, 5, 5, 9])):
        want = call(same)
        assert torch.equal(call(starts), want) and torch.isfinite(want).all(), starts
        assert torch.equal(call(starts, q_starts=int32(list(range(n + 1)))), call(same, q_starts=int32(list(range(n + 1))))), starts
    # the third, 7 .. 15, begins in the first, 4 .. 9; the fourth begins at its end
    got, want = call([4, 9, 7, 15, n]), call([4, 9, 9, 15, n], lengths=int32([300, 700, 0, 400]))
    assert (got.float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()


@pytest.mark.parametrize("heads", [2, 66])
def test_many_overlapping_prefixes(B, heads):
    # more than a wave looks at at once, of which every other one overlaps all before it: row tiles of the live ones only
    n, P = 90, 150
    prefix = [40 + (i * 37) % 300 for i in range(P)]
    cache, prefix_table, table, k, v = filled(B, prefix, [5 + i % 30 for i in range(n)], 1, 64, 16, 5)
    q, own = normal(1, n, heads, 64), int32([5 + i % 30 for i in range(n)])
    work = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")

    def call(starts):
        work.fill_(255)
        return B.ap_attention_shared(cache, q, prefix_table, int32(prefix), table, own, prefix_starts=int32(starts), work=work)
    owners = [min(i * n // 60, n) for i in range(61)]
    starts = owners[:60] + [n if i % 2 else 0 for i in range(60, P + 1)]
    same = owners[:60] + [owners[59]] * (P + 1 - 60)             # from there on starts descend, or begin at 0
    got, want = call(starts), call(same)
    assert torch.equal(got, want) and torch.isfinite(got).all()


@pytest.mark.parametrize("heads", [8, 40])                       # prefixes of few rows on average, and of many
@pytest.mark.parametrize("seed", range(8))
def test_tokens_have_one_sequence(B, heads, seed):
    # sequences and prefixes whose starts make no sense: each token's result is that of its sequence and prefix by themselves
    S, T, P = (70, 9)[seed % 2], 90, 7
    cache, prefix_table, table, k, v = filled(B, [300, 20, 700, 90, 400, 1, 33], [1 + (i * 37) % 200 for i in range(S)], 1, 64, 16, 5)
    lengths, own = int32([300, 20, 700, 90, 400, 1, 33]), int32([1 + (i * 37) % 200 for i in range(S)])
    q, starts, prefix_starts = normal(1, T, heads, 64), U.senseless_starts(seed, S, T), U.senseless_starts(seed + 50, P, S)
    work = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    out = B.ap_attention_shared(cache, q, prefix_table, lengths, table, own, prefix_starts=int32(prefix_starts), q_starts=int32(starts), work=work, out=torch.full_like(q, 7.0))
    live, upto, prefixes = U.live_sequences(starts, T), 0, []
    for p, (a, b) in enumerate(zip(prefix_starts, prefix_starts[1:])):
        if 0 <= a < b <= S and 0 <= starts[a] < starts[b] <= T:
            if starts[a] >= upto:
                prefixes.append((p, a, b, starts[a], starts[b]))
            upto = max(upto, starts[b])
    rows = [i for _, a, b in live for i in range(a, b)]
    assert (out[[i for i in range(T) if i not in rows]] == 7).all()
    for s, a, b in live:
        for i in range(a, b):
            of = [p for p, s0, s1, t0, t1 in prefixes if s0 <= s < s1 and t0 <= i < t1]
            sees = int(own[s]) - (b - 1 - i)
            want = B.ap_attention_shared(cache, q[i:i + 1].contiguous(), prefix_table[of].contiguous(), lengths[of].contiguous(), table[s:s + 1].contiguous(), int32([sees]))
            assert (out[i].float() - want[0].float()).abs().max() <= 2.0 ** -9 * max(float(want.abs().max()), 2.0 ** -9), (i, s, of)
