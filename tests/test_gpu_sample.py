"""GPU tests of sampling against a plain 64-bit form, row by row."""
import pytest
import torch

import step_util as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2402_10517_amd import binding
    return binding


def cuda(x, dtype=torch.float32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def logits_of(seed, rows, V, half, masked=False, size=2.2):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, V), generator=g, device="cuda") * size
    if masked:
        x[torch.rand((rows, V), generator=g, device="cuda") < 0.3] = float("-inf")
    return x.half() if half else x


def uniform_of(seed, rows):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed)).cuda()


def check(B, logits, uniform, kept=torch.float32, **settings):
    """One call against the definition; and the same without probabilities, and again."""
    tokens, p = B.ap_sample(logits, uniform, probabilities=kept, **settings)
    assert torch.equal(tokens, B.ap_sample(logits, uniform, **settings)[0])
    again = B.ap_sample(logits, uniform, probabilities=kept, **settings)
    assert torch.equal(tokens, again[0]) and torch.equal(p, again[1])
    want_tokens, want = S.sample(logits, uniform, **settings)
    # a weight in 64 bits over a sum whose parts are off by 2^-42 of the greatest, rounded once
    got = p.double().cpu()
    assert torch.equal(got > 0, want.to(kept) > 0), "others are kept: %d instead of %d" % (int((got > 0).sum()), int((want > 0).sum()))
    eps, least = (S.HALF_EPS16, S.SUBNORMAL16) if kept == torch.float16 else (2.0 ** -24, 2.0 ** -150)
    assert ((got - want).abs() <= (eps + logits.shape[1] * 2.0 ** -42) * want + least).all()
    assert torch.equal(tokens.cpu(), want_tokens), (tokens.cpu() != want_tokens).nonzero().flatten().tolist()
    return tokens, p


SIZES = [1, 2, 7, 8, 9, 63, 511, 512, 513, 1000, 4097, 8191, 8192, 8193, 16384, 16385, 32000, 32003, 65537]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", SIZES)
def test_sizes(B, V, half):
    rows = 6
    logits, u = logits_of(V, rows, V, half), uniform_of(V, rows)
    t = cuda([0.7, 1.0, 1.3, 0.0, 0.9, 2.0])
    check(B, logits, u, temperature=t)
    check(B, logits, u, temperature=t, top_k=cuda([1, 5, 50, 50, 300, V], torch.int32), kept=torch.float16)
    check(B, logits, u, temperature=t, top_p=cuda([0.3, 0.9, 0.95, 0.5, 0.999, 0.7]))
    check(B, logits, u, temperature=t, min_p=cuda([0.3, 0.01, 0.05, 0.5, 0.0, 0.7]))
    check(B, logits, u, temperature=t, top_k=cuda([1, 5, 50, 50, 300, 2000], torch.int32), top_p=cuda([0.3, 0.9, 0.95, 0.5, 0.8, 0.7]),
          min_p=cuda([0.3, 0.01, 0.05, 0.5, 0.0, 0.002]), kept=torch.float16)


@pytest.mark.parametrize("rows", [1, 2, 33, 64, 257, 513])
def test_rows(B, rows):
    logits, u = logits_of(rows, rows, 5000, True, masked=True), uniform_of(rows, rows)
    g = torch.Generator().manual_seed(rows)
    draw = lambda lo, hi: (lo + (hi - lo) * torch.rand(rows, generator=g)).cuda()  # noqa: E731
    k = torch.randint(0, 400, (rows,), generator=g).int().cuda()
    check(B, logits, u, temperature=draw(0.3, 2), top_k=k, top_p=draw(0.2, 1.1), min_p=draw(-0.1, 0.2))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V,rows", [(131071, 2), (131072, 40), (262144, 1), (1 << 20, 2)])
def test_large_vocabularies(B, V, rows, half):
    logits, u = logits_of(V, rows, V, half, masked=True), uniform_of(V, rows)
    t = torch.linspace(0.5, 1.5, rows).cuda()
    check(B, logits, u, temperature=t, top_p=torch.linspace(0.8, 0.99, rows).cuda())
    check(B, logits, u, temperature=t, top_k=torch.linspace(30, 60000, rows).int().cuda(), top_p=torch.linspace(0.99, 0.5, rows).cuda())
    check(B, logits, u, temperature=t, min_p=torch.linspace(0.1, 0.001, rows).cuda())


@pytest.mark.parametrize("V", [100, 3000, 20000, 140000])
def test_equal_logits_go_by_their_number(B, V):
    x = torch.zeros((5, V), device="cuda")
    x[1, ::3] = 1.0
    x[2, 1::2] = -0.0                                             # the same number as 0
    x[3] = torch.arange(V, device="cuda").remainder(5).float()
    x[4] = -7.25
    for u in (0.0, 0.37, 0.999999):
        uu = torch.full((5,), u).cuda()
        check(B, x, uu, top_k=cuda([7, V // 3 + 2, V // 2 + 1, V // 5 + 3, 1], torch.int32))
        check(B, x.half(), uu, top_k=cuda([V - 1, 1, 3, V // 10, 64], torch.int32))
        # dyadic shares of weights of 1: sums and borders are exact
        check(B, torch.zeros_like(x), uu, top_p=cuda([0.5, 0.25, 0.125, 0.75, 1.0]))
        check(B, x, uu, top_k=cuda([64, 64, 64, 64, 64], torch.int32), top_p=cuda([0.5, 0.25, 1.0, 0.375, 0.75]))


def test_more_equal_logits_than_a_list_holds(B):
    # many tokens in one first bin, at several logits next to each other, and one far above
    V = 60000
    x = 1.0 + torch.randint(0, 9, (4, V), generator=torch.Generator().manual_seed(1)).float().cuda() * 2.0 ** -22
    x[2, 777] = 30.0
    x[3] = -40.0 + torch.randn(V, generator=torch.Generator().manual_seed(2)).cuda() * 3
    x[3, 5] = 20.0
    u = cuda([0.2, 0.9, 0.99999, 0.5])
    check(B, x, u, top_k=cuda([10000, 30001, 20000, 25000], torch.int32))
    check(B, x, u, top_k=cuda([10000, 30001, 20000, 25000], torch.int32), top_p=cuda([0.31, 0.77, 0.9, 0.99]))
    check(B, x[:2].contiguous(), u[:2].contiguous(), top_p=cuda([0.31, 0.77]))


def test_settings_that_keep_everything_or_one(B):
    V = 4001
    logits, u = logits_of(1, 8, V, False), uniform_of(2, 8)
    everything = check(B, logits, u)
    for settings in (dict(top_k=cuda([0, -1, V, V + 5, 2 ** 31 - 1, -2 ** 31, 0, V], torch.int32)), dict(top_p=cuda([1.0, 1.5, float("inf"), float("nan"), 1, 2, 3, 4])),
                     dict(min_p=cuda([0.0, -1.0, float("nan"), -float("inf"), 0, 0, 0, 0])), dict(temperature=cuda([1.0] * 8))):
        got = check(B, logits, u, **settings)
        assert torch.equal(got[0], everything[0]) and torch.equal(got[1], everything[1])
    best = logits.argmax(1)
    for settings in (dict(top_k=cuda([1] * 8, torch.int32)), dict(top_p=cuda([0.0, -1.0, -float("inf"), 1e-30, 1e-9, 0, 0, 0])), dict(min_p=cuda([1.0, 2.0, float("inf"), 1.0, 1, 1, 1, 1])),
                     dict(temperature=cuda([0.0, -0.0, -1.0, float("nan"), -float("inf"), 1e-40, 1e-30, 1e-6]))):
        tokens, p = check(B, logits, u, **settings)
        assert torch.equal(tokens, best) and (p.gather(1, best[:, None]) == 1).all() and int((p > 0).sum()) == 8


def test_temperatures(B):
    logits, u = logits_of(1, 6, 3001, False), uniform_of(3, 6)
    check(B, logits, u, temperature=cuda([1e-3, 0.05, 10.0, 1e4, 1e30, 1.0]))
    check(B, logits, u, temperature=cuda([1e-3, 0.05, 10.0, 1e4, 3e38, 1.0]), top_k=cuda([100] * 6, torch.int32))
    # an infinite one: all weights are 1
    tokens, p = B.ap_sample(logits, u, temperature=cuda([float("inf")] * 6), probabilities=torch.float32)
    assert (p == p[0, 0]).all() and torch.equal(tokens.cpu(), (u.cpu().double() * 3001).floor().long())


def test_uniform_numbers_at_their_ends(B):
    V = 700
    logits = logits_of(1, 7, V, True, masked=True)
    u = cuda([0.0, -0.5, 1.0, 2.0, float("nan"), 1 - 2.0 ** -24, float("-inf")])
    check(B, logits, u, top_p=cuda([0.9] * 7))
    tokens, p = B.ap_sample(logits, u, probabilities=torch.float32, top_p=cuda([0.9] * 7))
    kept = [r.nonzero().flatten().tolist() for r in p]
    assert [int(t) for t in tokens] == [kept[0][0], kept[1][0], kept[2][-1], kept[3][-1], kept[4][-1], kept[5][-1], kept[6][0]]


def test_infinities_and_nan(B):
    V = 900
    inf, nan = float("inf"), float("nan")
    x = logits_of(1, 9, V, False)
    x[0, ::2] = nan
    x[1] = -inf
    x[2] = nan
    x[3, [5, 77, 800]] = inf
    x[4, :] = -inf
    x[4, 33] = -3e38
    x[5, [0, 1]] = cuda([3.4e38, -3.4e38])
    x[6, 1:] = nan
    x[7, 3] = inf
    x[7, 4:] = nan
    x[8] = cuda([-3.4e38]).expand(V)
    u = uniform_of(5, 9)
    for logits in (x, x.half()):
        check(B, logits, u)
        check(B, logits, u, top_k=cuda([5, 3, 2, 2, 10, 2, 5, 5, 7], torch.int32))
        check(B, logits, u, top_p=cuda([0.5] * 9), temperature=cuda([1.0, 1, 1, 2, 1, 1e30, 1, 1, 3]))
        check(B, logits, u, temperature=cuda([0.0] * 9), min_p=cuda([0.5] * 9))
    tokens, p = B.ap_sample(x, u, probabilities=torch.float32)
    assert tokens[1] == -1 and tokens[2] == -1 and not p[1:3].any() and int(tokens[3]) in (5, 77, 800) and tokens[7] == 3


def test_strides_and_places(B):
    V = 1003
    wide = logits_of(1, 5, V + 9, True)
    u, t, k = uniform_of(1, 5), cuda([0.8] * 5), cuda([40] * 5, torch.int32)
    for at in (0, 1, 5, 8):
        part = wide[:, at:at + V]
        got, want = check(B, part, u, temperature=t, top_k=k), check(B, part.contiguous(), u, temperature=t, top_k=k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p = torch.full((5, V), 7.0, dtype=torch.float16, device="cuda")
    tokens, back = B.ap_sample(wide[:, :V], u, temperature=t, top_k=k, probabilities=p)
    assert back.data_ptr() == p.data_ptr() and torch.equal(p, B.ap_sample(wide[:, :V], u, temperature=t, top_k=k, probabilities=torch.float16)[1])
    one = B.ap_sample(wide[:1, :V].expand(5, -1), u, temperature=t, top_k=k)[0]            # one row of logits, several draws
    assert torch.equal(one, check(B, wide[:1, :V].expand(5, -1).contiguous(), u, temperature=t, top_k=k)[0])


def test_rows_far_apart(B):
    far = torch.empty((1 << 31) + 4096, dtype=torch.float16, device="cuda")
    x = far.as_strided((3, 1500), (1 << 30, 1))
    x.copy_(logits_of(1, 3, 1500, True))
    check(B, x, uniform_of(1, 3), top_p=cuda([0.9] * 3))


def test_tokens_follow_their_probabilities(B):
    V, n = 50, 20000
    logits = logits_of(3, 1, V, False, size=1.5)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    tokens, p = B.ap_sample(logits.expand(n, -1), torch.rand(n, generator=g, device="cuda"), top_k=cuda([20] * n, torch.int32), probabilities=torch.float32)
    share = torch.bincount(tokens, minlength=V).double() / n
    # the standard deviation of a share is sqrt(p (1 - p) / n); 5 of them, 50 tokens
    assert ((share - p[0].double()).abs() <= 5 * (p[0].double() / n).sqrt() + 1e-9).all()


def test_probabilities_are_what_verification_takes(B):
    Sq, N, V = 6, 3, 3001
    logits = logits_of(1, Sq * (N + 1), V, True)
    draft_logits = (logits.view(Sq, N + 1, V)[:, :N].float() + 0.3 * logits_of(2, Sq * N, V, False).view(Sq, N, V)).half().reshape(Sq * N, V)
    t = lambda n: cuda([0.9] * n)  # noqa: E731
    drafted, draft = B.ap_sample(draft_logits, uniform_of(3, Sq * N), temperature=t(Sq * N), top_p=cuda([0.95] * (Sq * N)), probabilities=torch.float32)
    _, target = B.ap_sample(logits, uniform_of(4, Sq * (N + 1)), temperature=t(Sq * (N + 1)), top_p=cuda([0.95] * (Sq * (N + 1))), probabilities=torch.float32)
    noise = torch.empty((Sq, V), device="cuda").exponential_()
    tokens, accepted = B.ap_verify(target.view(Sq, N + 1, V), draft.view(Sq, N, V), drafted.view(Sq, N), torch.rand((Sq, N), device="cuda"), noise)
    assert ((accepted >= 0) & (accepted <= N)).all()
    for s in range(Sq):
        n = int(accepted[s])
        assert torch.equal(tokens[s, :n], drafted.view(Sq, N)[s, :n]) and target.view(Sq, N + 1, V)[s, n, tokens[s, n]] > 0


def test_streams(B):
    logits, u, p = logits_of(1, 30, 20000, True), uniform_of(1, 30), cuda([0.9] * 30)
    want = B.ap_sample(logits, u, top_p=p, probabilities=torch.float32)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [B.ap_sample(logits, u, top_p=p, probabilities=torch.float32, stream=(side, other)[i % 2]) for i in range(6)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in got)


def test_tensors_that_do_not_fit_are_refused(B):
    logits, u = logits_of(1, 4, 100, True), uniform_of(1, 4)
    call = lambda **kw: B.ap_sample(**dict(dict(logits=logits, uniform=u), **kw))  # noqa: E731
    call()
    for bad in (dict(logits=logits.cpu()), dict(logits=logits.double()), dict(logits=logits[0]), dict(logits=logits.t()), dict(uniform=u[:3]), dict(uniform=u.double()),
                dict(uniform=u.cpu()), dict(temperature=u.half()), dict(top_k=u), dict(top_k=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(top_p=u[:2]),
                dict(min_p=u.cpu()), dict(probabilities=logits.cpu()), dict(probabilities=logits[:2]), dict(probabilities=torch.float64), dict(probabilities=logits.double())):
        with pytest.raises(AssertionError):
            call(**bad)
    with pytest.raises(B.ApError):
        call(logits=torch.zeros((1, (1 << 20) + 1), dtype=torch.float16, device="cuda"), uniform=u[:1])
    with pytest.raises(TypeError):
        call(uniform=None)
    assert call(logits=logits[:0], uniform=u[:0])[0].shape == (0,)


def test_probabilities_that_do_not_fit_are_refused(B):
    x, u = logits_of(1, 4, 100, False), uniform_of(1, 4)
    before = x.clone()
    with pytest.raises(AssertionError):
        B.ap_sample(x, u, probabilities=torch.empty((100, 4), device="cuda"))
    with pytest.raises(B.ApError):                              # the logits themselves
        B.ap_sample(x, u, probabilities=x)
    both = torch.empty(1000, device="cuda")
    both[:400] = x.flatten()
    with pytest.raises(B.ApError):                              # the last row
        B.ap_sample(both[:400].view(4, 100), u, probabilities=both[399:799].view(4, 100))
    tokens, p = B.ap_sample(both[:400].view(4, 100), u, probabilities=both[400:800].view(4, 100))
    assert torch.equal(x, before) and torch.equal(tokens, B.ap_sample(x, u)[0]) and torch.equal(p, B.ap_sample(x, u, probabilities=torch.float32)[1])
