"""GPU tests of the norms around a block against a plain 64-bit form."""
import pytest
import torch

import step_util as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2402_10517_amd import binding
    return binding


def normal(seed, *shape, size=1.0, dtype=torch.float16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)


def check(got, want, bound, what):
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad), what + ": NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got.double()[inf], want[inf]), what + ": infinities"
    fine = ~(bad | inf)
    share = ((got.double() - want).abs()[fine] / bound[fine]).max().item() if fine.any() else 0.0
    assert share <= 1.0, "%s: error is %.3f of its bound" % (what, share)


def rounded(x, bound, type):
    """The bound of a value within `bound` of x that is then rounded to `type`."""
    eps, least = (S.HALF_EPS16, S.SUBNORMAL16) if type == torch.float16 else (S.EPS32, 2.0 ** -150)
    return bound + eps * (x.abs() + bound) + least


def norm_case(B, x, residual, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, scale=1.0, eps=1e-6, centred=False, post=None, **kw):
    out, r = B.ap_norm(x, residual, weight, bias, post_weight, post_bias, post, gate, scale, eps, centred, **kw)
    type = residual.dtype if residual is not None else torch.float32
    if x is None:
        given = residual
        assert r is None or torch.equal(r, residual)
    else:
        y, bound = x.double(), torch.zeros_like(x, dtype=torch.float64)
        if post or (post is None and (post_weight is not None or post_bias is not None)):
            y, bound = S.norm(x, post_weight, post_bias, eps, centred)
        g = scale * (1.0 if gate is None else gate.double())
        want, bound = g * y, abs(g) * (bound + 2 * S.EPS32 * y.abs())
        if residual is not None:
            want, bound = want + residual.double(), bound + S.EPS32 * abs(g) * y.abs()
        bound = bound + S.EPS32 * want.abs() + 2.0 ** -149          # computed in binary32
        want = torch.where(want.abs() > torch.finfo(type).max, want.sign() * torch.inf, want)
        if r is None:
            assert residual is None
            r = want.float()
            bound_in = bound
        else:
            check(r, want, rounded(torch.nan_to_num(want, posinf=0, neginf=0), bound, type), "residual")
            bound_in = None
        given = r
        if bound_in is not None:                                  # the norm's input is not seen: binary32, as its output would be
            want, bound = S.norm(given, weight, bias, eps, centred)
            root = (given.double() - (given.double().mean(1, keepdim=True) if centred else 0)).square().mean(1, keepdim=True).add(eps).sqrt()
            w = 1.0 if weight is None else weight.double().abs()
            spread = 2 * rounded(given.double(), bound_in, type).amax(1, keepdim=True) / root
            check(out, want, rounded(want, bound + spread * (w + want.abs()), torch.float16), "norm")
            return out, None
    if out is not None:
        want, bound = S.norm(given, weight, bias, eps, centred)
        check(out, want, rounded(want, bound, torch.float16), "norm")
    return out, r


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("columns", [1, 2, 7, 8, 9, 63, 64, 65, 511, 512, 513, 520, 1023, 4096, 5120, 5121, 8191, 8192, 8193, 8200, 11008, 16384, 16385, 16392, 28672, 32767, 32768])
def test_columns(B, columns, centred, half):
    T = 3
    x, residual = normal(1, T, columns), normal(2, T, columns, size=5, dtype=torch.float16 if half else torch.float32)
    w, b = normal(3, columns) + 1, normal(4, columns)
    norm_case(B, x, residual, w, b if centred else None, centred=centred)
    norm_case(B, x, residual, w, b, post_weight=normal(5, columns), post_bias=b.flip(0), gate=normal(6, T, columns), scale=-0.7, centred=centred)
    norm_case(B, None, residual, w, centred=centred)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("tokens,columns", [(256, 4104), (257, 4096), (257, 4097), (257, 4104), (300, 5121), (261, 6201), (258, 8192)])
def test_many_rows_of_many_columns(B, tokens, columns, centred, half):
    x, r = normal(columns, tokens, columns), normal(1, tokens, columns, size=3, dtype=torch.float16 if half else torch.float32)
    w, b, pw, pb = (normal(i, columns) for i in range(2, 6))
    norm_case(B, x, r, w, b, pw, pb, normal(6, tokens, columns), centred=centred)


@pytest.mark.parametrize("tokens", [1, 2, 5, 64, 300, 2049])
@pytest.mark.parametrize("half", [False, True])
def test_tokens(B, tokens, half):
    x, residual = normal(1, tokens, 777), normal(2, tokens, 777, size=5, dtype=torch.float16 if half else torch.float32)
    norm_case(B, x, residual, normal(3, 777))
    norm_case(B, x, residual, normal(3, 777), post_weight=normal(4, 777), gate=normal(5, 1, 777), centred=True)


def test_more_rows_than_workgroups(B):
    T = (1 << 20) + 77
    x, residual = normal(1, T, 9), normal(2, T, 9, dtype=torch.float32)
    norm_case(B, x, residual, normal(3, 9))


def test_parts_that_are_left_out(B):
    x, residual, w = normal(1, 5, 640), normal(2, 5, 640, dtype=torch.float32), normal(3, 640)
    out, r = norm_case(B, x, None, w)                                 # a norm alone
    assert r is None
    out, r = norm_case(B, x, None, None, post=True, gate=normal(4, 5, 640))
    out, r = B.ap_norm(x, residual, normed=False, scale=0.25)
    assert out is None and torch.equal(r, torch.add(residual, x.float(), alpha=0.25))
    out, r = B.ap_norm(None, residual, w)
    assert r is None
    kept = torch.zeros_like(residual)
    assert B.ap_norm(None, residual, w, residual_out=kept)[1] is not None and torch.equal(kept, residual)
    kept = torch.zeros_like(x)
    out, r = B.ap_norm(x, None, w, residual_out=kept, scale=2.0)     # the output's type without a residual
    assert torch.equal(kept, x * 2)
    assert B.ap_norm(x, None, normed=False) == (None, None)
    assert B.ap_norm(x[:0], residual[:0], w)[0].shape == (0, 640)


def test_strides_and_places(B):
    T, K = 9, 515
    wide, r = normal(1, T, 3 * K), normal(2, T, K + 5, dtype=torch.float32)
    w, gate = normal(3, K), normal(4, T, 2 * K)
    for at in (0, 1, 3, 8):
        x, res, g = wide[:, at:at + K], r[:, at % 5:at % 5 + K], gate[:, at:at + K]
        want = norm_case(B, x.contiguous(), res.contiguous(), w, gate=g.contiguous())
        got = norm_case(B, x, res, w, gate=g)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        to, kept = torch.full((T, K + 3), 7.0, dtype=torch.float16, device="cuda"), torch.full((T, K + 3), 7.0, device="cuda")
        B.ap_norm(x, res, w, gate=g, out=to[:, 1:K + 1], residual_out=kept[:, 2:K + 2])
        assert torch.equal(to[:, 1:K + 1], want[0]) and torch.equal(kept[:, 2:K + 2], want[1])
        assert (to[:, 0] == 7).all() and (to[:, K + 1:] == 7).all() and (kept[:, :2] == 7).all() and (kept[:, K + 2:] == 7).all()
    # every other row; rows of one memory; in place
    x, res = wide[::2, :K], r[::2, :K]
    got, want = B.ap_norm(x, res, w), B.ap_norm(x.contiguous(), res.contiguous(), w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = B.ap_norm(wide[:1, :K].expand(T, -1), r[:1, :K].expand(T, -1), w)
    assert torch.equal(one[0], one[0][:1].expand(T, -1))
    for columns in (K, 512, 5000, 20000):
        x, res, w = normal(5, 4, columns), normal(6, 4, columns, dtype=torch.float32), normal(7, columns)
        want = B.ap_norm(x, res, w, post_weight=w)
        got = B.ap_norm(x, res, w, post_weight=w, out=x, residual_out=res)
        assert torch.equal(x, want[0]) and torch.equal(res, want[1]) and got[0].data_ptr() == x.data_ptr()


def test_rows_far_apart(B):
    # row offsets beyond 32 bits
    far = torch.empty((1 << 31) + 4096, dtype=torch.float16, device="cuda")
    x = far.as_strided((3, 640), (1 << 30, 1))
    x.copy_(normal(1, 3, 640))
    residual, w = normal(2, 3, 640, dtype=torch.float32), normal(3, 640)
    got, want = B.ap_norm(x, residual, w), B.ap_norm(x.contiguous(), residual, w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("centred", [False, True])
def test_values(B, centred):
    K, w = 1000, normal(3, 1000)
    ones = torch.ones(K, dtype=torch.float16, device="cuda")
    for size in (0.0, 1e-30, 1e-20, 1e-3, 1.0, 1e4, 1e20, 1e30, 1e37):                  # sums of squares outside binary32
        norm_case(B, None, normal(1, 2, K, size=size, dtype=torch.float32), w, eps=1e-6, centred=centred)
        if size:
            norm_case(B, None, normal(1, 2, K, size=size, dtype=torch.float32), w, eps=0.0, centred=centred)
    big = normal(1, 2, K, size=30000).clamp(-65504, 65504)
    norm_case(B, big, normal(2, 2, K, dtype=torch.float16), w, post_weight=ones, centred=centred)
    norm_case(B, big, big, w, scale=3.0, centred=centred)                                 # a binary16 residual overflows
    offset = normal(1, 2, K, dtype=torch.float32) + 3000.0                                # a mean far above the differences
    norm_case(B, None, offset, w, centred=centred)
    same = torch.full((2, K), 1234.5, device="cuda")
    out, _ = B.ap_norm(None, same, w, bias=w, centred=centred)
    if centred:
        assert torch.equal(out, w.expand(2, -1))
    # NaN and infinities stay in their row
    r = normal(1, 4, K, dtype=torch.float32)
    r[1, 5], r[2, 999] = float("nan"), float("inf")
    norm_case(B, normal(2, 4, K), r, w, centred=centred)


def test_streams_and_graphs(B):
    x, residual, w = normal(1, 33, 5120), normal(2, 33, 5120, dtype=torch.float32), normal(3, 5120)
    want = B.ap_norm(x, residual, w, post_weight=w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        out, r = B.ap_norm(x, residual, w, post_weight=w, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want[0]) and torch.equal(r, want[1])


def test_tensors_that_do_not_fit_are_refused(B):
    x, residual, w = normal(1, 4, 64), normal(2, 4, 64, dtype=torch.float32), normal(3, 64)
    call = lambda **kw: B.ap_norm(**dict(dict(x=x, residual=residual, weight=w), **kw))  # noqa: E731
    call()
    for bad in (dict(x=x.float()), dict(x=x.cpu()), dict(x=x[:3]), dict(residual=residual.double()), dict(residual=residual[:, :63]), dict(weight=w.float()), dict(weight=w[:63]),
                dict(bias=w[None]), dict(post_weight=w.cpu()), dict(gate=x[:2]), dict(gate=x.float()), dict(out=residual), dict(residual_out=x), dict(x=x.t()),
                dict(x=x[0]), dict(out=x.t())):
        if bad.keys() == {"bias"}:
            continue
        with pytest.raises(AssertionError):
            call(**bad)
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(B.ApError):
            call(**bad)
    with pytest.raises(B.ApError):
        B.ap_norm(normal(1, 2, 32769), None)
    with pytest.raises(TypeError):
        B.ap_norm(None, None)


def test_rows_that_are_written_lie_apart(B):
    x, r = normal(1, 3, 64), normal(2, 3, 64, dtype=torch.float32)
    for bad in (dict(out=x[:1].expand(3, -1)), dict(residual_out=r[:1].expand(3, -1)), dict(out=torch.empty(256, dtype=torch.float16, device="cuda").as_strided((3, 64), (32, 1)))):
        with pytest.raises(B.ApError):
            B.ap_norm(x, r, **bad)
    assert B.ap_norm(x[:1], r[:1], out=torch.empty_like(x)[:1].expand(1, -1))[0].shape == (1, 64)


def ends_of_binary32(columns):
    """Rows of binary32 values at the ends of their range, none of them infinite."""
    g = torch.Generator().manual_seed(columns)
    most, least = torch.finfo(torch.float32).max, 2.0 ** -149
    rows = torch.zeros((9, columns), dtype=torch.float64)
    x = torch.randn((9, columns), generator=g, dtype=torch.float64)
    rows[0] = 1.0
    rows[0, columns // 2] = 3e38
    rows[1] = most
    rows[2] = most * x[2].sign()
    rows[3] = (x[3] * 1e38).clamp(-most, most)
    rows[4] = x[4] * 1e-37
    rows[5] = (x[5] * 2 ** 20).round() * least
    rows[6, columns // 3] = least
    rows[7] = x[7] * 1e-44
    rows[8] = x[8] * 2.0 ** 63
    return rows.float()


def check_ends(B, r, w, eps, centred, x=None):
    out, kept = B.ap_norm(x, r.cuda(), w, eps=eps, centred=centred)
    given = r if x is None else kept.cpu()
    want, bound = S.norm(given, w.cpu(), None, eps, centred)
    if centred:
        # The mean is a multiple of 2^-149, the least number of binary32: off by 2^-150, and the differences are exact from there on.  With s that share of their root mean
        # square, and d one of them, (d + s r) / sqrt(r^2 + s^2 r^2) is within s + s^2 / 2 |d| / r of d / r, and s^2 / 2 <= 2 s up to s = 4: beyond the half of a step there is none.
        d = given.double() - given.double().mean(1, keepdim=True)
        spread = d.square().mean(1, keepdim=True).sqrt()
        share = 2.0 ** -150 / torch.where(spread == 0, torch.ones_like(spread), spread)
        bound = bound + share * w.cpu().double().abs() + 2 * share * want.abs()
    check(out.cpu(), want, rounded(want, bound, torch.float16), "norm")


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("columns", [1, 3, 8, 200, 1000, 5121, 8192, 20000, 32768])
def test_rows_at_the_ends_of_binary32(B, columns, eps):
    r, w = ends_of_binary32(columns), normal(3, columns, size=0.2) + 0.5
    rows = [i for i in range(9) if eps > 0 or bool(r[i].any())]
    check_ends(B, r[rows], w, eps, False)
    check_ends(B, r[rows], w, eps, False, x=normal(4, len(rows), columns))


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("columns", [2, 3, 8, 200, 1000, 5121, 8192, 20000, 32768])
def test_centred_rows_at_the_ends_of_binary32(B, columns, eps):
    r, w = ends_of_binary32(columns), normal(3, columns, size=0.2) + 0.5
    most = torch.finfo(torch.float32).max
    g = torch.Generator().manual_seed(columns)
    r[1] = most * (1 - torch.rand(columns, generator=g) / 2)       # sums of eight beyond binary32
    more = torch.full((2, columns), -most)                        # differences beyond it
    more[0, columns // 2] = most
    more[1] = torch.where(torch.rand(columns, generator=g) < 0.1, most, -most)
    more[1, 0], more[1, 1] = most, -most
    r = torch.cat([r, more])
    rows = [i for i in range(len(r)) if eps > 0 or bool((r[i] != r[i, 0]).any())]
    check_ends(B, r[rows], w, eps, True)
    check_ends(B, r[rows], w, eps, True, x=normal(4, len(rows), columns))


def test_vectors_of_one_row(B):
    x, residual, w, b = normal(1, 4, 64), normal(2, 4, 64, dtype=torch.float32), normal(3, 64), normal(4, 64)
    want = B.ap_norm(x, residual, w, b, w, b)
    got = B.ap_norm(x, residual, w[None], b[None], w.view(8, 8), b[None])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for bad in (dict(bias=torch.stack([b, b])), dict(bias=torch.stack([b, b], dim=1)[:, 0]), dict(bias=b[:63]), dict(bias=b.float())):
        with pytest.raises(AssertionError):
            B.ap_norm(x, residual, w, **bad)


@pytest.mark.parametrize("tokens,columns,centred", [(1, 4096, False), (33, 5121, True), (300, 8192, False)])
def test_captured_and_replayed(B, tokens, columns, centred):
    x, residual, w, b = normal(1, tokens, columns), normal(2, tokens, columns, dtype=torch.float32), normal(3, columns), normal(4, columns)
    call = lambda: B.ap_norm(x, residual, w, b, post_weight=w, gate=w[None], scale=0.5, centred=centred)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(call())
    for seed in range(5, 9):
        x.copy_(normal(seed, tokens, columns))
        residual.copy_(normal(seed + 10, tokens, columns, dtype=torch.float32))
        for graph in graphs:
            graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[0]) and torch.equal(r, want[1]) for o, r in outs), seed
