"""Plain 64-bit forms of the decoder operators, and the error bounds of the kernels against them."""
import random

import torch

EPS32, HALF_EPS16, SUBNORMAL16 = 2.0 ** -24, 2.0 ** -11, 2.0 ** -25


def codes_of(x):
    """(codes, low, step) of rows of binary16 values, in the library's binary32 arithmetic: all three are exact there."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = ((high - low) / torch.full_like(low, 15.0)).half()
    s = step.float()
    codes = torch.where(s > 0, (x - low) / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(x)).round().clamp(0, 15)
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    nan = torch.full_like(low, float("nan"))
    return codes, torch.where(bad, nan, low), torch.where(bad, nan, s)


def cache_values(x):
    """What the cache stands for, in 64 bits."""
    codes, low, step = codes_of(x)
    return low.double() + step.double() * codes.double()


def rotate(x, rotary, positions, interleaved):
    """64-bit rotation of (tokens, heads, head_dim)."""
    out = x.double().clone()
    if rotary is None:
        return out
    half = rotary.shape[1] // 2
    cos, sin = rotary[positions, None, :half].double(), rotary[positions, None, half:].double()
    at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., at[0]].double(), x[..., at[1]].double()
    out[..., at[0]], out[..., at[1]] = a * cos - b * sin, b * cos + a * sin
    return out


def attention(q, k, v, scale, sees, low_k=None, low_v=None):
    """One sequence: q (n, heads, D), k, v (m, kv_heads, D), 64-bit; query i sees the first sees[i] keys.  Returns (out, bound): the
    bound is of a kernel with binary32 scores and sums and weights of the values good to HALF_EPS16 that rounds its result to binary16.

    A score of D products summed in any order of at most 16 dependent sums of partial sums is off by 16 EPS32 times the sum of the magnitudes that
    enter it, the same for sums over keys.  low_k, low_v: those magnitudes where they are more than |k|, |v| (values coded with an offset)."""
    n, H, D = q.shape
    m, G, _ = k.shape
    out, bound = torch.zeros((n, H, D), dtype=torch.float64, device=q.device), torch.zeros((n, H, D), dtype=torch.float64, device=q.device)
    if m == 0 or n == 0:
        return out, bound + SUBNORMAL16
    mask = torch.arange(m, device=q.device)[None, :] < sees[:, None].to(q.device)
    for h in range(H):
        kh, vh = k[:, h // (H // G)], v[:, h // (H // G)]
        mk, mv = (kh if low_k is None else low_k[:, h // (H // G)]).abs(), (vh if low_v is None else low_v[:, h // (H // G)]).abs()
        s = (q[:, h] @ kh.t()) * scale
        s = torch.where(mask, s, torch.full_like(s, float("-inf")))
        top = s.amax(1, keepdim=True)
        p = torch.where(mask, torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top)), torch.zeros_like(s))
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
        vals = torch.where(mask[:, :, None], vh[None], torch.zeros_like(vh[None])) if not torch.isfinite(vh).all() else None
        out[:, h] = (p[:, :, None] * vals).sum(1) if vals is not None else p @ vh
        # score error in the exponent (and its own size: the product with log2 e, the exponential's rounding), both ways through the normalisation
        size = (q[:, h].abs() @ torch.nan_to_num(mk).t()) * abs(scale)
        size = torch.where(mask, torch.nan_to_num(size, posinf=0.0), torch.zeros_like(size)).amax(1, keepdim=True)
        rel = 2 * (16 + 4) * EPS32 * size + HALF_EPS16 + 64 * EPS32
        mass = torch.nan_to_num(p) @ torch.nan_to_num(mv, posinf=0.0)
        # weights below the normal range of binary16 are off by SUBNORMAL16; the sum of weights is at least 1
        small = SUBNORMAL16 * torch.nan_to_num(mv, posinf=0.0).amax(0, keepdim=True) * mask.sum(1, keepdim=True) / torch.where(total == 0, torch.ones_like(total), total)
        bound[:, h] = HALF_EPS16 * out[:, h].abs() + rel * mass + small + SUBNORMAL16
    return out, bound


def check(got, want, bound, what=""):
    got = got.double()
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad), "%s NaN in other places: %d instead of %d" % (what, int(torch.isnan(got).sum()), int(bad.sum()))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what + " infinities"
    ok = ~(bad | inf)
    worst = ((got - want).abs()[ok] / bound[ok]).max().item() if ok.any() else 0.0
    assert worst <= 1.0, "%s error is %.3f of its bound" % (what, worst)
    return worst


def page_table(lengths, page, seed=0, extra=3, fill=-1, width=None):
    """Tables of pages in no order and the number of pages."""
    rng = random.Random(seed)
    need = [-(-n // page) for n in lengths]
    order = list(range(sum(need) + extra))
    rng.shuffle(order)
    table = torch.full((len(lengths), width or max(need + [1])), fill, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table, len(order)


def slots_of(table, page, sequence, first, last):
    t = torch.arange(first, last)
    return table[sequence, t // page].long() * page + t % page


def starts(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)


def live_sequences(starts, tokens):
    """(sequence, first token, end) of those that have tokens: starts in order and in range, not before the end of an earlier one."""
    live, upto = [], 0
    for s, (a, b) in enumerate(zip(starts, starts[1:])):
        if 0 <= a < b <= tokens:
            if a >= upto:
                live.append((s, a, b))
            upto = max(upto, b)
    return live


def senseless_starts(seed, sequences, tokens):
    """Starts of which some descend, leave the tokens or lie inside earlier sequences."""
    g = torch.Generator().manual_seed(seed)
    draw = lambda n: int(torch.randint(0, n, (1,), generator=g))  # noqa: E731
    starts = sorted(draw(tokens + 1) for _ in range(sequences + 1))
    for _ in range((1, 2, 6, 20)[seed % 4]):
        starts[draw(sequences + 1)] = (draw(tokens + 1), 0, tokens, -3, tokens + 5, 2 ** 31 - 1, -2 ** 31)[draw(7)]
    return starts
