"""Plain 64-bit forms of the operators around a decoder step (shared prefixes, norms, sampling), and the error bounds of the kernels against them."""
import torch

import decode_util as U

EPS32, HALF_EPS16, SUBNORMAL16 = U.EPS32, U.HALF_EPS16, U.SUBNORMAL16


def shared_attention(q, k, v, scale, sees, low_k, low_v):
    """One sequence over its prefix and its own keys: q (n, heads, D), k, v (m, kv_heads, D), 64-bit, query i sees the first sees[i] keys.  (out, bound).

    The bound is of a kernel with binary32 scores and sums (a sum of products is off by 16 EPS32 of the magnitudes that enter it, low_k and low_v with
    offsets), with values rounded to binary16 and weights kept to 16 bits (2^-17), that rounds its result to binary16.  A weight below 2^-21 of the greatest is a subnormal
    number of binary16: off by 2^-25 2^-7 of the greatest at least, which is a share of at most 2^-32 of the sum of weights per key."""
    n, H, D = q.shape
    m, G, _ = k.shape
    if m == 0 or n == 0:
        return torch.zeros_like(q), torch.full_like(q, SUBNORMAL16)
    group = H // G
    mask = torch.arange(m, device=q.device)[None, :] < sees[:, None].to(q.device)
    k, v, low_k, low_v = (x.transpose(0, 1).contiguous() for x in (k, v, low_k, low_v))            # (G, m, D)
    rows = q.view(n, G, group, D).permute(1, 2, 0, 3).reshape(G, group * n, D)
    seen = mask.repeat(group, 1)[None]
    s = torch.matmul(rows, k.transpose(1, 2).contiguous()) * scale
    s = torch.where(seen, s, torch.full_like(s, float("-inf")))
    top = s.amax(2, keepdim=True)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top)), torch.zeros_like(s))
    total = p.sum(2, keepdim=True)
    total = torch.where(total == 0, torch.ones_like(total), total)
    p = p / total
    # a NaN or an infinity reaches the rows that see it
    values = torch.where(torch.isnan(v), torch.zeros_like(v), v)
    out = torch.matmul(p, values)
    hit = torch.matmul(seen.double().expand(G, -1, -1).contiguous(), torch.isnan(v).double()) + (torch.isnan(s) & seen).any(2, keepdim=True)
    out = torch.where(hit > 0, torch.full_like(out, float("nan")), out)
    size = torch.matmul(rows.abs(), torch.nan_to_num(low_k).abs().transpose(1, 2).contiguous()) * abs(scale)
    size = torch.where(seen, size, torch.zeros_like(size)).amax(2, keepdim=True)
    magnitude = torch.nan_to_num(low_v).abs()
    mass = torch.matmul(torch.nan_to_num(p), magnitude)
    rel = 2 * (16 + 4) * EPS32 * size + HALF_EPS16 + 2 * 2.0 ** -17 + 64 * EPS32
    small = 2.0 ** -32 * torch.matmul(seen.double().expand(G, -1, -1).contiguous(), magnitude)
    bound = HALF_EPS16 * torch.nan_to_num(out).abs() + rel * mass + small + SUBNORMAL16
    back = lambda x: x.view(G, group, n, D).permute(2, 0, 1, 3).reshape(n, H, D)  # noqa: E731
    return back(out), back(bound)


def norm(v, weight, bias, eps, centred):
    """64-bit norm of rows, and the bound of the kernel's error against it where the rows are exact.

    Sums over a row: a mean of squares from binary32 sums of up to 32 products is off by 33 EPS32 of itself, the inverse of its root by half of that; its rounding to
    binary32 is half an EPS32 more, the inverse root 2 (one in the last place), and a product and the sum with the bias round once each.  A mean is off by 4 EPS32 of the mean magnitude, and so is each difference from it, whose
    square adds twice the relative error."""
    v = v.double()
    slack = torch.zeros_like(v[:, :1])
    if centred:
        slack = 4 * EPS32 * v.abs().mean(1, keepdim=True)
        v = v - v.mean(1, keepdim=True)
    root = torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    w = 1.0 if weight is None else weight.double()
    y = v / root * w
    spread = v.square().mean(1, keepdim=True).sqrt()
    shift = slack / torch.where(spread == 0, torch.ones_like(spread), spread)                     # of the differences, relative
    bound = y.abs() * (24 * EPS32 + 2 * shift) + slack / root * abs(w) + 2.0 ** -126
    if bias is not None:
        y = y + bias.double()
        bound = bound + EPS32 * (y.abs() + bias.double().abs())
    return y, bound


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, probabilities in 64 bits), row by row from the definition.  Sums are of 64-bit numbers: cases keep away from borders that they could move."""
    rows, V = logits.shape
    tokens, out = [], torch.zeros((rows, V), dtype=torch.float64)
    logits = logits.detach().cpu().double()
    of = lambda x, r, none: none if x is None else float(x[r])  # noqa: E731
    for r in range(rows):
        x = torch.where(torch.isnan(logits[r]), torch.full((V,), float("-inf"), dtype=torch.float64), logits[r])
        t, k, p, low, u = of(temperature, r, 1.0), of(top_k, r, 0), of(top_p, r, 1.0), of(min_p, r, 0.0), float(uniform[r])
        if bool((x == float("inf")).any()):
            x = torch.where(x == float("inf"), torch.zeros_like(x), torch.full_like(x, float("-inf")))
        there = torch.isfinite(x)
        if not there.any():
            tokens.append(-1)
            continue
        order = torch.sort(x, descending=True, stable=True).indices
        order = order[there[order]]
        if not t > 0:
            tokens.append(int(order[0]))
            out[r, order[0]] = 1.0
            continue
        w = torch.exp((x[order] - x[order[0]]) / t)
        n = len(order)
        if 0 < k < n:
            n = int(k)
        if p < 1:
            upto = w[:n].cumsum(0)
            n = int(((upto - w[:n]) < p * upto[-1]).sum().clamp(min=1))
        if low > 0:
            n = max(1, min(n, int((w >= min(low, 1.0)).sum())))
        out[r, order[:n]] = w[:n]
        upto = out[r].cumsum(0)
        kept = torch.sort(order[:n]).values
        passed = kept[upto[kept] > u * upto[-1]] if u < 1 else kept[:0]
        tokens.append(int(passed[0]) if len(passed) else int(kept[out[r, kept] > 0][-1]))
        out[r] /= upto[-1]
    return torch.tensor(tokens), out
