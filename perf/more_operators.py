"""More operators of a decoder step, as cases for timing them: attention of a batch whose sequences share prefixes in the 4-bit cache, norms
around a block with its gate, scale and residual, and sampling from logits.

Head layouts and columns are those of the decoder layers that the benchmark's matrices come from (4096, 5120 and 8192 columns: 32, 40 and
64 heads of 128, the last with 8 key heads) and smaller ones.  Activations are binary16, the residual binary32 or binary16; every case is drawn from
its seed alone, its lengths from the case itself.

With `own` false the operators are computed in elementary torch operations (in binary32; sampling in 64 bits, as the borders of what is kept
are sums of many weights), with it true by the library.
"""
import math
import random

import torch

own = False

KEY_OUTLIERS = 8.0                  # keys have a few channels much larger than the others


def listed():
    return [
        # Four chats that start with the same instructions, one new token each, a 7B layer with a key head per head: mostly latency.
        {"name": "shared_4x1000", "kind": "shared", "prefixes": 1, "sequences": 4, "queries": 1, "prefix": 1000, "longest": 61, "ragged": False,
         "heads": 32, "kv_heads": 32, "head_dim": 128, "page": 64},
        # Drafted tokens of 24 sequences of three tasks, each with its own instructions and examples; heads of 64, some batch places idle.
        {"name": "shared_drafts", "kind": "shared", "prefixes": 3, "sequences": 24, "queries": 5, "prefix": 3001, "longest": 500, "ragged": True,
         "heads": 16, "kv_heads": 4, "head_dim": 64, "page": 16},
        # A full batch of a 70B layer behind one long system prompt.
        {"name": "shared_64x8192", "kind": "shared", "prefixes": 1, "sequences": 64, "queries": 1, "prefix": 8192, "longest": 1023, "ragged": True,
         "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 64},
        # Questions about two long documents: the most work.
        {"name": "shared_documents", "kind": "shared", "prefixes": 2, "sequences": 48, "queries": 3, "prefix": 65536, "longest": 257, "ragged": True,
         "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 128},
        # The norm before a block of a 7B layer, one token: nothing but latency.
        {"name": "norm_1_token", "kind": "norm", "tokens": 1, "columns": 4096, "half": False, "centred": False, "post": False, "gate": "none",
         "fused": False},
        # A prompt through a layer with norms on both sides of the block and a gate per channel; an odd number of columns, binary16 residual.
        {"name": "norm_odd", "kind": "norm", "tokens": 1531, "columns": 5121, "half": True, "centred": True, "post": True, "gate": "channel",
         "fused": False},
        # Packed prompts of a 70B layer, a gate per value, the block's output as a view of a wider projection: the most work.
        {"name": "norm_prompts", "kind": "norm", "tokens": 8192, "columns": 8192, "half": False, "centred": False, "post": True, "gate": "value",
         "fused": True},
        # One sequence, ordinary settings, logits as the last product leaves them.
        {"name": "sample_1", "kind": "sample", "rows": 1, "vocabulary": 32000, "half": True, "kept": "none", "masked": False, "settings": "ordinary"},
        # The drafting model's tokens of a batch with the probabilities that verification wants; a large vocabulary of an odd size.
        {"name": "sample_64", "kind": "sample", "rows": 64, "vocabulary": 131071, "half": True, "kept": "float", "masked": True, "settings": "ordinary"},
        # A server's batch: every request has its own settings, greedy ones among them; binary32 logits.
        {"name": "sample_settings", "kind": "sample", "rows": 300, "vocabulary": 32003, "half": False, "kept": "half", "masked": True, "settings": "each"},
        # A large batch without a limit to the tokens but temperature.
        {"name": "sample_plain", "kind": "sample", "rows": 96, "vocabulary": 50021, "half": False, "kept": "none", "masked": False, "settings": "temperature"},
    ]


def _spread(rng, lo, hi):
    """A whole number in lo..hi, uniform in its logarithm."""
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    kind = rng.choice(["shared", "shared", "norm", "sample", "sample"])
    while True:
        if kind == "shared":
            kv = rng.choice([1, 2, 3, 4, 8, 8, 32, 40])
            heads = kv * (1 if kv > 8 else rng.choice([1, 2, 3, 4, 5, 7, 8]))
            prefixes = rng.choice([1, 1, 1, 2, 3, 5])
            c = {"kind": kind, "prefixes": prefixes, "sequences": max(prefixes, _spread(rng, 1, 128)), "queries": rng.choice([1, 1, 1, 2, 3, 5, 8]),
                 "prefix": _spread(rng, 17, 65536), "longest": _spread(rng, 8, 4096), "ragged": rng.random() < 0.7, "heads": heads, "kv_heads": kv,
                 "head_dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128, 256])}
            most = "shared_documents"
        elif kind == "norm":
            c = {"kind": kind, "tokens": _spread(rng, 1, 8192), "columns": _spread(rng, 64, 16384), "half": rng.random() < 0.5,
                 "centred": rng.random() < 0.4, "post": rng.random() < 0.5, "gate": rng.choice(["none", "none", "channel", "value"]),
                 "fused": rng.random() < 0.4}
            if rng.random() < 0.6:
                c["columns"] = (c["columns"] + 63) // 64 * 64
            most = "norm_prompts"
        else:
            c = {"kind": kind, "rows": _spread(rng, 1, 300), "vocabulary": _spread(rng, 1000, 131071), "half": rng.random() < 0.5,
                 "kept": rng.choice(["none", "float", "half"]), "masked": rng.random() < 0.5, "settings": rng.choice(["ordinary", "each", "temperature"])}
            most = "sample_settings"
        limit, w = work(next(x for x in listed() if x["name"] == most)), work(c)
        if kind == "sample" and w["bytes"] <= max(limit["bytes"], work(next(x for x in listed() if x["name"] == "sample_64"))["bytes"]):
            return c
        if w["bytes"] <= limit["bytes"] and w["flops"] <= limit["flops"]:
            return c


def _layout(case):
    """Of a shared case: sequences of each prefix, prefix lengths, (query tokens, own keys) of each sequence."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    P, S = case["prefixes"], case["sequences"]
    if case["ragged"] and P > 1:
        cuts = sorted(rng.sample(range(1, S), P - 1))
        sizes = [b - a for a, b in zip([0] + cuts, cuts + [S])]
    else:
        sizes = [S // P + (1 if i < S % P else 0) for i in range(P)]
    prefix = [case["prefix"] if i == 0 or not case["ragged"] else rng.randint(1, case["prefix"]) for i in range(P)]
    sequences = []
    for i in range(S):
        n = case["queries"]
        if case["ragged"] and i:
            n = 0 if rng.random() < 0.06 else rng.randint(1, n)
        length = case["longest"] if i == 0 or not case["ragged"] else rng.randint(1, case["longest"])
        sequences.append((n, max(n, length)))
    return sizes, prefix, sequences


def work(case):
    if case["kind"] == "norm":
        n = case["tokens"] * case["columns"]
        each = 4 + 2 * (2 if case["half"] else 4) + (2 if case["gate"] == "value" else 0)
        return {"bytes": n * each + 2 * case["columns"] * (2 + 2 * case["centred"] + 2 * case["post"]), "flops": n * (6 + 4 * case["post"] + 3 * case["centred"])}
    if case["kind"] == "sample":
        n = case["rows"] * case["vocabulary"]
        return {"bytes": n * ((2 if case["half"] else 4) + {"none": 0, "half": 2, "float": 4}[case["kept"]]), "flops": 6 * n}
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    sizes, prefix, sequences = _layout(case)
    at, pairs = 0, 0
    for size, m in zip(sizes, prefix):
        for n, own_keys in sequences[at:at + size]:
            pairs += n * (m + own_keys) - n * (n - 1) // 2
        at += size
    tokens, keys = sum(n for n, _ in sequences), sum(prefix) + sum(m for n, m in sequences if n)
    return {"bytes": keys * G * (D + 8) + 4 * tokens * H * D, "flops": 4 * H * D * pairs}


# ---------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _table(lengths, order, page):
    """Pages of each row, taken from the end of `order`; -1 behind them."""
    need = [-(-n // page) for n in lengths]
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    return table


def _slots(table, lengths, page):
    rows = [table[i, torch.arange(n) // page].long() * page + torch.arange(n) % page for i, n in enumerate(lengths)]
    return torch.cat(rows)


def _shared_inputs(case, seed):
    gen, G, D, P = _generator(seed), case["kv_heads"], case["head_dim"], case["page"]
    sizes, prefix, sequences = _layout(case)
    lengths = [m for _, m in sequences]
    pages = sum(-(-n // P) for n in prefix + lengths) + 3
    order = list(range(pages))
    random.Random(P + pages).shuffle(order)
    prefix_table, table = _table(prefix, order, P), _table(lengths, order, P)
    slots = torch.cat([_slots(prefix_table, prefix, P), _slots(table, lengths, P)]).cuda()
    q = _normal(gen, sum(n for n, _ in sequences), case["heads"], D)
    k, v = _normal(gen, len(slots), G, D), _normal(gen, len(slots), G, D)
    k[:, :, D // 3] *= KEY_OUTLIERS
    return q, k, v, slots, prefix_table, table, pages


def _norm_inputs(case, seed):
    gen, T, K = _generator(seed), case["tokens"], case["columns"]
    wide = (K + 7) // 8 * 4 if case["fused"] else 0                                  # the rest of a wider projection, of which x is a view
    x = _normal(gen, T, wide + K)[:, wide:]
    residual = torch.randn((T, K), generator=gen, device="cuda") * 3
    residual[:, ::97] *= 20                                                          # a residual stream has channels far above the others
    if case["half"]:
        residual = residual.half()
    weights = {"weight": 1 + 0.2 * _normal(gen, K)}
    if case["post"]:
        weights["post_weight"] = 0.3 + 0.1 * _normal(gen, K)
    if case["centred"]:
        weights["bias"] = 0.1 * _normal(gen, K)
        if case["post"]:
            weights["post_bias"] = 0.1 * _normal(gen, K)
    gate = None
    if case["gate"] != "none":
        gate = _normal(gen, T if case["gate"] == "value" else 1, K)
    return x, residual, gate, weights


def _sample_inputs(case, seed):
    gen, S, V = _generator(seed), case["rows"], case["vocabulary"]
    logits = torch.randn((S, V), generator=gen, device="cuda") * 2.2
    peaks = torch.randint(0, V, (S, 12), generator=gen, device="cuda")               # a few tokens that the model is nearly sure of
    logits.scatter_(1, peaks, 6 + 6 * torch.rand((S, 12), generator=gen, device="cuda"))
    if case["masked"]:                                                               # a grammar forbids tokens
        logits.masked_fill_(torch.rand((S, V), generator=gen, device="cuda") < 0.3, -math.inf)
    rng, settings = random.Random(seed), {}
    settings["temperature"] = [rng.uniform(0.6, 1.3) for _ in range(S)]
    if case["settings"] != "temperature":
        settings["top_k"] = [rng.choice([40, 50, 64, 1000])] * S
        settings["top_p"] = [rng.choice([0.9, 0.95])] * S
    if case["settings"] == "each":
        settings["temperature"] = [0.0 if rng.random() < 0.15 else t for t in settings["temperature"]]
        settings["top_k"] = [rng.choice([0, 0, 1, 20, 50, 400, 5000, V]) for _ in range(S)]
        settings["top_p"] = [rng.choice([1.0, 0.5, rng.uniform(0.7, 0.999)]) for _ in range(S)]
        settings["min_p"] = [rng.choice([0.0, 0.0, 0.05, rng.uniform(0.001, 0.2)]) for _ in range(S)]
    settings = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in settings.items()}
    uniform = torch.rand(S, generator=gen, device="cuda")
    return logits.half() if case["half"] else logits, uniform, settings


PROBABILITIES = {"none": None, "float": torch.float32, "half": torch.float16}


def prepare(case, seed):
    state = {"kind": case["kind"], "own": own}
    if own:
        from paper_2402_10517_amd import binding as B
        state["B"] = B
    if case["kind"] == "shared":
        q, k, v, slots, prefix_table, table, pages = _shared_inputs(case, seed)
        sizes, prefix, sequences = _layout(case)
        G, D, P = case["kv_heads"], case["head_dim"], case["page"]
        int32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        queries = [n for n, _ in sequences]
        state.update(q=q, page=P, prefix_table=prefix_table.cuda(), prefix_lengths=int32(prefix), prefix_starts=int32(_starts(sizes)),
                     table=table.cuda(), lengths=int32([m for _, m in sequences]), q_starts=int32(_starts(queries)), scale=D ** -0.5,
                     longest_prefix=max(prefix), longest=max(m for _, m in sequences), most=max(queries),
                     most_shared=max(sum(queries[a:b]) for a, b in zip(_starts(sizes), _starts(sizes)[1:])))
        if own:
            state["cache"] = B.KVCache(pages, G, D, page_tokens=P)
            B.ap_cache_append(state["cache"], k, v, slots)
        else:
            state["cache"] = {side: _plain_codes(x, slots, pages * P) for side, x in (("k", k), ("v", v))}
    elif case["kind"] == "norm":
        x, residual, gate, weights = _norm_inputs(case, seed)
        state.update(x=x, residual=residual, gate=gate, weights=weights, centred=case["centred"], scale=0.5 if case["post"] else 1.0)
    else:
        logits, uniform, settings = _sample_inputs(case, seed)
        state.update(logits=logits, uniform=uniform, settings=settings, kept=PROBABILITIES[case["kept"]])
    return state


# ---------------------------------------------------------------------------------------------------- plain forms


def _plain_codes(x, slots, places):
    """16 evenly spaced values per token and head, from its least value on, at their places: (codes, least value, step)."""
    out = [torch.zeros((places,) + x.shape[1:2] + (n,), dtype=t, device="cuda") for n, t in ((x.shape[2], torch.uint8), (1, torch.float16), (1, torch.float16))]
    x = x.float()
    low, high = x.amin(dim=2, keepdim=True), x.amax(dim=2, keepdim=True)
    step = ((high - low) / torch.full_like(low, 15.0)).half()
    divisor = torch.where(step > 0, step.float(), torch.ones_like(low))
    codes = torch.where(step > 0, (x - low) / divisor, torch.zeros_like(x)).round().clamp(0, 15)
    out[0][slots], out[1][slots], out[2][slots] = codes.to(torch.uint8), low.half(), step
    return out


def _plain_keys(state, side, table, longest):
    """(rows, kv heads, longest, head_dim): what the cache holds for the first keys of each row of the table."""
    t = torch.arange(longest, device="cuda")
    slots = (table[:, t // state["page"]].long().clamp(min=0) * state["page"] + t % state["page"])
    codes, low, step = (x[slots] for x in state["cache"][side])
    return (codes.float() * step.float() + low.float()).transpose(1, 2).contiguous()


def _plain_softmax_sums(q, k, v, seen, scale):
    """q (rows, kv heads, n, D), k, v (rows, kv heads, m, D), seen (rows, 1, n, m): maximum, sum of weights and sums of values."""
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    score = torch.where(seen, score, torch.full((), -math.inf, device="cuda"))
    top = score.amax(dim=3, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return top, p.sum(dim=3, keepdim=True), torch.matmul(p, v)


def _plain_places(starts, most, tokens):
    """Token numbers (rows, most) of the rows of `starts`, and which of them there are."""
    at = starts[:-1, None].long() + torch.arange(most, device="cuda")
    return at.clamp(max=tokens - 1), at < starts[1:, None]


def _plain_shared(s):
    q, H, D = s["q"].float(), s["q"].shape[1], s["q"].shape[2]
    T, G = len(q), s["cache"]["k"][0].shape[1]
    joined = []
    prefix_starts = s["q_starts"][s["prefix_starts"].long()]
    for table, lengths, longest, starts, most, causal in (
            (s["prefix_table"], s["prefix_lengths"], s["longest_prefix"], prefix_starts, s["most_shared"], False),
            (s["table"], s["lengths"], s["longest"], s["q_starts"], s["most"], True)):
        places, there = _plain_places(starts, most, T)
        rows = q[places].view(len(places), most, G, H // G, D).transpose(1, 2).reshape(len(places), G, most * (H // G), D)
        sees = lengths[:, None].long().expand(-1, most)
        if causal:                                        # the last token of a sequence sees its last key
            sees = sees - (starts[1:, None] - starts[:-1, None]) + 1 + torch.arange(most, device="cuda")
        seen = torch.arange(longest, device="cuda") < sees[:, :, None]
        seen = seen.repeat_interleave(H // G, dim=1)[:, None]
        parts = _plain_softmax_sums(rows, _plain_keys(s, "k", table, longest), _plain_keys(s, "v", table, longest), seen, s["scale"])
        parts = [x.view(len(places), G, most, H // G, -1).transpose(1, 2)[there].reshape(-1, H, x.shape[3]) for x in parts]
        joined.append([torch.zeros((T, H, x.shape[2]), device="cuda").index_copy(0, places[there], x) for x in parts])
    (m0, l0, o0), (m1, l1, o1) = joined
    top = torch.maximum(m0, m1)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w0, w1 = torch.exp(m0 - top), torch.exp(m1 - top)
    total = l0 * w0 + l1 * w1
    return ((o0 * w0 + o1 * w1) / torch.where(total == 0, torch.ones_like(total), total)).half()


EPS = 1e-6


def _plain_normed(x, weight, bias, centred):
    if centred:
        x = x - x.mean(dim=1, keepdim=True)
    x = x / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS) * weight.float()
    return x if bias is None else x + bias.float()


def _plain_norm(s):
    w, y = s["weights"], s["x"].float()
    if "post_weight" in w:
        y = _plain_normed(y, w["post_weight"], w.get("post_bias"), s["centred"])
    if s["gate"] is not None:
        y = y * s["gate"].float()
    residual = (s["residual"].float() + s["scale"] * y).to(s["residual"].dtype)
    return _plain_normed(residual.float(), w["weight"], w.get("bias"), s["centred"]).half(), residual


def _plain_sample(s):
    """In 64 bits: what is kept ends where a sum of many weights passes a limit."""
    x = s["logits"].double()
    rows, V = x.shape
    column = {k: v.double()[:, None] for k, v in s["settings"].items()}
    t = column["temperature"]
    ordered, order = torch.sort(x, dim=1, descending=True, stable=True)             # the lowest index first among equals
    w = torch.exp((ordered - ordered[:, :1]) / torch.where(t > 0, t, torch.ones_like(t)))
    place = torch.arange(V, device="cuda")[None, :]
    keep = (place == 0) | (t > 0)
    if "top_k" in column:
        k = torch.where(column["top_k"] > 0, column["top_k"], torch.full_like(t, V))
        keep &= place < k
    if "top_p" in column:
        kept = torch.where(keep, w, torch.zeros_like(w))
        upto = kept.cumsum(dim=1)
        keep &= (upto - kept < column["top_p"] * upto[:, -1:]) | (column["top_p"] >= 1)
    if "min_p" in column:
        keep &= w >= column["min_p"]
    kept = torch.zeros_like(w).scatter(1, order, torch.where(keep, w, torch.zeros_like(w)))
    upto = kept.cumsum(dim=1)
    total = upto[:, -1:]
    token = (upto <= s["uniform"].double()[:, None] * total).sum(dim=1)
    return token if s["kept"] is None else (token, (kept / total).to(s["kept"]))


def run(state):
    s = state
    if not s["own"]:
        return {"shared": _plain_shared, "norm": _plain_norm, "sample": _plain_sample}[s["kind"]](s)
    B = s["B"]
    if s["kind"] == "shared":
        return B.ap_attention_shared(s["cache"], s["q"], s["prefix_table"], s["prefix_lengths"], s["table"], s["lengths"],
                                     prefix_starts=s["prefix_starts"], q_starts=s["q_starts"], scale=s["scale"],
                                     max_prefix=s["longest_prefix"], max_length=s["longest"])
    if s["kind"] == "norm":
        return B.ap_norm(s["x"], s["residual"], gate=s["gate"], scale=s["scale"], eps=EPS, centred=s["centred"], **s["weights"])
    tokens, probabilities = B.ap_sample(s["logits"], s["uniform"], probabilities=s["kept"], **s["settings"])
    return tokens if s["kept"] is None else (tokens, probabilities)


# ---------------------------------------------------------------------------------------------------- definition in 64 bits


def _exact_values(x):
    """What the cache stands for, from the definition: low + step * nearest of 0..15, low and step binary16."""
    x = x.double()
    low, high = x.min(dim=-1, keepdim=True).values, x.max(dim=-1, keepdim=True).values
    step = ((high - low) / 15).half().double()
    code = torch.nan_to_num((x - low) / step, nan=0.0).round().clamp(0, 15)
    return low + step * code


def _exact_shared(case, seed):
    q, k, v, _, _, _, _ = _shared_inputs(case, seed)
    sizes, prefix, sequences = _layout(case)
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    own_at, key_at, row, s = sum(prefix), 0, 0, 0
    for size, m in zip(sizes, prefix):
        pk, pv = (_exact_values(x[key_at:key_at + m]).transpose(0, 1) for x in (k, v))                  # (G, m, D)
        key_at += m
        for n, length in sequences[s:s + size]:
            sk, sv = (torch.cat([p, _exact_values(x[own_at:own_at + length]).transpose(0, 1)], dim=1) for p, x in ((pk, k), (pv, v)))
            own_at += length
            if n:
                rows = q[row:row + n].double().view(n, G, H // G, D).permute(1, 2, 0, 3)                # (G, group, n, D)
                score = torch.matmul(rows, sk.transpose(1, 2)[:, None]) * D ** -0.5
                late = torch.ones((n, m + length), dtype=torch.bool, device="cuda").triu(m + length - n + 1)
                p = torch.softmax(score.masked_fill(late, -math.inf), dim=3)
                out[row:row + n] = torch.matmul(p, sv[:, None]).permute(2, 0, 1, 3).reshape(n, H, D)
            row += n
        s += size
    return out


def _exact_norm(case, seed):
    x, residual, gate, w = _norm_inputs(case, seed)

    def normed(a, weight, bias):
        mean = a.mean(dim=1, keepdim=True) if case["centred"] else 0.0
        spread = torch.linalg.vector_norm(a - mean, dim=1, keepdim=True) / case["columns"] ** 0.5
        y = (a - mean) * weight.double() / torch.hypot(spread, torch.full_like(spread, EPS ** 0.5))
        return y if bias is None else y + bias.double()

    y = x.double()
    if case["post"]:
        y = normed(y, w["post_weight"], w.get("post_bias"))
    if gate is not None:
        y = y * gate.double()
    r = residual.double() + (0.5 if case["post"] else 1.0) * y
    return normed(r.half().double() if case["half"] else r, w["weight"], w.get("bias")), r


def _exact_sample(case, seed):
    logits, _, settings = _sample_inputs(case, seed)
    out = torch.zeros(logits.shape, dtype=torch.float64, device="cuda")
    for r in range(case["rows"]):
        x = logits[r].double()
        t, k, p, low = (float(settings[n][r]) if n in settings else d for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)))
        if t <= 0:
            out[r, (x == x.max()).nonzero()[0, 0]] = 1.0
            continue
        chosen = torch.softmax(x / t, dim=0)
        chosen, index = torch.sort(chosen[torch.isfinite(x)], descending=True, stable=True)[0], torch.sort(x, descending=True, stable=True)[1]
        n = min(int(k), len(chosen)) if k > 0 else len(chosen)
        if p < 1:
            mass = chosen[:n].cumsum(0)
            n = min(n, 1 + int((mass < p * mass[-1]).sum()))
        n = max(1, min(n, int((chosen >= low * chosen[0]).sum())))
        out[r, index[:n]] = chosen[:n] / chosen[:n].sum()
    return out


def exact(case, seed):
    if case["kind"] == "shared":
        return _exact_shared(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(case, seed)
    return None if case["kept"] == "none" else (None, _exact_sample(case, seed))
