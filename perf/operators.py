"""The operators of a decoder step beside the any-precision products, as cases for timing them: keys and values rotated and
appended to a paged 4-bit cache, attention of new tokens over that cache, causal attention over packed prompts, and verification
of drafted tokens.

Head layouts are those of the decoder layers that the benchmark's matrices come from (4096, 5120 and 8192 columns: 32, 40 and 64
heads of 128, the last with 8 key heads: its 1024 x 8192 matrix) and smaller ones.  Activations are binary16 like everywhere
in the library; every case is drawn from its seed alone, its lengths from the case itself.

With `own` false the operators are computed in elementary torch operations in binary32, with it true by the library.
"""
import math
import random

import torch

own = False

ROTARY_BASE = 10000.0
KEY_OUTLIERS = 8.0                  # keys have a few channels much larger than the others


def listed():
    return [
        # One new token of one sequence through a 7B layer: nothing but latency.
        {"name": "append_1_token", "kind": "append", "sequences": 1, "longest": 1, "past": 1000, "heads": 32, "kv_heads": 32, "head_dim": 128,
         "rot_dim": 128, "interleaved": False, "fused": True, "padded": False, "page": 64},
        # Five prompts of a 70B layer enter the cache at once, q, k and v as views of the fused projection's output.
        {"name": "append_prompts", "kind": "append", "sequences": 5, "longest": 3001, "past": 0, "heads": 64, "kv_heads": 8, "head_dim": 128,
         "rot_dim": 128, "interleaved": False, "fused": True, "padded": True, "page": 64},
        # The most ordinary call: one query over a thousand tokens of a 7B layer, a key head per head.
        {"name": "cached_1x1000", "kind": "cached", "sequences": 1, "queries": 1, "longest": 1000, "ragged": False, "heads": 32, "kv_heads": 32,
         "head_dim": 128, "page": 64},
        # A batch of chats of different lengths through a 70B layer, some batch places idle.
        {"name": "cached_ragged_32", "kind": "cached", "sequences": 32, "queries": 1, "longest": 4099, "ragged": True, "heads": 64, "kv_heads": 8,
         "head_dim": 128, "page": 64},
        # Up to four drafted tokens and one more of each of eight sequences, heads of 64.
        {"name": "cached_drafts_8x5", "kind": "cached", "sequences": 8, "queries": 5, "longest": 16001, "ragged": True, "heads": 16, "kv_heads": 4,
         "head_dim": 64, "page": 16},
        # Two long documents: few rows, a long axis.
        {"name": "cached_long", "kind": "cached", "sequences": 2, "queries": 1, "longest": 131072, "ragged": False, "heads": 64, "kv_heads": 8,
         "head_dim": 128, "page": 128},
        # A short prompt through a 7B layer.
        {"name": "prompt_64", "kind": "prompt", "sequences": 1, "longest": 64, "prefix": 0, "ragged": False, "heads": 32, "kv_heads": 32,
         "head_dim": 128, "fused": True},
        # Prompts of different lengths in one call, through a 13B layer.
        {"name": "prompt_packed", "kind": "prompt", "sequences": 6, "longest": 2047, "prefix": 0, "ragged": True, "heads": 40, "kv_heads": 40,
         "head_dim": 128, "fused": True},
        # The next 500 tokens of prompts that are computed piece by piece, heads of 64.
        {"name": "prompt_pieces", "kind": "prompt", "sequences": 3, "longest": 500, "prefix": 7000, "ragged": True, "heads": 16, "kv_heads": 4,
         "head_dim": 64, "fused": False},
        # One long prompt through a 70B layer: the most work.
        {"name": "prompt_8192", "kind": "prompt", "sequences": 1, "longest": 8192, "prefix": 0, "ragged": False, "heads": 64, "kv_heads": 8,
         "head_dim": 128, "fused": True},
        # Four drafted tokens of one sequence, probabilities as a sampler leaves them.
        {"name": "verify_1", "kind": "verify", "sequences": 1, "drafts": 4, "vocabulary": 32000, "half": False, "ragged": False},
        # A batch of sequences with up to seven drafts each and a large vocabulary of an odd size, binary16 probabilities.
        {"name": "verify_64", "kind": "verify", "sequences": 64, "drafts": 7, "vocabulary": 131071, "half": True, "ragged": True},
    ]


def _spread(rng, lo, hi):
    """A whole number in lo..hi, uniform in its logarithm."""
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8, 8, 32, 40])
    group = 1 if kv > 8 else rng.choice([1, 2, 3, 4, 5, 7, 8])
    return {"heads": kv * group, "kv_heads": kv, "head_dim": rng.choice([64, 128, 128])}


def draw(rng):
    kind = rng.choice(["append", "cached", "cached", "prompt", "prompt", "verify"])
    while True:
        if kind == "append":
            c = dict({"kind": kind, "sequences": _spread(rng, 1, 64), "longest": rng.choice([1, 1, rng.randint(2, 9), _spread(rng, 10, 8191)]),
                      "past": rng.choice([0, rng.randint(1, 8000)])}, **_heads(rng))
            c["rot_dim"] = rng.choice([0, c["head_dim"] // 2, c["head_dim"], c["head_dim"]])
            c.update(interleaved=rng.random() < 0.3, fused=rng.random() < 0.6, padded=rng.random() < 0.4, page=rng.choice([16, 32, 64, 128]))
        elif kind == "cached":
            c = dict({"kind": kind, "sequences": _spread(rng, 1, 64), "queries": rng.choice([1, 1, 1, 2, 3, 5, 8, 17]),
                      "longest": _spread(rng, 17, 131072), "ragged": rng.random() < 0.7, "page": rng.choice([16, 32, 64, 128])}, **_heads(rng))
        elif kind == "prompt":
            c = dict({"kind": kind, "sequences": _spread(rng, 1, 16), "longest": _spread(rng, 1, 8192), "prefix": rng.choice([0, 0, _spread(rng, 1, 8192)]),
                      "ragged": rng.random() < 0.7}, **_heads(rng))
            c["fused"] = c["prefix"] == 0 and rng.random() < 0.6
        else:
            return {"kind": kind, "sequences": _spread(rng, 1, 64), "drafts": rng.randint(1, 8), "vocabulary": _spread(rng, 1000, 131071),
                    "half": rng.random() < 0.5, "ragged": rng.random() < 0.5}
        most = {"append": "append_prompts", "cached": "cached_long", "prompt": "prompt_8192"}[kind]
        limit = work(next(x for x in listed() if x["name"] == most))
        w = work(c)
        if w["bytes"] <= limit["bytes"] and w["flops"] <= limit["flops"]:
            return c


def _lengths(case):
    """What a case's sequences hold: append, prompt: (new tokens, tokens before them); cached: (query tokens, tokens in the cache)."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n, longest = case["sequences"], case["longest"]
    if case["kind"] == "append":
        return [(longest if i == 0 else rng.randint(1, longest), case["past"] and rng.randint(1, case["past"])) for i in range(n)]
    if case["kind"] == "cached":
        out = []
        for i in range(n):
            length = longest if i == 0 or not case["ragged"] else 0 if rng.random() < 0.08 else rng.randint(1, longest)
            out.append((rng.randint(1, case["queries"]) if case["ragged"] else case["queries"], length))
        return out
    return [(longest if i == 0 or not case["ragged"] else rng.randint(0, longest), case["prefix"] and rng.randint(0, case["prefix"])) for i in range(n)]


def _pairs(queries, keys):
    """Pairs of a causal sequence whose last query sees all keys."""
    seen = [max(0, keys - queries + 1 + i) for i in (0, queries - 1)] if queries else [0, 0]
    rows = min(queries, keys)
    return (seen[1] + seen[1] - rows + 1) * rows // 2


def work(case):
    if case["kind"] == "verify":
        row = case["vocabulary"] * (2 if case["half"] else 4)
        return {"bytes": case["sequences"] * (2 * row + 4 * case["vocabulary"] + 32 * case["drafts"]), "flops": 3 * case["sequences"] * case["vocabulary"]}
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    lengths = _lengths(case)
    new = sum(a for a, _ in lengths)
    if case["kind"] == "append":                 # q, k, v read; q, k and the cache's values written; the cache's bytes both ways
        return {"bytes": new * (2 * D * (H + 2 * G) + 2 * D * (H + 3 * G) + 2 * G * (D + 8) + 4 * case["rot_dim"]),
                "flops": new * (3 * case["rot_dim"] * (H + G) + 12 * D * G)}
    if case["kind"] == "cached":
        return {"bytes": sum(b for _, b in lengths) * G * (D + 8) + 4 * new * H * D, "flops": 4 * H * D * sum(_pairs(a, b) for a, b in lengths)}
    keys = sum(a + b for a, b in lengths)
    return {"bytes": 4 * new * H * D + 4 * keys * G * D, "flops": 4 * H * D * sum(_pairs(a, a + b) for a, b in lengths)}


# ---------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)


def _qkv(gen, tokens, H, G, D, fused):
    """q, k, v of (tokens, heads, head_dim): views of one projection's output, or tensors of their own."""
    if fused:
        x = _normal(gen, tokens, H + 2 * G, D)
        q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    else:
        q, k, v = _normal(gen, tokens, H, D), _normal(gen, tokens, G, D), _normal(gen, tokens, G, D)
    k[:, :, D // 3] *= KEY_OUTLIERS
    return q, k, v


def _pages(case, lengths):
    """A page table (sequence, page) of pages in no order, and the number of pages."""
    P = case["page"]
    rng = random.Random(len(lengths) * 1000 + P)
    need = [-(-n // P) for n in lengths]
    order = list(range(sum(need) + 3))
    rng.shuffle(order)
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table, len(order)


def _slots(table, sequence, first, last, page):
    """Cache places of tokens first..last-1 of a sequence."""
    t = torch.arange(first, last)
    return table[sequence, t // page].long() * page + t % page


def _rotary(rows, rot_dim):
    """(position, rot_dim): cosines, then sines, of position / base^(2 i / rot_dim)."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * ROTARY_BASE ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().cuda()


def _append_inputs(case, seed):
    gen, H, G, D = _generator(seed), case["heads"], case["kv_heads"], case["head_dim"]
    lengths = _lengths(case)
    table, pages = _pages(case, [a + b for a, b in lengths])
    slots = torch.cat([_slots(table, i, b, a + b, case["page"]) for i, (a, b) in enumerate(lengths)])
    if case["padded"]:
        slots[-(len(slots) // 9 + 1):] = -1      # the tail of a padded batch is not kept
    positions = torch.cat([torch.arange(b, a + b) for a, b in lengths])
    q, k, v = _qkv(gen, len(slots), H, G, D, case["fused"])
    rotary = _rotary(int(positions.max()) + 1, case["rot_dim"]) if case["rot_dim"] else None
    return q, k, v, positions.cuda(), slots.cuda(), rotary, pages


def _cached_inputs(case, seed):
    gen, H, G, D = _generator(seed), case["heads"], case["kv_heads"], case["head_dim"]
    lengths = _lengths(case)
    table, pages = _pages(case, [b for _, b in lengths])
    slots = torch.cat([_slots(table, i, 0, b, case["page"]) for i, (_, b) in enumerate(lengths)]).cuda()
    q = _normal(gen, sum(a for a, _ in lengths), H, D)
    _, k, v = _qkv(gen, len(slots), 0, G, D, False)
    return q, k, v, slots, table, pages


def _prompt_inputs(case, seed):
    gen, H, G, D = _generator(seed), case["heads"], case["kv_heads"], case["head_dim"]
    lengths = _lengths(case)
    queries, keys = sum(a for a, _ in lengths), sum(a + b for a, b in lengths)
    if case["fused"]:
        return _qkv(gen, queries, H, G, D, True)
    q, (_, k, v) = _normal(gen, queries, H, D), _qkv(gen, keys, 0, G, D, False)
    return q, k, v


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _verify_inputs(case, seed):
    gen, S, N, V = _generator(seed), case["sequences"], case["drafts"], case["vocabulary"]
    logits = torch.randn((S, N + 1, V), generator=gen, device="cuda") * 2.5
    target = torch.softmax(logits, dim=2)
    logits[:, :N] += torch.randn((S, N, V), generator=gen, device="cuda") * 0.4     # the model at fewer bits
    draft = torch.softmax(logits[:, :N], dim=2)
    del logits
    if case["half"]:
        target, draft = target.half(), draft.half()
    drafted = torch.multinomial(draft.reshape(S * N, V).float(), 1, generator=gen).reshape(S, N)
    uniform = torch.rand((S, N), generator=gen, device="cuda")
    noise = torch.empty((S, V), device="cuda").exponential_(generator=gen)
    rng = random.Random(seed)
    counts = [rng.randint(0, N) if case["ragged"] else N for _ in range(S)]
    return target, draft, drafted, uniform, noise, torch.tensor(counts, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    kind, state = case["kind"], {"kind": case["kind"], "own": own}
    if own:
        from paper_2402_10517_amd import binding as B
        state["B"] = B
    G, D = case.get("kv_heads"), case.get("head_dim")
    if kind == "append":
        q, k, v, positions, slots, rotary, pages = _append_inputs(case, seed)
        state.update(q=q, k=k, v=v, positions=positions, slots=slots, rotary=rotary, interleaved=case["interleaved"])
        if own:
            state["cache"] = B.KVCache(pages, G, D, page_tokens=case["page"])
        else:
            state["cache"] = _plain_cache(pages * case["page"], G, D)
    elif kind == "cached":
        q, k, v, slots, table, pages = _cached_inputs(case, seed)
        lengths = _lengths(case)
        state.update(q=q, table=table.cuda(), scale=D ** -0.5, page=case["page"], counts=[a for a, _ in lengths], keys=[b for _, b in lengths])
        state["lengths"] = torch.tensor(state["keys"], dtype=torch.int32, device="cuda")
        state["starts"] = None                   # as many query tokens in every sequence
        if len(set(state["counts"])) > 1:
            state["starts"] = torch.tensor(_starts(state["counts"]), dtype=torch.int32, device="cuda")
        state["longest"] = max(state["keys"])
        if own:
            state["cache"] = B.KVCache(pages, G, D, page_tokens=case["page"])
            B.ap_cache_append(state["cache"], k, v, slots)
        else:
            state["cache"] = _plain_cache(pages * case["page"], G, D)
            step = 1 << 16
            for i in range(0, len(slots), step):
                _plain_store(state["cache"], slots[i:i + step], k[i:i + step], v[i:i + step])
    elif kind == "prompt":
        q, k, v = _prompt_inputs(case, seed)
        lengths = _lengths(case)
        state.update(q=q, k=k, v=v, scale=D ** -0.5, queries=_starts([a for a, _ in lengths]), keys=_starts([a + b for a, b in lengths]))
        state["q_starts"] = torch.tensor(state["queries"], dtype=torch.int32, device="cuda")
        state["k_starts"] = torch.tensor(state["keys"], dtype=torch.int32, device="cuda")
    else:
        target, draft, drafted, uniform, noise, counts = _verify_inputs(case, seed)
        state.update(target=target, draft=draft, drafted=drafted, uniform=uniform, noise=noise, counts=counts)
    return state


# ---------------------------------------------------------------------------------------------------- plain forms


def _plain_cache(places, G, D):
    return {"k": torch.zeros((places, G, D), dtype=torch.uint8, device="cuda"), "v": torch.zeros((places, G, D), dtype=torch.uint8, device="cuda"),
            "k_low": torch.zeros((places, G, 1), dtype=torch.float16, device="cuda"), "v_low": torch.zeros((places, G, 1), dtype=torch.float16, device="cuda"),
            "k_scale": torch.zeros((places, G, 1), dtype=torch.float16, device="cuda"),
            "v_scale": torch.zeros((places, G, 1), dtype=torch.float16, device="cuda")}


def _plain_codes(x):
    """16 evenly spaced values per token and head, from its least value on: (codes, least value, step)."""
    x = x.float()
    low, high = x.amin(dim=2, keepdim=True), x.amax(dim=2, keepdim=True)
    scale = ((high - low) / torch.full_like(low, 15.0)).half()
    step = scale.float()
    codes = torch.where(step > 0, (x - low) / torch.where(step > 0, step, torch.ones_like(step)), torch.zeros_like(x)).round().clamp(0, 15)
    return codes.to(torch.uint8), low.half(), scale


def _plain_store(cache, slots, k, v):
    kept = slots >= 0
    for side, x in (("k", k), ("v", v)):
        codes, low, scale = _plain_codes(x[kept])
        cache[side][slots[kept]] = codes
        cache[side + "_low"][slots[kept]] = low
        cache[side + "_scale"][slots[kept]] = scale


def _plain_values(cache, side, slots):
    return cache[side][slots].float() * cache[side + "_scale"][slots].float() + cache[side + "_low"][slots].float()


def _plain_rotate(x, rows, interleaved):
    """x (tokens, heads, head_dim), rows (tokens, rot_dim) of the rotary table; the channels after rot_dim stay."""
    if rows is None:
        return x.clone()
    half = rows.shape[1] // 2
    cos, sin = rows[:, None, :half], rows[:, None, half:]
    out = x.float()
    part = out[:, :, :2 * half]
    first, second = (part[:, :, 0::2], part[:, :, 1::2]) if interleaved else (part[:, :, :half], part[:, :, half:])
    a, b = first * cos - second * sin, second * cos + first * sin
    if interleaved:
        rotated = torch.stack([a, b], dim=3).flatten(2)
    else:
        rotated = torch.cat([a, b], dim=2)
    return torch.cat([rotated, out[:, :, 2 * half:]], dim=2).half()


def _plain_attention(q, k, v, scale):
    """q (queries, heads, head_dim), k, v (keys, kv heads, head_dim) in binary32; the last query sees all keys."""
    n, H, D = q.shape
    m, G, _ = k.shape
    if m == 0 or n == 0:
        return torch.zeros_like(q)
    out = torch.empty_like(q)
    row = torch.arange(n, device=q.device)[:, None] + (m - n)
    seen = torch.arange(m, device=q.device)[None, :] <= row
    for g in range(G):
        heads = slice(g * (H // G), (g + 1) * (H // G))
        score = torch.matmul(q[:, heads].transpose(0, 1), k[:, g].t()) * scale
        score = score.masked_fill(~seen, float("-inf"))
        top = score.amax(dim=2, keepdim=True)
        p = torch.exp(score - torch.where(top == float("-inf"), torch.zeros_like(top), top))
        total = p.sum(dim=2, keepdim=True)
        o = torch.matmul(p, v[:, g]) / torch.where(total == 0, torch.ones_like(total), total)
        out[:, heads] = o.transpose(0, 1)
    return out


def _run_plain(s):
    if s["kind"] == "append":
        rows = None if s["rotary"] is None else s["rotary"][s["positions"]]
        q, k = _plain_rotate(s["q"], rows, s["interleaved"]), _plain_rotate(s["k"], rows, s["interleaved"])
        _plain_store(s["cache"], s["slots"], k, s["v"])
        kept = (s["slots"] >= 0)[:, None, None]
        at = s["slots"].clamp(min=0)
        back = [torch.where(kept, _plain_values(s["cache"], side, at), torch.zeros((), device="cuda")).half() for side in ("k", "v")]
        return q, k, back[0], back[1]
    if s["kind"] == "cached":
        out, at = [], 0
        for i, (n, m) in enumerate(zip(s["counts"], s["keys"])):
            t = torch.arange(m, device="cuda")
            slots = s["table"][i, t // s["page"]].long() * s["page"] + t % s["page"]
            out.append(_plain_attention(s["q"][at:at + n].float(), _plain_values(s["cache"], "k", slots), _plain_values(s["cache"], "v", slots),
                                        s["scale"]).half())
            at += n
        return torch.cat(out)
    if s["kind"] == "prompt":
        out = []
        for q0, q1, k0, k1 in zip(s["queries"], s["queries"][1:], s["keys"], s["keys"][1:]):
            out.append(_plain_attention(s["q"][q0:q1].float(), s["k"][k0:k1].float(), s["v"][k0:k1].float(), s["scale"]).half())
        return torch.cat(out)
    target, draft, drafted, counts = s["target"], s["draft"], s["drafted"], s["counts"].long()
    S, N, V = draft.shape
    p = target[:, :N].gather(2, drafted[:, :, None]).squeeze(2).float()
    q = draft.gather(2, drafted[:, :, None]).squeeze(2).float()
    place = torch.arange(N, device="cuda")[None, :]
    accepted = ((s["uniform"] * q < p) & (place < counts[:, None])).long().cumprod(dim=1).sum(dim=1)
    row = torch.arange(S, device="cuda")
    full = target[row, accepted].float()
    rest = (full - draft[row, accepted.clamp(max=N - 1)].float()).clamp(min=0)
    refused = (accepted < counts)[:, None] & (rest.amax(dim=1, keepdim=True) > 0)
    ratio = torch.where(refused, rest, full) / s["noise"]
    best = ratio.amax(dim=1, keepdim=True)
    token = torch.where(ratio == best, torch.arange(V, device="cuda")[None, :], V).amin(dim=1)
    place = torch.arange(N + 1, device="cuda")[None, :]
    tokens = torch.where(place < accepted[:, None], torch.cat([drafted, drafted[:, :1]], dim=1), -1)
    return torch.where(place == accepted[:, None], token[:, None], tokens), accepted.int()


def run(state):
    s = state
    if not s["own"]:
        return _run_plain(s)
    B = s["B"]
    if s["kind"] == "append":
        q, k = B.ap_cache_append(s["cache"], s["k"], s["v"], s["slots"], q=s["q"], positions=s["positions"], rotary=s["rotary"],
                                 interleaved=s["interleaved"])
        return (q, k) + B.ap_cache_read(s["cache"], s["slots"])
    if s["kind"] == "cached":
        return B.ap_attention_cached(s["cache"], s["q"], s["table"], s["lengths"], q_starts=s["starts"], max_length=s["longest"], scale=s["scale"])
    if s["kind"] == "prompt":
        return B.ap_attention_prompt(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], scale=s["scale"])
    return B.ap_verify(s["target"], s["draft"], s["drafted"], s["uniform"], s["noise"], counts=s["counts"])


# ---------------------------------------------------------------------------------------------------- definition in 64 bits


def _exact_values(x):
    """What the cache stands for, from the definition: low + step * nearest of 0..15, low and step binary16."""
    x = x.double()
    low, high = x.min(dim=-1, keepdim=True).values, x.max(dim=-1, keepdim=True).values
    step = ((high - low) / 15).half().double()
    code = torch.nan_to_num((x - low) / step, nan=0.0).round().clamp(0, 15)
    return low + step * code


def _exact_attention(q, k, v, scale):
    """One head: q (n, D), k, v (m, D) in 64 bits."""
    n, m = len(q), len(k)
    out = torch.zeros_like(q)
    first = max(0, n - m)                        # queries before it see nothing
    if first == n:
        return out
    score = (q[first:] @ k.t()) * scale
    late = torch.ones_like(score, dtype=torch.bool).triu(m - n + first + 1)
    out[first:] = torch.softmax(score.masked_fill(late, -math.inf), dim=1) @ v
    return out


def _exact_sequences(q, k, v, queries, keys, scale):
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    group = q.shape[1] // k.shape[1]
    for q0, q1, k0, k1 in zip(queries, queries[1:], keys, keys[1:]):
        for h in range(q.shape[1]):
            out[q0:q1, h] = _exact_attention(q[q0:q1, h].double(), k[k0:k1, h // group].double(), v[k0:k1, h // group].double(), scale)
    return out


def exact(case, seed):
    if case["kind"] == "verify":
        return None                              # whole numbers
    scale = case["head_dim"] ** -0.5
    lengths = _lengths(case)
    if case["kind"] == "prompt":
        q, k, v = _prompt_inputs(case, seed)
        return _exact_sequences(q, k, v, _starts([a for a, _ in lengths]), _starts([a + b for a, b in lengths]), scale)
    if case["kind"] == "cached":
        q, k, v, _, _, _ = _cached_inputs(case, seed)
        return _exact_sequences(q, _exact_values(k), _exact_values(v), _starts([a for a, _ in lengths]), _starts([b for _, b in lengths]), scale)
    q, k, v, positions, slots, rotary, _ = _append_inputs(case, seed)
    values = torch.where((slots >= 0)[:, None, None], _exact_values(v), torch.zeros((), dtype=torch.float64, device="cuda"))
    q, k = q.double(), k.double()
    if rotary is None:
        return q, k, torch.where((slots >= 0)[:, None, None], _exact_values(k), torch.zeros((), dtype=torch.float64, device="cuda")), values
    R = case["rot_dim"]
    turn = torch.complex(rotary[positions, :R // 2].double(), rotary[positions, R // 2:].double())[:, None, :]
    even, odd = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    out = []
    for x in (q, k):
        z = torch.complex(x[:, :, even].contiguous(), x[:, :, odd].contiguous()) * turn
        x = x.clone()
        x[:, :, even], x[:, :, odd] = z.real, z.imag
        out.append(x)
    # the cached keys are codes of the rotated keys after their rounding: they jump where that rounding does, and have no 64-bit value
    return out[0], out[1], None, values
