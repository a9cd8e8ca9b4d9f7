"""The operators of a decoder step in one run, as a server calls them for a batch behind one prompt: eager and captured."""
import numpy as np
import pytest
import torch

import decode_util as U

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, D, PAGE, VOCABULARY, SEQUENCES, PREFIX, BITS = 8, 2, 64, 16, 1024, 40, 150, 6
HIDDEN, MLP = HEADS * D, 768


@pytest.fixture(scope="module")
def B():
    from paper_2402_10517_amd import binding
    return binding


class Layer:
    def __init__(self, B, rng):
        def packed(rows, columns, gain):
            w = (rng.standard_t(5, size=(rows, columns)) * gain / columns ** 0.5).astype(np.float32)
            idx, luts = B.ap_quantize(w, iters=2)
            return B.ap_pack(idx, luts)
        self.qkv, self.out = packed((HEADS + 2 * KV_HEADS) * D, HIDDEN, 1.5), packed(HIDDEN, HIDDEN, 0.7)
        self.up, self.down, self.head = packed(2 * MLP, HIDDEN, 1.0), packed(HIDDEN, MLP, 0.7), packed(VOCABULARY, HIDDEN, 3.0)
        one = lambda: torch.from_numpy((1 + 0.1 * rng.normal(size=HIDDEN)).astype(np.float16)).cuda()  # noqa: E731
        self.first, self.second, self.last, self.post = one(), one(), one(), one()


class Plain:
    """The norm in 64 bits."""

    @staticmethod
    def norm(x, w):
        x = x.double()
        return (x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * w.double()).half()


def inputs(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn((SEQUENCES, HIDDEN), generator=g, device="cuda") * 2, torch.rand(SEQUENCES, generator=g, device="cuda"))


class Session:
    def __init__(self, B):
        self.B, self.layer = B, Layer(B, np.random.default_rng(0))
        lengths = [1 + (7 * i) % 30 for i in range(SEQUENCES)]
        table, pages = U.page_table([PREFIX] + lengths, PAGE)
        self.cache = B.KVCache(pages, KV_HEADS, D, page_tokens=PAGE)
        g = torch.Generator(device="cuda")
        g.manual_seed(9)
        n = PREFIX + sum(lengths)
        self.old = [torch.randn((n, KV_HEADS, D), generator=g, device="cuda", dtype=torch.float16) for _ in range(2)]
        self.slots = torch.cat([U.slots_of(table, PAGE, i, 0, m) for i, m in enumerate([PREFIX] + lengths)]).cuda()
        self.new = torch.cat([U.slots_of(table, PAGE, 1 + i, m - 1, m) for i, m in enumerate(lengths)]).cuda()
        self.positions = torch.tensor([PREFIX + m - 1 for m in lengths]).cuda()
        self.rotary = B.rotary_table(PREFIX + 64, D)
        self.tables = (table[:1].cuda(), torch.tensor([PREFIX], dtype=torch.int32).cuda(), table[1:].contiguous().cuda(), torch.tensor(lengths, dtype=torch.int32).cuda())
        self.temperature, self.top_k = torch.full((SEQUENCES,), 0.8).cuda(), torch.full((SEQUENCES,), 30, dtype=torch.int32).cuda()
        self.top_p, self.min_p = torch.full((SEQUENCES,), 0.95).cuda(), torch.full((SEQUENCES,), 0.01).cuda()
        self.work = torch.empty(HIDDEN * 2 * MLP * 4, dtype=torch.uint8, device="cuda")

    def fill(self):
        self.cache.buf.fill_(255)
        self.B.ap_cache_append(self.cache, *self.old, self.slots)

    def step(self, residual, uniform):
        """One token of every sequence: all operators, each result that leaves one."""
        B, w = self.B, self.layer
        h, _ = B.ap_norm(None, residual, w.first)
        h = B.ap_gemm(w.qkv, BITS, h, work=self.work).view(SEQUENCES, HEADS + 2 * KV_HEADS, D)
        q, k = B.ap_cache_append(self.cache, h[:, HEADS:HEADS + KV_HEADS], h[:, HEADS + KV_HEADS:], self.new, q=h[:, :HEADS], positions=self.positions, rotary=self.rotary)
        attended = B.ap_attention_shared(self.cache, q, *self.tables)
        block = B.ap_gemm(w.out, BITS, attended.view(SEQUENCES, HIDDEN), work=self.work)
        h, after = B.ap_norm(block, residual, w.second, post_weight=w.post, scale=0.5)
        gate, up = B.ap_gemm(w.up, BITS, h, work=self.work).chunk(2, dim=1)
        down = B.ap_gemm(w.down, BITS, (torch.nn.functional.silu(gate.float()) * up.float()).half(), work=self.work)
        last, final = B.ap_norm(down, after, w.last)
        logits = B.ap_gemm(w.head, BITS, last, work=self.work)
        tokens, p = B.ap_sample(logits, uniform, temperature=self.temperature, top_k=self.top_k, top_p=self.top_p, min_p=self.min_p, probabilities=torch.float32)
        return q, k, attended, block, h, after, down, last, final, logits, tokens, p


def test_a_step_behind_a_shared_prompt(B):
    session = Session(B)
    session.fill()
    residual, uniform = inputs(1)
    q, k, attended, block, h, after, down, last, final, logits, tokens, p = session.step(residual, uniform)
    # the same keys through the cached attention, prefix and own pages in one table (the prefix does not fill its last page: its keys are appended again)
    lengths = session.tables[3].tolist()
    table, pages = U.page_table([PREFIX + m for m in lengths], PAGE)
    cache = B.KVCache(pages, KV_HEADS, D, page_tokens=PAGE)
    at, order = PREFIX, []
    for m in lengths:
        order += list(range(PREFIX)) + list(range(at, at + m))
        at += m
    slots = torch.cat([U.slots_of(table, PAGE, i, 0, PREFIX + m) for i, m in enumerate(lengths)]).cuda()
    keys, values = (x[torch.tensor(order).cuda()] for x in session.old)
    B.ap_cache_append(cache, keys, values, slots)
    new = torch.cat([U.slots_of(table, PAGE, i, PREFIX + m - 1, PREFIX + m) for i, m in enumerate(lengths)]).cuda()
    first = Plain.norm(residual, session.layer.first)
    fused = B.ap_gemm(session.layer.qkv, BITS, B.ap_norm(None, residual, session.layer.first)[0]).view(SEQUENCES, -1, D)
    B.ap_cache_append(cache, k, fused[:, HEADS + KV_HEADS:], new)
    want = B.ap_attention_cached(cache, q, table.cuda(), torch.tensor([PREFIX + m for m in lengths], dtype=torch.int32).cuda())
    assert (attended.float() - want.float()).abs().max() <= 2.0 ** -9 * want.abs().max()
    # norms: a rounding of binary16 either way
    near = lambda a, b: ((a.float() - b.float()).abs() <= 2.0 ** -10 * b.float().abs() + 2.0 ** -24).all()  # noqa: E731
    assert near(B.ap_norm(None, residual, session.layer.first)[0], first)
    x = block.double()
    y = x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * session.layer.post.double()
    assert torch.allclose(after.double(), residual.double() + 0.5 * y, rtol=2.0 ** -20, atol=2.0 ** -20)
    assert near(h, Plain.norm(after, session.layer.second)) and near(last, Plain.norm(final, session.layer.last))
    assert torch.equal(final, after + down.float())
    assert ((p > 0).sum(1) <= 30).all() and ((p.double().sum(1) - 1).abs() < 1e-6).all() and (p.gather(1, tokens[:, None]) > 0).all()


def test_a_step_captured_and_replayed(B):
    session = Session(B)
    session.fill()
    residual, uniform = inputs(1)
    session.step(residual, uniform)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        session.step(residual, uniform)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = session.step(residual, uniform)
    other = torch.cuda.CUDAGraph()                               # a second one, of the same workspace and inputs
    with torch.cuda.graph(other):
        more = session.step(residual, uniform)
    for seed in (5, 6, 7, 8):
        fresh = inputs(seed)
        residual.copy_(fresh[0])
        uniform.copy_(fresh[1])
        session.fill()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        session.fill()
        other.replay()
        again = [o.clone() for o in more]
        session.fill()
        want = session.step(residual, uniform)
        for name, a, b, c in zip("q k attended block h after down last final logits tokens p".split(), got, again, want):
            assert torch.equal(a, c) and torch.equal(b, c), (seed, name)
