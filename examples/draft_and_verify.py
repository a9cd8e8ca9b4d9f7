"""Decoding that drafts and verifies with one stored model: tokens are drafted at few bits and verified at all of them.

A small decoder with random weights (quantised once by ap_quantize, so that its 3-bit and 8-bit models are kin) runs the library's
operators as a server would:

  prompt   ap_gemm, ap_cache_append (rotation and 4-bit cache), ap_attention_prompt over packed prompts of different lengths
  draft    one token per sequence and step at `draft_bits`: ap_gemv, ap_cache_append, ap_attention_cached
  verify   the drafts of all sequences at once at 8 bits, several tokens per sequence; their keys and values replace those of the
           draft in the cache; ap_verify says how many stand and draws the token after them

Needs a GPU:  python examples/draft_and_verify.py [--draft-bits 4] [--drafts 4] [--tokens 64]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_10517_amd import binding as B  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM, LAYERS, VOCABULARY, PAGE = 8, 2, 64, 2, 1024, 16
HIDDEN, MLP = HEADS * HEAD_DIM, 1024


def packed(rng, rows, columns, gain):
    w = (rng.standard_t(5, size=(rows, columns)) * gain / columns ** 0.5).astype(np.float32)
    idx, luts = B.ap_quantize(w, iters=3)
    return B.ap_pack(idx, luts)


class Decoder:
    """Weights, and the cache of one layer each."""

    def __init__(self, seed, pages, positions):
        rng = np.random.default_rng(seed)
        self.embedding = torch.from_numpy(rng.normal(size=(VOCABULARY, HIDDEN)).astype(np.float16)).cuda()
        self.layers = [{"qkv": packed(rng, (HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN, 1.5), "out": packed(rng, HIDDEN, HIDDEN, 0.7),
                        "up": packed(rng, 2 * MLP, HIDDEN, 1.0), "down": packed(rng, HIDDEN, MLP, 0.7),
                        "cache": B.KVCache(pages, KV_HEADS, HEAD_DIM, page_tokens=PAGE)} for _ in range(LAYERS)]
        self.head = packed(rng, VOCABULARY, HIDDEN, 3.0)
        self.rotary = B.rotary_table(positions, HEAD_DIM)

    def forward(self, bits, tokens, positions, slots, attend):
        """Probabilities after each of `tokens`; attend(layer's cache, q, k, v) is the attention of the call."""
        x = self.embedding[tokens].float()
        for layer in self.layers:
            h = B.ap_gemm(layer["qkv"], bits, norm(x)).view(len(tokens), HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = h[:, :HEADS], h[:, HEADS:HEADS + KV_HEADS], h[:, HEADS + KV_HEADS:]
            q, k = B.ap_cache_append(layer["cache"], k, v, slots, q=q, positions=positions, rotary=self.rotary)
            x = x + B.ap_gemm(layer["out"], bits, attend(layer["cache"], q, k, v).view(len(tokens), HIDDEN)).float()
            gate, up = B.ap_gemm(layer["up"], bits, norm(x)).float().chunk(2, dim=1)
            x = x + B.ap_gemm(layer["down"], bits, (torch.nn.functional.silu(gate) * up).half()).float()
        return torch.softmax(B.ap_gemm(self.head, bits, norm(x)).float(), dim=1)


def norm(x):
    return (x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6)).half()


def sample(p):
    return (p / torch.empty_like(p).exponential_()).argmax(dim=1)


class Session:
    """Sequences that are decoded together.  lengths: tokens whose keys and values are in the cache; last: the token after them."""

    def __init__(self, decoder, prompts, room):
        self.decoder, n = decoder, len(prompts)
        width = -(-room // PAGE)
        assert n * width <= decoder.layers[0]["cache"].pages
        pages = torch.randperm(n * width, generator=torch.Generator().manual_seed(1)).int()
        self.tables, self.room = pages.view(n, width).cuda(), room
        counts = torch.tensor([len(p) for p in prompts], dtype=torch.int32)
        starts = torch.cat([torch.zeros(1, dtype=torch.int32), counts.cumsum(0).int()]).cuda()
        positions = torch.cat([torch.arange(len(p)) for p in prompts]).cuda()
        sequence = torch.repeat_interleave(torch.arange(n), counts.long()).cuda()
        p = decoder.forward(8, torch.cat([torch.as_tensor(p) for p in prompts]).cuda(), positions, self.slots(sequence, positions),
                            lambda cache, q, k, v: B.ap_attention_prompt(q, k, v, starts))
        self.lengths = counts.cuda()
        self.last = sample(p[starts[1:].long() - 1])
        self.tokens = [list(t) + [int(x)] for t, x in zip(prompts, self.last)]

    def slots(self, sequence, positions):
        return self.tables[sequence, positions // PAGE].long() * PAGE + positions % PAGE

    def run(self, bits, tokens):
        """The model over the next tokens (sequences, n), whose keys and values go to the cache behind `lengths`."""
        sequences, n = tokens.shape
        positions = (self.lengths.long()[:, None] + torch.arange(n, device="cuda")).flatten()
        slots = self.slots(torch.arange(sequences, device="cuda").repeat_interleave(n), positions)
        p = self.decoder.forward(bits, tokens.flatten(), positions, slots,
                                 lambda cache, q, k, v: B.ap_attention_cached(cache, q, self.tables, self.lengths + n, max_length=self.room))
        return p.view(sequences, n, VOCABULARY)

    def step(self, draft_bits, drafts):
        """Drafts, verifies and keeps what stands; returns the number of accepted drafts of each sequence."""
        tokens, draft, lengths = [self.last], [], self.lengths
        for _ in range(drafts):
            p = self.run(draft_bits, tokens[-1][:, None])[:, 0]
            draft.append(p)
            tokens.append(sample(p))
            self.lengths = self.lengths + 1
        self.lengths = lengths                                  # the draft's keys and values are written over
        target = self.run(8, torch.stack(tokens, dim=1))
        drafted = torch.stack(tokens[1:], dim=1)
        new, accepted = B.ap_verify(target, torch.stack(draft, dim=1), drafted, torch.rand(drafted.shape, device="cuda"),
                                    torch.empty((len(drafted), VOCABULARY), device="cuda").exponential_())
        self.lengths = lengths + accepted + 1
        self.last = new.gather(1, accepted.long()[:, None]).squeeze(1)
        for kept, row, count in zip(self.tokens, new.tolist(), accepted.tolist()):
            kept.extend(row[:count + 1])
        return accepted


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--draft-bits", type=int, default=4)
    parser.add_argument("--drafts", type=int, default=4)
    parser.add_argument("--tokens", type=int, default=64, help="new tokens of each sequence, at least")
    args = parser.parse_args()
    torch.manual_seed(0)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, VOCABULARY, size=n) for n in (5, 33, 70, 1)]
    room = 70 + args.tokens + 2 * (args.drafts + 1)
    session = Session(Decoder(0, len(prompts) * -(-room // PAGE), room), prompts, room)
    steps = accepted = 0
    while min(len(t) - len(p) for t, p in zip(session.tokens, prompts)) < args.tokens and max(map(len, session.tokens)) + args.drafts < room:
        accepted += int(session.step(args.draft_bits, args.drafts).sum())
        steps += 1
    print("%d steps of %d drafts at %d bits: %.0f %% accepted, %.2f tokens per sequence and step" %
          (steps, args.drafts, args.draft_bits, 100 * accepted / (steps * args.drafts * len(prompts)), 1 + accepted / (steps * len(prompts))))


if __name__ == "__main__":
    main()
