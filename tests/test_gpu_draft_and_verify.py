"""The example that drafts and verifies with one stored model, on a GPU."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("draft_and_verify", os.path.join(ROOT, "examples", "draft_and_verify.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def decoder(example):
    return example.Decoder(0, 4 * 8, 128)


PROMPTS = [np.arange(n) % 1000 for n in (5, 33, 70, 1)]


def test_drafts_of_the_target_itself_stand(example, decoder):
    torch.manual_seed(1)
    session = example.Session(decoder, PROMPTS, 128)
    accepted = sum(int(session.step(8, 4).sum()) for _ in range(8))
    # the same model, but for the rounding of sums in products of other batch sizes: a refusal is rare
    assert accepted >= 0.9 * 8 * 4 * 4
    for tokens, prompt, length in zip(session.tokens, PROMPTS, session.lengths.tolist()):
        assert len(tokens) == length + 1 and np.array_equal(tokens[:len(prompt)], prompt) and 0 <= min(tokens) and max(tokens) < example.VOCABULARY


def test_fewer_bits_are_accepted_less_and_leave_the_cache_the_target_s(example, decoder):
    torch.manual_seed(2)
    session = example.Session(decoder, PROMPTS, 128)
    share = {}
    for bits in (6, 3):
        share[bits] = sum(int(session.step(bits, 3).sum()) for _ in range(4)) / (4 * 4 * 3)
    assert 0.0 < share[3] < share[6] <= 1.0
    # The first layer's keys and values depend on nothing but the tokens and the model: what the steps left in its cache is what the target's own pass over the same
    # tokens leaves there, not the draft's.  Products of other batch sizes differ by a step of binary16, which takes a code across to the next where the value
    # lies within 2^-10 of their middle: fewer than one in a hundred.  (Codes of the 3-bit model are others in most places.)
    def first_layer(s):
        lengths = s.lengths.tolist()
        slots = torch.cat([s.slots(torch.full((n,), i, device="cuda"), torch.arange(n, device="cuda")) for i, n in enumerate(lengths)])
        return example.B.ap_cache_read(decoder.layers[0]["cache"], slots)
    kept = first_layer(session)
    fresh = first_layer(example.Session(decoder, [t[:-1] for t in session.tokens], 128))
    for a, b in zip(kept, fresh):
        step = (b.amax(-1, keepdim=True) - b.amin(-1, keepdim=True)).float() / 15
        assert ((a.float() - b.float()).abs() > step / 2).float().mean().item() < 0.01
