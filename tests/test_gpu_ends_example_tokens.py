"""The example's fine-tuning step where tokens are none: sequences without any, and indices behind the vocabulary."""
import pytest
import torch

from test_gpu_block_example import load
from test_gpu_ends_together import make

pytestmark = pytest.mark.gpu


def run(token):
    ex = load()
    gen = torch.Generator(device="cuda").manual_seed(6)
    t = make(ex, gen, True)
    h = torch.randn((33, 256), generator=gen, device="cuda")
    loss, norm = t.step(h, token, ex.rotation(33, 64), 1e-2)
    return loss, norm, list(t.grads.values())


def test_tokens_behind_the_vocabulary_count_as_none():
    token = torch.arange(33, device="cuda").int()
    token[:10] = -1
    want = run(token)
    token[:10] = 512
    got = run(token)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(torch.equal(a, b) for a, b in zip(got[2], want[2]))


def test_a_sequence_without_tokens():
    loss, norm, grads = run(torch.full((33,), -1, dtype=torch.int32, device="cuda"))
    assert float(loss) == 0 and float(norm[0]) == 0 and not any(bool(g.any()) for g in grads)
