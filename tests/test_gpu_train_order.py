"""The order in which the gradient of embeddings adds, bit for bit: sorted
tokens in chunks, a chunk's terms of a row by ascending position, then the
chunks' sums over four wavefronts in turn, and these in order."""

import pytest
import torch

import ops_ref as ref
import paper_2609_25442_amd as wb
from gpu_util import say

pytestmark = pytest.mark.gpu


def in_order(d, tokens, rows, scale):
    """The gradient in fp32, one addition after the other."""
    count = len(tokens)
    chunk = 16
    while chunk < 256 and count > chunk * 512:
        chunk *= 2
    keys, order = torch.sort(torch.where((tokens >= 0) & (tokens < rows), tokens, rows), stable=True)
    out = torch.zeros(rows, d.shape[1])
    starts = [0] + (torch.nonzero(keys[1:] != keys[:-1])[:, 0] + 1).tolist() + [count]
    for lo, hi in zip(starts, starts[1:]):
        if keys[lo] == rows:
            continue
        parts, at = [], lo
        while at < hi:
            end = min(hi, (at // chunk + 1) * chunk)
            part = torch.zeros(d.shape[1])
            for t in order[at:end].tolist():
                part = part + d[t]
            parts.append(part)
            at = end
        waves = [parts[0]] + [torch.zeros(d.shape[1]) for _ in range(3)]
        for i, part in enumerate(parts[1:]):
            waves[i % 4] = waves[i % 4] + part
        total = waves[0]
        if len(parts) > 1:
            for w in waves[1:]:
                total = total + w
        out[keys[lo]] = total * torch.tensor(scale)
    return out


@pytest.mark.parametrize("count,vocab", [(1, 3), (15, 2), (16, 1), (17, 1), (200, 3), (3000, 7), (8192, 300), (8193, 2), (20000, 40), (40000, 3)])
def test_embedding_gradient_adds_in_its_order(count, vocab):
    say("order", count, vocab)
    g = torch.Generator().manual_seed(count)
    tokens = torch.randint(0, vocab + 1, (count,), generator=g)  # one of them outside
    tokens = torch.where(torch.rand(count, generator=g) < 0.4, 0, tokens)
    for cols, scale in ((9, 1.0), (8, -1.7)):
        d = ref.randn(count, cols, seed=cols) * 10.0 ** torch.randint(-3, 4, (count, 1), generator=g)
        got = wb.embedding_backward(d.cuda(), tokens.cuda(), vocab, scale=scale)
        assert torch.equal(got.cpu(), in_order(d, tokens, vocab, scale))


def test_a_row_of_one_chunk_is_added_by_ascending_position():
    """The terms cancel but for the order's roundings."""
    d = torch.tensor([[2.0 ** 24], [1.0], [1.0], [-2.0 ** 24], [3.0]]).repeat(1, 8)
    got = wb.embedding_backward(d.cuda(), torch.zeros(5, dtype=torch.int64, device="cuda"), 1)
    assert torch.all(got == 3.0)
