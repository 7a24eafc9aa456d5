"""Ends of sections whose fp32 gradients pass 4 GB (more than 2^30 entries): lm_heads in several slabs for that reason alone, hidden states in several blocks.  Against 64 bits, piece by piece of the
gradient, the first and the last rows by themselves; bounds as in test_gpu_head_large.py: the norm of independent roundings to bf16 stays below 2^-7 of the norm."""
import pytest
import torch

from paper_2605_10501_amd import binding as B
from test_gpu_head_large import _exact, _near

pytestmark = pytest.mark.gpu


def _inputs(n, d, vocab, std):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    h = torch.empty(n, d, device="cuda").normal_(0, 1, generator=g).bfloat16()
    w = torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16).normal_(0, std, generator=g)
    labels = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[0], labels[1], labels[2], labels[3] = vocab - 1, 0, -1, vocab // 2
    return h, w, labels, torch.empty(n, device="cuda").normal_(0, 1, generator=g)


def _check(n, d, vocab, std, block):
    h, w, labels, g = _inputs(n, d, vocab, std)
    logp, d_h, d_w = _exact(h, w, labels, g)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w, token_block=block)
    assert (out["logp"].double() - logp).abs().max().item() < 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256)      # |h| . |w| below 20
    for got, ref in ((out["d_h"], d_h), (got_w, d_w)):
        rows = len(ref)
        for a, b in [(rows * i // 16, rows * (i + 1) // 16) for i in range(16)] + [(0, 2), (rows - 1, rows)]:
            _near(got[a:b], ref[a:b], 2.0 ** -7)


# 4.6 GB; exactly 4 GB, where the size of a descriptor wraps to nothing
@pytest.mark.parametrize("n,d,vocab", [(64, 8192, 151936), (50, 4096, 262144)])
def test_gradient_of_a_large_lm_head(n, d, vocab):
    _check(n, d, vocab, 0.01, 0)


def test_gradient_of_many_hidden_states():
    """One block of as many tokens as there may be: 4.4 GB of sums would be one, if a block were as long as it is asked to be."""
    _check(270000, 4096, 1024, 0.01, 270000)
