"""bf16 ends of sections whose hidden size is no multiple of 64: their gradients by every tile of the products, ragged in every direction, in several parts and slabs, and in one piece where the
generic kernels are asked for.  Bounds as in test_gpu_head.py."""
import numpy as np
import pytest
import torch

from oracle import head as oracle
from paper_2605_10501_amd import binding as B
from test_gpu_head import Case, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile", [0, 256, 128, 128128, 128256, 64128, 64064, -1])
@pytest.mark.parametrize("n,d,vocab", [(300, 200, 1000), (45, 8, 4104), (700, 328, 2568), (1, 72, 8)])
@pytest.mark.parametrize("fp32_dz", [False, True])
def test_every_tile(tile, n, d, vocab, fp32_dz):
    c = Case("bf16", n, d, vocab)
    g = c.normal((n,))
    ref = oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.0, f64(g))
    h, w, labels, g = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels), c.dev(g, True)
    try:
        B.k_gemm_config(tile)
        d_w, only_w = torch.zeros(vocab, d, device="cuda"), torch.zeros(vocab, d, device="cuda")
        out = B.token_logprobs_backward(h, w, labels, g, d_w=d_w, fp32_dz=fp32_dz)
        only_h = B.token_logprobs_backward(h, w, labels, g, fp32_dz=fp32_dz)["d_h"]
        B.token_logprobs_backward(h, w, labels, g, d_w=only_w, need_d_h=False, fp32_dz=fp32_dz)
    finally:
        B.k_gemm_config(0)
    assert np.all(np.abs(f64(out["logp"]) - ref["logp"]) <= c.delta())
    c.check_gradients(ref, out["d_h"], d_w)
    assert torch.equal(only_h, out["d_h"]) and torch.equal(only_w, d_w)


@pytest.mark.parametrize("n", [1, 70, 700])
def test_few_tokens_of_a_large_vocabulary(n):
    """d_h in many parts of the vocabulary, the last one ragged."""
    from test_gpu_head_large import _exact, _inputs, _near
    d, vocab = 1000, 100008
    h, w, labels, g = _inputs(torch.bfloat16, max(n, 4), d, vocab, seed=n)
    h, labels, g, w = h[-n:].contiguous(), labels[-n:].contiguous(), g[-n:].contiguous(), (w * 0.1).contiguous()
    labels[-1] = vocab - 1
    logp, d_h, d_w = _exact(h, w, labels, g)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w)
    assert (out["logp"].double() - logp).abs().max().item() < 2.0 ** -24 * (2 * d * 30 + 4 * 30 + 256)
    _near(out["d_h"], d_h, 2.0 ** -7)
    _near(got_w, d_w, 2.0 ** -7)


def test_a_long_block_of_a_wide_head():
    """More tokens in one block than the tiles' products reach in fp32 (a preference loss of 16000 tokens of 65528): products with 64-bit offsets."""
    n, d, vocab = 16000, 65528, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.empty(n, d, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g)
    w = torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16).normal_(0, 0.002, generator=g)
    labels = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[::3] = -1
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.preference_loss_forward_backward(h, w, labels, B.Batch([0, n // 2, n]), 0.01, d_w=d_w)
    ok, sign = (labels >= 0).double(), torch.where(torch.arange(n, device="cuda") < n // 2, 1.0, -1.0).double()
    lq = torch.cat([torch.log_softmax(x.double() @ w.double().T, 1) for x in h.split(2000)])
    at = labels.long().clamp(min=0)[:, None]
    margin = (lq.gather(1, at)[:, 0] * ok * sign).sum()
    slope = -0.01 * torch.sigmoid(-0.01 * margin) * ok * sign
    dz = (-lq.exp()).scatter_add_(1, at, torch.ones_like(ok)[:, None]) * slope[:, None]
    assert abs(out["margin"].item() - margin.item()) <= n * 2.0 ** -24 * (2 * d * 2 + 256)                      # |h| . |w| below 2 (each token's bound, all of one sign)
    for a in range(0, n, 2000):
        exact = dz[a:a + 2000] @ w.double()
        assert ((out["d_h"][a:a + 2000].double() - exact).norm() <= 2.0 ** -7 * exact.norm()).item()
    exact = sum(x.T @ y.double() for x, y in zip(dz.split(2000), h.split(2000)))
    assert ((d_w.double() - exact).norm() <= 2.0 ** -7 * exact.norm()).item()
