"""Ends of sections at sizes where a block's exponentials or logits lie in several slabs (more than 4 GB for a block's tokens), d_h is summed in several parts, and tokens
go in several blocks by themselves; against 64 bits, a block of rows at a time.  Bounds as in test_gpu_head.py, by norm: roundings to bf16 that are independent (2^-7 of the norm),
fp32 sums of 64 products and their exponentials (2^-17)."""
import pytest
import torch

from paper_2605_10501_amd import binding as B

pytestmark = pytest.mark.gpu


def _inputs(dtype, n, d, vocab, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.empty(n, d, device="cuda").normal_(0, 1, generator=g)
    w = torch.empty(vocab, d, device="cuda").normal_(0, 0.2, generator=g)
    labels = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[:2], labels[2:4], labels[4:900:3] = vocab - 1, 0, -1                       # the last column, the first, tokens left out
    return h.to(dtype), w.to(dtype), labels, torch.empty(n, device="cuda").normal_(0, 1, generator=g)


def _exact(h, w, labels, g, rows=1024):
    """logp, d_h, d_w of sum g logp in 64 bits."""
    w64, ok = w.double(), labels >= 0
    logp, d_h, d_w = torch.zeros(len(g), device="cuda", dtype=torch.float64), torch.zeros(h.shape, device="cuda", dtype=torch.float64), torch.zeros(w.shape, device="cuda", dtype=torch.float64)
    at = torch.nonzero(ok).view(-1)
    for i in range(0, at.numel(), rows):
        a = at[i:i + rows]
        lq = torch.log_softmax(h[a].double() @ w64.T, 1)
        r = torch.arange(a.numel(), device="cuda")
        logp[a] = lq[r, labels[a].long()]
        dz = lq.exp_().neg_()
        dz[r, labels[a].long()] += 1.0
        dz *= g[a].double()[:, None]
        d_h[a] = dz @ w64
        d_w += dz.T @ h[a].double()
    return logp, d_h, d_w


def _near(got, ref, tol):
    assert torch.isfinite(got).all() and ((got.double() - ref).norm() <= tol * ref.norm()).item(), ((got.double() - ref).norm() / ref.norm()).item()


@pytest.mark.parametrize("dtype,n,d,vocab", [(torch.bfloat16, 8200, 64, 270336 + 8), (torch.bfloat16, 8200, 40, 140000), (torch.float32, 4200, 40, 270336)])
def test_several_slabs(dtype, n, d, vocab):
    h, w, labels, g = _inputs(dtype, n, d, vocab)
    logp, d_h, d_w = _exact(h, w, labels, g)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w)
    assert (out["logp"].double() - logp).abs().max().item() < 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256)      # |h| . |w| below 20
    tol = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -17
    _near(out["d_h"], d_h, tol)
    _near(got_w, d_w, tol)
    assert torch.equal(B.token_logprobs(h, w, labels), out["logp"])                   # (a forward pass has other slabs)
    half_w = torch.zeros(vocab, d, device="cuda")
    half = B.token_logprobs_backward(h, w, labels, g, d_w=half_w, token_block=4096)
    assert torch.equal(half["logp"], out["logp"])
    _near(half["d_h"], d_h, tol)
    _near(half_w, d_w, tol)


def test_top_logits_in_several_blocks_and_slabs():
    """Logits of 4 GB in blocks of tokens; one block of all tokens has several slabs."""
    n, d, vocab = 6000, 64, 200000
    h, w, _, _ = _inputs(torch.bfloat16, n, d, vocab)
    h, w = torch.round(h * 4) / 4, torch.round(w * 64) / 64                            # exact fp32 sums
    for block in (0, 6000):
        values, ids, lse = B.top_logits(h, w, 40, token_block=block)
        for i in range(0, n, 1500):
            z = h[i:i + 1500].double() @ w.double().T
            assert (torch.logsumexp(z, 1) - lse[i:i + 1500].double()).abs().max().item() < 1e-5
            s, at = torch.sort(z, dim=1, descending=True, stable=True)
            assert torch.equal(values[i:i + 1500].double(), s[:, :40]) and torch.equal(ids[i:i + 1500].long(), at[:, :40])


@pytest.mark.parametrize("n", [1, 70, 700])
def test_few_tokens_of_a_large_vocabulary(n):
    """d_h in many parts of the vocabulary."""
    d, vocab = 1536, 151936
    h, w, labels, g = _inputs(torch.bfloat16, max(n, 4), d, vocab, seed=n)
    h, labels, g, w = h[-n:].contiguous(), labels[-n:].contiguous(), g[-n:].contiguous(), (w * 0.1).contiguous()
    labels[-1] = 151935
    logp, d_h, d_w = _exact(h, w, labels, g)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w)
    assert (out["logp"].double() - logp).abs().max().item() < 2.0 ** -24 * (2 * d * 30 + 4 * 30 + 256)
    _near(out["d_h"], d_h, 2.0 ** -7)
    _near(got_w, d_w, 2.0 ** -7)
    again_w = torch.zeros(vocab, d, device="cuda")
    again = B.token_logprobs_backward(h, w, labels, g, d_w=again_w)
    assert torch.equal(again_w, got_w) and torch.equal(again["d_h"], out["d_h"])        # the same bits


def test_many_rows_of_one_id():
    """Rows of d_w that many tokens share: a label of 600 tokens, one of 300, one of 20, the rest once or twice; and more rows than one launch looks through."""
    for n in (2000, 9000):
        h, w, labels, g = _inputs(torch.bfloat16, n, 128, 4096, seed=n)
        labels[:600], labels[700:1000], labels[1000:1020] = 7, 8, 4095
        logp, d_h, d_w = _exact(h, w, labels, g)
        got_w = torch.zeros(4096, 128, device="cuda")
        out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w)
        _near(out["d_h"], d_h, 2.0 ** -8)                                             # (the labels' part is completed in fp32: one rounding, that of d_h)
        _near(got_w, d_w, 2.0 ** -8)
        for v in (7, 8, 4095):
            _near(got_w[v], d_w[v], 2.0 ** -8)
