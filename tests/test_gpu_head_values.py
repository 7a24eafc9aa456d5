"""Ends of sections where values are not as usual: NaN among the logits of a token that counts, entries of equal value, entries that are next to nothing beside the teacher's whole
vocabulary; and the same bits from the same call where many tokens meet a small lm_head."""
import numpy as np
import pytest
import torch

from oracle import head as oracle
from paper_2605_10501_amd import binding as B
from test_gpu_head import U, Case, f64

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 64), ("bf16", 40), ("fp32", 40)]


def _calls(c, h, w, d_w=None):
    """All losses of the case's labels, and log-probabilities, forward and backward: dicts.  Three pairs of sequences."""
    n = c.n
    labels, x = c.labels.cuda(), torch.full((n,), -5.0, device="cuda")
    cu = B.Batch([0, n // 6, n // 3, n // 2, 2 * n // 3, 5 * n // 6, n])
    ones = torch.ones(n, device="cuda")
    return (dict(logp=B.token_logprobs(h, w, labels)), B.token_logprobs_backward(h, w, labels, ones, d_w=d_w), B.policy_loss_forward_backward(h, w, labels, x, ones, ref_logp=x, kl_coef=0.1),
            B.preference_loss_forward_backward(h, w, labels, cu, 0.1, ref_logp=x), B.policy_loss_forward_backward(h, w, labels, x, -ones, need_d_h=False))


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("vocab", [328, 4360])
def test_nan_in_hidden_states_of_a_token_that_counts(dtype, d, vocab):
    c = Case(dtype, 60, d, vocab)
    at = int(torch.nonzero(c.ok)[5])
    pair = at // 20
    bad = c.h.clone()
    bad[at, d // 2] = float("nan")
    others = torch.ones(60, dtype=torch.bool, device="cuda")
    others[at] = False
    fine, got = _calls(c, c.h.cuda(), c.w.cuda()), _calls(c, bad.cuda(), c.w.cuda())
    for a, b in zip(fine, got):
        for k in a:
            if k == "d_h" and a[k] is not None:
                assert torch.isnan(b[k][at]).all()
            elif k in ("logp", "loss_tok"):
                assert torch.isnan(b[k][at]) and torch.equal(a[k][others], b[k][others])
            elif k == "margin":
                assert torch.isnan(b[k][pair]) and all(torch.equal(a[k][i], b[k][i]) for i in range(3) if i != pair)
            elif k == "loss":
                assert torch.isnan(b[k]) and torch.isfinite(a[k])
        if "margin" not in a and a.get("d_h") is not None:                              # (a pair's gradients all go by its margin)
            assert torch.equal(a["d_h"][others], b["d_h"][others])


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("vocab", [328, 4360])
@pytest.mark.parametrize("which", ["a label's", "another"])
def test_nan_in_a_row_of_the_lm_head(dtype, d, vocab, which):
    c = Case(dtype, 60, d, vocab)
    ok = c.ok.cuda()
    used = set(c.labels.tolist())
    row = int(c.labels[c.ok][3]) if which == "a label's" else next(v for v in range(vocab // 2, vocab) if v not in used)
    c.w[row, 0] = float("nan")
    for out in _calls(c, c.dev(c.h, True), c.w.cuda()):
        assert torch.isnan(out["logp"][ok]).all() and torch.all(out["logp"][~ok] == 0)
        if "loss" in out:
            assert torch.isnan(out["loss"])
        if "loss_tok" in out:
            assert torch.isnan(out["loss_tok"][ok]).all() and torch.all(out["loss_tok"][~ok] == 0)
        if out.get("d_h") is not None:
            assert torch.isnan(out["d_h"][ok]).all() and torch.all(out["d_h"][~ok] == 0)
    ids, top = c.labels.cuda()[:, None].contiguous(), torch.zeros(60, 1, device="cuda")
    kd = B.topk_kd_loss_forward_backward(c.dev(c.h, True), c.w.cuda(), ids, top)
    assert torch.isnan(kd["kl_tok"][ok]).all() and torch.all(kd["kl_tok"][~ok] == 0) and torch.isnan(kd["loss"])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 72), ("fp32", 72)])
def test_order_of_equal_entries(dtype, d):
    """A teacher's logits that are equal (they were stored in few bits): what is computed does not depend on the places they stand in.  (Sums of equal numbers are the same in any order.)"""
    n, vocab, k = 50, 4104, 100
    c = Case(dtype, n, d, vocab, left_out=False)
    h, w = c.h.cuda(), c.w.cuda()
    ids = torch.stack([torch.randperm(vocab, generator=c.g)[:k] for _ in range(n)]).to(torch.int32)
    top = torch.full((n, k), 3.0).cuda()
    first = None
    for i in range(4):
        order = torch.randperm(k, generator=c.g) if i else torch.arange(k)
        d_w = torch.zeros(vocab, d, device="cuda")
        out = B.topk_kd_loss_forward_backward(h, w, ids[:, order].contiguous().cuda(), top, d_w=d_w)
        out["d_w"] = d_w
        first = first or out
        assert all(torch.equal(out[x], first[x]) for x in out)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 72), ("fp32", 72)])
@pytest.mark.parametrize("k", [2, 40])
def test_entries_that_are_next_to_nothing(dtype, d, k):
    """lse_teacher far above the entries: a token's probabilities sum to e^-away.  Its KL and its gradient go to zero with them."""
    away = torch.tensor([0.5, 10.0, 30.0, 60.0, 69.0, 70.0, 80.0, 87.0, 88.5, 95.0, 103.0, 150.0, 1e4, 0.0])
    n, vocab = len(away), 4104
    c = Case(dtype, n, d, vocab, left_out=False)
    ids = torch.stack([torch.randperm(vocab, generator=c.g)[:k] for _ in range(n)]).to(torch.int32)
    top = c.normal((n, k), 2.0)
    lse = torch.logsumexp(top, 1) + away
    ref = oracle.topk_kd(f64(c.h), f64(c.w), f64(ids), f64(top), 1.0, 1.0, f64(lse))
    h, w = c.h.cuda(), c.w.cuda()
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.topk_kd_loss_forward_backward(h, w, ids.cuda(), top.cuda(), lse.cuda(), loss_scale=1.0, d_w=d_w)
    # a token's terms, each off by the logarithms' errors (of p: those of numbers as large as lse, too), of its mass; what fp32 does not hold is left out: 2^-100 of a token
    mass, big = np.exp(-f64(away)), np.abs(f64(lse)) + 20
    tol = mass * (c.delta() + U * (64 + 8 * big) * (1 + np.abs(f64(away)) + 20)) + 2.0 ** -100 * (big + 100)
    assert np.all(np.abs(f64(out["kl_tok"]) - ref["kl_tok"]) <= tol)
    got, size = f64(out["d_h"]), np.linalg.norm(f64(c.w), axis=1).max()
    # by norm: dz of a token is off by U (64 + 8 big) of itself beside what the other tests allow, and |dz| <= 2 mass
    for t in range(n):
        allowed = (2.0 ** -7 if dtype == "bf16" else 40 * c.delta()) * np.linalg.norm(ref["d_h"][t]) + 2 * mass[t] * U * (64 + 8 * big[t]) * size + 2.0 ** -99 * size
        assert np.isfinite(got[t]).all() and np.linalg.norm(got[t] - ref["d_h"][t]) <= allowed
    got = f64(d_w)
    assert np.isfinite(got).all() and np.linalg.norm(got - ref["d_w"]) <= (2.0 ** -7 if dtype == "bf16" else 40 * c.delta()) * np.linalg.norm(ref["d_w"])


@pytest.mark.parametrize("n,d,vocab", [(20000, 72, 1032), (20000, 72, 1024), (9000, 40, 4104), (20000, 128, 1032)])
def test_many_tokens_of_a_small_lm_head_have_the_same_bits(n, d, vocab):
    c = Case("bf16", n, d, vocab)
    g = c.normal((n,)).cuda()
    h, w, labels = c.dev(c.h, True), c.w.cuda(), c.labels.cuda()
    first = None
    for need in (True, True, True, False, False):
        d_w = torch.zeros(vocab, d, device="cuda")
        out = B.token_logprobs_backward(h, w, labels, g, d_w=d_w, need_d_h=need)
        first = first or (out, d_w)
        assert torch.equal(d_w, first[1]) and torch.equal(out["logp"], first[0]["logp"]) and (not need or torch.equal(out["d_h"], first[0]["d_h"]))
