"""bf16 ends of sections that keep the gradient of their logits in two bf16 numbers, against the oracle (64 bits) and against themselves.

Bounds as in test_gpu_head.py, with another rounding of dz: what the first number lacks is at most half a step, 2^-8 of dz, and the second number is off by 2^-8 of that, so 2^-16 in all, and no
hidden states are rounded again.  Twice as many terms in a sum: (2 n + 2) U of d_w, 2 V U of d_h.  d_h itself is rounded to bf16 when it is stored."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import head as oracle
from paper_2605_10501_amd import binding as B
from test_gpu_head import U, Case, f64

pytestmark = pytest.mark.gpu
SHAPES = [(45, 72, 328), (1, 64, 8), (2, 128, 1000), (130, 192, 2056), (300, 64, 4104), (513, 128, 648)]


def _check(c, ref, d_h, d_w, slack=0.0):
    delta, h, w, dz, at = c.delta(), f64(c.h), f64(c.w), np.abs(ref["dz"]), ref["at"]
    off = (2 * delta + 4 * U) * (dz + ref["selected"] * np.abs(ref["scale"])[:, None]) + dz * np.reshape(slack, (-1, 1)) + 2.0 ** -16 * dz
    if d_h is not None:
        bound = np.zeros_like(h)
        bound[at] = (off + 2 * c.vocab * U * dz) @ np.abs(w)
        got = f64(d_h)
        bound += 2.0 ** -8 * (np.abs(ref["d_h"]) + bound) + 1e-38
        assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref["d_h"]) <= bound)
        assert np.all(got[np.setdiff1d(np.arange(c.n), at)] == 0)
    if d_w is not None:
        bound = (off + (2 * c.n + 2) * U * dz).T @ np.abs(h[at])
        got = f64(d_w)
        bound += 2 * U * np.abs(got) + 1e-38
        assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref["d_w"]) <= bound)
        assert np.linalg.norm(got - ref["d_w"]) <= (2.0 ** -16 + 40 * delta + np.max(slack, initial=0.0)) * np.linalg.norm(ref["d_w"]) + 1e-37


@pytest.mark.parametrize("n,d,vocab", SHAPES)
@pytest.mark.parametrize("block", [0, 40])
def test_log_probabilities(n, d, vocab, block):
    c = Case("bf16", n, d, vocab, t=0.6)
    g = c.normal((n,))
    ref = oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 0.6, f64(g))
    h, w, labels, g = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels), c.dev(g, True)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, temperature=0.6, d_w=d_w, fp32_dz=True, token_block=block)
    assert np.all(np.abs(f64(out["logp"]) - ref["logp"]) <= c.delta())
    _check(c, ref, out["d_h"], d_w)
    other = torch.zeros(vocab, d, device="cuda")
    again = B.token_logprobs_backward(h, w, labels, g, temperature=0.6, d_w=other, need_d_h=False, fp32_dz=True, token_block=block)
    assert torch.equal(other, d_w) and torch.equal(again["logp"], out["logp"])
    assert torch.equal(B.token_logprobs_backward(h, w, labels, g, temperature=0.6, fp32_dz=True, token_block=block)["d_h"], out["d_h"])


@pytest.mark.parametrize("k", [1, 33, 128])
@pytest.mark.parametrize("n,d,vocab", SHAPES)
def test_entries(n, d, vocab, k):
    """Many entries of a token, none of them far above the others: where the roundings of a bf16 gradient show most."""
    k = min(k, vocab)
    c = Case("bf16", n, d, vocab, t=1.5, left_out=False)
    ids = torch.stack([torch.randperm(vocab, generator=c.g)[:k] for _ in range(n)]).to(torch.int32)
    top = c.normal((n, k), 0.3)
    if n > 8:
        ids[3], ids[4, k // 2:] = -1, vocab
    ref = oracle.topk_kd(f64(c.h), f64(c.w), f64(ids), f64(top), 1.5, 1.0 / n)
    c.ok = torch.from_numpy(np.isin(np.arange(n), ref["at"]))
    h, w = c.dev(c.h, True), c.dev(c.w)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.topk_kd_loss_forward_backward(h, w, ids.cuda(), top.cuda(), temperature=1.5, d_w=d_w, fp32_dz=True)
    assert np.all(np.abs(f64(out["kl_tok"]) - ref["kl_tok"]) <= c.delta() + U * (64 + 8 * np.abs(ref["kl_tok"])))
    _check(c, ref, out["d_h"], d_w)


@pytest.mark.parametrize("n,d,vocab", SHAPES)
def test_policy_and_preference_losses(n, d, vocab):
    c = Case("bf16", n, d, vocab)
    logp = torch.from_numpy(oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.0)["logp"])
    old, refp, adv = (logp + 0.05).float(), (logp + c.normal((n,), 0.2)).float(), c.normal((n,))
    h, w, labels = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels)
    ref = oracle.policy(f64(c.h), f64(c.w), f64(c.labels), f64(old), f64(adv), 0.2, 0.3, 0.1, f64(refp), None, 1.0, 0.25)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.policy_loss_forward_backward(h, w, labels, c.dev(old, True), c.dev(adv, True), clip_low=0.2, clip_high=0.3, ref_logp=c.dev(refp, True), kl_coef=0.1, loss_scale=0.25, d_w=d_w, fp32_dz=True)
    tol = (c.delta() + 8 * U) * 2 * np.exp(1.0) * (1 + np.abs(f64(adv)))
    assert np.all(np.abs(f64(out["loss_tok"]) - ref["loss_tok"]) <= tol)
    slope = ref["grad"][ref["at"]]
    slack = (c.delta() + 8 * U) * ref["steep"][ref["at"]] / np.where(slope == 0, 1.0, np.abs(slope))
    _check(c, ref, out["d_h"], d_w, slack)
    cut = [0, n // 5, n // 2, n // 2 + n // 7, n]
    ref = oracle.preference(f64(c.h), f64(c.w), f64(c.labels), cut, 0.2, 0.1, f64(refp), 1.0, 0.5)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.preference_loss_forward_backward(h, w, labels, B.Batch(cut), 0.2, ref_logp=c.dev(refp, True), label_smoothing=0.1, d_w=d_w, fp32_dz=True)
    tol = n * c.delta() + 4 * U * np.abs(ref["margin"])
    assert np.all(np.abs(f64(out["margin"]) - ref["margin"]) <= tol) and abs(out["loss"].item() - ref["loss"]) <= 0.2 * tol.sum() + 16 * U
    _check(c, ref, out["d_h"], d_w, 0.2 * n * c.delta() + 16 * U)


def test_an_fp32_head_and_a_forward_pass():
    """An fp32 head has nothing to choose; a forward pass takes the choice, and has the loss of the backward pass.  The C entry turns the choice down for fp32."""
    c = Case("fp32", 50, 72, 328)
    h, w, labels, g = c.dev(c.h), c.dev(c.w), c.dev(c.labels), torch.ones(50, device="cuda")
    a, b = B.token_logprobs_backward(h, w, labels, g), B.token_logprobs_backward(h, w, labels, g, fp32_dz=True)
    assert all(torch.equal(a[k], b[k]) for k in a)
    cfg, ws = B._head(h, w, 1.0, 1.0, 0)[0], B.workspace(B.head_workspace_bytes(w, 50))
    cfg.dtype |= 256
    assert B._fn("ms_token_logprobs")(C.byref(cfg), 50, h.data_ptr(), labels.data_ptr(), g.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) != 0
    assert "bad dtype" in B.lib().ms_last_error().decode()
    c = Case("bf16", 50, 64, 328)
    h, w, labels = c.dev(c.h), c.dev(c.w), c.dev(c.labels)
    old, adv = torch.full((50,), -5.0, device="cuda"), torch.ones(50, device="cuda")
    a, b = (B.policy_loss_forward_backward(h, w, labels, old, adv, need_d_h=need, fp32_dz=True) for need in (True, False))
    assert torch.equal(a["loss"], b["loss"]) and torch.equal(a["logp"], b["logp"])


@pytest.mark.parametrize("n,d,vocab", [(8200, 64, 140000), (600, 1536, 151936)])
def test_several_slabs_and_parts(n, d, vocab):
    from test_gpu_head_large import _exact, _inputs, _near
    h, w, labels, g = _inputs(torch.bfloat16, n, d, vocab)
    w = (w * (64 / d) ** 0.5).contiguous()
    logp, d_h, d_w = _exact(h, w, labels, g, rows=512)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w, fp32_dz=True)
    assert (out["logp"].double() - logp).abs().max().item() < 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256)
    _near(out["d_h"], d_h, 2.0 ** -8)                                                     # rounded once
    _near(got_w, d_w, 2.0 ** -15)                                                         # dz to 2^-16 of itself, fp32 sums and exponentials to 2^-17


def test_in_a_graph_with_a_workspace_that_held_other_things():
    c = Case("bf16", 200, 128, 2056)
    h, w, labels, g = c.dev(c.h), c.w.cuda(), c.labels.cuda(), c.normal((200,)).cuda()
    ws = torch.empty(B.head_workspace_bytes(w, 200, fp32_dz=True), dtype=torch.uint8, device="cuda")
    d_w = torch.zeros(2056, 128, device="cuda")
    ws.fill_(0)
    first = B.token_logprobs_backward(h, w, labels, g, d_w=d_w, ws=ws, fp32_dz=True)
    graph, got_w = torch.cuda.CUDAGraph(), torch.zeros_like(d_w)
    with torch.cuda.graph(graph):
        got_w.zero_()
        out = B.token_logprobs_backward(h, w, labels, g, d_w=got_w, ws=ws, fp32_dz=True)
    for fill in (0xff, 0x7f, 1):
        ws.fill_(fill)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got_w, d_w) and all(torch.equal(out[k], first[k]) for k in out)
