"""Losses, log-probabilities and top logits at the end of a section against the oracle (64 bits).

Bounds, u = 2^-24: a logit of d products is off by at most d u sum |h w| (any order of fp32 sums) <= d u A, A the largest |h| . |w| of a row and the
vocabulary; a log-probability by twice that over T, and by the rounding of what goes into the exponentials and the sum over the
vocabulary's strips: delta = u (2 d A / T + 4 max |z| / T + 256).  Gradients of the logits, dz = c q, and c (q - p) at the selected ids, are off by c q (2 delta + 4 u) (there: c times
that), by what c itself is off, and for a bf16 head by half a step of bf16 (2^-8) once where they are stored; sums of up to V or n products by V u, n u of the sum of magnitudes; the row's factor times the
hidden states is rounded to bf16 too (d_w), and d_h when it is stored.  Roundings that are independent add up like their squares: the norm of the
difference stays below 2^-7 of the norm (three of them, each uniform within half a step: 2^-8 sqrt(3 / 3))."""
import numpy as np
import pytest
import torch

from oracle import head as oracle
from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy().astype(np.int64)


class Case:
    """Hidden states, lm_head and labels; a third of the tokens are left out, with NaN for hidden states."""

    def __init__(self, dtype, n, d, vocab, seed=0, std=0.1, t=1.0, left_out=True):
        self.g = torch.Generator().manual_seed(seed * 1000 + n + d + vocab)
        self.n, self.d, self.vocab, self.t, self.dtype = n, d, vocab, t, dtype
        self.h = torch.empty(n, d).normal_(0, 1, generator=self.g).to(TYPES[dtype])
        self.w = torch.empty(vocab, d).normal_(0, std, generator=self.g).to(TYPES[dtype])
        self.labels = torch.randint(0, vocab, (n,), generator=self.g, dtype=torch.int32)
        if left_out and n > 1:
            out = torch.rand(n, generator=self.g) < 0.33
            self.labels[out] = torch.where(torch.rand(n, generator=self.g) < 0.5, -100, vocab).to(torch.int32)[out]
        self.ok = (self.labels >= 0) & (self.labels < vocab)

    def dev(self, x, nan_where_left_out=False):
        x = x.clone()
        if nan_where_left_out:
            x[~self.ok] = float("nan")
        return x.cuda()

    def normal(self, shape, std=1.0):
        return torch.empty(shape).normal_(0, std, generator=self.g)

    def delta(self):
        h, w = f64(self.h), f64(self.w)
        a = np.abs(h).max(0) @ np.abs(w).max(0) if h.size else 0.0
        a = min(a, float(np.linalg.norm(h, axis=1).max(initial=0.0) * np.linalg.norm(w, axis=1).max()))
        z = float(np.abs(h @ w.T).max(initial=0.0)) / self.t
        return U * (2 * self.d * a / self.t + 4 * z + 256)

    def check_gradients(self, ref, d_h, d_w, before=None, slack=0.0):
        """d_w against ref's on top of `before`; slack: by how much of itself c is off, [rows] or a number."""
        bf, delta = self.dtype == "bf16", self.delta()
        h, w, dz, at = f64(self.h), f64(self.w), np.abs(ref["dz"]), ref["at"]
        off = (2 * delta + 4 * U) * (dz + ref["selected"] * np.abs(ref["scale"])[:, None]) + dz * np.reshape(slack, (-1, 1))
        bound_h = np.zeros_like(h)
        bound_h[at] = (off + (2.0 ** -8 if bf else 0) * dz + self.vocab * U * dz) @ np.abs(w)
        bound_w = (off + (2.0 ** -7 + 2.0 ** -16 if bf else 0) * dz + (self.n + 2) * U * dz).T @ np.abs(h[at])
        if d_h is not None:
            got = f64(d_h)
            bound_h += (2.0 ** -8 if bf else U) * (np.abs(ref["d_h"]) + bound_h) + 1e-38
            assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref["d_h"]) <= bound_h), np.abs(got - ref["d_h"]).max()
            out = np.setdiff1d(np.arange(self.n), at)
            assert np.all(got[out] == 0)
            norm = np.linalg.norm(ref["d_h"])
            assert np.linalg.norm(got - ref["d_h"]) <= (2.0 ** -7 if bf else 40 * delta) * norm + 1e-37
        if d_w is not None:
            got = f64(d_w) - (0 if before is None else f64(before))
            bound_w += U * (2 * np.abs(f64(d_w)) + (0 if before is None else np.abs(f64(before)))) + 1e-38
            assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref["d_w"]) <= bound_w), np.abs(got - ref["d_w"]).max()
            if before is None:
                assert np.linalg.norm(got - ref["d_w"]) <= (2.0 ** -7 if bf else 40 * delta) * np.linalg.norm(ref["d_w"]) + 1e-37


# hidden sizes that a multiple of 64 makes fast and others; vocabularies of part of a strip, of several tiles and odd ones
SHAPES = [("fp32", 45, 72, 328), ("fp32", 1, 128, 1024), ("fp32", 293, 128, 1024), ("bf16", 45, 72, 328), ("bf16", 1, 64, 8), ("bf16", 2, 128, 1000), ("bf16", 130, 192, 2056),
          ("bf16", 300, 64, 4104), ("bf16", 513, 128, 648)]


@pytest.mark.parametrize("t", [1.0, 0.6])
@pytest.mark.parametrize("dtype,n,d,vocab", SHAPES)
def test_log_probabilities(dtype, n, d, vocab, t):
    c = Case(dtype, n, d, vocab, t=t)
    g = c.normal((n,))
    ref = oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), t, f64(g))
    h, w, labels = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels)
    logp = B.token_logprobs(h, w, labels, temperature=t)
    assert np.all(np.abs(f64(logp) - ref["logp"]) <= c.delta()) and np.all(f64(logp)[~c.ok.numpy()] == 0)
    before = c.normal((vocab, d)).cuda()
    d_w = before.clone()
    out = B.token_logprobs_backward(h, w, labels, c.dev(g, True), temperature=t, d_w=d_w)
    assert torch.equal(out["logp"], logp)
    c.check_gradients(ref, out["d_h"], d_w, before)
    d_w = torch.zeros_like(before)
    assert B.token_logprobs_backward(h, w, labels, c.dev(g, True), temperature=t, d_w=d_w, need_d_h=False)["d_h"] is None
    c.check_gradients(ref, None, d_w)
    c.check_gradients(ref, B.token_logprobs_backward(h, w, labels, c.dev(g, True), temperature=t)["d_h"], None)


@pytest.mark.parametrize("kl,weighted", [(0.0, False), (0.1, True)])
@pytest.mark.parametrize("dtype,n,d,vocab", SHAPES)
def test_policy_loss(dtype, n, d, vocab, kl, weighted):
    c = Case(dtype, n, d, vocab)
    logp = torch.from_numpy(oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.0)["logp"])
    # away from the borders of the clip, which 1e-3 of a logarithm would not cross
    step = c.normal((n,), 0.3)
    step = torch.where((step - np.log(1.3)).abs() < 0.02, step + 0.05, torch.where((step - np.log(0.8)).abs() < 0.02, step - 0.05, step))
    old = (logp - step).float()
    refp = (logp + c.normal((n,), 0.2)).float()
    adv, weights = c.normal((n,)), torch.rand(n, generator=c.g)
    adv[n // 2] = 0.0
    ref = oracle.policy(f64(c.h), f64(c.w), f64(c.labels), f64(old), f64(adv), 0.2, 0.3, kl, f64(refp), f64(weights) if weighted else None, 1.0, 0.25)
    h, w, labels = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels)
    args = dict(clip_low=0.2, clip_high=0.3, ref_logp=c.dev(refp, True) if kl else None, kl_coef=kl, weights=c.dev(weights, True) if weighted else None, loss_scale=0.25)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.policy_loss_forward_backward(h, w, labels, c.dev(old, True), c.dev(adv, True), d_w=d_w, **args)
    # ratios of e^1 at most, times advantages
    tol = (c.delta() + 8 * U) * 2 * np.exp(1.0) * (1 + np.abs(f64(adv)))
    assert np.all(np.abs(f64(out["loss_tok"]) - ref["loss_tok"]) <= tol)
    assert abs(out["loss"].item() - ref["loss"]) <= 0.25 * (tol.sum() + 64 * U * np.abs(ref["loss_tok"]).sum())
    assert np.all(np.abs(f64(out["logp"]) - ref["logp"]) <= c.delta())
    slope = ref["grad"][ref["at"]]
    c.check_gradients(ref, out["d_h"], d_w, slack=(c.delta() + 8 * U) * ref["steep"][ref["at"]] / np.where(slope == 0, 1.0, np.abs(slope)))
    only = B.policy_loss_forward_backward(h, w, labels, c.dev(old, True), c.dev(adv, True), need_d_h=False, **args)
    assert torch.equal(only["loss"], out["loss"]) and torch.equal(only["loss_tok"], out["loss_tok"]) and only["d_h"] is None


@pytest.mark.parametrize("eps,with_ref", [(0.0, True), (0.1, False)])
@pytest.mark.parametrize("dtype,n,d,vocab", SHAPES)
def test_preference_loss(dtype, n, d, vocab, eps, with_ref):
    c = Case(dtype, n, d, vocab)
    cut = [0, n // 5, n // 2, n // 2, n // 2, n // 2 + n // 7, n, n, n]                   # a pair with one side, one without any, one empty
    c.labels[n // 2:n // 2 + 1] = -1
    c.ok = (c.labels >= 0) & (c.labels < vocab)
    logp = torch.from_numpy(oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.3)["logp"])
    refp = (logp + c.normal((n,), 0.3)).float() if with_ref else None
    beta = 0.2 if with_ref else 0.002
    c.t = 1.3
    ref = oracle.preference(f64(c.h), f64(c.w), f64(c.labels), cut, beta, eps, f64(refp), 1.3, 0.25)
    h, w, labels = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.preference_loss_forward_backward(h, w, labels, B.Batch(cut), beta, ref_logp=c.dev(refp, True) if with_ref else None, label_smoothing=eps, temperature=1.3, d_w=d_w)
    tol = n * c.delta() + 4 * U * np.abs(ref["margin"])
    assert np.all(np.abs(f64(out["margin"]) - ref["margin"]) <= tol)
    assert abs(out["loss"].item() - ref["loss"]) <= beta * tol.sum() + 16 * U
    more = beta * n * c.delta() + 16 * U                                                  # what the margin's error does to a slope, relative
    c.check_gradients(ref, out["d_h"], d_w, slack=more)


@pytest.mark.parametrize("k", [1, 5, 64, 128])
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("dtype,n,d,vocab", SHAPES)
def test_entries(dtype, n, d, vocab, whole, k):
    k = min(k, vocab)
    c = Case(dtype, n, d, vocab, t=1.5, left_out=False)
    ids = torch.stack([torch.randperm(vocab, generator=c.g)[:k] for _ in range(n)]).to(torch.int32)
    top = c.normal((n, k), 3.0)
    if n > 8:
        ids[3], ids[4, k // 2:], top[5] = -1, vocab, -float("inf")                       # none, few, none above -inf
        ids[6, k - 1] = ids[6, 0]                                                        # the same twice: the first counts
        top[7, 0] = -float("inf")
        top[4, k // 2:] = float("nan")
    lse = torch.logsumexp(torch.where(torch.isfinite(top), top, -1e30) / 1.5, 1).clamp(min=0) + 0.4 if whole else None
    ref = oracle.topk_kd(f64(c.h), f64(c.w), f64(ids), f64(top), 1.5, 1.0 / n, f64(lse))
    c.ok = torch.from_numpy(np.isin(np.arange(n), ref["at"]))
    h, w = c.dev(c.h, True), c.dev(c.w)
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.topk_kd_loss_forward_backward(h, w, ids.cuda(), top.cuda(), lse.cuda() if whole else None, temperature=1.5, d_w=d_w)
    tol = c.delta() + U * (64 + 8 * np.abs(ref["kl_tok"]))
    assert np.all(np.abs(f64(out["kl_tok"]) - ref["kl_tok"]) <= tol), np.abs(f64(out["kl_tok"]) - ref["kl_tok"]).max()
    assert abs(out["loss"].item() - ref["loss"]) <= tol.mean() + 64 * U * abs(ref["loss"])
    c.check_gradients(ref, out["d_h"], d_w)
    only = B.topk_kd_loss_forward_backward(h, w, ids.cuda(), top.cuda(), lse.cuda() if whole else None, temperature=1.5, need_d_h=False)
    assert torch.equal(only["kl_tok"], out["kl_tok"])


def _grid(c):
    """Products whose fp32 sums are exact: equal logits are equal in any order of the sums."""
    c.h, c.w = (torch.round(c.h.float() * 4) / 4).to(c.h.dtype), (torch.round(c.w.float() * 64) / 64).to(c.w.dtype)


@pytest.mark.parametrize("k", [1, 7, 64, 128])
@pytest.mark.parametrize("dtype,n,d,vocab", SHAPES + [("bf16", 3, 64, 20000), ("fp32", 3, 8, 20000)])
def test_top_logits(dtype, n, d, vocab, k):
    k = min(k, vocab)
    c = Case(dtype, n, d, vocab, t=0.8, left_out=False)
    _grid(c)
    values, ids, lse = oracle.top_logits(f64(c.h), f64(c.w), k, 0.8)
    got = B.top_logits(c.h.cuda(), c.w.cuda(), k, temperature=0.8)
    assert np.array_equal(f64(got[0]), values) and np.array_equal(f64(got[1]), ids)
    assert np.all(np.abs(f64(got[2]) - lse) <= c.delta())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_top_logits_of_equal_and_ordered_rows(dtype):
    """All logits equal (the first ids), rising (the last), falling, all of a strip above the rest, minus infinity but for a few."""
    vocab, d, k = 1032, 64, 100
    z = torch.stack([torch.zeros(vocab), torch.arange(vocab) / 8.0, -torch.arange(vocab) / 8.0, (torch.arange(vocab) // 64 == 5) * 1.0 - 0.25 * (torch.arange(vocab) % 3)])
    w = torch.zeros(vocab, d)
    w[:, :4] = z.T
    w = w.to(TYPES[dtype])
    h = torch.eye(4, d).to(TYPES[dtype])
    values, ids, lse = oracle.top_logits(f64(h), f64(w), k, 1.0)
    got = B.top_logits(h.cuda(), w.cuda(), k)
    assert np.array_equal(f64(got[0]), values) and np.array_equal(f64(got[1]), ids) and np.allclose(f64(got[2]), lse, rtol=1e-6)
    w[7:, 0] = -float("inf")                                                             # 7 of them are finite; the others come by their ids
    got = B.top_logits(torch.eye(1, d).to(TYPES[dtype]).cuda(), torch.nan_to_num(w, neginf=-1e30).to(w.dtype).cuda(), 9)
    assert f64(got[1]).tolist() == [list(range(9))] and got[2].item() == pytest.approx(np.log(7), rel=1e-6)


def test_top_logits_with_nan():
    h, w = torch.ones(2, 64).bfloat16(), torch.randn(520, 64).bfloat16()
    w[77, 3] = float("nan")
    values, ids, lse = B.top_logits(h.cuda(), w.cuda(), 20)
    assert torch.isnan(lse).all() and ((ids >= -1) & (ids < 520)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gap", [20.0, 60.0, 300.0, 3000.0])
def test_labels_far_below_the_largest_logit(dtype, gap):
    """The reference of a row is its label's logit: others may be far above it, in one strip or in several, also in the last."""
    vocab, d, n = 712, 64, 6
    w = torch.zeros(vocab, d)
    w[:, 0] = torch.randn(vocab, generator=torch.Generator().manual_seed(3)) * 0.5
    w[100, 1], w[700, 1], w[101, 1], w[300, 2] = 1.0, 1.0, 0.9, 1.0
    h = torch.zeros(n, d)
    h[:, 0] = 1.0
    h[0, 1] = h[1, 1] = h[2, 2] = gap
    h[4, 1], h[4, 2] = gap, gap * 0.5
    h[5, 1] = -gap
    c = Case(dtype, n, d, vocab, left_out=False)
    c.h, c.w = h.to(TYPES[dtype]), w.to(TYPES[dtype])
    c.labels = torch.tensor([5, 700, 6, 7, 300, 100], dtype=torch.int32)
    g = torch.tensor([1.0, -1, 0.5, 1, -0.25, 2])
    ref = oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.0, f64(g))
    d_w = torch.zeros(vocab, d, device="cuda")
    out = B.token_logprobs_backward(c.h.cuda(), c.w.cuda(), c.labels.cuda(), g.cuda(), d_w=d_w)
    assert np.all(np.abs(f64(out["logp"]) - ref["logp"]) <= c.delta())
    c.check_gradients(ref, out["d_h"], d_w)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 40), ("fp32", 40)])
def test_nothing_counts_and_empty_calls(dtype, d):
    c = Case(dtype, 70, d, 264)
    c.labels[:] = -1
    c.ok[:] = False
    h, w, labels, x = c.dev(c.h, True), c.w.cuda(), c.labels.cuda(), torch.full((70,), float("nan"), device="cuda")
    d_w = torch.ones(264, d, device="cuda")
    for out in (B.policy_loss_forward_backward(h, w, labels, x, x, ref_logp=x, kl_coef=0.1, weights=x, d_w=d_w), B.token_logprobs_backward(h, w, labels, x, d_w=d_w),
                B.preference_loss_forward_backward(h, w, labels, B.Batch([0, 30, 70]), 0.1, ref_logp=x, d_w=d_w),
                B.topk_kd_loss_forward_backward(h, w, torch.full((70, 3), -1, dtype=torch.int32, device="cuda"), x[:, None].repeat(1, 3), lse_teacher=x, d_w=d_w)):
        assert out.get("loss", torch.zeros(())).item() == 0 and torch.all(out["d_h"] == 0) and all(torch.all(v == 0) for v in out.values())
    assert torch.all(d_w == 1)
    none = torch.empty(0, d, dtype=TYPES[dtype], device="cuda")
    i0, f0 = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    assert B.policy_loss_forward_backward(none, w, i0, f0, f0, d_w=d_w)["loss"].item() == 0
    out = B.preference_loss_forward_backward(none, w, i0, B.Batch([0, 0, 0]), 0.1, d_w=d_w)
    assert out["loss"].item() == 0 and out["margin"].tolist() == [0.0]
    assert B.topk_kd_loss_forward_backward(none, w, i0.view(0, 3), f0.view(0, 3), d_w=d_w)["loss"].item() == 0
    assert B.token_logprobs(none, w, i0).numel() == 0 and B.top_logits(none, w, 3)[0].shape == (0, 3) and torch.all(d_w == 1)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 72), ("fp32", 72)])
def test_token_blocks_and_gradient_over_the_states(dtype, d):
    """Blocks of 40 of 97 tokens: every token's numbers are those of one block; d_h may take the states' place."""
    c = Case(dtype, 97, d, 1032)
    old, adv = c.normal((97,)) - 7, c.normal((97,))
    h, w, labels = c.dev(c.h), c.w.cuda(), c.labels.cuda()
    ids, top = torch.stack([torch.randperm(1032, generator=c.g)[:9] for _ in range(97)]).to(torch.int32).cuda(), c.normal((97, 9)).cuda()

    def run(block):
        d_w = [torch.zeros(1032, d, device="cuda") for _ in range(3)]
        return (B.policy_loss_forward_backward(h, w, labels, old.cuda(), adv.cuda(), d_w=d_w[0], token_block=block), B.topk_kd_loss_forward_backward(h, w, ids, top, d_w=d_w[1], token_block=block),
                B.token_logprobs_backward(h, w, labels, adv.cuda(), d_w=d_w[2], token_block=block), d_w, B.top_logits(h, w, 9, token_block=block))
    one, many = run(0), run(40)
    for a, b in zip(one[:3], many[:3]):
        assert all(torch.equal(a[k], b[k]) for k in a)
    assert all(torch.equal(a, b) for a, b in zip(one[4], many[4]))
    for a, b in zip(one[3], many[3]):                                                    # three sums of a few terms instead of one: fp32 sums in another order
        assert ((a - b).abs() <= 97 * U * 16 * a.abs().max()).all()
    x = h.clone()
    lib, cfg = B._fn("ms_token_logprobs_backward"), B._head(x, w, 1.0, 1.0, 40)[0]
    ws = B.workspace(B.head_workspace_bytes(w, 97, token_block=40))
    a = adv.cuda()
    assert lib(B.C.byref(cfg), 97, x.data_ptr(), labels.data_ptr(), a.data_ptr(), None, x.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(x, one[2]["d_h"])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 72)])
def test_streams_and_graphs(dtype, d):
    """Two calls at once on two streams, and two captured graphs replayed in turn with eager work between, against the calls one by one; inputs change between
    replays."""
    c = Case(dtype, 200, d, 2056)
    old, adv = (c.normal((200,)) - 7).cuda(), c.normal((200,)).cuda()
    h, w, labels = c.dev(c.h), c.w.cuda(), c.labels.cuda()
    ids, top = torch.randint(0, 2056, (200, 20), generator=c.g, dtype=torch.int32).cuda(), c.normal((200, 20)).cuda()
    cu = B.Batch([0, 50, 90, 150, 200])

    def calls(h, d_w):
        return (B.policy_loss_forward_backward(h, w, labels, old, adv, d_w=d_w[0]), B.topk_kd_loss_forward_backward(h, w, ids, top, d_w=d_w[1]),
                B.preference_loss_forward_backward(h, w, labels, cu, 0.1, d_w=d_w[2]), dict(zip("abc", B.top_logits(h, w, 20))), dict(a=B.token_logprobs(h, w, labels)))

    def zeros():
        return [torch.zeros(2056, d, device="cuda") for _ in range(3)]

    def same(a, b, wa, wb):
        assert all(torch.equal(x[k], y[k]) for x, y in zip(a, b) for k in x) and all(torch.equal(x, y) for x, y in zip(wa, wb))
    streams = [torch.cuda.Stream() for _ in range(2)]
    d_ws = [zeros() for _ in range(3)]
    eager = calls(h, d_ws[2])
    torch.cuda.synchronize()
    outs = []
    for s, d_w in zip(streams, d_ws):
        with torch.cuda.stream(s):
            outs.append(calls(h, d_w))
    torch.cuda.synchronize()
    for out, d_w in zip(outs, d_ws):
        same(out, eager, d_w, d_ws[2])
    xs, grads, graphs, res = [h.clone(), (h.float() * 0.5).to(h.dtype)], [zeros(), zeros()], [], []
    for x, d_w in zip(xs, grads):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for v in d_w:
                v.zero_()
            res.append(calls(x, d_w))
        graphs.append(graph)
    for i in range(3):
        for j in (0, 1):
            graphs[j].replay()
        torch.cuda.synchronize()
        for x, out, d_w in zip(xs, res, grads):
            ref = zeros()
            same(out, calls(x, ref), d_w, ref)
        for x in xs:
            x.mul_(1.25)


def test_sections_learn_through_them():
    """As they are used: a teacher section's top logits, a student section distilled from them; with every entry, that is the whole-teacher loss."""
    cfg_t, cfg_s = wl.workload("c1").teacher, wl.workload("c1").student
    cfg_t, cfg_s = wl.scaled(cfg_t, vocab=128), wl.scaled(cfg_s, vocab=128)
    batch = B.Batch([0, 20, 53, 60])
    wt, ws = wl.section_weights(cfg_t, 0, "t", "cuda"), wl.section_weights(cfg_s, 0, "s", "cuda")
    head_t, head_s = (wl.normal(0, f"head.{n}", (128, c.d_model), 0.1, device="cuda") for n, c in (("t", cfg_t), ("s", cfg_s)))
    x = wl.randint(0, "ids", 60, 0, 128, "cuda")
    h_t, h_s = B.section_forward(cfg_t, wt, batch, x), B.section_forward(cfg_s, ws, batch, x)
    top, ids, lse = B.top_logits(h_t, head_t, 128, temperature=1.5)
    d_w, d_w_kd = torch.zeros_like(head_s), torch.zeros_like(head_s)
    out = B.topk_kd_loss_forward_backward(h_s, head_s, ids, top, lse, temperature=1.5, d_w=d_w)
    grads, grads_kd = B.zero_grads(ws), B.zero_grads(ws)
    B.section_forward_backward(cfg_s, ws, grads, batch, x, d_h_out=out["d_h"])
    kd = wl.KDConfig(128, cfg_t.d_model, cfg_s.d_model, 1.5, 64, "fp32")
    ref = B.section_forward_backward(cfg_s, ws, grads_kd, batch, x, kd=kd, w_teacher=head_t, w_student=head_s, h_teacher=h_t, d_w_student=d_w_kd)
    assert out["loss"].item() == pytest.approx(ref["loss"].item(), rel=1e-4)
    pairs = [(d_w, d_w_kd)] + [(grads["layers"][0][k], grads_kd["layers"][0][k]) for k in ("w_qkv", "w_o", "w_up", "w_down", "norm1_g")]
    for a, b in pairs:                                                                   # fp32 throughout
        assert ((a - b).norm() <= 1e-4 * b.norm()).item()
    # a frozen reference scores the tokens, the policy learns from them: at the same weights all ratios are 1, and the gradient is the plain policy gradient's
    labels = torch.roll(x, -1)
    old = B.token_logprobs(h_s, head_s, labels)
    adv = wl.normal(0, "adv", (60,), device="cuda")
    a = B.policy_loss_forward_backward(h_s, head_s, labels, old, adv, ref_logp=old, kl_coef=0.1, loss_scale=1.0)
    b = B.token_logprobs_backward(h_s, head_s, labels, -adv)
    assert torch.allclose(a["d_h"], b["d_h"], rtol=1e-5, atol=1e-6) and a["loss"].item() == pytest.approx(-adv.sum().item(), rel=1e-4, abs=1e-4)


# every tile of the products, ragged rows, columns and rows that do not count; the generic kernels on the same sizes; -1: logits stored in fp32
@pytest.mark.parametrize("tile", [256, 128, 128128, 128256, 64128, 64064, -1])
@pytest.mark.parametrize("n,d,vocab", [(300, 192, 1000), (45, 64, 4104), (700, 320, 2568)])
def test_every_tile(tile, n, d, vocab):
    c = Case("bf16", n, d, vocab)
    g = c.normal((n,))
    ref = oracle.token_logprobs(f64(c.h), f64(c.w), f64(c.labels), 1.0, f64(g))
    h, w, labels, g = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels), c.dev(g, True)
    free = B.token_logprobs(h, w, labels)
    t = Case("bf16", n, d, vocab, left_out=False)
    _grid(t)
    values, ids, lse = oracle.top_logits(f64(t.h), f64(t.w), 20, 1.0)
    try:
        B.k_gemm_config(tile)
        d_w = torch.zeros(vocab, d, device="cuda")
        out = B.token_logprobs_backward(h, w, labels, g, d_w=d_w)
        only = B.token_logprobs(h, w, labels)
        top = B.top_logits(t.h.cuda(), t.w.cuda(), 20)
    finally:
        B.k_gemm_config(0)
    assert np.all(np.abs(f64(out["logp"]) - ref["logp"]) <= c.delta()) and torch.equal(only, out["logp"])
    assert tile < 0 or torch.equal(free, only)                                           # all tiles add up in one order
    c.check_gradients(ref, out["d_h"], d_w)
    assert np.array_equal(f64(top[0]), values) and np.array_equal(f64(top[1]), ids) and np.all(np.abs(f64(top[2]) - lse) <= t.delta())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 72), ("fp32", 72)])
@pytest.mark.parametrize("n,vocab,k", [(137, 2056, 3), (90, 4104, 100), (1, 264, 9)])
def test_a_workspace_holds_whatever_it_held(monkeypatch, dtype, d, n, vocab, k):
    """The same bits with a workspace of zeros, of NaN, of large numbers and of what another call left behind."""
    c = Case(dtype, n, d, vocab)
    old, adv = (c.normal((n,)) - 7).cuda(), c.normal((n,)).cuda()
    h, w, labels = c.dev(c.h), c.w.cuda(), c.labels.cuda()
    ids, top = torch.randint(-1, vocab, (n, k), generator=c.g, dtype=torch.int32).cuda(), c.normal((n, k)).cuda()
    cu = B.Batch([0, n // 3, n])
    one = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")

    def calls(fill):
        def workspace(nbytes, device="cuda", tag=None):
            assert nbytes <= one.numel()
            if fill is not None:
                one.fill_(fill)
            return one[:max(int(nbytes), 256)]
        monkeypatch.setattr(B, "workspace", workspace)
        d_w = [torch.zeros(vocab, d, device="cuda") for _ in range(4)]
        out = [B.policy_loss_forward_backward(h, w, labels, old, adv, ref_logp=old, kl_coef=0.1, d_w=d_w[0]), B.topk_kd_loss_forward_backward(h, w, ids, top, d_w=d_w[1]),
               B.preference_loss_forward_backward(h, w, labels, cu, 0.1, d_w=d_w[2]), B.token_logprobs_backward(h, w, labels, adv, d_w=d_w[3]), dict(enumerate(B.top_logits(h, w, k))),
               dict(a=B.token_logprobs(h, w, labels))]
        return out, d_w
    ref = calls(0)
    for fill in (0xff, 0x7f, None):
        got = calls(fill)
        for a, b in zip(ref[0], got[0]):
            assert all(torch.equal(a[x], b[x]) for x in a)
        assert all(torch.equal(a, b) for a, b in zip(ref[1], got[1]))


# logits in tiles of 64 and of 128, ragged in every direction, and of more hidden numbers than one accumulator takes
@pytest.mark.parametrize("n,d,vocab", [(700, 72, 1992), (1300, 136, 1032), (4100, 40, 2056), (530, 8, 2560), (290, 1032, 4104)])
def test_many_rows_in_fp32(n, d, vocab):
    test_log_probabilities("fp32", n, d, vocab, 0.6)
    c = Case("fp32", n, d, vocab)
    h, w, labels = c.dev(c.h, True), c.dev(c.w), c.dev(c.labels)
    a, b = B.token_logprobs(h, w, labels), B.token_logprobs(h, w, labels, token_block=520)
    assert np.all(np.abs(f64(a) - f64(b)) <= 2 * c.delta())                              # (fewer rows than a few hundred have products of another order)
