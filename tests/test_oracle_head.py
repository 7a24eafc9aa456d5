"""The oracle of the losses at the end of a section: gradients against differences, closed forms, and the whole-teacher loss that distillation from
all of a teacher's logits has to be."""
import numpy as np
import pytest

from conftest import fd_grad
from oracle import head
from oracle.kd import kd_loss_forward_backward


def _case(rng, n=7, d=5, vocab=11):
    h, w = rng.normal(size=(n, d)), rng.normal(size=(vocab, d))
    labels = rng.integers(0, vocab, n)
    labels[[1, 4]] = -100, vocab
    return h, w, labels


def _check(f, out, h, w):
    """Central differences with steps of 1e-6: about 1e-9 off for values of order one."""
    for x, g in ((h, out["d_h"]), (w, out["d_w"])):
        for i in range(0, x.size, 3):
            idx = np.unravel_index(i, x.shape)
            assert abs(fd_grad(f, x, idx) - g[idx]) < 1e-7 * max(1.0, abs(g[idx])), idx


def test_given_gradient(rng):
    h, w, labels = _case(rng)
    g = rng.normal(size=7)
    _check(lambda: np.sum(g * head.token_logprobs(h, w, labels, 0.7)["logp"]), head.token_logprobs(h, w, labels, 0.7, g), h, w)


@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_gradient(rng, kl):
    h, w, labels = _case(rng)
    old = head.token_logprobs(h, w, labels, 1.3)["logp"] + rng.normal(size=7) * 0.4
    ref, adv, weights = old + 0.1, rng.normal(size=7), rng.uniform(0.5, 1, 7)
    a = (labels, old, adv, 0.2, 0.3, kl, ref, weights, 1.3, 0.5)
    out = head.policy(h, w, *a)
    assert out["loss_tok"][1] == 0 and out["grad"][4] == 0
    _check(lambda: head.policy(h, w, *a)["loss"], out, h, w)


@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_preference_gradient(rng, eps):
    h, w, labels = _case(rng)
    ref = rng.normal(size=7) - 2
    a = (labels, [0, 2, 4, 4, 7], 0.3, eps, ref, 1.1, 0.5)
    out = head.preference(h, w, *a)
    _check(lambda: head.preference(h, w, *a)["loss"], out, h, w)
    assert head.preference(h, w, np.full(7, -1), *a[1:])["loss"] == 0                            # no token counts: no pair does
    even = head.preference(h, w, labels, [0, 0, 0], 1.0)                                         # an empty pair
    assert even["margin"].tolist() == [0.0] and even["loss"] == 0


@pytest.mark.parametrize("whole", [False, True])
def test_entries_gradient(rng, whole):
    h, w, _ = _case(rng)
    ids = np.array([rng.permutation(11)[:4] for _ in range(7)])
    top = rng.normal(size=(7, 4)) * 2
    ids[0, 2], ids[1, 1], ids[2], top[3, 1] = ids[0, 0], 11, -1, -np.inf
    lse = np.log(np.exp(np.where(np.isfinite(top), top, 0) / 1.4).sum(1)) + 0.5 if whole else None
    out = head.topk_kd(h, w, ids, top, 1.4, 0.5, lse)
    assert out["kl_tok"][2] == 0 and 2 not in out["at"]
    _check(lambda: head.topk_kd(h, w, ids, top, 1.4, 0.5, lse)["loss"], out, h, w)


def test_all_entries_are_the_whole_teacher(rng):
    h, w, _ = _case(rng)
    h_t, w_t = rng.normal(size=(7, 3)), rng.normal(size=(11, 3))
    top, ids, lse = head.top_logits(h_t, w_t, 11, 1.7)
    assert np.all(np.diff(top, axis=1) <= 0)
    ref = kd_loss_forward_backward(h_t, h, w_t, w, 1.7, 0.3)
    for given in (None, lse):
        out = head.topk_kd(h, w, ids, top, 1.7, 0.3, given)
        for a, b in (("loss", "loss"), ("kl_tok", "kl_tok"), ("d_h", "d_h_s"), ("d_w", "d_w_s")):
            np.testing.assert_allclose(out[a], ref[b], rtol=1e-11, atol=1e-13)


def test_equal_logits_come_by_their_ids():
    _, ids, lse = head.top_logits(np.ones((1, 2)), np.array([[0.0, 1], [1, 0], [1, 1], [1, 0]]), 4, 1.0)
    assert ids.tolist() == [[2, 0, 1, 3]] and lse[0] == pytest.approx(np.log(3 * np.e + np.e ** 2))
