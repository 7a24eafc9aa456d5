"""Calls at the end of a section that are turned down, by what they say, before anything is launched: none of this needs a GPU.  And the workspace's plan."""
import ctypes as C

import pytest
import torch

from paper_2605_10501_amd import binding as B


P = 1 << 40                                           # a pointer that nobody follows; the tests' matrices lie megabytes apart
H, W, DH, DW = P, P + (1 << 28), P + (2 << 28), P + (3 << 28)
BIG = 1 << 45


def cfg(**over):
    a = dict(vocab=1024, hidden=128, dtype=B.MS_BF16, token_block=0, temperature=1.0, loss_scale=1.0, w_dev=W)
    a.update(over)
    return B._HeadCfg(*[a[n] for n, _ in B._HeadCfg._fields_])




def top(c, n=4, k=8, h=H, out=P, ws=P, size=BIG):
    return B._fn("ms_top_logits")(C.byref(c), n, h, k, out, out, out, ws, size, None)


def tkd(c, n=4, k=8, ids=P, loss=P, h=H, d_h=DH, d_w=None, ws=P, size=BIG):
    return B._fn("ms_topk_kd_loss_forward_backward")(C.byref(c), n, h, k, ids, P, None, loss, None, d_h, d_w, ws, size, None)


def policy(c, n=4, low=0.2, high=0.2, kl=0.0, ref=None, labels=P, loss=P, d_w=DW, size=BIG):
    pc = B._PolicyCfg(low, high, kl)
    return B._fn("ms_policy_loss_forward_backward")(C.byref(c), C.byref(pc), n, P, labels, P, ref, P, None, loss, None, None, None, d_w, P, size, None)


def pref(c, cu=(0, 2, 4), n=4, beta=0.1, eps=0.0, labels=P, size=BIG, dev=P):
    host = (C.c_int32 * len(cu))(*cu)
    b, pc = B.BatchC(n, len(cu) - 1, C.c_void_p(dev), host), B._PreferenceCfg(beta, eps)
    return B._fn("ms_preference_loss_forward_backward")(C.byref(c), C.byref(pc), C.byref(b), H, labels, None, P, None, None, DH, None, P, size, None)


def logp(c, n=4, labels=P, out=P, size=BIG):
    return B._fn("ms_token_logprobs")(C.byref(c), n, P, labels, out, P, size, None)


def logp_back(c, d_logp=P, d_h=DH, n=4):
    return B._fn("ms_token_logprobs_backward")(C.byref(c), n, P, P, d_logp, None, d_h, None, P, BIG, None)


@pytest.mark.parametrize("call", [top, tkd, policy, pref, logp, logp_back])
@pytest.mark.parametrize("over,says", [
    (dict(dtype=7), "bad dtype"), (dict(vocab=0), "must be positive"), (dict(vocab=1020), "multiples of 8"), (dict(hidden=100), "multiples of 8"), (dict(hidden=1 << 17), "hidden size over"),
    (dict(temperature=0.0), "temperature"), (dict(temperature=float("nan")), "temperature"), (dict(temperature=1e-42), "temperature"), (dict(loss_scale=float("inf")), "loss_scale"),
    (dict(token_block=12), "token_block"), (dict(token_block=-8), "token_block"), (dict(w_dev=None), "null lm_head"), (dict(w_dev=W + 4), "16-byte aligned")])
def test_configurations(call, over, says):
    assert call(cfg(**over)) != 0
    assert says in B.lib().ms_last_error().decode()


@pytest.mark.parametrize("d_h,d_w", [(H + 16, None), (H - 16, None), (W + 16, None), (W - 16, None), (DH, DH + 512), (None, H + 16), (None, W), (None, W - 1024 * 128 * 4 + 16), (DW + 16, DW)])
def test_gradients_over_something_else(d_h, d_w):
    assert tkd(cfg(), d_h=d_h, d_w=d_w) != 0
    assert "overlap" in B.lib().ms_last_error().decode()
    assert tkd(cfg(), d_h=H, d_w=None, size=8) != 0 and "workspace" in B.lib().ms_last_error().decode()       # over the states: what comes after is checked
    assert tkd(cfg(), d_h=H + 4 * 128 * 2, d_w=W - 1024 * 128 * 4, size=8) != 0 and "workspace" in B.lib().ms_last_error().decode()


@pytest.mark.parametrize("call,says", [
    (lambda: top(cfg(), k=0), "k must be"), (lambda: top(cfg(), k=129), "k must be"), (lambda: top(cfg(vocab=8), k=9), "k must be"), (lambda: top(cfg(), n=-1), "negative token count"),
    (lambda: top(cfg(), out=None), "null pointer"), (lambda: top(cfg(), h=None), "null pointer"), (lambda: top(cfg(), h=H + 8), "16-byte aligned"), (lambda: top(cfg(), size=16), "workspace 16 <"),
    (lambda: top(cfg(), ws=None), "null pointer"), (lambda: tkd(cfg(), k=0), "k must be"), (lambda: tkd(cfg(), k=200), "k must be"), (lambda: tkd(cfg(), ids=None), "null pointer"),
    (lambda: tkd(cfg(), loss=None), "loss_dev"), (lambda: tkd(cfg(), d_h=DH + 2), "16-byte aligned"), (lambda: tkd(cfg(), size=100), "workspace 100 <"),
    (lambda: policy(cfg(), low=1.5), "clip_low"), (lambda: policy(cfg(), low=-0.1), "clip_low"), (lambda: policy(cfg(), high=float("nan")), "clip_high"), (lambda: policy(cfg(), kl=-1.0), "kl_coef"),
    (lambda: policy(cfg(), kl=0.1), "kl_coef without ref_logp"), (lambda: policy(cfg(), labels=None), "null pointer"), (lambda: policy(cfg(), loss=None), "loss_dev"),
    (lambda: policy(cfg(), d_w=DW + 4), "16-byte aligned"), (lambda: policy(cfg(), size=64), "workspace 64 <"),
    (lambda: pref(cfg(), cu=(0, 2, 3, 4)), "no pairs"), (lambda: pref(cfg(), cu=(0, 3, 2)), "cu_seqlens"), (lambda: pref(cfg(), cu=(1, 2, 4)), "from 0 to"), (lambda: pref(cfg(), cu=(0, 5, 4)), "must not decrease"),
    (lambda: pref(cfg(), beta=0.0), "beta"), (lambda: pref(cfg(), eps=1.0), "label_smoothing"), (lambda: pref(cfg(), dev=None), "null cu_seqlens"), (lambda: pref(cfg(), size=64), "workspace 64 <"),
    (lambda: pref(cfg(hidden=65536), cu=(0, 2, 40000), n=40000), "in one block"),
    (lambda: logp(cfg(), out=None), "null pointer"), (lambda: logp(cfg(), labels=None), "null pointer"), (lambda: logp(cfg(), size=8), "workspace 8 <"),
    (lambda: logp_back(cfg(), d_logp=None), "null pointer"), (lambda: logp_back(cfg(), d_h=None), "null pointer")])
def test_arguments(call, says):
    assert call() != 0
    assert says in B.lib().ms_last_error().decode()


def test_the_binding_checks_its_tensors():
    h, w = torch.zeros(4, 64), torch.zeros(16, 64)
    for f in (lambda: B.top_logits(h, w, 3), lambda: B.token_logprobs(h, w, torch.zeros(4, dtype=torch.int32)), lambda: B.top_logits(h.double(), w, 3), lambda: B.top_logits([1], w, 3),
              lambda: B.topk_kd_loss_forward_backward(h, w, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3))):
        with pytest.raises(ValueError, match="expected"):
            f()


def test_workspace_grows_with_the_call():
    q = lambda **k: B._fn("ms_head_workspace_bytes")(C.byref(cfg(**{a: b for a, b in k.items() if a in dict(B._HeadCfg._fields_)})), k.get("n", 100), k.get("k", 0), k.get("back", 1))
    assert 0 < q(back=0) < q() < q(k=64) and q(n=200) > q()
    assert q(n=100000, token_block=64) < q(n=100000)
    assert q(vocab=-8) == 0 and q(n=-1) == 0 and q(k=129) == 0 and q(token_block=-8) == 0
    for c in (cfg(vocab=151936, hidden=1536), cfg(vocab=32000, hidden=1024), cfg(vocab=1024, dtype=B.MS_F32)):
        for n in (1, 7, 4096, 32768, 200000):
            need = B._fn("ms_head_workspace_bytes")(C.byref(c), n, 64, 1)
            assert 0 < need < 40 << 30
            assert 0 < B._fn("ms_top_logits_workspace_bytes")(C.byref(c), n, 64) < 16 << 30


@pytest.mark.parametrize("vocab,hidden,dtype", [(151936, 1536, "bf16"), (32000, 1024, "bf16"), (32000, 64, "bf16"), (32000, 72, "bf16"), (1024, 128, "fp32"), (151936, 512, "fp32")])
@pytest.mark.parametrize("k", [0, 64])
@pytest.mark.parametrize("block", [0, 40, 4096])
def test_memory_for_many_tokens_serves_fewer(vocab, hidden, dtype, k, block):
    c = C.byref(cfg(vocab=vocab, hidden=hidden, dtype=B.MS_F32 if dtype == "fp32" else B.MS_BF16, token_block=block))
    ns = [*range(0, 700), *range(700, 9000, 13), *range(9000, 140000, 397)]
    queries = [lambda n, b=b: B._fn("ms_head_workspace_bytes")(c, n, k, b) for b in (0, 1)]
    queries.append(lambda n: B._fn("ms_preference_workspace_bytes")(c, n, n // 2, 1) if k == 0 and n < 100000 else 0)
    queries.append(lambda n: B._fn("ms_top_logits_workspace_bytes")(c, n, k) if k else 0)
    for q in queries:
        need = [q(n) for n in ns]
        assert all(a <= b or b == 0 for a, b in zip(need, need[1:]))
