"""Distillation from stored logits and preference losses where a block's exponentials or logits, or the lm_head's gradient, lie in several slabs: entries and labels on both sides of the slabs' border and
in the last column, and gradients that are put together from all slabs.  Against 64 bits a block of rows at a time; bounds as in test_gpu_head_large.py."""
import pytest
import torch

from paper_2605_10501_amd import binding as B
from test_gpu_head_large import _exact, _inputs, _near

pytestmark = pytest.mark.gpu
# by the tokens' exponentials (their entries' logits dot products of their own, and by marks), by logits in fp32 (bf16 and fp32), by the gradient of the lm_head
SIZES = [(torch.bfloat16, 8200, 64, 270336 + 8, 7), (torch.bfloat16, 7200, 1536, 300000, 100), (torch.bfloat16, 8200, 40, 140000, 64), (torch.float32, 4200, 40, 270336, 64),
         (torch.bfloat16, 70, 8192, 151936, 64)]


def _border(dtype, n, d, vocab):
    """The first column of the second slab, as the plan has it: slabs are as wide as reach allows, of equal numbers of 256 columns."""
    reach = 2 ** 32 - 2 ** 20
    ez = 2 if dtype == torch.bfloat16 and d % 64 == 0 else 4
    rows = (n + 15) // 16 * 16
    wide = min(reach // ((4 if dtype == torch.bfloat16 else 2) * d) - 512, reach // (ez * (rows + 256))) // 256 * 256
    slabs = -(-vocab // wide)
    assert slabs > 1
    return (-(-vocab // slabs) + 255) // 256 * 256


def _scaled(dtype, n, d, vocab):
    h, w, labels, g = _inputs(dtype, n, d, vocab)
    return h, (w * (64 / max(d, 64)) ** 0.5).contiguous(), labels, g                     # logits as large as at 64 columns


def _tol(dtype):
    return 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -17


@pytest.mark.parametrize("dtype,n,d,vocab,k", SIZES)
@pytest.mark.parametrize("whole", [False, True])
def test_entries_over_several_slabs(dtype, n, d, vocab, k, whole):
    h, w, labels, g = _scaled(dtype, n, d, vocab)
    cut = _border(dtype, n, d, vocab)
    gen = torch.Generator(device="cuda").manual_seed(5)
    step = vocab // k
    ids = (torch.arange(k, device="cuda") * step + torch.randint(0, step, (n, k), generator=gen, device="cuda")).int()                                   # rising, distinct
    for j, v in enumerate((cut - 1, cut, cut + 1, vocab - 1, 0)):                         # beside the border, in the last column, in the first
        at = torch.arange(j, n, 5, device="cuda")
        place = min(v // step, k - 1)
        ids[at, place] = v
    ids = torch.where(labels[:, None] >= 0, ids, -1)
    ids = ids.gather(1, torch.argsort(torch.rand(n, k, generator=gen, device="cuda"), 1))   # in any order
    top = torch.empty(n, k, device="cuda").normal_(0, 2, generator=gen)
    lse = torch.logsumexp(top.double(), 1).float() + 0.3 if whole else None
    ok = labels >= 0
    w64, kl = w.double(), torch.zeros(n, device="cuda", dtype=torch.float64)
    d_h, d_w = torch.zeros(n, d, device="cuda", dtype=torch.float64), torch.zeros(vocab, d, device="cuda", dtype=torch.float64)
    rows = torch.nonzero(ok).view(-1)
    for a in rows.split(512):
        lq = torch.log_softmax(h[a].double() @ w64.T, 1)
        lp = top[a].double() - (torch.logsumexp(top[a].double(), 1) if lse is None else lse[a].double())[:, None]
        p = torch.exp(lp)
        kl[a] = (p * (lp - lq.gather(1, ids[a].long()))).sum(1)
        dz = (lq.exp_() * p.sum(1, keepdim=True)).scatter_add_(1, ids[a].long(), -p) / n
        d_h[a] = dz @ w64
        d_w += dz.T @ h[a].double()
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.topk_kd_loss_forward_backward(h, w, ids, top, lse, d_w=got_w)
    tol = 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256 + 64 + 8 * kl.abs())                    # |h| . |w| below 20
    assert ((out["kl_tok"].double() - kl).abs() <= tol).all() and torch.all(out["kl_tok"][~ok] == 0)
    assert abs(out["loss"].item() - kl.sum().item() / n) <= tol.mean().item() + 2.0 ** -18 * abs(kl.sum().item()) / n
    _near(out["d_h"], d_h, _tol(dtype))
    _near(got_w, d_w, _tol(dtype))
    assert torch.all(out["d_h"][~ok] == 0)
    chosen = torch.unique(torch.tensor([0, cut - 1, cut, cut + 1, vocab - 1], device="cuda"))
    _near(got_w[chosen], d_w[chosen], _tol(dtype))
    only = B.topk_kd_loss_forward_backward(h, w, ids, top, lse, need_d_h=False)             # (a forward pass has other slabs, or none)
    assert torch.equal(only["kl_tok"], out["kl_tok"])


@pytest.mark.parametrize("dtype,n,d,vocab", [s[:4] for s in SIZES])
def test_preference_loss_over_several_slabs(dtype, n, d, vocab):
    h, w, labels, _ = _scaled(dtype, n, d, vocab)
    cut = _border(dtype, n, d, vocab)
    labels[5:9] = torch.tensor([cut - 1, cut, cut + 1, vocab - 1], dtype=torch.int32, device="cuda")
    cu = [0, n // 3, n // 2, n - n // 4, n]
    beta = 0.02 / n ** 0.5
    ok, logp, sign = labels >= 0, torch.zeros(n, device="cuda", dtype=torch.float64), torch.ones(n, device="cuda", dtype=torch.float64)
    w64 = w.double()
    for a in torch.nonzero(ok).view(-1).split(512):
        lq = torch.log_softmax(h[a].double() @ w64.T, 1)
        logp[a] = lq.gather(1, labels[a].long()[:, None])[:, 0]
    del lq, w64
    for i in (1, 3):
        sign[cu[i]:cu[i + 1]] = -1
    ref = (logp + 0.3 * torch.sin(torch.arange(n, device="cuda"))).float()
    diff = (logp - ref.double()) * sign * ok
    margin = torch.stack([diff[:cu[2]].sum(), diff[cu[2]:].sum()])
    slope = -0.5 * beta * torch.sigmoid(-beta * margin)                                    # loss_scale 1 / pairs
    g = torch.where(torch.arange(n, device="cuda") < cu[2], slope[0], slope[1]) * sign
    _, d_h, d_w = _exact(h, w, labels, g.float(), rows=512)
    got_w = torch.zeros(vocab, d, device="cuda")
    out = B.preference_loss_forward_backward(h, w, labels, B.Batch(cu), beta, ref_logp=ref, d_w=got_w)
    delta = 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256)
    assert (out["logp"].double() - logp).abs().max().item() < delta
    assert (out["margin"].double() - margin).abs().max().item() <= n * delta + 2.0 ** -22 * margin.abs().max().item()
    loss = torch.nn.functional.softplus(-beta * margin).mean().item()
    assert abs(out["loss"].item() - loss) <= beta * n * delta + 2.0 ** -20
    _near(out["d_h"], d_h, _tol(dtype) + beta * n * delta)
    _near(got_w, d_w, _tol(dtype) + beta * n * delta)
    assert torch.all(out["d_h"][~ok] == 0)


def test_forward_passes_over_several_slabs():
    """More logits than one launch takes (2^34): a token's numbers are those of blocks with one slab, logits of entries by marks among them."""
    n, d, vocab, k = 65536, 1024, 262144 + 8, 128
    h, w, labels, _ = _scaled(torch.bfloat16, n, d, vocab)
    cut = (-(-vocab // 2) + 255) // 256 * 256                                             # two slabs
    labels[5:9] = torch.tensor([cut - 1, cut, cut + 1, vocab - 1], dtype=torch.int32, device="cuda")
    logp = B.token_logprobs(h, w, labels)
    assert torch.equal(logp, B.token_logprobs(h, w, labels, token_block=4096))
    a = torch.arange(1024, device="cuda")
    lq = torch.log_softmax(h[a].double() @ w.double().T, 1)
    ref = torch.where(labels[a] >= 0, lq.gather(1, labels[a].long().clamp(min=0)[:, None])[:, 0], 0.0)
    delta = 2.0 ** -24 * (2 * d * 20 + 4 * 20 + 256)
    assert ((logp[a].double() - ref).abs() <= delta).all()
    gen = torch.Generator(device="cuda").manual_seed(6)
    step = vocab // k
    ids = (torch.arange(k, device="cuda") * step + torch.randint(0, step, (n, k), generator=gen, device="cuda")).int()
    ids[0::3, min(cut // step, k - 1)], ids[1::3, (cut - 1) // step], ids[2::3, k - 1] = cut, cut - 1, vocab - 1
    top = torch.empty(n, k, device="cuda").normal_(0, 2, generator=gen)
    one, many = (B.topk_kd_loss_forward_backward(h, w, ids, top, need_d_h=False, token_block=b) for b in (0, 4096))
    assert torch.equal(one["kl_tok"], many["kl_tok"])
    lp = torch.log_softmax(top[a].double(), 1)
    kl = (lp.exp() * (lp - lq.gather(1, ids[a].long()))).sum(1)
    assert ((one["kl_tok"][a].double() - kl).abs() <= delta + 2.0 ** -24 * (64 + 8 * kl.abs())).all()
