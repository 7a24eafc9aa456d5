"""What is measured of the operators at the end of a decoder section that train it on something else than a whole teacher.

All of them take hidden states and an lm_head and meet the vocabulary inside:

* top: a frozen teacher's k largest logits of each token, their ids and the log-sum-exp, as they are stored for later distillation.
* tkd: distillation from such stored logits, forward and backward.
* logp: log-probabilities of given tokens, as a frozen reference or a behaviour policy reports them.
* policy: clipped policy loss with a KL term towards a reference, forward and backward.
* pref: preference loss over pairs of sequences (log ratios to a reference), forward and backward.

`own` selects the framework's kernels; without it `run` is the plain form.  Hidden sizes and vocabularies are those of the decoder
configurations in workloads.py; token counts run from one token to the largest packed micro-batch.  The gradient of an lm_head is
accumulated in fp32; that of a bf16 lm_head is compared in bf16, the type of the products that it is a sum of.
"""
import math

import torch

own = False
DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
# hidden size, vocabulary, type
HEADS = {"c1_teacher": (256, 1024, "fp32"), "c1_student": (128, 1024, "fp32"),
         "c2_teacher": (2048, 32000, "bf16"), "c2_student": (1024, 32000, "bf16"),
         "c5_teacher": (4096, 151936, "bf16"), "c5_student": (1536, 151936, "bf16")}
STD = 0.02                                            # of the lm_heads
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
BETA, SMOOTHING = 0.1, 0.05


def listed():
    return [
        # the teacher's best candidates for one token: reads the lm_head, latency is all else that it costs
        dict(name="top_token", kind="top", cfg="c5_teacher", n=1, k=64, t=1.0),
        # a short fp32 batch
        dict(name="top_fp32", kind="top", cfg="c1_teacher", n=293, k=20, t=2.0),
        # a document through the widest teacher
        dict(name="top_teacher", kind="top", cfg="c5_teacher", n=4096, k=64, t=1.0),
        # one more token of a sequence that a reference scores
        dict(name="logp_token", kind="logp", cfg="c5_student", n=1, seqs=1, share=1.0, t=1.0),
        # a sequence of odd length with its prompt left out
        dict(name="logp_odd", kind="logp", cfg="c2_student", n=777, seqs=1, share=0.7, t=1.0),
        # four short samples in fp32, some of the tokens padding
        dict(name="tkd_fp32", kind="tkd", cfg="c1_student", n=293, k=20, t=1.0, whole=False),
        # one sample of odd length, probabilities over the teacher's whole vocabulary
        dict(name="tkd_odd", kind="tkd", cfg="c2_student", n=1031, k=33, t=2.0, whole=True),
        # the largest micro-batch at the largest vocabulary
        dict(name="tkd_student", kind="tkd", cfg="c5_student", n=32768, k=64, t=1.0, whole=False),
        # a few answers of a small policy, forty in a hundred tokens are prompt
        dict(name="policy_odd", kind="policy", cfg="c2_student", n=2053, seqs=5, share=0.6, t=1.0),
        # sixteen answers of the largest student
        dict(name="policy_student", kind="policy", cfg="c5_student", n=16384, seqs=16, share=0.75, t=1.0),
        # three short pairs
        dict(name="pref_odd", kind="pref", cfg="c2_student", n=1337, seqs=6, share=0.6, t=1.0),
        # eight pairs of answers to long prompts
        dict(name="pref_student", kind="pref", cfg="c5_student", n=8192, seqs=16, share=0.5, t=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "logp", "tkd", "tkd", "policy", "policy", "pref", "pref"])
    t = rng.choice([1.0, 1.0, 0.7, 2.0])
    if kind == "top":
        cfg = rng.choice(list(HEADS))
        return dict(kind=kind, cfg=cfg, n=_log_int(rng, 1, 4096), k=_log_int(rng, 1, 128), t=t)
    cfg = rng.choice([c for c in HEADS if c.endswith("student")])
    if kind == "tkd":
        return dict(kind=kind, cfg=cfg, n=_log_int(rng, 1, 32768), k=_log_int(rng, 1, 128), t=t, whole=rng.random() < 0.5)
    n = _log_int(rng, 2, 32768 if kind == "logp" else 16384)
    seqs = 2 * rng.randint(1, max(1, min(8, n // 4)))
    return dict(kind=kind, cfg=cfg, n=n, seqs=seqs, share=round(rng.uniform(0.3, 1.0), 2), t=t)


# ------------------------------------------------------------------ inputs
def _lengths(case):
    """Lengths of the packed sequences: uneven, their sum is n."""
    n, seqs = case["n"], case["seqs"]
    part = [1.0 + 0.7 * math.sin(1.0 + 2.3 * i) for i in range(seqs)]
    cuts = [round(n * sum(part[:i]) / sum(part)) for i in range(seqs + 1)]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _scored(case):
    """Tokens of each sequence that count: its last ones."""
    return [max(1, round(case["share"] * m)) if m else 0 for m in _lengths(case)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    (d, vocab, dtype), n, kind = HEADS[case["cfg"]], case["n"], case["kind"]
    dt = BF16 if dtype == "bf16" else F32

    def normal(shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=F32, device=DEV).normal_(mean, std, generator=gen)

    def uniform(shape, lo=0.0, hi=1.0):
        return torch.empty(shape, dtype=F32, device=DEV).uniform_(lo, hi, generator=gen)

    s = dict(case=case, kind=kind)
    if kind == "top":
        # values on a grid so coarse that fp32 sums of their products have no rounding in any order: then logits that are equal
        # are so everywhere, and which of them comes first is decided by their ids
        s["h"] = (torch.round(normal((n, d)) * 8) / 8).to(dt)
        s["w"] = (torch.round(normal((vocab, d), STD) * 512) / 512).to(dt)
        return s
    s["w"] = normal((vocab, d), STD).to(dt)
    if kind != "logp":
        s["d_w"] = torch.zeros((vocab, d), dtype=F32, device=DEV)
    lift = 1.0 / (STD * STD * d)                      # hidden states lean towards the row of what follows, as trained ones do
    if kind == "tkd":
        k = case["k"]
        gap = 1 + torch.exp(uniform((n, k)) * math.log(vocab / k)).long().clamp_(max=max(1, vocab // k - 1))
        ids = (torch.cumsum(gap, 1) + (uniform((n, 1)) * vocab).long()) % vocab                 # distinct within a row
        top = normal((n, 1), 2.0, 18.0) - torch.cumsum(-0.3 * torch.log(uniform((n, k), 1e-6)), 1)
        s["lse"] = torch.logsumexp(top / case["t"], 1) + 0.5 * uniform((n,)) if case["whole"] else None
        few = torch.arange(k, device=DEV) >= torch.where(uniform((n, 1)) < 0.1, (uniform((n, 1)) * k).long() + 1, k)
        few |= uniform((n, 1)) > (0.97 if n > 8 else 1.5)                                       # padding: a row without entries
        s["ids"] = torch.where(few, -1, ids).to(torch.int32)
        s["top"] = torch.where(few, float("nan"), top)
        h = normal((n, d))
        for j in range(min(k, 3)):
            h.add_(s["w"][ids[:, j]].float() * (uniform((n, 1), 1.0, 9.0) / (1 + j)), alpha=lift)
        s["h"] = h.to(dt)
        return s
    labels = torch.exp(uniform((n,)) * math.log(vocab)).long().clamp_(1, vocab) - 1             # as frequent as words are
    s["h"] = (normal((n, d)) + s["w"][labels].float() * uniform((n, 1), 3.0, 14.0) * lift).to(dt)
    lens, scored = _lengths(case), _scored(case)
    seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV), output_size=n)
    ends = torch.tensor(lens, device=DEV).cumsum(0)
    counts = ends[seq] - torch.arange(n, device=DEV) <= torch.tensor(scored, device=DEV)[seq]
    s["labels"] = torch.where(counts, labels, -100).to(torch.int32)
    if kind == "logp":
        return s
    # about what this model itself says of the tokens (over a large vocabulary the logits of all others are as good as normal)
    z = (s["h"].float() * s["w"][labels].float()).sum(1) / case["t"]
    rest = math.log(vocab) + 0.5 * (STD / case["t"] * s["h"].float().norm(dim=1)).square()
    lse = torch.logaddexp(rest, z) if vocab > 4096 else torch.logsumexp(s["h"].float() @ s["w"].float().t() / case["t"], 1)
    logp = z - lse
    # what training has changed since the reference: some of it goes one way for a whole sequence
    s["ref_logp"] = torch.where(counts, logp + normal((n,), 0.3) + normal((len(lens),), 0.05)[seq], float("nan"))
    if kind == "policy":
        # ratios keep clear of the clip's borders, where the last digit of a logarithm decides
        near, far = uniform((n,), -0.15, 0.15), uniform((n,), 0.32, 0.6) * torch.where(uniform((n,)) < 0.5, -1.0, 1.0)
        s["old_logp"] = torch.where(counts, logp + torch.where(uniform((n,)) < 0.8, near, far), float("nan"))
        s["adv"] = torch.where(counts, normal((len(lens),))[seq], float("nan"))
        s["weights"] = 1.0 / (len(lens) * torch.tensor(scored, device=DEV, dtype=F32)[seq])     # mean over a sequence's tokens, then over sequences
        return s
    s["cu"], s["seq"], s["batch"] = [0] + [int(v) for v in ends], seq, None
    return s


# ------------------------------------------------------------------ plain forms
def _plain_lse(z):
    m = z.amax(1, keepdim=True)
    return m + torch.log(torch.exp(z - m).sum(1, keepdim=True))


def _plain_top(s):
    z = s["h"].float() @ s["w"].float().t()
    lse = _plain_lse(z / s["case"]["t"])[:, 0]
    top, ids = torch.sort(z, dim=1, descending=True, stable=True)
    k = s["case"]["k"]
    return dict(top=top[:, :k].contiguous(), ids=ids[:, :k].to(torch.int32), lse=lse)


def _plain_grads(s, h, w, dz):
    """Gradients of hidden states and lm_head from those of the logits."""
    dh = (dz @ w).to(s["h"].dtype)
    s["d_w"] += dz.t() @ h
    return dict(d_h=dh, d_w=s["d_w"].to(s["w"].dtype))


def _plain_tkd(s):
    t, n = s["case"]["t"], s["case"]["n"]
    ok = s["ids"] >= 0
    some = ok.any(1, keepdim=True)
    h, w = torch.where(some, s["h"].float(), 0.0), s["w"].float()
    top = torch.where(ok, s["top"] / t, -math.inf)
    lse_t = torch.where(some, _plain_lse(torch.where(some, top, 0.0)), 0.0) if s["lse"] is None else s["lse"][:, None]
    log_p = top - lse_t
    p = torch.exp(log_p)
    z = (h @ w.t()).mul_(1 / t)
    lse = _plain_lse(z)
    at = s["ids"].long().clamp(min=0)
    log_q = z.gather(1, at) - lse
    kl = torch.where(ok, p * (log_p - log_q), 0.0).sum(1)
    dz = z.sub_(lse).exp_().mul_(p.sum(1, keepdim=True)).scatter_add_(1, at, -p).mul_(1 / (n * t))
    return dict(loss=kl.sum() / n, kl=kl, **_plain_grads(s, h, w, dz))


def _plain_logp(s):
    ok = s["labels"] >= 0
    at = s["labels"].long().clamp(min=0)[:, None]
    h, w = torch.where(ok[:, None], s["h"].float(), 0.0), s["w"].float()
    z = (h @ w.t()).mul_(1 / s["case"]["t"])
    lse = _plain_lse(z)
    return ok, at, h, w, z, lse, torch.where(ok, (z.gather(1, at) - lse)[:, 0], 0.0)


def _plain_label_grads(s, parts, g):
    """Gradients from those of the tokens' log-probabilities."""
    _, at, h, w, z, lse, _ = parts
    dz = z.sub_(lse).exp_().mul_(-g[:, None]).scatter_add_(1, at, g[:, None]).mul_(1 / s["case"]["t"])
    return _plain_grads(s, h, w, dz)


def _plain_policy(s):
    parts = _plain_logp(s)
    ok, logp = parts[0], parts[-1]
    old, ref, adv = (torch.where(ok, s[k], 0.0) for k in ("old_logp", "ref_logp", "adv"))
    ratio = torch.exp(logp - old)
    inside = torch.where(adv > 0, ratio <= 1 + CLIP_HIGH, ratio >= 1 - CLIP_LOW)
    gain = torch.where(inside, ratio, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)) * adv
    away = torch.exp(ref - logp)
    weight = torch.where(ok, s["weights"], 0.0)
    loss = weight * (KL * (away - (ref - logp) - 1) - gain)
    g = weight * (KL * (1 - away) - torch.where(inside, ratio * adv, 0.0))
    return dict(loss=loss.sum(), loss_tok=loss, logp=logp, **_plain_label_grads(s, parts, g))


def _plain_pref(s):
    parts = _plain_logp(s)
    ok, logp = parts[0], parts[-1]
    diff = torch.where(ok, logp - s["ref_logp"], 0.0)
    pairs = len(s["cu"]) // 2
    of_seq = torch.zeros(2 * pairs, dtype=F64, device=DEV).index_add_(0, s["seq"], diff.double()).view(-1, 2)
    margin = (of_seq[:, 0] - of_seq[:, 1]).float()
    x = BETA * margin
    log_win, log_lose = -torch.log1p(torch.exp(-x)), -torch.log1p(torch.exp(x))
    loss = -((1 - SMOOTHING) * log_win + SMOOTHING * log_lose)
    slope = BETA / pairs * (SMOOTHING * torch.sigmoid(x) - (1 - SMOOTHING) * torch.sigmoid(-x))
    g = torch.where(ok, torch.stack((slope, -slope), 1).view(-1)[s["seq"]], 0.0)
    return dict(loss=loss.mean(), margin=margin, logp=logp, **_plain_label_grads(s, parts, g))


# ------------------------------------------------------------------ one pass
def run(s):
    kind, case = s["kind"], s["case"]
    if not own:
        if kind == "top":
            return _plain_top(s)
        if kind == "tkd":
            return _plain_tkd(s)
        if kind == "logp":
            return dict(logp=_plain_logp(s)[-1])
        return _plain_policy(s) if kind == "policy" else _plain_pref(s)
    from paper_2605_10501_amd import binding as B
    t = case["t"]
    if kind == "top":
        top, ids, lse = B.top_logits(s["h"], s["w"], case["k"], temperature=t)
        return dict(top=top, ids=ids, lse=lse)
    if kind == "logp":
        return dict(logp=B.token_logprobs(s["h"], s["w"], s["labels"], temperature=t))
    if kind == "tkd":
        out = B.topk_kd_loss_forward_backward(s["h"], s["w"], s["ids"], s["top"], lse_teacher=s["lse"], temperature=t, d_w=s["d_w"])
        keep = dict(loss=out["loss"], kl=out["kl_tok"])
    elif kind == "policy":
        out = B.policy_loss_forward_backward(s["h"], s["w"], s["labels"], s["old_logp"], s["adv"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                                             ref_logp=s["ref_logp"], kl_coef=KL, weights=s["weights"], temperature=t, loss_scale=1.0, d_w=s["d_w"])
        keep = {k: out[k] for k in ("loss", "loss_tok", "logp")}
    else:
        s["batch"] = s["batch"] or B.Batch(s["cu"])                       # packed once, as its program keeps it
        out = B.preference_loss_forward_backward(s["h"], s["w"], s["labels"], s["batch"], beta=BETA, ref_logp=s["ref_logp"],
                                                 label_smoothing=SMOOTHING, temperature=t, d_w=s["d_w"])
        keep = {k: out[k] for k in ("loss", "margin", "logp")}
    return dict(keep, d_h=out["d_h"], d_w=s["d_w"].to(s["w"].dtype))


# ------------------------------------------------------------------ necessary work
def work(case):
    (d, vocab, dtype), n, kind = HEADS[case["cfg"]], case["n"], case["kind"]
    es = 2 if dtype == "bf16" else 4
    if kind == "top":
        return dict(bytes=(n + vocab) * d * es + n * (8 * case["k"] + 4), flops=2.0 * n * vocab * d)
    rows = n if kind == "tkd" else sum(_scored(case))
    if kind == "logp":
        return dict(bytes=(rows + vocab) * d * es + 8 * n, flops=2.0 * rows * vocab * d)
    # the lm_head and the tokens that count are read, their gradients written (the lm_head's read, added to and given out)
    small = n * (8 * case["k"] + 8) if kind == "tkd" else 28 * n
    return dict(bytes=(rows + n + 2 * vocab) * d * es + 8 * vocab * d + small, flops=6.0 * rows * vocab * d)


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    n, t, kind = case["n"], case["t"], case["kind"]
    w, rows = s["w"].double(), 2048
    vocab, d = w.shape
    if kind == "top":
        top, lse = [], []
        for i in range(0, n, rows):
            z = s["h"][i:i + rows].double() @ w.T
            top.append(torch.topk(z, case["k"], dim=1).values)
            lse.append(torch.logsumexp(z / t, 1))
        return dict(top=torch.cat(top), ids=None, lse=torch.cat(lse))
    d_h, d_w = torch.zeros((n, d), dtype=F64, device=DEV), torch.zeros((vocab, d), dtype=F64, device=DEV)

    def blocks():
        """Tokens that count, a block at a time: where they are, their hidden states, the log-probabilities of everything."""
        have = (s["ids"] >= 0).any(1) if kind == "tkd" else s["labels"] >= 0
        at = torch.nonzero(have).view(-1)
        for i in range(0, at.numel(), rows):
            a = at[i:i + rows]
            h = s["h"][a].double()
            yield a, h, torch.log_softmax(h @ w.T / t, 1)

    def gradients(a, h, g):
        g = g / t
        d_h[a] = g @ w
        d_w.add_(g.T @ h)

    if kind == "tkd":
        kl = torch.zeros(n, dtype=F64, device=DEV)
        for a, h, log_q in blocks():
            full = torch.zeros_like(log_q)                                # the teacher's probabilities, spread over the vocabulary
            r, c = torch.nonzero(s["ids"][a] >= 0, as_tuple=True)
            y = torch.full(s["ids"][a].shape, -math.inf, dtype=F64, device=DEV)
            y[r, c] = s["top"][a][r, c].double() / t
            y = y - (torch.logsumexp(y, 1) if s["lse"] is None else s["lse"][a].double())[:, None]
            where = s["ids"][a][r, c].long()
            full[r, where] = torch.exp(y[r, c])
            kl[a] = torch.zeros_like(kl[a]).index_add_(0, r, full[r, where] * (y[r, c] - log_q[r, where]))
            gradients(a, h, (torch.exp(log_q) * full.sum(1, keepdim=True) - full) / n)
        return dict(loss=kl.sum() / n, kl=kl, d_h=d_h, d_w=d_w)
    logp = torch.zeros(n, dtype=F64, device=DEV)
    for a, _, log_q in blocks():
        logp[a] = log_q[torch.arange(a.numel(), device=DEV), s["labels"][a].long()]
    if kind == "logp":
        return dict(logp=logp)
    ok = s["labels"] >= 0
    if kind == "policy":
        r = torch.exp(logp - s["old_logp"].double())
        a = s["adv"].double()
        gain = torch.minimum(r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a)
        u = s["ref_logp"].double() - logp
        loss = torch.where(ok, s["weights"].double() * (KL * (torch.expm1(u) - u) - gain), 0.0)
        slope = torch.where(gain < r * a, 0.0, r * a)
        g = torch.where(ok, s["weights"].double() * (-KL * torch.expm1(u) - slope), 0.0)
        out = dict(loss=loss.sum(), loss_tok=loss, logp=logp)
    else:
        pairs = len(s["cu"]) // 2
        u = torch.where(ok, logp - s["ref_logp"].double(), 0.0)
        sums = torch.stack([u[a:b].sum() for a, b in zip(s["cu"], s["cu"][1:])])
        margin = sums[0::2] - sums[1::2]
        ls = torch.nn.functional.logsigmoid
        loss = -(1 - SMOOTHING) * ls(BETA * margin) - SMOOTHING * ls(-BETA * margin)
        win = torch.sigmoid(BETA * margin)
        slope = BETA / pairs * (win - (1 - SMOOTHING))
        g = torch.zeros(n, dtype=F64, device=DEV)
        for i, (a, b) in enumerate(zip(s["cu"], s["cu"][1:])):
            g[a:b] = slope[i // 2] * (1 - 2 * (i % 2))
        g = torch.where(ok, g, 0.0)
        out = dict(loss=loss.mean(), margin=margin, logp=logp)
    for a, h, log_q in blocks():
        q = -torch.exp(log_q)
        q[torch.arange(a.numel(), device=DEV), s["labels"][a].long()] += 1.0
        gradients(a, h, g[a][:, None] * q)
    return dict(out, d_h=d_h, d_w=d_w)
