"""Losses, log-probabilities and top logits at the end of a decoder section (oracle).

z = h w^T / T are a token's logits and q = softmax(z); every loss is a sum of terms of log q, so its gradient goes through
dz, then d_h = dz w and d_w = dz^T h:

  log-probability of a label l:  logp = ln q_l,                         dz = g / T (1_l - q)       for d loss / d logp = g
  teacher's entries (ids, t):    KL = sum p (ln p - ln q),              dz = scale / T (q sum p - p)
      p = e^(t / T - L), L = ln sum e^(t / T) over the entries, or given
  clipped policy loss:           r = e^(logp - old), u = ref - logp,    g = scale weight (-[inside] r A + kl (1 - e^u))
      weight (-min(r A, clip(r, 1 - low, 1 + high) A) + kl (e^u - u - 1))
  preference loss:               m = sum_chosen (logp - ref) - sum_rejected (logp - ref),  g = +- scale beta (s(x) - 1 + eps)
      -(1 - eps) ln s(x) - eps ln s(-x),  x = beta m

Tokens with a label outside the vocabulary, or without an entry, take no part.
"""
import numpy as np


def _log_softmax(z):
    m = np.max(z, axis=1, keepdims=True)
    return z - m - np.log(np.sum(np.exp(z - m), axis=1, keepdims=True))


def _gradients(h, w, at, dz):
    d_h = np.zeros_like(h)
    d_h[at] = dz @ w
    return d_h, dz.T @ h[at]


def top_logits(h, w, k, temperature):
    """(values, ids, lse): the k largest of h w^T, equal ones by their ids."""
    z = h @ w.T
    ids = np.argsort(-z, axis=1, kind="stable")[:, :k]
    m = np.max(z, axis=1)
    return np.take_along_axis(z, ids, 1), ids, m / temperature + np.log(np.sum(np.exp((z - m[:, None]) / temperature), axis=1))


def entries(ids, top, vocab, temperature, lse_teacher=None):
    """(p, counts) [n, k]: the teacher's probabilities of the entries that count; a token's first entry of an id does, if its id is in the vocabulary."""
    n, k = ids.shape
    p, counts = np.zeros((n, k)), np.zeros((n, k), dtype=bool)
    for t in range(n):
        seen = set()
        for j in range(k):
            if 0 <= ids[t, j] < vocab and ids[t, j] not in seen and top[t, j] > -np.inf:
                counts[t, j] = True
                seen.add(ids[t, j])
        y = top[t, counts[t]] / temperature
        if y.size:
            p[t, counts[t]] = np.exp(y - (np.max(y) + np.log(np.sum(np.exp(y - np.max(y)))) if lse_teacher is None else lse_teacher[t]))
    return p, counts


def topk_kd(h, w, ids, top, temperature, loss_scale, lse_teacher=None):
    n, vocab = h.shape[0], w.shape[0]
    p, counts = entries(ids, top, vocab, temperature, lse_teacher)
    at = np.nonzero(counts.any(1))[0]
    lq = _log_softmax(h[at] @ w.T / temperature)
    full, kl = np.zeros_like(lq), np.zeros(n)
    for i, t in enumerate(at):
        c = counts[t] & (p[t] > 0)
        full[i, ids[t, c]] = p[t, c]
        kl[t] = np.sum(p[t, c] * (np.log(p[t, c]) - lq[i, ids[t, c]]))
    dz = loss_scale / temperature * (np.exp(lq) * full.sum(1, keepdims=True) - full)
    d_h, d_w = _gradients(h, w, at, dz)
    return dict(loss=loss_scale * kl.sum(), kl_tok=kl, d_h=d_h, d_w=d_w, dz=dz, at=at, scale=loss_scale / temperature * full.sum(1), selected=full > 0)


def token_logprobs(h, w, labels, temperature, g=None):
    """dict(logp); with g = d loss / d logp, its gradients too (of the rows `at`: dz, and scale: dz = scale q but where selected).  g may be a
    function of logp."""
    n, vocab = h.shape[0], w.shape[0]
    at = np.nonzero((labels >= 0) & (labels < vocab))[0]
    lq = _log_softmax(h[at] @ w.T / temperature)
    logp = np.zeros(n)
    logp[at] = lq[np.arange(at.size), labels[at]]
    out = dict(logp=logp)
    if g is not None:
        grad = g(logp) if callable(g) else g
        dz = -np.exp(lq)
        dz[np.arange(at.size), labels[at]] = -np.expm1(logp[at])
        dz *= grad[at, None] / temperature
        out["d_h"], out["d_w"] = _gradients(h, w, at, dz)
        selected = np.zeros(dz.shape, dtype=bool)
        selected[np.arange(at.size), labels[at]] = True
        out.update(grad=np.where(np.isin(np.arange(n), at), grad, 0.0), dz=dz, at=at, scale=-grad[at] / temperature, selected=selected)
    return out


def policy(h, w, labels, old, adv, low, high, kl=0.0, ref=None, weights=None, temperature=1.0, loss_scale=1.0):
    n, vocab = h.shape[0], w.shape[0]
    ok = (labels >= 0) & (labels < vocab)
    loss_tok, steep = np.zeros(n), np.zeros(n)

    def gradient(logp):
        g = np.zeros(n)
        for t in np.nonzero(ok)[0]:
            r, a, wt = np.exp(logp[t] - old[t]), adv[t], 1.0 if weights is None else weights[t]
            gain = min(r * a, np.clip(r, 1 - low, 1 + high) * a)
            term, slope = -gain, -r * a if gain == r * a else 0.0
            if kl:
                u = ref[t] - logp[t]
                term += kl * (np.expm1(u) - u)
                slope -= kl * np.expm1(u)
            loss_tok[t], g[t] = wt * term, loss_scale * wt * slope
            steep[t] = loss_scale * wt * (abs(r * a) + (kl * np.exp(ref[t] - logp[t]) if kl else 0.0))     # at least |d slope / d logp|
        return g
    out = token_logprobs(h, w, labels, temperature, gradient)
    return dict(out, loss_tok=loss_tok, loss=loss_scale * loss_tok.sum(), steep=steep)


def preference(h, w, labels, cu, beta, eps=0.0, ref=None, temperature=1.0, loss_scale=1.0):
    n, vocab, pairs = h.shape[0], w.shape[0], (len(cu) - 1) // 2
    ok = (labels >= 0) & (labels < vocab)
    margin, terms = np.zeros(pairs), np.zeros(pairs)

    def gradient(logp):
        g = np.zeros(n)
        diff = np.where(ok, logp - (0.0 if ref is None else np.where(ok, ref, 0.0)), 0.0)
        for i in range(pairs):
            a, b, c = cu[2 * i:2 * i + 3]
            if not ok[a:c].any():
                continue
            margin[i] = diff[a:b].sum() - diff[b:c].sum()
            x = beta * margin[i]
            terms[i] = (1 - eps) * np.logaddexp(0.0, -x) + eps * np.logaddexp(0.0, x)
            slope = loss_scale * beta * (eps * np.exp(-np.logaddexp(0.0, -x)) - (1 - eps) * np.exp(-np.logaddexp(0.0, x)))
            g[a:b], g[b:c] = slope, -slope
        return np.where(ok, g, 0.0)
    out = token_logprobs(h, w, labels, temperature, gradient)
    return dict(out, margin=margin, loss=loss_scale * terms.sum())
