"""What is measured of three groups of operators that decoder sections are made of.

* qkn: RMSNorm of every query and key head of a packed qkv tensor and its rotation to the token's position, in one pass;
  as a frozen teacher runs it (forward) and as a student trains through it (forward and backward).
* emb: embedding rows times a scale, and the gradient of the table as sums over the tokens sorted by id.
* fp8: what a frozen teacher computes with its matrices in 8 bits, e4m3 with one power-of-two scale for each block of 128
  (weights: 128 x 128, activations: 128 of a row): weights laid out, a linear layer, a whole SwiGLU feed-forward block.

`own` selects the framework's kernels; without it `run` is the plain form.  Sizes are those of the decoder configurations
in workloads.py, token counts run from one token to the largest packed micro-batch.
"""
import math

import torch

from paper_2605_10501_amd import workloads as wl

own = False
DEV = "cuda"
BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
EPS = 1e-6
E4M3_MAX = 448.0
# d_model, query heads, key/value heads, head_dim, d_ffn, vocabulary
DECODERS = {"c1_teacher": (256, 4, 4, 64, 688, 1024), "c1_student": (128, 2, 2, 64, 344, 1024),
            "c2_teacher": (2048, 16, 4, 128, 5504, 32000), "c2_student": (1024, 8, 2, 128, 2816, 32000),
            "c5_teacher": (4096, 32, 8, 128, 11008, 151936), "c5_student": (1536, 12, 2, 128, 8960, 151936)}
MAX_POS = 16384                                       # the longest document of a pack


def listed():
    return [
        # the latest token of one sequence: latency is all it costs
        dict(name="qkn_token", kind="qkn", cfg="c5_teacher", dtype="bf16", n=1, train=False),
        # the fp32 student's heads on four short samples, forward and backward
        dict(name="qkn_fp32", kind="qkn", cfg="c1_student", dtype="fp32", n=293, train=True),
        # a student's micro-batch of odd length, forward and backward
        dict(name="qkn_student", kind="qkn", cfg="c5_student", dtype="bf16", n=20011, train=True),
        # the widest teacher on the largest micro-batch
        dict(name="qkn_teacher", kind="qkn", cfg="c5_teacher", dtype="bf16", n=32768, train=False),
        # fp32 embedding of a padded batch: one id takes a third of the tokens, some (image places) are outside the table
        dict(name="emb_padded", kind="emb", cfg="c1_student", dtype="fp32", n=293, ids="padded", scale=math.sqrt(128)),
        # the student's embedding on the largest micro-batch, ids as frequent as words are
        dict(name="emb_student", kind="emb", cfg="c5_student", dtype="bf16", n=32768, ids="text", scale=math.sqrt(1536)),
        # laying out a matrix of the teacher's feed-forward block in 8 bits, once per matrix
        dict(name="fp8_weights", kind="weights", cfg="c5_teacher", matrix="up", dtype="bf16"),
        # one token through the widest projection: reads the weights, computes next to nothing
        dict(name="fp8_token", kind="linear", cfg="c5_teacher", matrix="up", dtype="bf16", m=1, residual=False),
        # a contraction that ends inside a block, onto an fp32 residual stream
        dict(name="fp8_odd", kind="linear", cfg="c1_teacher", matrix="down", dtype="fp32", m=293, residual=True),
        # the attention's projections on one 4096-token document
        dict(name="fp8_qkv", kind="linear", cfg="c5_teacher", matrix="qkv", dtype="bf16", m=4096, residual=False),
        # norm, gate and up, SwiGLU, down on a single sample and on the largest micro-batch
        dict(name="ffn_sample", kind="ffn", cfg="c2_teacher", m=777),
        dict(name="ffn_teacher", kind="ffn", cfg="c5_teacher", m=32768),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["qkn", "qkn", "emb", "emb", "linear", "linear", "ffn", "weights"])
    if kind == "qkn":
        cfg = rng.choice(list(DECODERS))
        return dict(kind=kind, cfg=cfg, dtype="fp32" if cfg.startswith("c1") else rng.choice(["bf16", "bf16", "fp32"]),
                    n=_log_int(rng, 1, 32768), train=rng.random() < 0.6)
    if kind == "emb":
        cfg = rng.choice(list(DECODERS))
        return dict(kind=kind, cfg=cfg, dtype="fp32" if cfg.startswith("c1") else "bf16", n=_log_int(rng, 1, 32768),
                    ids=rng.choice(["text", "text", "even", "padded"]), scale=rng.choice([1.0, math.sqrt(DECODERS[cfg][0])]))
    # (a contraction over 344 is no multiple of 16: the products take rows of whole 16-byte pieces)
    cfg = rng.choice([c for c in DECODERS if c != "c1_student"])
    if kind == "linear":
        return dict(kind=kind, cfg=cfg, matrix=rng.choice(["qkv", "o", "up", "down"]), dtype=rng.choice(["bf16", "bf16", "fp32"]),
                    m=_log_int(rng, 1, 32768), residual=rng.random() < 0.4)
    if kind == "ffn":
        return dict(kind=kind, cfg=cfg, m=_log_int(rng, 1, 32768))
    return dict(kind=kind, cfg=cfg, matrix=rng.choice(["qkv", "o", "up", "down"]), dtype=rng.choice(["bf16", "fp32"]))


def _matrix(case, which=None):
    """(outputs, inputs) of one of a layer's four matrices."""
    d, nq, nkv, hd, f, _ = DECODERS[case["cfg"]]
    return {"qkv": ((nq + 2 * nkv) * hd, d), "o": (d, nq * hd), "up": (2 * f, d), "down": (d, f)}[which or case["matrix"]]


def _dtype(case):
    return BF16 if case["dtype"] == "bf16" else F32


# ------------------------------------------------------------------ inputs
def _ids(case, gen):
    vocab, n = DECODERS[case["cfg"]][5], case["n"]
    u = torch.rand(n, generator=gen, device=DEV, dtype=F64)
    if case["ids"] == "even":
        ids = (u * vocab).long()
    else:                                             # log-uniform: id k about as often as the k-th most frequent word
        ids = torch.exp(u * math.log(vocab)).long() - 1
    ids = ids.clamp_(0, vocab - 1)
    if case["ids"] == "padded":
        v = torch.rand(n, generator=gen, device=DEV)
        ids = torch.where(v < 0.35, torch.zeros_like(ids), torch.where(v > 0.9, torch.full_like(ids, -1), ids))
    return ids.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    d, nq, nkv, hd, f, vocab = DECODERS[case["cfg"]]

    def normal(shape, std=1.0, mean=0.0, dtype=BF16):
        return torch.empty(shape, dtype=F32, device=DEV).normal_(mean, std, generator=gen).to(dtype)

    s = dict(kind=kind, case=case)
    if kind == "qkn":
        n, dt = case["n"], _dtype(case)
        s["heads"] = (nq, nkv, hd)
        s["x"] = normal((n, (nq + 2 * nkv) * hd), 1.5, dtype=dt)
        s["g_q"], s["g_k"] = normal((hd,), 0.1, 1.0, dt), normal((hd,), 0.1, 1.0, dt)
        s["pos"] = (torch.arange(n, device=DEV) % (1 + MAX_POS * 3 // 4) + (MAX_POS // 4 - 1) * (n == 1)).to(torch.int32)
        angle = torch.arange(MAX_POS, device=DEV, dtype=F64)[:, None] * 1e4 ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=F64) / hd)
        s["table"] = torch.stack((angle.cos(), angle.sin()), -1).to(F32)
        if case["train"]:
            s["dy"] = normal(s["x"].shape, dtype=dt)
            s["dg_q"], s["dg_k"] = (torch.zeros(hd, dtype=F32, device=DEV) for _ in range(2))
    elif kind == "emb":
        dt = _dtype(case)
        s["ids"] = _ids(case, gen)
        s["table"] = normal((vocab, d), 0.02, dtype=dt)
        s["dx"] = normal((case["n"], d), dtype=dt)
        s["d_table"] = torch.zeros((vocab, d), dtype=F32, device=DEV)
    elif kind == "weights":
        s["w"] = normal(_matrix(case), 0.02, dtype=_dtype(case))
    else:
        def plan(which):                              # a matrix as a program keeps it: codes and exponents
            return _quantize(normal(_matrix(case, which), 0.02), 128)
        m = case["m"]
        n_in = _matrix(case)[1] if kind == "linear" else d
        x = normal((m, n_in), dtype=F32)
        x[:, ::211] *= 20.0                           # a few channels are far larger than the others
        x[m // 2:m // 2 + (m > 8)] = 0.0              # a padding row
        if kind == "linear":
            s["x"], s["w"] = x.to(_dtype(case)), plan(case["matrix"])
            s["residual"] = normal((m, _matrix(case)[0]), dtype=F32) if case["residual"] else None
        else:
            s["x"], s["g"] = x, normal((d,), 0.02, 1.0)
            s["up"], s["down"] = plan("up"), plan("down")
    return s


# ------------------------------------------------------------------ plain forms
def _rows_rms(t):
    return torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)


def _rotate(t, cos, sin):
    lo, hi = t.chunk(2, -1)
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1)


def _qkn_plain(s):
    nq, nkv, hd = s["heads"]
    n, dt = s["x"].shape[0], s["x"].dtype
    x = s["x"].float().view(n, -1, hd)
    cos, sin = s["table"][s["pos"].long()].unbind(-1)
    cos, sin = cos[:, None], sin[:, None]
    xh, gains = x[:, :nq + nkv], torch.cat((s["g_q"].float().expand(nq, hd), s["g_k"].float().expand(nkv, hd)))
    r = _rows_rms(xh)
    y = torch.cat((_rotate(xh * r * gains, cos, sin), x[:, nq + nkv:]), 1)
    out = dict(y=y.view(n, -1).to(dt))
    if s["case"]["train"]:
        dy = s["dy"].float().view(n, -1, hd)
        dn = _rotate(dy[:, :nq + nkv], cos, -sin)
        xn = xh * r
        t = dn * gains
        dx = torch.cat((r * (t - xn * (t * xn).mean(-1, keepdim=True)), dy[:, nq + nkv:]), 1)
        dg = (dn * xn).sum(0)
        s["dg_q"] += dg[:nq].sum(0)
        s["dg_k"] += dg[nq:].sum(0)
        out.update(dx=dx.view(n, -1).to(dt), dg_q=s["dg_q"], dg_k=s["dg_k"])
    return out


def _emb_plain(s):
    scale, ids, table = s["case"]["scale"], s["ids"].long(), s["table"]
    inside = ((ids >= 0) & (ids < table.shape[0]))[:, None]
    at = ids.clamp(0, table.shape[0] - 1)
    x = torch.where(inside, table[at].float() * scale, 0.0).to(table.dtype)
    s["d_table"].index_add_(0, at, torch.where(inside, s["dx"].float() * scale, 0.0))
    return dict(x=x, d_table=s["d_table"])


def _blocks(x, rows):
    """x [r, c] in blocks of `rows` x 128, padded with zeros: [blocks down, rows, blocks across, 128]."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % rows))
    return x.view(-1, rows, x.shape[1] // 128, 128)


def _quantize(x, rows):
    """Codes [r, c] and one exponent byte (2^(byte - 127)) per block, rows of them padded to whole words: the least power
    of two that brings the block's largest value to 448 or below; 1 for a block of zeros."""
    b = _blocks(x.float(), rows)
    mant, e = torch.frexp(b.abs().amax((1, 3)))
    e = torch.where(mant == 0, 0, e - 9 + (mant > 0.875).int()).clamp(min=-127)
    q = torch.ldexp(b, -e[:, None, :, None]).reshape(b.shape[0] * rows, -1)[:x.shape[0], :x.shape[1]].to(E4M3)
    return q.contiguous(), torch.nn.functional.pad(e + 127, (0, -e.shape[1] % 4), value=127).to(torch.uint8)


def _value(q, e, rows):
    """The fp32 values of codes and exponents."""
    n = -(-q.shape[1] // 128)
    return torch.ldexp(_blocks(q.float(), rows), (e[:, :n].int() - 127)[:, None, :, None]).reshape(-1, 128 * n)[:q.shape[0], :q.shape[1]]


def _linear_plain(x, w, residual=None):
    y = _value(*_quantize(x, 1), 1) @ _value(*w, 128).t()
    return y if residual is None else y + residual


def _ffn_plain(s):
    h = s["x"] * _rows_rms(s["x"]) * s["g"].float()
    gate, up = _linear_plain(h, s["up"]).chunk(2, -1)
    return _linear_plain(gate * torch.sigmoid(gate) * up, s["down"]).to(BF16)


# ------------------------------------------------------------------ one pass
def run(s):
    kind = s["kind"]
    if not own:
        if kind == "qkn":
            return _qkn_plain(s)
        if kind == "emb":
            return _emb_plain(s)
        if kind == "weights":
            return _quantize(s["w"], 128)
        if kind == "linear":
            return _linear_plain(s["x"], s["w"], s["residual"]).to(BF16 if s["residual"] is None else F32)
        return _ffn_plain(s)
    from paper_2605_10501_amd import binding as B
    if kind == "qkn":
        a = (*s["heads"], s["g_q"], s["g_k"], EPS, s["pos"], s["table"])
        out = dict(y=B.k_qk_norm_rope_forward(s["x"], *a))
        if s["case"]["train"]:
            out.update(dx=B.k_qk_norm_rope_backward(s["dy"], s["x"], *a, s["dg_q"], s["dg_k"]), dg_q=s["dg_q"], dg_k=s["dg_k"])
        return out
    if kind == "emb":
        x = B.k_embedding_scaled_forward(s["ids"], s["table"], s["case"]["scale"])
        return dict(x=x, d_table=B.k_embedding_sorted_backward(s["ids"], s["dx"], s["case"]["scale"], s["d_table"]))
    if kind == "weights":
        return B.k_fp8_quantize(s["w"], block_rows=128)
    if kind == "linear":
        return B.k_gemm_fp8(*B.k_fp8_quantize(s["x"]), *s["w"], residual=s["residual"])
    h = B.k_norm_fp8(s["x"], s["g"], EPS)
    return B.k_gemm_fp8(*B.k_gemm_fp8_swiglu(*h, *s["up"]), *s["down"])


# ------------------------------------------------------------------ necessary work
def _distinct(case):
    """Expected number of table rows that a batch touches."""
    vocab, n = DECODERS[case["cfg"]][5], case["n"]
    if case["ids"] == "even":
        return vocab * -math.expm1(n * math.log1p(-1.0 / vocab))
    k = torch.arange(1, vocab, dtype=F64)
    p = torch.log1p(1.0 / k) / math.log(vocab) * (0.55 if case["ids"] == "padded" else 1.0)
    return float((1.0 - (1.0 - p.clamp(max=1 - 1e-12)).pow(n)).sum())


def work(case):
    kind = case["kind"]
    d, nq, nkv, hd, f, vocab = DECODERS[case["cfg"]]
    if kind == "qkn":
        es, n, heads = (2 if case["dtype"] == "bf16" else 4), case["n"], nq + nkv
        row, all_ = heads * hd * es, (nq + 2 * nkv) * hd * es
        size = n * (2 * all_ + 4) + min(n, MAX_POS) * hd * 4
        return dict(bytes=size + (n * (2 * all_ + row) if case["train"] else 0), flops=n * heads * hd * (26.0 if case["train"] else 8.0))
    if kind == "emb":
        es, n, rows = (2 if case["dtype"] == "bf16" else 4), case["n"], _distinct(case)
        return dict(bytes=8 * n + rows * d * (es + 8) + 2 * n * d * es, flops=3.0 * n * d)
    if kind == "weights":
        r, c = _matrix(case)
        return dict(bytes=r * c * ((2 if case["dtype"] == "bf16" else 4) + 1), flops=2.0 * r * c)
    m = case["m"]
    if kind == "linear":
        n, k = _matrix(case)
        return dict(bytes=m * k * (2 if case["dtype"] == "bf16" else 4) + n * k + m * n * (8 if case["residual"] else 2), flops=2.0 * m * n * k)
    return dict(bytes=m * d * 6 + 3 * d * f, flops=6.0 * m * d * f)


# ------------------------------------------------------------------ the same in 64 bits
def _round_e4m3(y):
    """Values (448 at most) to the nearest number of 4 significant bits, steps of 2^-9 at least; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _held(x, rows):
    """(codes' values, the numbers they stand for) of x in 64 bits."""
    r, c = x.shape
    out, val = torch.empty_like(x), torch.empty_like(x)
    for j in range(0, c, 128):
        cols = x[:, j:j + 128]
        top = torch.nn.functional.pad(cols.abs().amax(1), (0, -r % rows)).view(-1, rows).amax(1)
        scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX))), 1.0).repeat_interleave(rows)[:r, None]
        out[:, j:j + 128] = _round_e4m3(cols / scale)
        val[:, j:j + 128] = out[:, j:j + 128] * scale
    return out, val


def _plan64(w):
    q, e = w
    scale = torch.exp2(e.double() - 127).repeat_interleave(128, 0).repeat_interleave(128, 1)
    return q.float().double() * scale[:q.shape[0], :q.shape[1]]


def _by_rows(x, f, step=4096):
    return torch.cat([f(x[i:i + step]) for i in range(0, x.shape[0], step)])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "weights":
        return _by_rows(s["w"], lambda w: _held(w.double(), 128)[0]), None
    if kind == "emb":
        scale, ids, vocab = case["scale"], s["ids"].long(), s["table"].shape[0]
        x = torch.zeros(s["dx"].shape, dtype=F64, device=DEV)
        grad = torch.zeros(s["table"].shape, dtype=F64, device=DEV)
        keep = torch.nonzero((ids >= 0) & (ids < vocab)).view(-1)
        x[keep] = scale * s["table"][ids[keep]].double()
        grad.index_add_(0, ids[keep], scale * s["dx"][keep].double())
        return dict(x=x, d_table=grad)
    if kind == "linear":
        w = _plan64(s["w"])
        y = _by_rows(s["x"], lambda x: _held(x.double(), 1)[1] @ w.T)
        return y if s["residual"] is None else y + s["residual"].double()
    if kind == "ffn":
        up, down, g = _plan64(s["up"]), _plan64(s["down"]), s["g"].double()

        def block(x):
            x = x.double()
            x = x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS) * g
            gu = _held(x, 1)[1] @ up.T
            f = gu.shape[1] // 2
            return _held(gu[:, :f] / (1 + torch.exp(-gu[:, :f])) * gu[:, f:], 1)[1] @ down.T
        return _by_rows(s["x"], block)
    nq, nkv, hd = s["heads"]
    x = s["x"].double()
    n, half = x.shape[0], hd // 2
    c, si = (s["table"][s["pos"].long(), :, i].double() for i in (0, 1))
    y, dgs = x.clone(), {"q": torch.zeros(hd, dtype=F64, device=DEV), "k": torch.zeros(hd, dtype=F64, device=DEV)}
    dx = s["dy"].double().clone() if case["train"] else None
    for h in range(nq + nkv):
        at, name = slice(h * hd, (h + 1) * hd), "q" if h < nq else "k"
        g, xh = s["g_" + name].double(), x[:, at]
        inv = 1 / torch.sqrt((xh * xh).sum(1, keepdim=True) / hd + EPS)
        v = xh * inv * g
        y[:, at] = torch.cat((v[:, :half] * c - v[:, half:] * si, v[:, :half] * si + v[:, half:] * c), 1)
        if case["train"]:
            d = s["dy"][:, at].double()
            d = torch.cat((d[:, :half] * c + d[:, half:] * si, d[:, half:] * c - d[:, :half] * si), 1)
            dgs[name] += (d * xh * inv).sum(0)
            dx[:, at] = inv * (d * g) - xh * inv ** 3 * (d * g * xh).sum(1, keepdim=True) / hd
    return dict(y=y, dx=dx, dg_q=dgs["q"], dg_k=dgs["k"]) if case["train"] else dict(y=y)
