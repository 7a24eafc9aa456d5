"""Decoder sections with options (scaled embeddings, query / key norms, 8-bit matrices) against a plain decoder in 64 bits with autograd."""
import ctypes as C

import pytest
import torch

from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import workloads as wl
from test_gpu_fp8 import quantized, values

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def config(dtype, **over):
    base = dict(arch="decoder", dtype=dtype, n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=500)
    return wl.SectionConfig(**{**base, **over})


def gains(cfg, seed, device="cuda"):
    return [{k: wl.normal(seed, f"{k}{i}", (cfg.head_dim,), 0.2, 1.0, cfg.torch_dtype, device) for k in ("q_norm_g", "k_norm_g")} for i in range(cfg.n_layers)]


def rms(x, g, eps):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * g


def rows_in_8_bits(x):
    """x as rows quantised in blocks of 128 hold it."""
    codes, b = quantized(x, 1)
    return codes * torch.exp2(b.double() - 127).repeat_interleave(128, 1)[:, :x.shape[1]]


def decoder(cfg, w, ids, cu, scale=1.0, norms=None, held=lambda x: x):
    """h_out of the decoder in 64 bits; held: what an input of a matrix becomes."""
    n, hd, nq, nkv = len(ids), cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads
    x = w["embedding"][ids] * scale
    pos = torch.cat([torch.arange(b - a) for a, b in zip(cu[:-1], cu[1:])])
    ang = pos[:, None].double() * cfg.rope_base ** (-2.0 * torch.arange(hd // 2, dtype=F64) / hd)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    seq = torch.repeat_interleave(torch.arange(len(cu) - 1), torch.tensor([b - a for a, b in zip(cu[:-1], cu[1:])]))
    mask = (seq[:, None] == seq[None]) & (pos[:, None] >= pos[None])

    def rot(t):
        lo, hi = t.chunk(2, -1)
        return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)
    for li, l in enumerate(w["layers"]):
        qkv = (held(rms(x, l["norm1_g"], cfg.norm_eps)) @ l["w_qkv"].T).view(n, -1, hd)
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
        if norms:
            q, k = rms(q, norms[li]["q_norm_g"], cfg.norm_eps), rms(k, norms[li]["k_norm_g"], cfg.norm_eps)
        q, k = rot(q), rot(k).repeat_interleave(nq // nkv, 1)
        p = torch.einsum("qhd,khd->hqk", q, k) / hd ** 0.5
        p = torch.softmax(p.masked_fill(~mask, -torch.inf), -1)
        o = torch.einsum("hqk,khd->qhd", p, v.repeat_interleave(nq // nkv, 1)).reshape(n, -1)
        x = x + held(o) @ l["w_o"].T
        g, u = (held(rms(x, l["norm2_g"], cfg.norm_eps)) @ l["w_up"].T).chunk(2, -1)
        x = x + held(g / (1 + torch.exp(-g)) * u) @ l["w_down"].T
    return rms(x, w["final_norm_g"], cfg.norm_eps)


def as64(obj, grad=False):
    if isinstance(obj, dict):
        return {k: as64(v, grad) for k, v in obj.items() if v is not None}
    if isinstance(obj, list):
        return [as64(v, grad) for v in obj]
    return obj.detach().cpu().to(F64).requires_grad_(grad)


def off(got, ref):
    return float((got.cpu().double() - ref).norm() / ref.norm())


LENGTHS = [37, 1, 64, 21]


def data(cfg, seed=4):
    batch = B.Batch(wl.cu_seqlens_of(LENGTHS))
    w = wl.section_weights(cfg, seed, "so", "cuda")
    w["layers"] = [{k: (v * 3 if k.startswith("w_") else v) for k, v in lw.items()} for lw in w["layers"]]
    ids = wl.randint(seed, "ids", batch.n_tokens, 0, cfg.vocab, "cuda")
    ids[5:9] = 7
    return batch, w, ids, wl.normal(seed, "dh", (batch.n_tokens, cfg.d_model), 1.0, 0.0, cfg.torch_dtype, "cuda")


# fp32: products of 688 terms and four layers' worth of them; 64 bits are off by nothing.  bf16: about a dozen roundings of 2^-9 (rms 2^-9 / sqrt 3 each) in
# a row, that is 4e-3; the gradients twice as many
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol,tol_grad", [("fp32", 2e-6, 5e-6), ("bf16", 1e-2, 2e-2)])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_training_with_norms_and_scale(dtype, tol, tol_grad, head_dim):
    cfg = config(dtype, head_dim=head_dim)
    batch, w, ids, dh = data(cfg)
    norms, scale = gains(cfg, 4), 6.5
    opt = B.SectionOptions(embed_scale=scale, qk_norm=True, layers=norms)
    grads = B.zero_grads(w)
    ngrads = [{k: torch.zeros(cfg.head_dim, device="cuda") for k in l} for l in norms]
    out = B.section_forward_backward(cfg, w, grads, batch, ids, d_h_out=dh, options=opt, option_grads=ngrads)
    w64, n64 = as64(w, True), as64(norms, True)
    h = decoder(cfg, w64, ids.cpu().long(), batch.cu, scale, n64)
    (h * dh.cpu().double()).sum().backward()
    assert off(out["h_out"], h.detach()) < tol
    assert torch.equal(B.section_forward(cfg, w, batch, ids, options=opt), out["h_out"])
    for k in ("embedding", "final_norm_g"):
        assert off(grads[k], w64[k].grad) < tol_grad, k
    for i in range(cfg.n_layers):
        for k in ("norm1_g", "w_qkv", "w_o", "norm2_g", "w_up", "w_down"):
            assert off(grads["layers"][i][k], w64["layers"][i][k].grad) < tol_grad, (i, k)
        for k in ("q_norm_g", "k_norm_g"):
            assert off(ngrads[i][k], n64[i][k].grad) < tol_grad, (i, k)


@pytest.mark.gpu
def test_embedding_gradient_repeats_bit_for_bit():
    cfg = config("bf16", n_layers=1)
    batch, w, ids, dh = data(cfg)
    ids[:] = 3                                                    # all tokens add to one row
    runs = []
    for _ in range(2):
        grads = B.zero_grads(w)
        B.section_forward_backward(cfg, w, grads, batch, ids, d_h_out=dh, options=B.SectionOptions(embed_scale=2.0))
        runs.append(grads["embedding"])
    assert torch.equal(runs[0], runs[1]) and bool(runs[0][3].any()) and not bool(runs[0][4:].any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_options_that_change_nothing(dtype):
    cfg = config(dtype)
    batch, w, ids, dh = data(cfg)
    plain, with_ = B.zero_grads(w), B.zero_grads(w)
    a = B.section_forward_backward(cfg, w, plain, batch, ids, d_h_out=dh)
    b = B.section_forward_backward(cfg, w, with_, batch, ids, d_h_out=dh, options=B.SectionOptions())
    assert torch.equal(a["h_out"], b["h_out"]) and torch.equal(B.section_forward(cfg, w, batch, ids, options=B.SectionOptions()), a["h_out"])
    assert torch.equal(plain["layers"][0]["norm1_g"], with_["layers"][0]["norm1_g"])
    # 64 equal signs at most in a row's sum: a few half steps of fp32
    assert torch.allclose(plain["embedding"], with_["embedding"], rtol=1e-5, atol=1e-5 * float(plain["embedding"].abs().max()))


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [LENGTHS, [1], [40, 9], [150, 63]])
@pytest.mark.parametrize("d_ffn", [688, 640])
def test_teacher_in_8_bits(lengths, d_ffn):
    cfg = config("bf16", d_ffn=d_ffn, n_layers=2)
    batch = B.Batch(wl.cu_seqlens_of(lengths))
    _, w, _, _ = data(cfg)
    ids = wl.randint(4, "ids8", batch.n_tokens, 0, cfg.vocab, "cuda")
    w8, layers = B.quantize_section(w)
    norms = gains(cfg, 5)
    opt = B.SectionOptions(embed_scale=3.0, qk_norm=True, fp8=True, layers=[{**a, **b} for a, b in zip(layers, norms)])
    h = B.section_forward(cfg, w8, batch, ids, options=opt)
    w64 = as64(w)
    for l, lw, lo in zip(w64["layers"], w8["layers"], layers):
        for k in ("qkv", "o", "up", "down"):
            l["w_" + k] = values(lw["w_" + k], lo["s_" + k], 128)
    ref = decoder(cfg, w64, ids.cpu().long(), batch.cu, 3.0, as64(norms), rows_in_8_bits)
    # Two pipelines that round differently in front of a quantisation (bf16: up to 2^-9 of a value; a step of e4m3 is 2^-3.5 of it in the mean) have
    # different codes where a tie lies between, and what that changes moves more codes behind it: in the end their quantisation errors, 2^-3 /
    # sqrt 12 / 1.44 = 2.5e-2 of an operand each, are independent, 3.5e-2 between the two, eight operands in two layers: up to 0.1.  The
    # measure is therefore the same definition with its operands moved by a bf16 rounding's worth before they are quantised.
    shift = torch.Generator().manual_seed(1)
    moved = decoder(cfg, w64, ids.cpu().long(), batch.cu, 3.0, as64(norms),
                    lambda x: rows_in_8_bits(x * (1 + 2.0 ** -9 * (2 * torch.rand(x.shape, generator=shift, dtype=F64) - 1))))
    floor = off(moved, ref)
    assert floor < 0.15 and off(h, ref) < 1.5 * floor
    assert torch.equal(h, by_kernels(cfg, w8, layers, norms, batch, ids, 3.0))


def by_kernels(cfg, w, scales, norms, batch, ids, embed_scale):
    """The 8-bit section from the kernel-level entry points: the same bits."""
    nq, nkv, hd, eps = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.norm_eps
    pos, table = B.k_positions(batch), B.k_rope_table(batch.max_seqlen, hd, cfg.rope_base)
    x = B.k_embedding_scaled_forward(ids, w["embedding"], embed_scale)
    for lw, ls, ln in zip(w["layers"], scales, norms):
        qkv = B.k_gemm_fp8(*B.k_norm_fp8(x, lw["norm1_g"], eps), lw["w_qkv"], ls["s_qkv"])
        qkv = B.k_qk_norm_rope_forward(qkv, nq, nkv, hd, ln["q_norm_g"], ln["k_norm_g"], eps, pos, table)
        o, _ = B.k_attention_forward(qkv, batch, nq, nkv, hd, True)
        x = B.k_gemm_fp8(*B.k_fp8_quantize(o), lw["w_o"], ls["s_o"], residual=x, c_fp32=True, fast_sums=True)
        act = B.k_gemm_fp8_swiglu(*B.k_norm_fp8(x, lw["norm2_g"], eps), lw["w_up"], ls["s_up"])
        x = B.k_gemm_fp8(*act, lw["w_down"], ls["s_down"], residual=x, c_fp32=True, fast_sums=True)
    return B.k_norm_forward(0, x, w["final_norm_g"], None, eps)[0]


@pytest.mark.gpu
def test_teacher_and_student_with_distillation_loss():
    """A step as it would be run: teacher in 8 bits, student with norms and scale trained on its states, optimizer step, all in one graph."""
    t, s = config("bf16", d_model=512, d_ffn=1408, n_layers=2), config("bf16", n_layers=1)
    kd = wl.KDConfig(s.vocab - 500 % 8, t.d_model, s.d_model, 1.0, 128)
    batch, tw, ids, _ = data(t)
    _, sw, _, _ = data(s, 6)
    tw8, layers = B.quantize_section(tw)
    topt = B.SectionOptions(embed_scale=t.d_model ** 0.5, fp8=True, layers=layers)
    norms = gains(s, 6)
    sopt = B.SectionOptions(embed_scale=s.d_model ** 0.5, qk_norm=True, layers=norms)
    wt, wst = (wl.normal(8, k, (kd.vocab, d), 0.02, 0.0, BF16, "cuda") for k, d in (("wt", t.d_model), ("ws", s.d_model)))
    grads, dws = B.zero_grads(sw), torch.zeros((kd.vocab, s.d_model), device="cuda")
    ngrads = [{k: torch.zeros(s.head_dim, device="cuda") for k in l} for l in norms]
    wsb = torch.empty(B.section_workspace_bytes(t, batch.n_tokens, batch.max_seqlen, False, topt), dtype=torch.uint8, device="cuda")
    wss = torch.empty(B.section_workspace_bytes(s, batch.n_tokens, batch.max_seqlen, True, sopt) + B.kd_workspace_bytes(kd, batch.n_tokens),
                      dtype=torch.uint8, device="cuda")

    def step():
        grads["embedding"].zero_()
        h_t = B.section_forward(t, tw8, batch, ids, ws=wsb, options=topt)
        out = B.section_forward_backward(s, sw, grads, batch, ids, kd=kd, w_teacher=wt, w_student=wst, h_teacher=h_t, d_w_student=dws, ws=wss,
                                         options=sopt, option_grads=ngrads)
        return out["loss"], out["h_out"], h_t
    want = [v.clone() for v in step()]
    emb = grads["embedding"].clone()
    assert bool(torch.isfinite(want[0])) and bool(emb.isfinite().all()) and bool(emb.any())
    assert all(bool(g.isfinite().all()) and bool(g.any()) for l in ngrads for g in l.values())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for _ in range(3):
        wsb.fill_(255), wss.fill_(255)                            # nothing is expected of the workspaces
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[1], got[1]) and torch.equal(want[2], got[2]) and torch.equal(want[0], got[0])
        assert torch.allclose(grads["embedding"], emb, rtol=2e-2, atol=2e-2 * float(emb.abs().max()))
        step()


def test_workspaces_do_not_shrink_with_more_tokens():
    cfg = config("bf16", d_model=128, d_ffn=2048, n_layers=1, vocab=50000)
    fake = [{"q_norm_g": None}]
    for o, bwd in ((B.SectionOptions(fp8=True, layers=fake), False), (B.SectionOptions(qk_norm=True, layers=fake), True)):
        last = 0
        for n in [*range(1, 140), 4096, 4097, 131071, 131072, 131073, 131200, 140000, 524288, 524289, 530000]:
            b = B.section_workspace_bytes(cfg, n, 1, bwd, o)
            assert b >= last > -1, n
            last = b
    f = B._fn("ms_k_embedding_sorted_backward_scratch_bytes")
    sizes = [f(n, d, 50000) for d in (8,) for n in range(130000, 132000)]
    assert sizes == sorted(sizes)


def test_refusals_before_anything_is_launched():
    lib = B.lib()
    p256 = lambda t: C.cast(C.c_void_p(256), t)

    def call(dtype="bf16", backward=False, layers=True, option_grads=True, scale=1.0, qk=0, fp8=0, field=None, **over):
        cfg = config(dtype, n_layers=1, **over)
        c = B._cfg_c(cfg)
        host = (C.c_int32 * 2)(0, 4)
        b = B.BatchC(4, 1, C.c_void_p(256), host)
        lp, lo = (B.LayerPtrs * 1)(), (B.LayerOptions * 1)()
        for f in B._LAYER_FIELDS:
            setattr(lp[0], f, 256)
        for f in B._OPTION_FIELDS:
            setattr(lo[0], f, None if f == field else 256)
        w = B.SectionPtrs(256, lp, 256, 256)
        o = B.SectionOptionsC(scale, qk, fp8, lo if layers else None)
        v = C.c_void_p(256)
        if backward:
            return lib.ms_section_forward_backward_with(C.byref(c), C.byref(o), lo if option_grads else None, C.byref(w), C.byref(w), C.byref(b), v, v, v,
                                                        None, None, None, None, None, None, v, C.c_size_t(16), None)
        return lib.ms_section_forward_with(C.byref(c), C.byref(o), C.byref(w), C.byref(b), v, v, v, C.c_size_t(16), None)
    assert call() == -3 and call(backward=True) == -3                        # everything but the workspace is right
    assert call(qk=1) == -3 and call(fp8=1) == -3 and call(qk=1, backward=True) == -3
    assert call(scale=float("nan")) == -1 and call(scale=float("inf")) == -1
    assert call(qk=1, layers=False) == -1 and call(fp8=1, layers=False) == -1
    for f in ("q_norm_g", "k_norm_g"):
        assert call(qk=1, field=f) == -1
    for f in ("s_qkv", "s_o", "s_up", "s_down"):
        assert call(fp8=1, field=f) == -1
    assert call(qk=1, backward=True, option_grads=False) == -1
    assert call(fp8=1, backward=True) == -4 and call(fp8=1, dtype="fp32") == -4 and call(fp8=1, d_ffn=344) == -4 and call(arch="encoder", vocab=0) == -4
    with pytest.raises(ValueError, match="each of 2 layers"):
        B.SectionOptions(qk_norm=True, layers=[{}]).check(config("bf16"))
    with pytest.raises(ValueError, match="q_norm_g"):
        B.SectionOptions(qk_norm=True, layers=[{}, {}]).check(config("bf16"))


def test_codes_go_with_their_option():
    cfg = config("bf16", n_layers=1)
    d, a, f = cfg.d_model, cfg.n_q_heads * cfg.head_dim, cfg.d_ffn
    sizes = {"w_qkv": (cfg.d_qkv, d), "w_o": (d, a), "w_up": (2 * f, d), "w_down": (d, f)}
    plain = {k: torch.empty(s, dtype=torch.bfloat16) for k, s in sizes.items()}
    codes = {k: torch.empty(s, dtype=torch.float8_e4m3fn) for k, s in sizes.items()}
    ids = torch.zeros(4, dtype=torch.int32)
    for k in sizes:                                                          # read as bf16, codes would end too early
        with pytest.raises(ValueError, match=k + ".*fp8=True"):
            B.section_forward(cfg, {"layers": [dict(plain, **{k: codes[k]})]}, None, ids)
        with pytest.raises(ValueError, match=k + ".*fp8=True"):
            B.section_forward_backward(cfg, {"layers": [dict(plain, **{k: codes[k]})]}, None, type("Batch", (), {"n_tokens": 4}), ids)
    with pytest.raises(ValueError, match="w_qkv"):
        B._check_matrices(cfg, {"layers": [plain]}, B.SectionOptions(fp8=True), None)
    with pytest.raises(ValueError, match="w_qkv"):
        B._check_matrices(cfg, {"layers": [dict(codes, w_qkv=codes["w_qkv"][1:])]}, B.SectionOptions(fp8=True), None)


def test_sizes_and_alignment_are_refused_before_anything_is_launched():
    """What the kernels behind the options would turn down in the middle of a section."""
    lib = B.lib()

    def call(qk=0, fp8=0, weights={}, options={}, backward=False, **over):
        cfg = config("bf16", n_layers=1, **over)
        c, host = B._cfg_c(cfg), (C.c_int32 * 2)(0, 4)
        b = B.BatchC(4, 1, C.c_void_p(256), host)
        lp, lo = (B.LayerPtrs * 1)(), (B.LayerOptions * 1)()
        for f in B._LAYER_FIELDS:
            setattr(lp[0], f, weights.get(f, 256))
        for f in B._OPTION_FIELDS:
            setattr(lo[0], f, options.get(f, 256))
        w, v = B.SectionPtrs(256, lp, 256, 256), C.c_void_p(256)
        o = B.SectionOptionsC(1.0, qk, fp8, lo)
        if backward:
            return lib.ms_section_forward_backward_with(C.byref(c), C.byref(o), lo, C.byref(w), C.byref(w), C.byref(b), v, v, v,
                                                        None, None, None, None, None, None, v, C.c_size_t(16), None)
        return lib.ms_section_forward_with(C.byref(c), C.byref(o), C.byref(w), C.byref(b), v, v, v, C.c_size_t(16), None)
    assert call(qk=1) == -3 and call(fp8=1) == -3                            # all is right but the workspace
    for f in ("q_norm_g", "k_norm_g"):
        assert call(qk=1, options={f: 264}) == -4 and call(qk=1, options={f: 264}, backward=True) == -4 and call(fp8=1, options={f: 264}) == -3
    for f in ("w_qkv", "w_o", "w_up", "w_down"):
        assert call(fp8=1, weights={f: 264}) == -4 and call(qk=1, weights={f: 264}) == -3
    for f in ("s_qkv", "s_o", "s_up", "s_down"):
        assert call(fp8=1, options={f: 258}) == -4 and call(fp8=1, options={f: 260}) == -3
    assert call(qk=1, head_dim=24) == -4 and call(qk=1, head_dim=520) == -4
    assert call(fp8=1, n_q_heads=1, n_kv_heads=1, head_dim=24) == -4


def test_pointers_of_embedding_and_norms_are_refused_before_anything_is_launched():
    """The sorted gradient is a backward call's last kernel, so that its refusal would leave all other gradients added up."""
    lib = B.lib()

    def call(qk=0, fp8=0, scale=1.0, weights={}, embedding=256, grad=256, final=256, backward=False, vocab=500):
        cfg = config("bf16", n_layers=1, vocab=vocab)
        c, host = B._cfg_c(cfg), (C.c_int32 * 2)(0, 4)
        b = B.BatchC(4, 1, C.c_void_p(256), host)
        lp, lo = (B.LayerPtrs * 1)(), (B.LayerOptions * 1)()
        for f in B._LAYER_FIELDS:
            setattr(lp[0], f, weights.get(f, 256))
        for f in B._OPTION_FIELDS:
            setattr(lo[0], f, 256)
        w, g, v = B.SectionPtrs(embedding, lp, final, 256), B.SectionPtrs(grad, lp, 256, 256), C.c_void_p(256)
        o = B.SectionOptionsC(scale, qk, fp8, lo)
        if backward:
            return lib.ms_section_forward_backward_with(C.byref(c), C.byref(o), lo, C.byref(w), C.byref(g), C.byref(b), v, v, v,
                                                        None, None, None, None, None, None, v, C.c_size_t(16), None)
        return lib.ms_section_forward_with(C.byref(c), C.byref(o), C.byref(w), C.byref(b), v, v, v, C.c_size_t(16), None)
    assert call() == -3 and call(backward=True) == -3 and call(fp8=1) == -3              # all is right but the workspace
    assert call(backward=True, grad=260) == -4 and b"embedding" in lib.ms_last_error()
    assert call(scale=2.0, embedding=264) == -4 and call(scale=2.0, embedding=264, backward=True) == -4
    assert call(embedding=264) == -3 and call(embedding=264, backward=True) == -3        # rows as they are may begin anywhere
    assert call(vocab=0, grad=260, backward=True) == -3                                  # not an embedding's
    assert call(final=264) == -4 and call(final=264, backward=True) == -4
    for f in ("norm1_g", "norm2_g"):
        assert call(fp8=1, weights={f: 264}) == -4 and f"layer 0".encode() in lib.ms_last_error()


def test_a_scale_without_an_embedding_is_refused():
    cfg, o = B._cfg_c(config("bf16", vocab=0)), B.SectionOptionsC(2.0, 0, 0, None)
    assert B.lib().ms_section_workspace_bytes_with(C.byref(cfg), C.byref(o), 4, 4, 0) == 0 and b"embeds nothing" in B.lib().ms_last_error()
    o.embed_scale = 1.0
    assert B.lib().ms_section_workspace_bytes_with(C.byref(cfg), C.byref(o), 4, 4, 0) > 0
    host, v = (C.c_int32 * 2)(0, 4), C.c_void_p(256)
    b, o.embed_scale = B.BatchC(4, 1, C.c_void_p(256), host), 2.0
    assert B.lib().ms_section_forward_with(C.byref(cfg), C.byref(o), None, C.byref(b), v, v, v, C.c_size_t(16), None) == -1
    assert b"embeds nothing" in B.lib().ms_last_error()


def test_refusals_name_their_reason():
    """The same code has several causes: each refusal comes from its own check."""
    lib, host = B.lib(), (C.c_int32 * 2)(0, 4)

    def why(qk=0, fp8=0, scale=1.0, dtype="bf16", backward=False, n_tokens=4, **over):
        c, lo = B._cfg_c(config(dtype, n_layers=1, **over)), (B.LayerOptions * 1)()
        o = B.SectionOptionsC(scale, qk, fp8, lo)
        cu = (C.c_int32 * 2)(0, n_tokens)
        b, v = B.BatchC(n_tokens, 1, C.c_void_p(256), cu), C.c_void_p(256)
        if backward:
            status = lib.ms_section_forward_backward_with(C.byref(c), C.byref(o), lo, None, None, C.byref(b), v, v, v, None, None, None, None, None, None, v,
                                                          C.c_size_t(16), None)
        else:
            status = lib.ms_section_forward_with(C.byref(c), C.byref(o), None, C.byref(b), v, v, v, C.c_size_t(16), None)
        return status, lib.ms_last_error().decode()
    for hd in (24, 96, 520):                                                  # whatever the options
        for qk, fp8 in ((0, 0), (1, 0), (0, 1), (1, 1)):
            status, text = why(qk, fp8, head_dim=hd)
            assert status == -4 and f"head_dim={hd}" in text
    for hd in (64, 80, 128):                                                  # the head sizes that there are suit every option: next come the weights
        for n_q in (1, 3):
            status, text = why(1, 1, head_dim=hd, n_q_heads=n_q, n_kv_heads=1)
            assert status == -1 and "null weights" in text
    assert why(fp8=1, d_ffn=344)[1].startswith("section: d_model=256 and d_ffn=344") and "forward-only" in why(fp8=1, backward=True)[1]
    assert "bf16" in why(fp8=1, dtype="fp32")[1] and "for decoders" in why(arch="encoder", vocab=0)[1] and "not finite" in why(scale=float("nan"))[1]
    assert "sorts" in why(backward=True, n_tokens=(1 << 24) + 8, n_q_heads=1, n_kv_heads=1, head_dim=64, dtype="fp32")[1]


@pytest.mark.gpu
def test_training_steps_with_the_optimizer_in_one_graph():
    """Teacher in 8 bits, student with norms and scale, distillation loss, AdamW: three replays are three eager steps.  Trained are the final gains, whose
    gradient has one order of sums, so that states and gains have to be equal; the table's update, behind attention's atomics, goes to a copy."""
    t, s = config("bf16", d_model=512, d_ffn=1408, n_layers=1), config("bf16", n_layers=1)
    kd = wl.KDConfig(s.vocab - 500 % 8, t.d_model, s.d_model, 1.0, 128)
    batch, tw, ids, _ = data(t)
    _, sw, _, _ = data(s, 6)
    tw8, layers = B.quantize_section(tw)
    topt, norms = B.SectionOptions(embed_scale=t.d_model ** 0.5, fp8=True, layers=layers), gains(s, 6)
    sopt = B.SectionOptions(embed_scale=s.d_model ** 0.5, qk_norm=True, layers=norms)
    wt, wst = (wl.normal(8, k, (kd.vocab, d), 0.02, 0.0, BF16, "cuda") for k, d in (("wt", t.d_model), ("ws", s.d_model)))
    grads, lr = B.zero_grads(sw), 0.05
    ngrads = [{k: torch.zeros(s.head_dim, device="cuda") for k in l} for l in norms]

    def fresh():
        sw["final_norm_g"].copy_(first)
        grads["final_norm_g"].zero_(), grads["embedding"].zero_()
        for k, st in state.items():
            st[0].copy_(start[k]), st[1].zero_(), st[2].zero_()
    first = sw["final_norm_g"].clone()
    start = {"final_norm_g": first.float(), "embedding": sw["embedding"].float()}
    state = {k: [v.clone(), torch.zeros_like(v), torch.zeros_like(v)] for k, v in start.items()}

    def step():
        h_t = B.section_forward(t, tw8, batch, ids, options=topt)
        out = B.section_forward_backward(s, sw, grads, batch, ids, kd=kd, w_teacher=wt, w_student=wst, h_teacher=h_t,
                                         d_w_student=torch.zeros((kd.vocab, s.d_model), device="cuda"), options=sopt, option_grads=ngrads)
        B.adamw_step(grads["final_norm_g"], *state["final_norm_g"], sw["final_norm_g"], 1, lr=lr, zero_grad=True)
        B.adamw_step(grads["embedding"], *state["embedding"], None, 1, lr=lr, zero_grad=True)
        return out["h_out"]
    want = []
    for _ in range(3):
        want.append((step().clone(), sw["final_norm_g"].clone(), state["final_norm_g"][0].clone()))
    assert not torch.equal(want[0][1], first) and not torch.equal(want[1][0], want[0][0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h = step()
    fresh()
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want[k][0]) and torch.equal(sw["final_norm_g"], want[k][1]) and torch.equal(state["final_norm_g"][0], want[k][2]), k
        B.section_forward(t, tw8, batch, ids, options=topt)               # the program's own work between the replays
    # three steps of moments with the first one's bias correction move a number by at most 1 + sqrt(1 + 0.81 / 0.95) + sqrt(1 + 0.81 / 0.95 + (0.81 / 0.95)^2)
    # = 3.97 lr (Cauchy's inequality), whatever its gradients; rows of ids that are not there stay
    moved = (state["embedding"][0] - start["embedding"]).abs()
    there = torch.zeros(s.vocab, dtype=torch.bool, device="cuda")
    there[ids.long()] = True
    assert bool(moved[there].any(1).all()) and not bool(moved[~there].any())
    assert float(moved.max()) < 4 * lr and not bool(grads["embedding"].any())


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [[1], [40, 9], [150, 63]])
@pytest.mark.parametrize("d_ffn", [688, 640])
def test_teacher_in_8_bits_with_fp32_sums(lengths, d_ffn):
    cfg = config("bf16", d_ffn=d_ffn, n_layers=2)
    batch = B.Batch(wl.cu_seqlens_of(lengths))
    _, w, _, _ = data(cfg)
    ids = wl.randint(4, "ids8", batch.n_tokens, 0, cfg.vocab, "cuda")
    w8, scales = B.quantize_section(w)
    norms, nq, nkv, hd, eps = gains(cfg, 5), cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.norm_eps
    layers = [{**a, **b} for a, b in zip(scales, norms)]
    h = B.section_forward(cfg, w8, batch, ids, options=B.SectionOptions(embed_scale=3.0, qk_norm=True, fp8=True, layers=layers, fp32_sums=True))
    pos, table = B.k_positions(batch), B.k_rope_table(batch.max_seqlen, hd, cfg.rope_base)
    x = B.k_embedding_scaled_forward(ids, w["embedding"], 3.0)
    for lw, ls in zip(w8["layers"], layers):
        qkv = B.k_gemm_fp8(*B.k_norm_fp8(x, lw["norm1_g"], eps), lw["w_qkv"], ls["s_qkv"], fp32_sums=True)
        qkv = B.k_qk_norm_rope_forward(qkv, nq, nkv, hd, ls["q_norm_g"], ls["k_norm_g"], eps, pos, table)
        x = B.k_gemm_fp8(*B.k_fp8_quantize(B.k_attention_forward(qkv, batch, nq, nkv, hd, True)[0]), lw["w_o"], ls["s_o"], residual=x, c_fp32=True)
        act = B.k_swiglu_fp8(B.k_gemm_fp8(*B.k_norm_fp8(x, lw["norm2_g"], eps), lw["w_up"], ls["s_up"], c_fp32=True))
        x = B.k_gemm_fp8(*act, lw["w_down"], ls["s_down"], residual=x, c_fp32=True)
    assert torch.equal(h, B.k_norm_forward(0, x, w["final_norm_g"], None, eps)[0])
    fast = B.section_forward(cfg, w8, batch, ids, options=B.SectionOptions(embed_scale=3.0, qk_norm=True, fp8=True, layers=layers))
    assert torch.equal(fast, by_kernels(cfg, w8, scales, norms, batch, ids, 3.0)) and not torch.equal(h, fast)


def test_workspace_of_fp32_sums():
    cfg, fake = config("bf16", n_layers=1), [{"q_norm_g": None}]
    size = lambda n, **o: B.section_workspace_bytes(cfg, n, n, False, B.SectionOptions(fp8=True, layers=fake, **o))
    sizes = [size(n, fp32_sums=True) for n in (1, 2, 63, 64, 65, 130, 4096)]
    assert sizes == sorted(sizes) and sizes[-1] >= 4096 * 2 * cfg.d_ffn * 4


def test_options_for_more_layers_than_there_are_are_refused():
    """Also where the section reads none of them."""
    cfg = config("bf16", n_layers=2)
    for o in (B.SectionOptions(embed_scale=2.0, layers=[{}] * 3), B.SectionOptions(qk_norm=True, layers=[{}] * 3)):
        with pytest.raises(ValueError, match="section of 2"):
            B.section_workspace_bytes(cfg, 8, 8, False, o)
    assert B.section_workspace_bytes(cfg, 8, 8, False, B.SectionOptions(embed_scale=2.0, layers=[{}])) > 0
