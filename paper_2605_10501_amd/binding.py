"""Thin ctypes binding of libmaestro_section.so (same names as the C ABI, minus the ms_ prefix).

Argument marshalling only: every step of the path runs inside the HIP library.  PyTorch
provides device memory and the current stream.  There is no CPU fallback: if the library is
missing, loading fails.
"""
import contextlib
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmaestro_section.so")
MS_F32, MS_BF16 = 0, 1
MS_DECODER, MS_ENCODER = 0, 1
_LAYER_FIELDS = ["norm1_g", "norm1_b", "w_qkv", "b_qkv", "w_o", "b_o",
                 "norm2_g", "norm2_b", "w_up", "b_up", "w_down", "b_down"]


class SectionConfigC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ["arch", "dtype", "n_layers", "d_model", "n_q_heads", "n_kv_heads",
                                         "head_dim", "d_ffn", "vocab"]] + [("norm_eps", C.c_float), ("rope_base", C.c_float)]


class LayerPtrs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _LAYER_FIELDS]


class SectionPtrs(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("layers", C.POINTER(LayerPtrs)),
                ("final_norm_g", C.c_void_p), ("final_norm_b", C.c_void_p)]


class BatchC(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("n_seqs", C.c_int32),
                ("cu_seqlens_dev", C.c_void_p), ("cu_seqlens_host", C.POINTER(C.c_int32))]


class KDConfigC(C.Structure):
    _fields_ = [("vocab", C.c_int32), ("h_teacher", C.c_int32), ("h_student", C.c_int32), ("chunk", C.c_int32),
                ("dtype", C.c_int32), ("temperature", C.c_float), ("loss_scale", C.c_float),
                ("w_teacher_dev", C.c_void_p), ("w_student_dev", C.c_void_p), ("token_block", C.c_int32)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built (python -m paper_2605_10501_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_10501_amd.build`")
        _lib = C.CDLL(LIB_PATH)
        _lib.ms_last_error.restype = C.c_char_p
        for name in ["ms_section_workspace_bytes", "ms_kd_workspace_bytes", "ms_k_norm_backward_scratch_bytes",
                     "ms_k_attention_backward_scratch_bytes", "ms_section_workspace_bytes_with"]:
            getattr(_lib, name).restype = C.c_size_t
    return _lib


def _check(status):
    if status != 0:
        raise RuntimeError(f"maestro_section error {status}: {lib().ms_last_error().decode()}")


def _p(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _on(device):
    """`device` as the current one: the library launches there, on its current stream."""
    same = device.type != "cuda" or device.index == torch.cuda.current_device()
    return contextlib.nullcontext() if same else torch.cuda.device(device)


def _dt(dtype):
    if dtype in ("bf16", torch.bfloat16, MS_BF16):
        return MS_BF16
    if dtype in ("fp32", torch.float32, MS_F32) and dtype is not False:
        return MS_F32
    raise ValueError(dtype)


def _tdt(dtype):
    return torch.bfloat16 if _dt(dtype) == MS_BF16 else torch.float32


class Batch:
    """A packed micro-batch: host and device copies of cu_seqlens."""

    def __init__(self, cu_seqlens, device="cuda"):
        self.cu = [int(v) for v in cu_seqlens]
        self.n_seqs = len(self.cu) - 1
        self.n_tokens = self.cu[-1] if self.cu else 0
        self.max_seqlen = max([b - a for a, b in zip(self.cu[:-1], self.cu[1:])], default=0)
        self._host = (C.c_int32 * len(self.cu))(*self.cu)
        self.cu_dev = torch.tensor(self.cu, dtype=torch.int32, device=device)

    def c(self):
        return BatchC(self.n_tokens, self.n_seqs, _p(self.cu_dev), self._host)


def _cfg_c(cfg):
    return SectionConfigC(MS_DECODER if cfg.arch == "decoder" else MS_ENCODER, _dt(cfg.dtype), cfg.n_layers, cfg.d_model,
                          cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.d_ffn, cfg.vocab, cfg.norm_eps, cfg.rope_base)


def _ptrs_c(cfg, w):
    layers = (LayerPtrs * cfg.n_layers)()
    for i, lw in enumerate(w["layers"]):
        for f in _LAYER_FIELDS:
            t = lw.get(f)
            setattr(layers[i], f, t.data_ptr() if t is not None else None)
    emb, fb = w.get("embedding"), w.get("final_norm_b")
    s = SectionPtrs(emb.data_ptr() if emb is not None else None, layers, w["final_norm_g"].data_ptr(),
                    fb.data_ptr() if fb is not None else None)
    s._keep = layers
    return s


def _kd_c(kd, w_teacher, w_student, loss_scale):
    return KDConfigC(kd.vocab, kd.h_teacher, kd.h_student, kd.chunk, _dt(kd.dtype), kd.temperature, loss_scale,
                     w_teacher.data_ptr(), w_student.data_ptr(), getattr(kd, "token_block", 0))


def zero_grads(weights):
    """fp32 zero buffers with the structure of `weights`."""
    def z(t):
        return torch.zeros(t.shape, dtype=torch.float32, device=t.device) if t is not None else None
    g = {k: z(v) for k, v in weights.items() if k != "layers"}
    g["layers"] = [{k: z(v) for k, v in lw.items()} for lw in weights["layers"]]
    return g


def workspace(nbytes, device="cuda", tag=None):
    """A byte buffer of at least nbytes, the caller's own (whatever the tag): PyTorch's allocator gives the memory to nobody else
    before the current stream is done with it, or while a graph that is being captured may be replayed.  One kept here
    would be shared by calls on two streams, a teacher's and a student's for instance."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


_OPTION_FIELDS = ["q_norm_g", "k_norm_g", "s_qkv", "s_o", "s_up", "s_down"]


class LayerOptions(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _OPTION_FIELDS]


class SectionOptionsC(C.Structure):
    _fields_ = [("embed_scale", C.c_float), ("qk_norm", C.c_int32), ("fp8", C.c_int32), ("layers", C.POINTER(LayerOptions))]


class SectionOptions:
    """Options of a decoder section: embed_scale; layers: one dict per layer with q_norm_g and k_norm_g ([head_dim], in the section's dtype) if
    qk_norm, and the scale bytes s_qkv, s_o, s_up, s_down of the matrices' codes if fp8 (see quantize_section).  fp32_sums: the products of
    8-bit matrices sum in fp32 throughout (k_gemm_fp8), at half the rate."""

    def __init__(self, embed_scale=1.0, qk_norm=False, fp8=False, layers=None, fp32_sums=False):
        self.embed_scale, self.qk_norm, self.fp8, self.layers = float(embed_scale), bool(qk_norm), bool(fp8), layers
        self.fp32_sums = bool(fp32_sums)
        if self.fp32_sums and not self.fp8:
            raise ValueError("fp32_sums is a choice for fp8 matrices")

    def check(self, cfg, device=None):
        if (self.qk_norm or self.fp8) and (self.layers is None or len(self.layers) != cfg.n_layers):
            raise ValueError(f"section options: expected a dict for each of {cfg.n_layers} layers")
        words = lambda k: (k + 511) // 512 * 4
        rows = lambda n: (n + 127) // 128
        d, a, f = cfg.d_model, cfg.n_q_heads * cfg.head_dim, cfg.d_ffn
        for lo in self.layers or ():
            for k in ("q_norm_g", "k_norm_g") if self.qk_norm else ():
                _need(k, lo.get(k), (_tdt(cfg.dtype),), (cfg.head_dim,), device)
            if self.fp8:
                for k, n, kin in (("s_qkv", cfg.d_qkv, d), ("s_o", d, a), ("s_up", 2 * f, d), ("s_down", d, f)):
                    _need(k, lo.get(k), (torch.uint8,), (rows(n), words(kin)), device)

    def c(self, cfg):
        o = SectionOptionsC(self.embed_scale, int(self.qk_norm), int(self.fp8) + int(self.fp32_sums), _layer_options(self.layers, cfg.n_layers))
        return o


def _layer_options(layers, n):
    if layers is None:
        return None
    if len(layers) > n:
        raise ValueError(f"section options: {len(layers)} layers' worth for a section of {n}")
    arr = (LayerOptions * n)()
    for i, lo in enumerate(layers):
        for f in _OPTION_FIELDS:
            t = lo.get(f)
            setattr(arr[i], f, t.data_ptr() if t is not None else None)
    return arr


def _check_matrices(cfg, weights, options, device):
    """Codes belong to sections with fp8, and nothing else does: a byte per number read as two would go past the end."""
    d, a, f = cfg.d_model, cfg.n_q_heads * cfg.head_dim, cfg.d_ffn
    for lw in weights["layers"]:
        for k, n, kin in (("w_qkv", cfg.d_qkv, d), ("w_o", d, a), ("w_up", 2 * f, d), ("w_down", d, f)):
            if options is not None and options.fp8:
                _need(k, lw.get(k), (torch.float8_e4m3fn,), (n, kin), device)
            elif lw.get(k) is not None and lw[k].dtype == torch.float8_e4m3fn:
                raise ValueError(f"{k}: 8-bit codes need SectionOptions(fp8=True) with their scales")


def quantize_section(weights):
    """(weights with w_qkv, w_o, w_up and w_down as e4m3 codes, their scale bytes as the layers of SectionOptions(fp8=True))."""
    out, layers = dict(weights, layers=[]), []
    for lw in weights["layers"]:
        lw, lo = dict(lw), {}
        for k in ("qkv", "o", "up", "down"):
            lw["w_" + k], lo["s_" + k] = k_fp8_quantize(lw["w_" + k], 128)
        out["layers"].append(lw)
        layers.append(lo)
    return out, layers


def section_workspace_bytes(cfg, max_tokens, max_seqlen, need_backward, options=None):
    c = _cfg_c(cfg)
    if options is not None:
        o = options.c(cfg)
        return lib().ms_section_workspace_bytes_with(C.byref(c), C.byref(o), max_tokens, max_seqlen, int(need_backward))
    return lib().ms_section_workspace_bytes(C.byref(c), max_tokens, max_seqlen, int(need_backward))


def kd_workspace_bytes(kd, max_tokens):
    c = KDConfigC(kd.vocab, kd.h_teacher, kd.h_student, kd.chunk, _dt(kd.dtype), kd.temperature, 1.0, None, None,
                  getattr(kd, "token_block", 0))
    return lib().ms_kd_workspace_bytes(C.byref(c), max_tokens)


def section_forward(cfg, weights, batch, x_in, h_out=None, ws=None, options=None):
    if options is not None:
        options.check(cfg, x_in.device)
    _check_matrices(cfg, weights, options, x_in.device)
    c, w, b = _cfg_c(cfg), _ptrs_c(cfg, weights), batch.c()
    if h_out is None:
        h_out = torch.empty((batch.n_tokens, cfg.d_model), dtype=_tdt(cfg.dtype), device=x_in.device)
    if ws is None:
        ws = workspace(section_workspace_bytes(cfg, batch.n_tokens, batch.max_seqlen, False, options), x_in.device)
    if options is not None:
        o = options.c(cfg)
        with _on(x_in.device):
            _check(lib().ms_section_forward_with(C.byref(c), C.byref(o), C.byref(w), C.byref(b), _p(x_in), _p(h_out), _p(ws),
                                                 C.c_size_t(ws.numel()), _stream()))
        return h_out
    with _on(x_in.device):
        _check(lib().ms_section_forward(C.byref(c), C.byref(w), C.byref(b), _p(x_in), _p(h_out), _p(ws),
                                        C.c_size_t(ws.numel()), _stream()))
    return h_out


def section_forward_backward(cfg, weights, grads, batch, x_in, d_h_out=None, kd=None, w_teacher=None, w_student=None,
                             h_teacher=None, d_w_student=None, loss_scale=None, want_d_x_in=False, ws=None, options=None,
                             option_grads=None):
    """Returns dict(h_out, loss, kl_tok, d_x_in); `grads` (and d_w_student) are accumulated in place.  option_grads: with
    SectionOptions(qk_norm=True), fp32 q_norm_g and k_norm_g of each layer, accumulated too."""
    if options is not None:
        options.check(cfg, x_in.device)
        if options.qk_norm:
            if option_grads is None or len(option_grads) != cfg.n_layers:
                raise ValueError(f"option_grads: expected a dict for each of {cfg.n_layers} layers")
            for lg in option_grads:
                for k in ("q_norm_g", "k_norm_g"):
                    _need("gradient of " + k, lg.get(k), (torch.float32,), (cfg.head_dim,), x_in.device)
    _check_matrices(cfg, weights, options, x_in.device)
    c, w, g, b = _cfg_c(cfg), _ptrs_c(cfg, weights), _ptrs_c(cfg, grads), batch.c()
    dev, n = x_in.device, batch.n_tokens
    h_out = torch.empty((n, cfg.d_model), dtype=_tdt(cfg.dtype), device=dev)
    need = section_workspace_bytes(cfg, n, batch.max_seqlen, True, options)
    loss = kl = kdc = None
    if kd is not None:
        kdc = _kd_c(kd, w_teacher, w_student, (1.0 / max(n, 1)) if loss_scale is None else loss_scale)
        need += kd_workspace_bytes(kd, n)
        loss = torch.zeros((), dtype=torch.float32, device=dev)
        kl = torch.empty((n,), dtype=torch.float32, device=dev)
    d_x_in = torch.empty_like(h_out) if (want_d_x_in and cfg.vocab == 0) else None
    if ws is None:
        ws = workspace(need, dev)
    if options is not None:
        o = options.c(cfg)
        with _on(dev):
            _check(lib().ms_section_forward_backward_with(
                C.byref(c), C.byref(o), _layer_options(option_grads, cfg.n_layers), C.byref(w), C.byref(g), C.byref(b), _p(x_in), _p(h_out),
                _p(d_h_out), C.byref(kdc) if kdc is not None else None, _p(h_teacher), _p(d_w_student), _p(loss), _p(kl), _p(d_x_in),
                _p(ws), C.c_size_t(ws.numel()), _stream()))
        return dict(h_out=h_out, loss=loss, kl_tok=kl, d_x_in=d_x_in)
    with _on(dev):
        _check(lib().ms_section_forward_backward(
            C.byref(c), C.byref(w), C.byref(g), C.byref(b), _p(x_in), _p(h_out), _p(d_h_out),
            C.byref(kdc) if kdc is not None else None, _p(h_teacher), _p(d_w_student), _p(loss), _p(kl), _p(d_x_in),
            _p(ws), C.c_size_t(ws.numel()), _stream()))
    return dict(h_out=h_out, loss=loss, kl_tok=kl, d_x_in=d_x_in)


def kd_loss_forward_backward(kd, w_teacher, w_student, h_teacher, h_student, loss_scale=None, need_d_h=True,
                             d_w_student=None, ws=None):
    """Returns dict(loss, kl_tok, d_h_s); d_w_student (fp32 [V, Hs]) is accumulated in place if given."""
    n, dev = h_student.shape[0], h_student.device
    kdc = _kd_c(kd, w_teacher, w_student, (1.0 / max(n, 1)) if loss_scale is None else loss_scale)
    loss = torch.zeros((), dtype=torch.float32, device=dev)
    kl = torch.empty((n,), dtype=torch.float32, device=dev)
    d_h = torch.empty_like(h_student) if need_d_h else None
    if ws is None:
        ws = workspace(kd_workspace_bytes(kd, n), dev)
    _check(lib().ms_kd_loss_forward_backward(C.byref(kdc), n, _p(h_teacher), _p(h_student), _p(loss), _p(kl), _p(d_h),
                                             _p(d_w_student), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return dict(loss=loss, kl_tok=kl, d_h_s=d_h)


KD_STATIC_SCRATCH_BYTES = 64 << 20


def kd_loss_forward_backward_static(kd, w_teacher, w_student, h_teacher, h_student, loss, kl_tok, d_h_student,
                                    d_w_student=None, loss_scale=None):
    """The allocation-free variant: every output is the caller's tensor, the scratch is the library's built-in array."""
    n = h_student.shape[0]
    kdc = _kd_c(kd, w_teacher, w_student, (1.0 / max(n, 1)) if loss_scale is None else loss_scale)
    _check(lib().ms_kd_loss_forward_backward_static(C.byref(kdc), n, _p(h_teacher), _p(h_student), _p(loss), _p(kl_tok),
                                                    _p(d_h_student), _p(d_w_student), _stream()))


def pack_microbatches(lengths, token_budget, policy=0):
    """Returns (order, mb_offsets, cu_seqlens_per_mb) as Python lists."""
    n = len(lengths)
    arr = (C.c_int32 * max(n, 1))(*lengths)
    order, offs, cus = (C.c_int32 * max(n, 1))(), (C.c_int32 * (n + 1))(), (C.c_int32 * max(2 * n, 1))()
    n_mb = C.c_int32(0)
    _check(lib().ms_pack_microbatches(arr, n, token_budget, policy, order, offs, C.byref(n_mb), cus))
    offs_l = [offs[i] for i in range(n_mb.value + 1)]
    out, pos = [], 0
    for m in range(n_mb.value):
        k = offs_l[m + 1] - offs_l[m]
        out.append([cus[pos + i] for i in range(k + 1)])
        pos += k + 1
    return [order[i] for i in range(offs_l[-1])], offs_l, out


class _MergerCfg(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("d_vit", C.c_int32), ("merge", C.c_int32), ("d_hidden", C.c_int32), ("d_llm", C.c_int32)]


class _MergerPtrs(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("w1", "b1", "w2", "b2")]


def _merger_c(w, merge):
    dh, din = w["w1"].shape
    return _MergerCfg(_dt(w["w1"].dtype), din // merge, merge, dh, w["w2"].shape[0])


def _merger_ptrs(t):
    return _MergerPtrs(*[_p(t[k]) for k in ("w1", "b1", "w2", "b2")])


def merger_workspace_bytes(w, n_groups, merge=4):
    c = _merger_c(w, merge)
    lib().ms_merger_workspace_bytes.restype = C.c_size_t
    return lib().ms_merger_workspace_bytes(C.byref(c), n_groups)


def merger_forward(w, h_vit, positions, x_llm, ws, merge=4):
    """Writes the projected visual rows into x_llm (in place) at `positions` (int32 device tensor)."""
    c, pw = _merger_c(w, merge), _merger_ptrs(w)
    _check(lib().ms_merger_forward(C.byref(c), C.byref(pw), positions.numel(), _p(h_vit), _p(positions), x_llm.shape[0], _p(x_llm),
                                   _p(ws), C.c_size_t(ws.numel()), _stream()))


def merger_backward(w, grads, h_vit, positions, d_x_llm, ws, merge=4):
    """Returns d_h_vit; `grads` (fp32 dict like w) is accumulated in place.  `ws` must be the forward call's workspace."""
    c, pw, pg = _merger_c(w, merge), _merger_ptrs(w), _merger_ptrs(grads)
    d_h = torch.empty_like(h_vit)
    _check(lib().ms_merger_backward(C.byref(c), C.byref(pw), C.byref(pg), positions.numel(), _p(h_vit), _p(positions),
                                    d_x_llm.shape[0], _p(d_x_llm), _p(d_h), _p(ws), C.c_size_t(ws.numel()), _stream()))
    return d_h


class _AdamWCfg(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("grad_scale", C.c_float), ("step", C.c_int32), ("zero_grad", C.c_int32)]


def adamw_step(grad, master, m, v, weight, step, lr, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, grad_scale=1.0,
               zero_grad=False):
    """In-place AdamW update of fp32 master / m / v from fp32 grad; `weight` (bf16 or fp32, or None) gets round(master)."""
    cfg = _AdamWCfg(lr, beta1, beta2, eps, weight_decay, grad_scale, step, int(zero_grad))
    dt = MS_F32 if weight is None else _dt(weight.dtype)
    _check(lib().ms_adamw_step(C.byref(cfg), dt, C.c_int64(master.numel()), _p(grad), _p(master), _p(m), _p(v), _p(weight),
                               _stream()))


def schedule_samples(tuples, interleave=True):
    """tuples: n x 6 times (Sec. 3.4).  Returns (order, makespan)."""
    n = len(tuples)
    flat = (C.c_double * max(6 * n, 1))(*[float(x) for t in tuples for x in t])
    order, mk = (C.c_int32 * max(n, 1))(), C.c_double(0.0)
    _check(lib().ms_schedule_samples(n, flat, int(bool(interleave)), order, C.byref(mk)))
    return [order[i] for i in range(n)], mk.value


def schedule_makespan(tuples, order, interleave=True):
    """Returns (makespan, critical_idle) of executing `tuples` in `order`."""
    n = len(tuples)
    flat = (C.c_double * max(6 * n, 1))(*[float(x) for t in tuples for x in t])
    arr = (C.c_int32 * max(n, 1))(*order)
    mk, idle = C.c_double(0.0), C.c_double(0.0)
    _check(lib().ms_schedule_makespan(n, flat, arr, int(bool(interleave)), C.byref(mk), C.byref(idle)))
    return mk.value, idle.value


# ------------------------------------------------------------------ kernel-level entry points
def k_gemm_config(tile=0, mfma16=-1):
    """Kernel selection of the bf16 GEMMs (tests, measurements): tile 0 / 128 / 256 / 256256 / 128128 / 128256 / 64128 / 64064 / -1, mfma16 -1 / 0 / 1."""
    _check(lib().ms_k_gemm_config(int(tile), int(mfma16)))


def k_gemm(a, b, trans_a=False, trans_b=False, c=None, c_fp32=False, accumulate=False, bias=None, residual=None,
           alpha=1.0, split_k=1, dtype=None):
    res_fp32 = residual is not None and residual.dtype == torch.float32 and a.dtype == torch.bfloat16
    """C[M,N] = alpha * A(m,k) B(n,k) (+bias) (+residual); a / b are 2-D tensors in their stored layout."""
    dt = _dt(dtype if dtype is not None else a.dtype)
    M, K = (a.shape[1], a.shape[0]) if trans_a else a.shape
    N = b.shape[1] if trans_b else b.shape[0]
    if c is None:
        c = torch.empty((M, N), dtype=torch.float32 if (c_fp32 or dt == MS_F32) else torch.bfloat16, device=a.device)
    _check(lib().ms_k_gemm(dt, int(trans_a), int(trans_b), M, N, K, C.c_float(alpha), _p(a), C.c_int64(a.stride(0)),
                           _p(b), C.c_int64(b.stride(0)), _p(c), C.c_int64(c.stride(0)), int(c_fp32), int(accumulate),
                           _p(bias), _p(residual), C.c_int64(residual.stride(0) if residual is not None else 0),
                           int(res_fp32), split_k, _stream()))
    return c


def k_gemm_swiglu(a, w, want_gate_up=True):
    """a[M,K], w[2F,K] (gate rows | up rows) -> (act[M,F], gate_up[M,2F] or None); bf16."""
    M, K = a.shape
    F = w.shape[0] // 2
    act = torch.empty((M, F), dtype=a.dtype, device=a.device)
    gu = torch.empty((M, 2 * F), dtype=a.dtype, device=a.device) if want_gate_up else None
    _check(lib().ms_k_gemm_swiglu(M, F, K, _p(a), C.c_int64(a.stride(0)), _p(w), C.c_int64(w.stride(0)), _p(act),
                                  C.c_int64(F), _p(gu), C.c_int64(2 * F), _stream()))
    return act, gu


def k_norm_forward(kind, x, g, b, eps):
    """x may be fp32 while g / b / y are bf16 (fp32 residual stream of a bf16 section)."""
    n, d = x.shape
    y = torch.empty((n, d), dtype=g.dtype, device=x.device)
    xf = int(x.dtype == torch.float32 and g.dtype == torch.bfloat16)
    rstd = torch.empty(n, dtype=torch.float32, device=x.device)
    mean = torch.empty(n, dtype=torch.float32, device=x.device) if kind == 1 else None
    _check(lib().ms_k_norm_forward(kind, _dt(g.dtype), xf, n, d, C.c_float(eps), _p(x), _p(g), _p(b), _p(y), _p(mean),
                                   _p(rstd), _stream()))
    return y, mean, rstd


def k_norm_backward(kind, dy, x, g, mean, rstd, add=None, dg=None, db=None):
    n, d = x.shape
    dx = torch.empty_like(dy)
    xf = int(x.dtype == torch.float32 and g.dtype == torch.bfloat16)
    dg = torch.zeros(d, dtype=torch.float32, device=x.device) if dg is None else dg
    db = (torch.zeros(d, dtype=torch.float32, device=x.device) if db is None else db) if kind == 1 else None
    sc = workspace(lib().ms_k_norm_backward_scratch_bytes(d), x.device, "norm")
    _check(lib().ms_k_norm_backward(kind, _dt(g.dtype), xf, n, d, _p(dy), _p(x), _p(g), _p(mean), _p(rstd), _p(add), _p(dx),
                                    _p(dg), _p(db), _p(sc), _stream()))
    return dx, dg, db


def k_positions(batch):
    pos = torch.empty(batch.n_tokens, dtype=torch.int32, device=batch.cu_dev.device)
    _check(lib().ms_k_positions(batch.n_tokens, batch.n_seqs, _p(batch.cu_dev), _p(pos), _stream()))
    return pos


def k_rope_table(max_pos, head_dim, base, device="cuda"):
    t = torch.empty((max_pos, head_dim // 2, 2), dtype=torch.float32, device=device)
    _check(lib().ms_k_rope_table(max_pos, head_dim, C.c_float(base), _p(t), _stream()))
    return t


def k_rope(x, n_heads, head_dim, pos, table, inverse=False):
    """In place on x[n, row_stride]."""
    _check(lib().ms_k_rope(_dt(x.dtype), x.shape[0], n_heads, head_dim, C.c_int64(x.stride(0)), _p(x), _p(pos), _p(table),
                           int(inverse), _stream()))
    return x


def k_act_forward(kind, up):
    n, f = up.shape[0], up.shape[1] // 2 if kind == 0 else up.shape[1]
    a = torch.empty((n, f), dtype=up.dtype, device=up.device)
    _check(lib().ms_k_act_forward(kind, _dt(up.dtype), n, f, _p(up), _p(a), _stream()))
    return a


def k_act_backward(kind, da, up):
    dup = torch.empty_like(up)
    _check(lib().ms_k_act_backward(kind, _dt(up.dtype), da.shape[0], da.shape[1], _p(da), _p(up), _p(dup), _stream()))
    return dup


def k_embedding_forward(ids, table, out_fp32=False):
    x = torch.empty((ids.shape[0], table.shape[1]), dtype=torch.float32 if out_fp32 else table.dtype, device=table.device)
    _check(lib().ms_k_embedding_forward(_dt(table.dtype), int(out_fp32), ids.shape[0], table.shape[1], table.shape[0],
                                        _p(ids), _p(table), _p(x), _stream()))
    return x


def k_embedding_backward(ids, dx, vocab, d_table=None):
    if d_table is None:
        d_table = torch.zeros((vocab, dx.shape[1]), dtype=torch.float32, device=dx.device)
    _check(lib().ms_k_embedding_backward(_dt(dx.dtype), ids.shape[0], dx.shape[1], vocab, _p(ids), _p(dx), _p(d_table),
                                         _stream()))
    return d_table


# The entry points below take device tensors of one device and check them here; outputs and scratch that are not given are allocated
# per call, so calls on several streams, devices or captured graphs share nothing.
def _args(*types):
    kinds = {"i": C.c_int32, "l": C.c_int64, "f": C.c_float, "p": C.c_void_p, "z": C.c_size_t}
    return [kinds[k] for k in "".join(types)]


_ARGTYPES = {
    "ms_k_qk_norm_rope_forward": _args("iiiiif", "plpppp", "ipl", "p"),
    "ms_k_qk_norm_rope_backward": _args("iiiiif", "plplpppp", "ipl", "pppp"),
    "ms_k_embedding_scaled_forward": _args("iiiiif", "pppp"),
    "ms_k_embedding_sorted_backward": _args("iiiif", "ppppzp"),
    "ms_k_fp8_quantize": _args("iiii", "plplplp"),
    "ms_k_norm_fp8": _args("iiiif", "ppplplp"),
    "ms_k_swiglu_fp8": _args("iii", "plplplp"),
    "ms_k_gemm_fp8": _args("iii", "plplplpl", "plipli", "p"),
    "ms_k_gemm_fp8_swiglu": _args("iii", "plplplpl", "plpl", "pzp"),
}
_SCRATCH = {
    "ms_k_qk_norm_rope_backward_scratch_bytes": _args("i"),
    "ms_k_embedding_sorted_backward_scratch_bytes": _args("iii"),
    "ms_k_gemm_fp8_swiglu_scratch_bytes": _args("iii"),
}
_fns = {}


def _fn(name):
    f = _fns.get(name)
    if f is None:
        f = getattr(lib(), name)
        f.argtypes = _ARGTYPES.get(name) or _SCRATCH[name]
        f.restype = C.c_size_t if name in _SCRATCH else C.c_int
        _fns[name] = f
    return f


def _call(name, dev, *args):
    """The library's entry point on the current stream of `dev`, which is made the current device for the call."""
    f, i = _fn(name), dev.index
    if i == torch._C._cuda_getDevice():
        status = f(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(dev):
            status = f(*args, torch._C._cuda_getCurrentRawStream(i))
    if status:
        _check(status)


def _need(name, t, dtypes, shape, device, rows=False):
    """t: a tensor of one of `dtypes` and of `shape` (None: any size) on `device` (None: any GPU), contiguous, or, with `rows`, a matrix
    whose rows are."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.shape == shape and t.is_cuda and (device is None or t.device == device) and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise ValueError(f"{name}: expected a tensor of {' or '.join(str(d) for d in dtypes)}, got {getattr(t, 'dtype', type(t).__name__)}")
    if t.dim() != len(shape) or any(s is not None and s != a for s, a in zip(shape, t.shape)):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name}: expected a tensor on {device or 'a GPU'}, got one on {t.device}")
    if not (t.is_contiguous() or (rows and t.stride(1) == 1 and t.stride(0) >= t.shape[1])):
        raise ValueError(f"{name}: expected {'rows with unit stride' if rows else 'a contiguous tensor'}, got strides {t.stride()}")


def _n_rows(t):
    return t.shape[0] if isinstance(t, torch.Tensor) and t.dim() == 2 else None


def _ld(t):
    """Elements between the rows of a matrix (a single row may carry any stride)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


_STORE, _F32, _I32 = (torch.bfloat16, torch.float32), (torch.float32,), (torch.int32,)


def _qkn_args(x, n_q_heads, n_kv_heads, head_dim, g_q, g_k, pos, table, what):
    n = _n_rows(x)
    _need(what, x, _STORE, (n, (n_q_heads + 2 * n_kv_heads) * head_dim), None, rows=True)
    dev = x.device
    _need("g_q", g_q, (x.dtype,), (head_dim,), dev)
    _need("g_k", g_k, (x.dtype,), (head_dim,), dev)
    _need("pos", pos, _I32, (n,), dev)
    _need("table", table, _F32, (table.shape[0] if isinstance(table, torch.Tensor) and table.dim() else None, head_dim // 2, 2), dev)
    return n, dev


def k_qk_norm_rope_forward(x, n_q_heads, n_kv_heads, head_dim, g_q, g_k, eps, pos, table, out=None):
    """RMSNorm (gains g_q / g_k) and rotation of the query and key heads of x [n, (n_q + 2 n_kv) head_dim]; V heads are copied.  out=x: in
    place.  pos, table: k_positions, k_rope_table."""
    n, dev = _qkn_args(x, n_q_heads, n_kv_heads, head_dim, g_q, g_k, pos, table, "x")
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif out is not x:
        _need("out", out, (x.dtype,), x.shape, dev, rows=True)
    _call("ms_k_qk_norm_rope_forward", dev, _dt(x.dtype), n, n_q_heads, n_kv_heads, head_dim, eps, x.data_ptr(), _ld(x), g_q.data_ptr(),
          g_k.data_ptr(), pos.data_ptr(), table.data_ptr(), table.shape[0], out.data_ptr(), _ld(out))
    return out


def k_qk_norm_rope_backward(dy, x, n_q_heads, n_kv_heads, head_dim, g_q, g_k, eps, pos, table, dg_q, dg_k, out=None):
    """Returns dx (V heads: dy's); x is the forward call's input.  dg_q / dg_k (fp32) are accumulated in place.  out=dy: in place."""
    n, dev = _qkn_args(x, n_q_heads, n_kv_heads, head_dim, g_q, g_k, pos, table, "x")
    _need("dy", dy, (x.dtype,), x.shape, dev, rows=True)
    _need("dg_q", dg_q, _F32, (head_dim,), dev)
    _need("dg_k", dg_k, _F32, (head_dim,), dev)
    if out is None:
        out = torch.empty_like(dy, memory_format=torch.contiguous_format)
    elif out is not dy:
        _need("out", out, (x.dtype,), x.shape, dev, rows=True)
    sc = dg_q.new_empty(_fn("ms_k_qk_norm_rope_backward_scratch_bytes")(head_dim) // 4)
    _call("ms_k_qk_norm_rope_backward", dev, _dt(x.dtype), n, n_q_heads, n_kv_heads, head_dim, eps, dy.data_ptr(), _ld(dy), x.data_ptr(),
          _ld(x), g_q.data_ptr(), g_k.data_ptr(), pos.data_ptr(), table.data_ptr(), table.shape[0], out.data_ptr(), _ld(out),
          dg_q.data_ptr(), dg_k.data_ptr(), sc.data_ptr())
    return out


def k_embedding_scaled_forward(ids, table, scale, out_fp32=False):
    """scale * table[ids]; ids outside the table give zeros."""
    _need("table", table, _STORE, (None, None), None)
    _need("ids", ids, _I32, (None,), table.device)
    n, (vocab, d) = ids.shape[0], table.shape
    x = table.new_empty((n, d), dtype=torch.float32) if out_fp32 else table.new_empty((n, d))
    _call("ms_k_embedding_scaled_forward", table.device, _dt(table.dtype), int(out_fp32), n, d, vocab, scale, ids.data_ptr(), table.data_ptr(), x.data_ptr())
    return x


def k_embedding_sorted_backward(ids, dx, scale, d_table):
    """d_table (fp32 [vocab, d], accumulated in place and returned) += scale * the sums of dx's rows by id, in an order that the ids alone fix."""
    _need("dx", dx, _STORE, (None, None), None)
    n, d = dx.shape
    _need("ids", ids, _I32, (n,), dx.device)
    _need("d_table", d_table, _F32, (None, d), dx.device)
    vocab = d_table.shape[0]
    sc = ids.new_empty((_fn("ms_k_embedding_sorted_backward_scratch_bytes")(n, d, vocab) + 3) // 4)
    _call("ms_k_embedding_sorted_backward", dx.device, _dt(dx.dtype), n, d, vocab, scale, ids.data_ptr(), dx.data_ptr(), d_table.data_ptr(),
          sc.data_ptr(), sc.numel() * 4)
    return d_table


def _codes(n, k, scale_rows, device):
    """Empty codes [n, k] and scale bytes (rows of whole words)."""
    return (torch.empty((n, k), dtype=torch.float8_e4m3fn, device=device),
            torch.empty((scale_rows, (k + 511) // 512 * 4), dtype=torch.uint8, device=device))


def k_fp8_quantize(x, block_rows=1):
    """(codes e4m3 [n, k], scale bytes): value = code * 2^(byte - 127), a byte per block of block_rows (1 or 128) x 128."""
    _need("x", x, _STORE, (None, None), None, rows=True)
    n, k = x.shape
    q, s = _codes(n, k, n if block_rows == 1 else (n + 127) // 128, x.device)
    _call("ms_k_fp8_quantize", x.device, _dt(x.dtype), block_rows, n, k, x.data_ptr(), _ld(x), q.data_ptr(), k, s.data_ptr(), s.shape[1])
    return q, s


def k_norm_fp8(x, g, eps):
    """Codes and scale bytes of RMSNorm(x) g; x may be fp32 while g is bf16."""
    _need("x", x, _STORE, (None, None), None)
    n, d = x.shape
    _need("g", g, (x.dtype, torch.bfloat16), (d,), x.device)
    q, s = _codes(n, d, n, x.device)
    _call("ms_k_norm_fp8", x.device, _dt(g.dtype), int(x.dtype == torch.float32), n, d, eps, x.data_ptr(), g.data_ptr(), q.data_ptr(), d,
          s.data_ptr(), s.shape[1])
    return q, s


def k_swiglu_fp8(gate_up):
    """Codes and scale bytes of silu(gate) * up, gate_up [n, 2 f]."""
    both = gate_up.shape[1] // 2 * 2 if isinstance(gate_up, torch.Tensor) and gate_up.dim() == 2 else None
    _need("gate_up", gate_up, _STORE, (None, both), None, rows=True)
    n, f = gate_up.shape[0], gate_up.shape[1] // 2
    q, s = _codes(n, f, n, gate_up.device)
    _call("ms_k_swiglu_fp8", gate_up.device, _dt(gate_up.dtype), n, f, gate_up.data_ptr(), _ld(gate_up), q.data_ptr(), f, s.data_ptr(), s.shape[1])
    return q, s


def _fp8_args(a, sa, w, sw):
    _need("a", a, (torch.float8_e4m3fn,), (None, None), None, rows=True)
    (m, k), dev = a.shape, a.device
    words = (k + 511) // 512 * 4
    _need("sa", sa, (torch.uint8,), (m, words), dev, rows=True)
    _need("w", w, (torch.float8_e4m3fn,), (None, k), dev, rows=True)
    _need("sw", sw, (torch.uint8,), ((w.shape[0] + 127) // 128, words), dev, rows=True)
    return m, w.shape[0], k, a.data_ptr(), _ld(a), sa.data_ptr(), _ld(sa), w.data_ptr(), _ld(w), sw.data_ptr(), _ld(sw)


def k_gemm_fp8(a, sa, w, sw, residual=None, c=None, c_fp32=None, fast_sums=False, fp32_sums=False):
    """a w^T (+ residual) of 8-bit operands as k_fp8_quantize makes them (a: block_rows=1, w: 128).  The result is bf16, or fp32 if c_fp32
    (by default: if the residual is); c: a tensor to write to, which may be the residual (else they must not overlap).  fast_sums: an fp32 result from the 8-bit
    matrix cores' sums, which a bf16 result has unless fp32_sums asks for an fp32 result's, at half the rate."""
    if fast_sums and fp32_sums:
        raise ValueError("k_gemm_fp8: fast_sums and fp32_sums exclude each other")
    args = _fp8_args(a, sa, w, sw)
    m, n, dev = args[0], args[1], a.device
    if residual is not None:
        _need("residual", residual, _STORE, (m, n), dev, rows=True)
    if c is None:
        f32 = residual is not None and residual.dtype == torch.float32 if c_fp32 is None else c_fp32
        c = torch.empty((m, n), dtype=torch.float32 if f32 else torch.bfloat16, device=dev)
    else:
        _need("c", c, _STORE, (m, n), dev, rows=True)
    kind = (2 if fast_sums else 1) if c.dtype == torch.float32 else 3 if fp32_sums else 0
    _call("ms_k_gemm_fp8", dev, *args, c.data_ptr(), _ld(c), kind, residual.data_ptr() if residual is not None else None,
          _ld(residual) if residual is not None else 0, int(residual is not None and residual.dtype == torch.float32))
    return c


def k_gemm_fp8_config(tile=0):
    """Tile of the 8-bit products (tests, measurements): 0 / 256256 / 256192 / 128128 / 128129 / 64128 / 64129 / 64064; 16016: the kernel without tiles."""
    _check(lib().ms_k_gemm_fp8_config(int(tile)))


def k_gemm_fp8_swiglu(a, sa, w, sw, fp32_sums=False):
    """Codes and scale bytes of silu(a wg^T) * (a wu^T), w [2 f, k] = gate rows, then up rows.  fp32_sums: as for k_gemm_fp8, with gate and up
    through memory."""
    args = _fp8_args(a, sa, w, sw)
    m, f, k, dev = args[0], args[1] // 2, args[2], a.device
    if args[1] % 2:
        raise ValueError(f"w: expected gate rows and as many up rows, got {args[1]}")
    if fp32_sums:
        return k_swiglu_fp8(k_gemm_fp8(a, sa, w, sw, c_fp32=True))
    q, s = _codes(m, f, m, dev)
    nb = _fn("ms_k_gemm_fp8_swiglu_scratch_bytes")(m, f, k)
    sc = torch.empty(nb, dtype=torch.uint8, device=dev) if nb else None
    _call("ms_k_gemm_fp8_swiglu", dev, m, f, *args[2:], q.data_ptr(), f, s.data_ptr(), s.shape[1], sc.data_ptr() if nb else None, nb)
    return q, s


def k_colsum(x, out=None):
    n, c = x.shape
    out = torch.zeros(c, dtype=torch.float32, device=x.device) if out is None else out
    sc = workspace(lib().ms_k_norm_backward_scratch_bytes(c), x.device, "norm")
    _check(lib().ms_k_colsum(_dt(x.dtype), n, c, _p(x), _p(out), _p(sc), _stream()))
    return out


def k_attention_forward(qkv, batch, n_q_heads, n_kv_heads, head_dim, causal):
    n = qkv.shape[0]
    o = torch.empty((n, n_q_heads * head_dim), dtype=qkv.dtype, device=qkv.device)
    lse = torch.empty((n_q_heads, n), dtype=torch.float32, device=qkv.device)
    _check(lib().ms_k_attention_forward(_dt(qkv.dtype), int(causal), n_q_heads, n_kv_heads, head_dim, n, batch.n_seqs,
                                        batch.max_seqlen, _p(batch.cu_dev), _p(qkv), _p(o), _p(lse), _stream()))
    return o, lse


def k_attention_backward(qkv, o, lse, d_o, batch, n_q_heads, n_kv_heads, head_dim, causal):
    n = qkv.shape[0]
    dqkv = torch.empty_like(qkv)
    sc = workspace(lib().ms_k_attention_backward_scratch_bytes(_dt(qkv.dtype), n_q_heads, n_kv_heads, head_dim, n),
                   qkv.device, "attn")
    _check(lib().ms_k_attention_backward(_dt(qkv.dtype), int(causal), n_q_heads, n_kv_heads, head_dim, n, batch.n_seqs,
                                         batch.max_seqlen, _p(batch.cu_dev), _p(qkv), _p(o), _p(lse), _p(d_o), _p(dqkv),
                                         _p(sc), _stream()))
    return dqkv


def k_mfma_probe(workgroups, iters, sink, random_operands=False, mfma16=False):
    _check(lib().ms_k_mfma_probe(workgroups, iters, int(random_operands), int(mfma16), _p(sink), _stream()))


def k_clock_monitor(microseconds, out):
    """out: int64[2] device tensor; launched on the current stream."""
    _check(lib().ms_k_clock_monitor(int(microseconds), _p(out), _stream()))


def k_copy(src, dst):
    _check(lib().ms_k_copy(_p(src), _p(dst), C.c_size_t(src.numel() * src.element_size()), _stream()))
    return dst


PROFILE_CLASSES = ["gemm_nt", "gemm_t", "attn_fwd", "attn_bwd", "norm_fwd", "norm_bwd", "act_fwd", "act_bwd", "rope",
                   "kd_stats", "kd_dz", "misc"]


def profile_enable(on):
    _check(lib().ms_profile_enable(int(on)))


def profile_read():
    """{class name: (launches, total_ms, total_work)} of the launches recorded since profile_enable(1)."""
    out = {}
    for i, name in enumerate(PROFILE_CLASSES):
        n, ms, work = C.c_int64(0), C.c_double(0), C.c_double(0)
        _check(lib().ms_profile_read(i, C.byref(n), C.byref(ms), C.byref(work)))
        out[name] = (n.value, ms.value, work.value)
    return out
