"""Query / key norms with rotation in one pass, against the definition in 64 bits and against differences."""
import pytest
import torch

from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import workloads as wl

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EPS = 1e-6
U = 2.0 ** -24                       # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def inputs(n, nq, nkv, hd, dtype, max_pos=97, device="cuda"):
    tag = f"qkn{n}.{nq}.{nkv}.{hd}"
    x = wl.normal(3, tag + "x", (n, (nq + 2 * nkv) * hd), 2.0, 0.0, dtype, device)
    dy = wl.normal(3, tag + "dy", x.shape, 1.0, 0.0, dtype, device)
    g_q, g_k = (wl.normal(3, tag + k, (hd,), 0.3, 1.0, dtype, device) for k in ("gq", "gk"))
    pos = (torch.arange(n, device=device) * 37 % max_pos).to(torch.int32)
    angle = torch.arange(max_pos, dtype=F64)[:, None] * 1e4 ** (-2.0 * torch.arange(hd // 2, dtype=F64) / hd)
    return x, dy, g_q, g_k, pos, torch.stack((angle.cos(), angle.sin()), -1).to(F32).to(device)


def rotate(t, c, s):
    lo, hi = t.chunk(2, -1)
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


def angles(pos, table):
    p = pos.long().cpu()
    inside = ((p >= 0) & (p < table.shape[0]))[:, None]
    cs = table.cpu().double()[p.clamp(0, table.shape[0] - 1)]
    return torch.where(inside, cs[..., 0], 1.0)[:, None], torch.where(inside, cs[..., 1], 0.0)[:, None]


def reference(x, dy, g_q, g_k, pos, table, nq, nkv, hd):
    """(y, dx, dg_q, dg_k) in 64 bits and what each one's fp32 rounding errors scale with."""
    n = x.shape[0]
    x, dy = x.cpu().double().view(n, -1, hd), dy.cpu().double().view(n, -1, hd)
    g = torch.cat((g_q.cpu().double().expand(nq, hd), g_k.cpu().double().expand(nkv, hd)))
    c, s = angles(pos, table)
    xh = x[:, :nq + nkv]
    r = 1 / torch.sqrt(xh.square().mean(-1, keepdim=True) + EPS)
    y, d = rotate(xh * r * g, c, s), rotate(dy[:, :nq + nkv], c, -s)
    xn, t = xh * r, d * g
    m = (t * xn).mean(-1, keepdim=True)
    dx = r * (t - xn * m)
    pair = lambda v: rotate(v.abs(), torch.ones_like(c), -torch.ones_like(c)).abs()   # |lo| + |hi| (and the half that differs)
    both = lambda v: torch.cat([v.abs()[..., :hd // 2] + v.abs()[..., hd // 2:]] * 2, -1)
    dabs = both(dy[:, :nq + nkv])
    e_y, e_dx = both(xh * r * g), r * (dabs * g.abs() + xn.abs() * (dabs * g.abs() * xn.abs()).mean(-1, keepdim=True))
    dg, e_dg = (d * xn), dabs * xn.abs()
    v = x[:, nq + nkv:]
    return dict(y=torch.cat((y, v), 1).reshape(n, -1), dx=torch.cat((dx, dy[:, nq + nkv:]), 1).reshape(n, -1),
                dg_q=dg[:, :nq].sum((0, 1)), dg_k=dg[:, nq:].sum((0, 1)),
                e_y=torch.cat((e_y, 0 * v), 1).reshape(n, -1), e_dx=torch.cat((e_dx, 0 * v), 1).reshape(n, -1),
                e_dg_q=e_dg[:, :nq].sum((0, 1)), e_dg_k=e_dg[:, nq:].sum((0, 1)))


def close(got, ref, scale, dtype, ulps, what):
    """Half a step of the output's type, and `ulps` fp32 half steps of what the sums are made of."""
    bound = half_step(dtype) * (1 + 1e-3) * ref.abs() + ulps * U * scale + 1e-30
    off = (got.cpu().double() - ref).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off / bound).max()):.3g} of the bound"


# an fp32 sum of hd squares in 16-element pieces and a tree, a reciprocal root, four products: under 64 half steps; the backward pass
# doubles that.  A gain's gradient: at most 400 terms per lane here, 64 / G lanes, 4 waves and the partial rows.
SHAPES = [(1, 1, 1, 16), (1, 32, 8, 128), (2, 12, 2, 128), (5, 3, 1, 80), (293, 2, 2, 64), (130, 7, 3, 256), (33, 5, 5, 48),
          (9, 2, 1, 512), (1031, 8, 2, 128), (4099, 4, 1, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,nq,nkv,hd", SHAPES)
def test_forward_and_backward(n, nq, nkv, hd, dtype):
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, dtype)
    pos[n // 2] = -1                                              # no position: not rotated
    pos[n // 3] = table.shape[0]
    ref = reference(x, dy, g_q, g_k, pos, table, nq, nkv, hd)
    a = (nq, nkv, hd, g_q, g_k, EPS, pos, table)
    close(B.k_qk_norm_rope_forward(x, *a), ref["y"], ref["e_y"], dtype, 64, "y")
    dg_q, dg_k = torch.full((hd,), 3.0, device="cuda"), torch.zeros(hd, device="cuda")
    dx = B.k_qk_norm_rope_backward(dy, x, *a, dg_q, dg_k)
    close(dx, ref["dx"], ref["e_dx"], dtype, 128, "dx")
    close(dg_q - 3.0, ref["dg_q"], ref["e_dg_q"] + 3, F32, 512, "dg_q")
    close(dg_k, ref["dg_k"], ref["e_dg_k"], F32, 512, "dg_k")
    again_q, again_k = torch.full((hd,), 3.0, device="cuda"), torch.zeros(hd, device="cuda")
    assert torch.equal(dx, B.k_qk_norm_rope_backward(dy, x, *a, again_q, again_k)) and torch.equal(dg_q, again_q) and torch.equal(dg_k, again_k)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_strided_rows(dtype):
    n, nq, nkv, hd = 77, 6, 2, 128
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, dtype)
    a = (nq, nkv, hd, g_q, g_k, EPS, pos, table)
    want = B.k_qk_norm_rope_forward(x, *a)
    wide = torch.full((n, x.shape[1] + 24), 7.0, dtype=dtype, device="cuda")
    wide[:, 8:8 + x.shape[1]] = x
    view = wide[:, 8:8 + x.shape[1]]
    assert torch.equal(B.k_qk_norm_rope_forward(view, *a), want)
    assert B.k_qk_norm_rope_forward(view, *a, out=view) is view
    assert torch.equal(view, want) and bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + x.shape[1]:] == 7).all())
    grads = [torch.zeros(hd, device="cuda") for _ in range(4)]
    dx = B.k_qk_norm_rope_backward(dy, x, *a, grads[0], grads[1])
    assert B.k_qk_norm_rope_backward(dy, x, *a, grads[2], grads[3], out=dy) is dy
    assert torch.equal(dx, dy) and torch.equal(grads[0], grads[2]) and torch.equal(grads[1], grads[3])
    one = torch.zeros(hd, device="cuda")                          # one gain for both kinds: one row takes both gradients
    B.k_qk_norm_rope_backward(wl.normal(3, f"qkn{n}.{nq}.{nkv}.{hd}dy", x.shape, 1.0, 0.0, dtype, "cuda"), x, *a, one, one)
    assert torch.allclose(one, grads[0] + grads[1], rtol=1e-5, atol=1e-4)


@pytest.mark.gpu
def test_zero_rows_infinities_and_large_values():
    n, nq, nkv, hd = 6, 2, 1, 64
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, BF16)
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, hd + 1] = float("inf")
    x[3] = 1e-30
    v_bits = x[:, 3 * hd:].view(torch.int16)
    v_bits[4] = 0x7FA5                                            # a NaN pattern in a V head is copied as it is
    a = (nq, nkv, hd, g_q, g_k, EPS, pos, table)
    y = B.k_qk_norm_rope_forward(x, *a)
    assert bool((y[0, :3 * hd] == 0).all())
    assert bool(y[1, :hd].isnan().all()) and not bool(y[1, hd:].isnan().any())
    assert not bool(y[2, :hd].isnan().any()) and not bool(y[2, 2 * hd:].isnan().any())
    assert bool(y[3].isfinite().all())
    assert torch.equal(y[:, 3 * hd:].view(torch.int16), v_bits)


@pytest.mark.gpu
def test_gradient_against_differences():
    n, nq, nkv, hd = 5, 3, 2, 64
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, F32)
    dg_q, dg_k = torch.zeros(hd, device="cuda"), torch.zeros(hd, device="cuda")
    dx = B.k_qk_norm_rope_backward(dy, x, nq, nkv, hd, g_q, g_k, EPS, pos, table, dg_q, dg_k).cpu().double()
    vx, vq, vk = (wl.normal(5, k, t.shape, 1.0, 0.0, F64) for k, t in (("vx", x), ("vq", g_q), ("vk", g_k)))
    f = lambda h: (reference(x.cpu().double() + h * vx, dy, g_q.cpu().double() + h * vq, g_k.cpu().double() + h * vk, pos, table, nq, nkv, hd)["y"]
                   * dy.cpu().double()).sum()
    h = 1e-5                                                      # differences of 64 bits: 1e-10 and what the kernel rounds, 1e-6
    want, got = (f(h) - f(-h)) / (2 * h), (dx * vx).sum() + (dg_q.cpu().double() * vq).sum() + (dg_k.cpu().double() * vk).sum()
    parts = (dx * vx).abs().sum() + (dg_q.cpu().double() * vq).abs().sum() + (dg_k.cpu().double() * vk).abs().sum()
    assert abs(got - want) <= 128 * U * parts + 1e-7 * parts


@pytest.mark.gpu
def test_replayed_graph_and_other_stream():
    n, nq, nkv, hd = 211, 12, 2, 128
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, BF16)
    a = (nq, nkv, hd, g_q, g_k, EPS, pos, table)
    dg_q, dg_k = torch.zeros(hd, device="cuda"), torch.zeros(hd, device="cuda")
    y0, dx0 = B.k_qk_norm_rope_forward(x, *a), B.k_qk_norm_rope_backward(dy, x, *a, dg_q, dg_k)
    ref = dg_q.clone(), dg_k.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(B.k_qk_norm_rope_forward(x, *a), y0)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dg_q.zero_(), dg_k.zero_()
        y, dx = B.k_qk_norm_rope_forward(x, *a), B.k_qk_norm_rope_backward(dy, x, *a, dg_q, dg_k)
    for _ in range(3):
        y.zero_(), dx.zero_()
        B.k_qk_norm_rope_forward(dy, *a)                          # the program's own work between the replays
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y0) and torch.equal(dx, dx0) and torch.equal(dg_q, ref[0]) and torch.equal(dg_k, ref[1])


@pytest.mark.gpu
def test_empty_batch():
    x, dy, g_q, g_k, pos, table = inputs(3, 2, 1, 64, BF16)
    a = (2, 1, 64, g_q, g_k, EPS, pos[:0], table)
    dg = [torch.ones(64, device="cuda") for _ in range(2)]
    assert B.k_qk_norm_rope_forward(x[:0], *a).shape == (0, 256)
    assert B.k_qk_norm_rope_backward(dy[:0], x[:0], *a, *dg).shape == (0, 256) and bool((dg[0] == 1).all())


def test_refusals_before_anything_is_launched():
    """Raw calls with made-up addresses: each is turned down on the host."""
    def fwd(dtype=1, n=4, nq=2, nkv=1, hd=64, eps=1e-6, x=4096, xs=256, gq=256, gk=256, pos=256, tab=256, mp=8, y=1 << 20, ys=256):
        return B._fn("ms_k_qk_norm_rope_forward")(dtype, n, nq, nkv, hd, eps, x, xs, gq, gk, pos, tab, mp, y, ys, None)

    def bwd(dy=4096, dys=256, x=1 << 20, xs=256, dx=1 << 21, dxs=256, dgq=256, dgk=512, sc=256):
        return B._fn("ms_k_qk_norm_rope_backward")(1, 4, 2, 1, 64, 1e-6, dy, dys, x, xs, 256, 256, 256, 256, 8, dx, dxs, dgq, dgk, sc, None)
    assert fwd(n=0) == 0
    for bad in (dict(x=None), dict(y=None), dict(gq=None), dict(pos=None), dict(tab=None), dict(dtype=2), dict(n=-1), dict(nq=0), dict(nkv=-1),
                dict(mp=0), dict(eps=float("nan")), dict(eps=-1.0), dict(y=4096 + 256), dict(x=4096, y=4096, ys=264)):
        assert fwd(**bad) == -1, bad
    for bad in (dict(hd=24), dict(hd=528), dict(x=4104), dict(xs=260), dict(gq=264), dict(ys=257)):
        assert fwd(**bad) in (-4, -2), bad
    for bad in (dict(xs=128), dict(ys=192)):
        assert fwd(**bad) == -2, bad
    for bad in (dict(dy=None), dict(sc=None), dict(dgq=None), dict(dx=(1 << 20) + 512), dict(dx=4096 + 64)):
        assert bwd(**bad) == -1, bad
    assert b"qk_norm_rope_backward" in B.lib().ms_last_error()


def test_binding_turns_down_wrong_tensors():
    x, dy, g_q, g_k, pos, table = inputs(3, 2, 1, 64, BF16, device="cpu")
    with pytest.raises(ValueError, match="on a GPU"):
        B.k_qk_norm_rope_forward(x, 2, 1, 64, g_q, g_k, EPS, pos, table)
    with pytest.raises(ValueError, match="shape"):
        B.k_qk_norm_rope_forward(x, 2, 2, 64, g_q, g_k, EPS, pos, table)
    with pytest.raises(ValueError, match="float16"):
        B.k_qk_norm_rope_forward(x.half(), 2, 1, 64, g_q, g_k, EPS, pos, table)


def test_dx_whose_v_heads_run_into_x_is_refused():
    """Out of place, dx's last V heads would be written over the first query heads of an x that begins behind its key heads."""
    def bwd(dx, dy=1 << 16, x=1 << 20):                           # 4 rows of (2 + 2) heads of 64 in bf16: 512 bytes, 384 of them query and key heads
        return B._fn("ms_k_qk_norm_rope_backward")(1, 4, 2, 1, 64, 1e-6, dy, 256, x, 256, 256, 256, 256, 256, 8, dx, 256, 256, 512, 256, None)
    x = 1 << 20
    for dx in (x - 2048 + 128, x - 2048 + 16, x + 3 * 512 + 384 - 16):
        assert bwd(dx) == -1 and b"dx overlaps x" in B.lib().ms_last_error(), dx


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_views_side_by_side_are_apart(dtype):
    n, nq, nkv, hd = 37, 3, 1, 64
    x, dy, g_q, g_k, pos, table = inputs(n, nq, nkv, hd, dtype)
    a, w = (nq, nkv, hd, g_q, g_k, EPS, pos, table), x.shape[1]
    want = B.k_qk_norm_rope_forward(x, *a)
    both = torch.full((n, 3 * w), 7.0, dtype=dtype, device="cuda")
    both[:, w:2 * w] = x
    for at in (0, 2 * w):                                         # in front of and behind its input in each row
        assert torch.equal(B.k_qk_norm_rope_forward(both[:, w:2 * w], *a, out=both[:, at:at + w]), want)
    assert torch.equal(both[:, w:2 * w], x)
    g = [torch.zeros(hd, device="cuda") for _ in range(4)]
    dx = B.k_qk_norm_rope_backward(dy, x, *a, g[0], g[1])
    both[:, :w] = dy
    assert torch.equal(B.k_qk_norm_rope_backward(both[:, :w], both[:, w:2 * w], *a, g[2], g[3], out=both[:, 2 * w:]), dx)
    assert torch.equal(g[0], g[2]) and torch.equal(g[1], g[3]) and torch.equal(both[:, w:2 * w], x) and torch.equal(both[:, :w], dy)
