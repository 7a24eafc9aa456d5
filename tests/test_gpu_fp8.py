"""8-bit operands and their products: codes and scales bit by bit, products against the operands' values in 64 bits."""
import ctypes as C

import pytest
import torch

from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import workloads as wl

BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
U = 2.0 ** -24


def normal(tag, shape, std=1.0, dtype=BF16, device="cuda"):
    return wl.normal(13, tag, shape, std, 0.0, dtype, device)


def round_e4m3(y):
    """64-bit values to e4m3: 4 significant bits, steps of 2^-9 at least, ties to even, NaN from infinities."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(y.isfinite(), torch.round(y / step) * step, torch.nan)


def quantized(x, rows):
    """(codes' values, scale bytes without padding) by the definition, in 64 bits on the CPU."""
    x = x.detach().cpu().double()
    n, k = x.shape
    codes, nb, kb = torch.empty_like(x), -(-n // rows), -(-k // 128)
    bytes_ = torch.empty((nb, kb), dtype=torch.int64)
    for b in range(kb):
        for a in range(nb):
            v = x[a * rows:(a + 1) * rows, b * 128:(b + 1) * 128]
            top = torch.where(v.isfinite(), v.abs(), 0.0).max()
            e = max(int(torch.ceil(torch.log2(top / 448))), -127) if top > 0 else 0
            codes[a * rows:(a + 1) * rows, b * 128:(b + 1) * 128] = round_e4m3(v / 2.0 ** e)
            bytes_[a, b] = e + 127
    return codes, bytes_


def values(q, s, rows):
    """What codes and scale bytes stand for, in 64 bits on the CPU."""
    scale = torch.exp2(s.cpu().double() - 127).repeat_interleave(rows, 0).repeat_interleave(128, 1)
    return q.cpu().float().double() * scale[:q.shape[0], :q.shape[1]]


def check_codes(q, s, x, rows):
    codes, bytes_ = quantized(x, rows)
    kb = bytes_.shape[1]
    assert torch.equal(s[:, :kb].cpu().long(), bytes_) and bool((s[:, kb:] == 127).all()) and s.shape[1] == (kb + 3) // 4 * 4
    got = q.cpu().float().double()
    assert torch.equal(got.isnan(), codes.isnan()) and torch.equal(got.nan_to_num(9e9), codes.nan_to_num(9e9))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("n,k", [(1, 16), (3, 128), (130, 144), (257, 688), (5, 4112), (128, 512)])
def test_codes_and_scales(n, k, rows, dtype):
    x = normal(f"q{n}.{k}", (n, k), 1.0, F32)
    x *= torch.exp2(torch.arange(n, device="cuda") % 37 - 18.0)[:, None]          # every scale its own
    x[:, 0] *= 100
    x[n // 2] = 0
    x = x.to(dtype)
    check_codes(*B.k_fp8_quantize(x, rows), x, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 128])
def test_codes_of_special_values(rows):
    n = 12
    x = torch.zeros((n, 256), dtype=F32, device="cuda")
    x[0, :5] = torch.tensor([float("inf"), -3.0, float("nan"), 448.0, 1e-3])
    x[1, 0] = 448.0                                                # the largest code exactly, and just above
    x[2, 0], x[2, 200] = 448.0 + 2 ** -15, 1.75 * 2.0 ** -100
    x[3, 0], x[3, 1] = 3.4e38, -1e38
    x[4, 0], x[4, 3] = 2.0 ** -126, 2.0 ** -130                    # smallest normal, subnormal numbers
    x[5, 0] = 2.0 ** -149
    x[6] = torch.arange(256, device="cuda") / 16 - 8               # ties
    x[7] = (torch.arange(256, device="cuda") - 128) * 2.0 ** -9
    x[8, 0], x[8, 1:40] = 448.0, (torch.arange(39, device="cuda") + 1) * 2.0 ** -10      # subnormal codes and their ties
    x[9] = float("nan")
    if rows == 1:
        check_codes(*B.k_fp8_quantize(x, 1), x, 1)
    else:
        for i in range(n):
            check_codes(*B.k_fp8_quantize(x[i:i + 1].clone(), 128), x[i:i + 1], 128)


@pytest.mark.gpu
def test_strided_rows_and_untouched_neighbours():
    wide = torch.full((70, 400), 7.0, dtype=BF16, device="cuda")
    wide[:, 16:16 + 272] = normal("sr", (70, 272))
    x = wide[:, 16:16 + 272]
    check_codes(*B.k_fp8_quantize(x), x.contiguous(), 1)
    q, s = torch.full((72, 304), 5, dtype=torch.uint8, device="cuda"), torch.full((72, 8), 9, dtype=torch.uint8, device="cuda")
    B._call("ms_k_fp8_quantize", x.device, 1, 1, 70, 272, x.data_ptr(), 400, q.data_ptr(), 304, s.data_ptr(), 8)
    check_codes(q[:70, :272].view(E4M3), s[:70, :4], x.contiguous(), 1)
    assert bool((q[70:] == 5).all()) and bool((q[:, 272:] == 5).all()) and bool((s[70:] == 9).all()) and bool((s[:, 4:] == 9).all())


def near_codes(q, s, ref, moved=1e-3, slack=0.0):
    """Codes of a computed operand: within half a step of e4m3 and what fp32 computing adds (a value that close to a tie may go either way)."""
    got = values(q, s, 1)
    top = torch.nn.functional.pad(ref.abs(), (0, -ref.shape[1] % 128)).view(ref.shape[0], -1, 128).amax(-1).repeat_interleave(128, 1)[:, :ref.shape[1]]
    # half a step of a normal code: 2^-4 relative; of a subnormal one: 2^-10 of a scale that is at most top / 224 (or, next to a power, twice that)
    bound = 2.0 ** -4 * ref.abs() * (1 + 1e-2) + 2.0 ** -10 * top / 224 * 1.01 + 1e-30
    assert bool(((got - ref).abs() <= bound + slack).all())
    scale = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-127))
    exact = torch.where(top > 0, round_e4m3(ref / scale) * scale, 0.0)
    # ulps of fp32 computing move a value over a tie at most once in some 10^4 times
    assert float((got != exact).double().mean()) <= moved


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(1, 128), (7, 688), (130, 4096), (33, 5104), (300, 512)])
def test_norm_and_quantise(n, d):
    for xt, gt in ((F32, BF16), (BF16, BF16), (F32, F32)):
        x, g = normal(f"nx{n}{d}", (n, d), 3.0, xt), 1 + normal(f"ng{d}", (d,), 0.1, F32)
        g = g.to(gt)
        x[n // 2, :] = 0
        xd = x.cpu().double()
        near_codes(*B.k_norm_fp8(x, g, 1e-6), xd / torch.sqrt(xd.square().mean(1, keepdim=True) + 1e-6) * g.cpu().double())


@pytest.mark.gpu
@pytest.mark.parametrize("n,f", [(1, 16), (5, 344 * 2), (129, 5504)])
def test_swiglu_and_quantise(n, f):
    for dt in (BF16, F32):
        gu = normal(f"gu{n}{f}", (n, 2 * f), 2.0, dt)
        g, u = gu.cpu().double().chunk(2, 1)
        near_codes(*B.k_swiglu_fp8(gu), g / (1 + torch.exp(-g)) * u)


def operands(m, n, k, tag=""):
    a, w = normal(f"a{m}{k}{tag}", (m, k), 1.0, F32), normal(f"w{n}{k}{tag}", (n, k), 0.05, F32)
    a *= torch.exp2(torch.arange(m, device="cuda") % 11 - 5.0)[:, None] * torch.exp2(torch.arange(k, device="cuda") // 128 % 5 - 2.0)
    w *= torch.exp2(torch.arange(n, device="cuda") // 128 % 5 - 2.0)[:, None] * torch.exp2(torch.arange(k, device="cuda") // 128 % 3 - 1.0)
    if m > 3:
        a[m // 2] = 0
    return B.k_fp8_quantize(a), B.k_fp8_quantize(w, 128)


def product(a, w):
    x, y = values(*a, 1).cuda(), values(*w, 128).cuda()
    return x @ y.t(), x.abs() @ y.abs().t()


def cut_off(a, w):
    """What the 8-bit matrix cores may cut off: of eight consecutive k, seven products lose less than 2^-13 of the largest each."""
    x, y = values(*a, 1).cuda().abs().float(), values(*w, 128).cuda().abs().float()
    x, y = (torch.nn.functional.pad(t, (0, -t.shape[1] % 8)) for t in (x, y))
    top = torch.zeros((x.shape[0], y.shape[0]), dtype=F64, device="cuda")
    for k in range(0, x.shape[1], 8):
        best = x[:, k, None] * y[None, :, k]
        for i in range(k + 1, k + 8):
            best = torch.maximum(best, x[:, i, None] * y[None, :, i])
        top += best
    return 7 * 2.0 ** -13 * top


def close(got, ref, size, k, what, extra=0.0):
    """Half a step of the output's type, and of the fp32 sum a step (rounded or cut off) for each eight k and one for each block."""
    bound = torch.finfo(got.dtype).eps / 2 * 1.001 * ref.abs() + (k / 8 + k / 128 + 16) * 2 * U * size + extra + 1e-30
    off = (got.double() - ref).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off / bound).max()):.3g} of the bound"


# one row of tiles and several, ragged in every direction, K within a block, at its end and behind it; more K tiles than a panel of scales
SHAPES = [(1, 16, 16), (1, 1, 128), (1, 4096, 2048), (2, 300, 688), (16, 24832, 512), (17, 129, 1024), (33, 8200, 272), (63, 1000, 4096), (64, 64, 144),
          (65, 256, 128), (100, 333, 688), (256, 256, 256), (257, 511, 1536), (300, 2048, 4112), (511, 130, 160), (777, 1280, 384), (1025, 768, 2048),
          (70, 64, 13968), (129, 300, 14000), (5, 40, 28000), (2049, 144, 272)]


@pytest.fixture
def fp8_tile():
    yield B.k_gemm_fp8_config
    B.k_gemm_fp8_config(0)


TILES = [256256, 128128, 128129, 64128, 64129, 64064]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [s for s in SHAPES if s[0] > 1])
def test_tiles_give_the_same_bits(m, n, k, fp8_tile):
    a, w = operands(m, n, k)
    ref, size = product(a, w)
    res = normal(f"r{m}{n}", (m, n), 1.0)
    first = None
    for tile in TILES:
        fp8_tile(tile)
        got = [B.k_gemm_fp8(*a, *w), B.k_gemm_fp8(*a, *w, residual=res, c_fp32=True, fast_sums=True), B.k_gemm_fp8(*a, *w, c_fp32=True)]
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(first, got)), tile
    close(first[0], ref, size, k, "bf16", cut_off(a, w))
    close(first[2], ref, size, k, "fp32")


@pytest.mark.gpu
@pytest.mark.parametrize("m,f,k", [(65, 128, 144), (257, 640, 256), (300, 256, 2048), (130, 384, 14000), (513, 512, 13840)])
def test_swiglu_tiles_give_the_same_bits(m, f, k, fp8_tile):
    a, w = operands(m, 2 * f, k)
    gu = B.k_gemm_fp8(*a, *w, c_fp32=True, fast_sums=True)
    q, s = B.k_swiglu_fp8(gu)
    for tile in (256256, 128128, 64128):
        fp8_tile(tile)
        q2, s2 = B.k_gemm_fp8_swiglu(*a, *w)
        assert torch.equal(s, s2) and torch.equal(q.view(torch.uint8), q2.view(torch.uint8)), tile


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(m, n, k):
    a, w = operands(m, n, k)
    ref, size = product(a, w)
    cut = cut_off(a, w)
    close(B.k_gemm_fp8(*a, *w), ref, size, k, "bf16", cut)
    fast = B.k_gemm_fp8(*a, *w, c_fp32=True, fast_sums=True)
    close(fast, ref, size, k, "fp32, fast sums", cut)
    assert torch.equal(fast.to(BF16), B.k_gemm_fp8(*a, *w))
    close(B.k_gemm_fp8(*a, *w, c_fp32=True), ref, size, k, "fp32")
    res32, res16 = normal(f"r{m}{n}", (m, n), 1.0, F32), normal(f"r{m}{n}", (m, n), 1.0)
    c = B.k_gemm_fp8(*a, *w, residual=res32)
    assert c.dtype == F32
    close(c, ref + res32.double(), size, k, "fp32 onto fp32", 2 * U * (ref.abs() + res32.double().abs()))
    close(B.k_gemm_fp8(*a, *w, residual=res16), ref + res16.double(), size, k, "bf16 onto bf16", cut + 2 * U * (ref.abs() + res16.double().abs()))
    into = res32.clone()
    assert B.k_gemm_fp8(*a, *w, residual=into, c=into) is into and torch.equal(into, c)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(20, 100, 272), (90, 100, 272), (300, 270, 688)])
def test_strided_operands_and_untouched_neighbours(m, n, k):
    a, w = operands(m, n, k)
    wide = lambda t, rows, cols, fill: torch.full((rows, cols), fill, dtype=torch.uint8, device="cuda")
    A, W = wide(a[0], m, k + 32, 0x7F), wide(w[0], n, k + 48, 0x7F)          # NaN codes behind the rows
    A[:, :k], W[:, :k] = a[0].view(torch.uint8), w[0].view(torch.uint8)
    SA, SW = wide(a[1], m, a[1].shape[1] + 4, 255), wide(w[1], w[1].shape[0], w[1].shape[1] + 8, 255)
    kb = -(-k // 128)
    SA[:, :kb], SW[:, :kb] = a[1][:, :kb], w[1][:, :kb]                       # NaN scales behind theirs
    want = B.k_gemm_fp8(*a, *w)
    C = torch.full((m + 1, n + 9), 3.0, dtype=BF16, device="cuda")
    words = a[1].shape[1]
    B.k_gemm_fp8(A[:, :k].view(E4M3), SA[:, :words], W[:, :k].view(E4M3), SW[:, :words], c=C[:m, 1:n + 1])
    assert torch.equal(C[:m, 1:n + 1], want)
    assert bool((C[m] == 3).all()) and bool((C[:, 0] == 3).all()) and bool((C[:, n + 1:] == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("m", [40, 300])
def test_nan_and_infinite_rows_stay_apart(m):
    a = normal("na", (m, 256), 1.0, F32)
    a[3, 7], a[m - 1, 200] = float("nan"), float("inf")
    qa, qw = B.k_fp8_quantize(a), B.k_fp8_quantize(normal("nw", (200, 256), 0.05), 128)
    c = B.k_gemm_fp8(*qa, *qw)
    assert bool(c[3].isnan().all()) and bool(c[m - 1].isnan().all()) and int(c.isnan().sum()) == 400


@pytest.mark.gpu
def test_rows_do_not_depend_on_the_batch():
    """Above 64 rows every tile adds up K in the same order."""
    a, w = operands(2100, 1536, 1040)
    for f32 in (False, True):
        full = B.k_gemm_fp8(*a, *w, c_fp32=f32)
        for m in (65, 130, 300, 700, 1500):
            assert torch.equal(B.k_gemm_fp8(a[0][:m], a[1][:m], *w, c_fp32=f32), full[:m]), m


@pytest.mark.gpu
@pytest.mark.parametrize("m,f,k", [(1, 16, 128), (5, 688, 256), (64, 5504, 512), (65, 128, 144), (200, 688, 256), (300, 256, 2048), (777, 1280, 272),
                                   (130, 384, 14000)])
def test_gate_up_swiglu(m, f, k):
    a, w = operands(m, 2 * f, k)
    ref, size = product(a, w)
    g, u = ref.cpu().chunk(2, 1)
    q, s = B.k_gemm_fp8_swiglu(*a, *w)
    assert q.shape == (m, f) and s.shape == (m, (f + 511) // 512 * 4)
    # Gate and up are off by at most eg and eu, silu's slope is at most 1.1, silu(g) at most |g|, and a code moves by (1 + 2^-3) of it.  How many codes move:
    # normal sums are off by 1.5e-5 of their deviation, so a sum of t deviations by 1.5e-5 / t of itself; a step is 2^-3.5 of a value in
    # the mean, so 1.7e-4 / t of the codes cross a tie; over the density 0.8 of small t that is 0.8 * 1.7e-4 * ln(1 / 1.7e-4) = 1.2e-3, for gate and up each
    eg, eu = (cut_off(a, w) + (k / 8 + k / 128 + 16) * 2 * U * size).cpu().chunk(2, 1)
    near_codes(q, s, g / (1 + torch.exp(-g)) * u, 1e-2, 1.125 * (1.1 * (u.abs() + eu) * eg + g.abs() * eu))
    gu = B.k_gemm_fp8(*a, *w, c_fp32=True, fast_sums=True)                    # the same numbers in two calls
    q2, s2 = B.k_swiglu_fp8(gu)
    assert torch.equal(s, s2) and torch.equal(q.view(torch.uint8), q2.view(torch.uint8))


@pytest.mark.gpu
def test_feed_forward_block_in_8_bits():
    """norm, gate and up, SwiGLU, down onto the residual, as a teacher layer runs them."""
    for m in (1, 50, 700):
        d, f = 512, 1408
        x, g = normal(f"fx{m}", (m, d), 1.0, F32), (1 + normal("fg", (d,), 0.1, F32)).to(BF16)
        up, down = B.k_fp8_quantize(normal("fu", (2 * f, d), 0.05), 128), B.k_fp8_quantize(normal("fd", (d, f), 0.05), 128)
        h = B.k_norm_fp8(x, g, 1e-6)
        act = B.k_gemm_fp8_swiglu(*h, *up)
        y = B.k_gemm_fp8(*act, *down, residual=x)
        gate, u = product(h, up)[0].chunk(2, 1)
        a64 = gate / (1 + torch.exp(-gate)) * u
        ref, size = product(act, down)
        close(y, ref + x.double(), size, f, "down", 2 * U * (ref.abs() + x.double().abs()))
        # the block as a whole: codes are off by 2^-4 at most each, independently: sums of f of them by 2^-4 of their root
        whole = a64 @ values(*down, 128).cuda().t()
        assert float((ref - whole).norm() / whole.norm()) < 2.0 ** -4


@pytest.mark.gpu
def test_replayed_graph_and_other_stream():
    a, w = operands(300, 512, 688)
    x = normal("gx", (300, 688))

    def block():
        return B.k_gemm_fp8(*B.k_fp8_quantize(x), *w), *B.k_gemm_fp8_swiglu(a[0][:40], a[1][:40], *w)
    want = block()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = block()
    torch.cuda.current_stream().wait_stream(side)
    same = lambda p, q: all(torch.equal(i.view(torch.uint8), j.view(torch.uint8)) for i, j in zip(p, q))
    assert same(want, got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = block()
    for _ in range(3):
        for t in out:
            t.view(torch.uint8).zero_()
        block()
        g.replay()
        torch.cuda.synchronize()
        assert same(want, out)


@pytest.mark.gpu
def test_empty_batch():
    _, w = operands(4, 64, 128)
    q, s = B.k_fp8_quantize(torch.zeros((0, 128), dtype=BF16, device="cuda"))
    assert q.shape == (0, 128) and B.k_gemm_fp8(q, s, *w).shape == (0, 64) and B.k_gemm_fp8_swiglu(q, s, *w)[0].shape == (0, 32)


def test_refusals_before_anything_is_launched():
    f = B._fn

    def quant(dtype=1, rows=1, n=4, k=128, x=256, ldx=128, q=512, ldq=128, s=256, lds=4):
        return f("ms_k_fp8_quantize")(dtype, rows, n, k, x, ldx, q, ldq, s, lds, None)

    def gemm(m=4, n=64, k=128, a=256, lda=128, sa=256, ldsa=4, w=256, ldw=128, sw=256, ldsw=4, c=256, ldc=64, r=None, ldr=0):
        return f("ms_k_gemm_fp8")(m, n, k, a, lda, sa, ldsa, w, ldw, sw, ldsw, c, ldc, 0, r, ldr, 0, None)

    def swiglu(m=4, F=64, k=128, a=256, ldsa=4, q=256, ldq=64, s=256, lds=4, sc=256, nb=1 << 20):
        return f("ms_k_gemm_fp8_swiglu")(m, F, k, a, 128, 256, ldsa, 256, 128, 256, 4, q, ldq, s, lds, sc, nb, None)
    assert quant(n=0) == 0 and gemm(m=0) == 0 and swiglu(m=0) == 0
    for call, bad in ((quant, dict(x=None)), (quant, dict(q=None)), (quant, dict(s=None)), (quant, dict(dtype=5)), (quant, dict(rows=64)),
                      (quant, dict(n=-1)), (quant, dict(k=0)), (gemm, dict(a=None)), (gemm, dict(sw=None)), (gemm, dict(c=None)), (gemm, dict(n=0)),
                      (gemm, dict(m=-1)), (swiglu, dict(q=None)), (swiglu, dict(F=0)), (swiglu, dict(F=1 << 30))):
        assert call(**bad) == -1, bad
    for call, bad in ((quant, dict(ldx=120)), (quant, dict(ldq=112)), (quant, dict(k=144, ldx=144, ldq=144, lds=0)), (gemm, dict(lda=112)), (gemm, dict(ldsa=0)),
                      (gemm, dict(k=528, lda=528, ldw=528)), (gemm, dict(ldc=63)), (gemm, dict(r=256, ldr=60)), (swiglu, dict(ldq=48)), (swiglu, dict(lds=0))):
        assert call(**bad) == -2, bad
    for call, bad in ((quant, dict(k=120)), (quant, dict(x=264)), (quant, dict(ldx=132)), (quant, dict(s=258)), (quant, dict(lds=6)), (gemm, dict(k=120)),
                      (gemm, dict(a=264)), (gemm, dict(lda=136)), (gemm, dict(ldw=1 << 25)), (gemm, dict(c=257)), (swiglu, dict(F=72, ldq=80)), (swiglu, dict(q=264))):
        assert call(**bad) == -4, bad
    assert swiglu(nb=100) == -3 and swiglu(sc=None) == -3 and b"scratch" in B.lib().ms_last_error()
    assert B.lib().ms_k_gemm_fp8_config(77) == -1 and B.lib().ms_k_gemm_fp8_config(0) == 0
    n = f("ms_k_norm_fp8")
    assert n(1, 0, 4, 128, float("nan"), 256, 256, 256, 128, 256, 4, None) == -1 and n(1, 0, 4, 128, 1e-6, 256, None, 256, 128, 256, 4, None) == -1
    assert n(1, 0, 4, 136, 1e-6, 256, 256, 256, 144, 256, 4, None) == -4 and n(1, 1, 4, 128, 1e-6, 256, 258, 256, 128, 256, 4, None) == -4
    assert f("ms_k_swiglu_fp8")(1, 4, 128, 256, 128, 256, 128, 256, 4, None) == -2


def test_a_residual_that_overlaps_the_result_is_refused():
    lib = B.lib()
    v, M, N, K = C.c_void_p, 8, 32, 128

    def call(c, ldc, c_fp32, r, ldr, r_fp32):
        return lib.ms_k_gemm_fp8(M, N, K, v(16), C.c_int64(K), v(16), C.c_int64(4), v(16), C.c_int64(K), v(16), C.c_int64(4), v(c), C.c_int64(ldc),
                                 c_fp32, v(r), C.c_int64(ldr), r_fp32, None)
    base = 1 << 20
    assert call(base, 64, 0, base + 2, 64, 0) == -1                         # one element on
    assert call(base, 64, 0, base + 128, 64, 0) == -1                       # one row on
    assert call(base, 64, 0, base, 96, 0) == -1                             # the same start, other rows
    assert call(base, 64, 1, base, 64, 0) == -1 and call(base, 64, 0, base, 32, 1) == -1          # the same start, another type
    assert call(base, 48, 0, base + 64, 48, 0) == -1                        # side by side in rows that hold one and a half


@pytest.mark.gpu
def test_residual_beside_the_result():
    a, sa = B.k_fp8_quantize(torch.randn(70, 128, device="cuda"))
    w, sw = B.k_fp8_quantize(torch.randn(32, 128, device="cuda"), 128)
    both = torch.randn(70, 64, device="cuda").to(torch.bfloat16)
    r = both[:, 32:]
    ref = B.k_gemm_fp8(a, sa, w, sw, residual=r.clone())
    B.k_gemm_fp8(a, sa, w, sw, residual=r, c=both[:, :32])
    assert torch.equal(both[:, :32], ref)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [s for s in SHAPES if s[0] > 1] + [(70, 191, 256), (70, 193, 256), (300, 448, 1152), (520, 1345, 384)])
def test_tile_of_192_outputs_gives_the_same_bits(m, n, k, fp8_tile):
    """Its wave columns begin and end inside the weights' scale blocks."""
    a, w = operands(m, n, k)
    res = normal(f"r{m}{n}", (m, n), 1.0)
    calls = [lambda: B.k_gemm_fp8(*a, *w), lambda: B.k_gemm_fp8(*a, *w, residual=res), lambda: B.k_gemm_fp8(*a, *w, residual=res, c_fp32=True, fast_sums=True)]
    fp8_tile(128128)
    want = [f() for f in calls]
    fp8_tile(256192)
    assert all(torch.equal(f(), x) for f, x in zip(calls, want))


@pytest.mark.gpu
def test_gate_up_weights_with_rows_far_apart():
    """2 f rows that one buffer descriptor does not reach: the scratch that the sizes ask for is enough."""
    f, k, ld = 1024, 256, (1 << 21) + (1 << 16)
    a, w = operands(300, 2 * f, k)
    far = torch.empty(2 * f * ld, dtype=torch.uint8, device="cuda").view(2 * f, ld)[:, :k].view(E4M3)
    far.copy_(w[0])
    for m in (1, 40, 64, 65, 300):
        x = a[0][:m], a[1][:m]
        want, got = B.k_gemm_fp8_swiglu(*x, *w), B.k_gemm_fp8_swiglu(*x, far, w[1])
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(want, got)), m


def test_scratch_of_the_sizes_is_enough_for_any_row_stride():
    f = B._fn
    need = f("ms_k_gemm_fp8_swiglu_scratch_bytes")(300, 1024, 256)

    def call(m, ldw, nb):                                                    # (nothing is there to launch on: what the host checks turn down is -3)
        return f("ms_k_gemm_fp8_swiglu")(m, 1024, 256, 256, 256, 256, 4, 256, ldw, 256, 4, 256, 1024, 256, 8, 256, nb, None)
    assert call(300, (1 << 21) + (1 << 16), need - 256) == -3 and call(40, 256, 40 * 8192 - 1) == -3
    assert need == 64 * 8192
    if not torch.cuda.is_available():
        assert call(300, (1 << 21) + (1 << 16), need) != -3


def test_gate_up_of_an_odd_number_of_columns_is_refused():
    """Rows of 48 numbers of which a view shows 33: 16 gates, 16 ups and one that would be left out."""
    with pytest.raises(ValueError, match="gate_up: expected shape"):
        B.k_swiglu_fp8(torch.zeros((3, 48), dtype=BF16)[:, :33])
    with pytest.raises(ValueError, match="on a GPU"):
        B.k_swiglu_fp8(torch.zeros((3, 48), dtype=BF16)[:, :32])


def some_codes(n, k, tag):
    """Codes of every kind but NaN."""
    c = (wl.uniform(13, tag, n * k) * 256).to(torch.uint8).view(n, k)
    return torch.where((c & 127) == 127, torch.full_like(c, 0x38), c).view(E4M3).cuda()


# bytes of both operands; where their product leaves fp32's normal numbers there is nothing to compare
@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(5, 48, 128), (100, 48, 144), (300, 256, 384)])
@pytest.mark.parametrize("ea,ew", [(0, 127), (127, 0), (1, 130), (2, 140), (3, 127), (127, 3), (3, 240), (240, 3), (246, 3), (3, 246), (0, 246), (246, 0), (100, 10),
                                   (246, 90), (90, 246)])
def test_scales_at_the_ends_of_their_range(ea, ew, m, n, k):
    sc = lambda rows, b: torch.full((rows, (k + 511) // 512 * 4), b, dtype=torch.uint8, device="cuda")
    a, w = (some_codes(m, k, f"sa{m}{k}"), sc(m, ea)), (some_codes(n, k, f"sw{n}{k}"), sc((n + 127) // 128, ew))
    ref, size = product(a, w)
    one = 2.0 ** (127 - ea), 2.0 ** (127 - ew)                               # to the codes' own values, in which cut_off computes in fp32
    cut = cut_off((a[0], sc(m, 127)), (w[0], sc(w[1].shape[0], 127))) / one[0] / one[1]
    close(B.k_gemm_fp8(*a, *w, c_fp32=True, fast_sums=True), ref, size, k, "fast sums", cut)
    # below 2^-124 a code times its scale is off by up to 2^-134, times the other operand's row
    rounded = (2.0 ** -134 * (ea < 3) * values(*w, 128).cuda().abs().sum(1)[None] + 2.0 ** -134 * (ew < 3) * values(*a, 1).cuda().abs().sum(1)[:, None])
    close(B.k_gemm_fp8(*a, *w, c_fp32=True), ref, size, k, "fp32 sums", rounded)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [6, 90])
def test_products_of_the_smallest_and_largest_numbers(m):
    """As the quantisers lay them out: bytes 0 .. 247."""
    x = normal(f"ends{m}", (m, 256), 1.0, F32).clamp(-3, 3)
    x[:, :128] *= torch.exp2(torch.arange(m, device="cuda") % 6 * 49.8 - 124.0)[:, None]
    x[1, 5] = 3.2e38                                                         # byte 247
    x[2, 7] = 2.0 ** -149
    w = normal("endw", (40, 256), 2.0 ** -12, F32)
    qa, qw = B.k_fp8_quantize(x), B.k_fp8_quantize(w, 128)
    assert int(qa[1][1, 0]) == 247 and int(qa[1].min()) <= 5
    ref, size = product(qa, qw)
    cut = 7 * 2.0 ** -13 * size
    close(B.k_gemm_fp8(*qa, *qw, c_fp32=True, fast_sums=True), ref, size, 256, "fast sums", cut)
    close(B.k_gemm_fp8(*qa, *qw, c_fp32=True), ref, size, 256, "fp32 sums", 2.0 ** -134 * values(*qw, 128).cuda().abs().sum(1)[None])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (17, 129, 1024), (100, 333, 688), (300, 2048, 4112), (2049, 144, 272), (777, 1280, 384)])
def test_bf16_results_from_fp32_sums(m, n, k):
    a, w = operands(m, n, k)
    ref, size = product(a, w)
    got = B.k_gemm_fp8(*a, *w, fp32_sums=True)
    close(got, ref, size, k, "bf16 from fp32 sums")                          # without what the 8-bit sums cut off
    assert got.dtype == BF16 and torch.equal(got, B.k_gemm_fp8(*a, *w, c_fp32=True).to(BF16))
    res = normal(f"r{m}{n}", (m, n), 1.0)
    assert torch.equal(B.k_gemm_fp8(*a, *w, residual=res, fp32_sums=True), B.k_gemm_fp8(*a, *w, residual=res, c_fp32=True).to(BF16))
    if n % 32 == 0:
        q, s = B.k_gemm_fp8_swiglu(*a, *w, fp32_sums=True)
        g, u = ref.cpu().chunk(2, 1)
        # fp32 sums move a value over a tie as seldom as other fp32 computing: their error of (k / 8 + ...) half steps at most reaches the codes as in
        # test_gate_up_swiglu
        eg, eu = ((k / 8 + k / 128 + 16) * 2 * U * size).cpu().chunk(2, 1)
        near_codes(q, s, g / (1 + torch.exp(-g)) * u, 1e-2, 1.125 * (1.1 * (u.abs() + eu) * eg + g.abs() * eu))


def test_one_kind_of_sums_is_asked_for():
    with pytest.raises(ValueError, match="exclude"):
        B.k_gemm_fp8(None, None, None, None, fast_sums=True, fp32_sums=True)
    with pytest.raises(ValueError, match="fp8"):
        B.SectionOptions(fp32_sums=True)
    f = B._fn("ms_k_gemm_fp8")
    call = lambda kind, ldc=64, c=256: f(4, 64, 128, 256, 128, 256, 4, 256, 128, 256, 4, c, ldc, kind, None, 0, 0, None)
    assert call(4) == -1 and call(-1) == -1 and call(3, 63) == -2
    assert call(3, c=257) == -4 and call(1, c=258) == -4                     # 3 is a bf16 result


def test_the_kernel_for_few_rows_can_be_asked_for(fp8_tile):
    """With any number of rows that one launch takes; more are refused."""
    fp8_tile(16016)
    f = B._fn("ms_k_gemm_fp8")
    assert f(65535 * 16 + 1, 64, 128, 256, 128, 256, 4, 256, 128, 256, 4, 1 << 30, 64, 0, None, 0, 0, None) == -4
    assert b"too large for one launch" in B.lib().ms_last_error()


@pytest.mark.gpu
def test_the_kernel_for_few_rows_with_many(fp8_tile):
    a, w = operands(700, 100, 688)
    ref, size = product(a, w)
    fp8_tile(16016)
    close(B.k_gemm_fp8(*a, *w), ref, size, 688, "bf16", cut_off(a, w))
    close(B.k_gemm_fp8(*a, *w, c_fp32=True), ref, size, 688, "fp32")
    a, w = operands(100, 256, 272)
    got = B.k_gemm_fp8_swiglu(*a, *w)
    fp8_tile(64128)
    assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(got, B.k_gemm_fp8_swiglu(*a, *w)))
