"""Scaled embedding rows and the table's gradient by sorted tokens, against sums in 64 bits."""
import pytest
import torch

from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import workloads as wl

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = 2.0 ** -24


def ids_of(kind, n, vocab):
    t = torch.arange(n)
    u = wl.uniform(11, f"ids{kind}{n}", n).double()
    return {"even": (u * vocab).long(), "one": torch.full((n,), vocab - 1), "few": (u * 3).long() % vocab,
            "text": torch.exp(u * torch.log(torch.tensor(float(vocab)))).long() - 1,
            "outside": torch.where(t % 3 == 0, torch.tensor(-7), torch.where(t % 3 == 1, torch.tensor(vocab), (u * vocab).long())),
            "none": torch.full((n,), -1), "runs": (t // 32) % vocab, "back": (vocab - 1 - t) % vocab}[kind].to(torch.int32)


def reference(ids, dx, scale, vocab):
    ids, dx = ids.cpu().long(), dx.cpu().double()
    keep = (ids >= 0) & (ids < vocab)
    ref, size = torch.zeros((vocab, dx.shape[1]), dtype=F64), torch.zeros((vocab, dx.shape[1]), dtype=F64)
    ref.index_add_(0, ids[keep], scale * dx[keep])
    size.index_add_(0, ids[keep], abs(scale) * dx[keep].abs())
    return ref, size


CASES = [(1, 8, 1, "one"), (1, 128, 1024, "even"), (2, 64, 7, "one"), (31, 40, 5, "few"), (32, 16, 3, "runs"), (33, 16, 3, "one"),
         (64, 16, 2, "runs"), (293, 128, 1024, "outside"), (500, 24, 511, "none"), (1024, 136, 512, "text"), (1025, 136, 513, "text"),
         (4099, 64, 32000, "text"), (5000, 32, 300000, "back"), (3001, 2056, 90, "even"), (2048, 128, 151936, "runs")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,vocab,kind", CASES)
def test_gradient(n, d, vocab, kind, dtype):
    ids = ids_of(kind, n, vocab).cuda()
    dx = wl.normal(2, f"dx{n}.{d}", (n, d), 1.0, 0.0, dtype, "cuda")
    start = wl.normal(2, f"t{d}", (vocab, d), 1.0, 0.0, F32, "cuda")
    got, scale = start.clone(), 11.3
    assert B.k_embedding_sorted_backward(ids, dx, scale, got) is got
    ref, size = reference(ids, dx, scale, vocab)
    # 32 terms of a piece, every eighth piece and eight sums, one product: a sum of m terms is off by at most (m / 8 + 48) half steps of
    # the terms' absolute sum; then one addition to what was there
    bound = (n / 8 / 32 + 48) * U * size + U * (ref + start.cpu().double()).abs() * 1.01
    off = (got.cpu().double() - (ref + start.cpu().double())).abs()
    assert bool((off <= bound).all()), float((off - bound).max())
    untouched = torch.ones(vocab, dtype=torch.bool)
    untouched[ids.cpu().long()[(ids.cpu() >= 0) & (ids.cpu() < vocab)]] = False
    assert torch.equal(got.cpu()[untouched], start.cpu()[untouched])
    again = start.clone()
    B.k_embedding_sorted_backward(ids, dx, scale, again)
    assert torch.equal(again, got)


@pytest.mark.gpu
@pytest.mark.parametrize("n,ids_kind", [(140_000, "text"), (600_000, "few"), (200_003, "outside")])
def test_gradient_of_long_batches(n, ids_kind):
    """Several workgroups of the sort with one, four and sixteen tokens a thread; integers, so that the sums are exact."""
    vocab, d = 40_000, 8
    ids = ids_of(ids_kind, n, vocab).cuda()
    dx = (torch.arange(n * d, device="cuda") % 7 - 3).view(n, d).to(BF16)
    got = torch.zeros((vocab, d), device="cuda")
    B.k_embedding_sorted_backward(ids, dx, 1.0, got)
    assert torch.equal(got.cpu().double(), reference(ids, dx, 1.0, vocab)[0])


@pytest.mark.gpu
def test_tables_past_32_bit_offsets():
    vocab, d = 70_000, 16_384                                     # 2^30.1 elements of fp32: 4.6 GB
    got = torch.zeros((vocab, d), device="cuda")
    ids = torch.tensor([vocab - 1, 3, vocab - 1, vocab], dtype=torch.int32, device="cuda")
    dx = torch.ones((4, d), dtype=BF16, device="cuda")
    B.k_embedding_sorted_backward(ids, dx, 0.5, got)
    assert bool((got[vocab - 1] == 1.0).all()) and bool((got[3] == 0.5).all()) and float(got.sum(dtype=F64)) == 1.5 * d
    x = B.k_embedding_scaled_forward(ids, got, 2.0)
    assert bool((x[0] == 2).all()) and bool((x[1] == 1).all()) and bool((x[3] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,vocab", [(1, 8, 1), (293, 128, 1024), (1025, 1536, 77), (7, 5000, 19)])
def test_forward(n, d, vocab):
    ids = ids_of("outside", n, vocab).cuda()
    for dtype in (BF16, F32):
        table = wl.normal(2, f"tab{vocab}{d}", (vocab, d), 0.02, 0.0, dtype, "cuda")
        for scale in (1.0, 39.19):
            s32 = torch.tensor(scale, dtype=F32).double()
            at = ids.cpu().long()
            ref = torch.zeros((n, d), dtype=F64)
            keep = (at >= 0) & (at < vocab)
            ref[keep] = s32 * table.cpu().double()[at[keep]]
            # the fp32 product of two fp32 (or a bf16 and an fp32) numbers rounds once, the store once
            assert torch.equal(B.k_embedding_scaled_forward(ids, table, scale).cpu(), ref.to(F32).to(dtype))
            if dtype == BF16:
                assert torch.equal(B.k_embedding_scaled_forward(ids, table, scale, out_fp32=True).cpu(), ref.to(F32))


@pytest.mark.gpu
def test_non_finite_gradients_stay_in_their_rows():
    ids = torch.tensor([4, 1, 4, -1, 2], dtype=torch.int32, device="cuda")
    dx = torch.ones((5, 16), dtype=BF16, device="cuda")
    dx[1, 3], dx[3] = float("inf"), float("nan")                   # the second belongs to no row
    got = B.k_embedding_sorted_backward(ids, dx, 1.0, torch.zeros((6, 16), device="cuda"))
    assert float(got[1, 3]) == float("inf") and int((~got.isfinite()).sum()) == 1


@pytest.mark.gpu
def test_replayed_graphs_do_not_share_scratch():
    vocab, d = 5000, 64
    made = []
    for k, n in enumerate((3000, 1500)):
        ids, dx = ids_of("text", n, vocab).cuda(), wl.normal(k, "g", (n, d), 1.0, 0.0, BF16, "cuda")
        made.append((ids, dx, B.k_embedding_sorted_backward(ids, dx, 2.0, torch.zeros((vocab, d), device="cuda")), torch.zeros((vocab, d), device="cuda")))
    graphs = []
    for ids, dx, _, out in made:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out.zero_()
            B.k_embedding_sorted_backward(ids, dx, 2.0, out)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, _, want, out in made:
            assert torch.equal(want, out)
            out.fill_(9.0)


@pytest.mark.gpu
def test_empty_batch():
    table = torch.ones((4, 8), device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert B.k_embedding_scaled_forward(none, table, 2.0).shape == (0, 8)
    assert bool((B.k_embedding_sorted_backward(none, torch.zeros((0, 8), device="cuda"), 2.0, table) == 1).all())


def test_refusals_before_anything_is_launched():
    need = B._fn("ms_k_embedding_sorted_backward_scratch_bytes")(100, 64, 50)
    assert need > 0 and B._fn("ms_k_embedding_sorted_backward_scratch_bytes")(1 << 25, 64, 50) == 0

    def bwd(dtype=1, n=100, d=64, vocab=50, ids=256, dx=256, dt=256, sc=256, nb=need):
        return B._fn("ms_k_embedding_sorted_backward")(dtype, n, d, vocab, 1.0, ids, dx, dt, sc, nb, None)

    def fwd(dtype=1, f32=0, n=100, d=64, vocab=50, ids=256, tab=256, x=256):
        return B._fn("ms_k_embedding_scaled_forward")(dtype, f32, n, d, vocab, 1.0, ids, tab, x, None)
    assert bwd(n=0) == 0 and fwd(n=0) == 0
    for bad in (dict(ids=None), dict(dx=None), dict(dt=None), dict(sc=None), dict(dtype=7), dict(n=-1), dict(d=0), dict(vocab=0)):
        assert bwd(**bad) == -1, bad
    assert bwd(nb=need - 1) == -3 and b"scratch" in B.lib().ms_last_error()
    for bad in (dict(d=60), dict(dx=264), dict(dt=260), dict(n=(1 << 24) + 1)):
        assert bwd(**bad) == -4, bad
    for bad in (dict(ids=None), dict(tab=None), dict(x=None), dict(dtype=-1), dict(vocab=-3)):
        assert fwd(**bad) == -1, bad
    assert fwd(d=12) == -4 and fwd(tab=264) == -4
