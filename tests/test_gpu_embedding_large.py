"""The table's gradient for large batches: pieces of 32 places, dx read with and without the non-temporal policy.  dx holds small integers, so that the
sums are exact in any order.  tests/test_embedding_plan.py checks that the cases take these kernels."""
import pytest
import torch

from paper_2605_10501_amd import binding as B
from test_gpu_embedding_sorted import ids_of

F32, F64 = torch.float32, torch.float64
# tokens (no multiple of 32 but one), columns, vocabulary, ids, type, places of a piece, non-temporal
CASES = [(32771, 1536, 151, kind, "bf16", 32, True) for kind in ("one", "runs", "few", "text", "outside", "none")] + [
    (33001, 768, 151, kind, "fp32", 32, True) for kind in ("one", "few", "text", "outside")] + [
    (22013, 1600, vocab, kind, "bf16", 32, False) for vocab, kind in ((3, "one"), (40000, "text"), (700, "runs"), (40000, "back"), (151, "outside"))] + [
    (22013, 800, vocab, kind, "fp32", 32, False) for vocab, kind in ((3, "few"), (40000, "even"), (700, "runs"))] + [
    (33056, 2056, 1033, "runs", "bf16", 32, True), (17001, 4096, 517, "text", "fp32", 32, True), (140_003, 264, 400, "text", "bf16", 32, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,vocab,kind,dtype,tile,stream", CASES)
def test_gradient(n, d, vocab, kind, dtype, tile, stream):
    t = torch.bfloat16 if dtype == "bf16" else F32
    ids = ids_of(kind, n, vocab).cuda()
    row, col = torch.arange(n, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    dx = ((row * 31 + col * 7 + row // 32) % 7 - 3).to(t)
    start = ((torch.arange(vocab, device="cuda")[:, None] + col) % 5).to(F32)
    got = start.clone()
    B.k_embedding_sorted_backward(ids, dx, 2.0, got)
    # |sums| <= 6 * 140003 + 4 < 2^24: exact in fp32
    want, keep = start.to(F64), (ids >= 0) & (ids < vocab)
    want.index_add_(0, ids[keep].long(), 2.0 * dx[keep].to(F64))
    assert torch.equal(got.to(F64), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
def test_gradient_of_normal_values_repeats(dtype):
    n, d, vocab = 32771, 1536 if dtype == torch.bfloat16 else 768, 500
    ids = ids_of("text", n, vocab).cuda()
    dx = torch.randn((n, d), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(dtype)
    runs = [B.k_embedding_sorted_backward(ids, dx, 1.7, torch.zeros((vocab, d), device="cuda")) for _ in range(3)]
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])
    want, size = (torch.zeros((vocab, d), dtype=F64, device="cuda").index_add_(0, ids.long(), 1.7 * v) for v in (dx.to(F64), dx.to(F64).abs()))
    # 32 terms of a piece, every fourth piece in eights, four sums and a product: at most (pieces / 4 + 48) half steps of the absolute sum
    assert bool(((runs[0].to(F64) - want).abs() <= (n / 32 / 4 + 48) * 2.0 ** -24 * size * 1.01).all())
