"""The balance loss, the counts and the gradient against 64 bits and differences.

Errors: a probability is within 4 2^-22 of itself (two roundings of an exponential of 2 ulp, the sum of at most 1024 of them in a tree
of depth 10 and lanes of 32, a division and a product); the loss a weighted sum of them in fp32 per block: 2^-17 covers a thousand tokens to a
block.  The gradient is g p (slope - dot) whose bracket is relative to the largest slope."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def run(logits, ids, mask, grad=0.5):
    T, E = logits.shape
    loss, slope = torch.full((1,), -7.0, device="cuda"), torch.empty(E, device="cuda")
    counts = torch.full((E,), -7, dtype=torch.int32, device="cuda")
    ws = torch.empty(sgdb.sgdb_balance_loss_workspace_bytes(T, E), dtype=torch.uint8, device="cuda").fill_(255)
    sgdb.sgdb_balance_loss(logits, ids, mask, loss, counts, slope, ws)
    dlogits = torch.full_like(logits, 55.0)
    sgdb.sgdb_balance_loss_backward(torch.full((1,), grad, device="cuda"), logits, mask, slope, dlogits)
    return loss, counts, dlogits


def reference(logits, ids, mask):
    """Loss as a function of the logits in 64 bits (for autograd), counts."""
    T, E = logits.shape
    kept = torch.ones(T, dtype=torch.bool, device="cuda") if mask is None else mask != 0
    n, k = int(kept.sum()), ids.size(1)
    chosen = ids[kept].reshape(-1).long()
    counts = torch.bincount(chosen[(chosen >= 0) & (chosen < E)], minlength=E)
    if n == 0:
        return torch.nan_to_num(logits.double()).mul(0.0).sum(), counts
    x = logits[kept]
    p = torch.where(torch.isneginf(x).all(1, keepdim=True), 0.0, torch.softmax(torch.where(torch.isneginf(x).all(1, keepdim=True), 0.0, x), 1))
    return E * ((counts.double() / (n * k)) * (p.sum(0) / n)).sum(), counts


SIZES = [(1, 1, 1), (1, 8, 2), (3, 9, 4), (33, 2, 1), (64, 64, 8), (1000, 7, 3), (257, 130, 5), (100, 1024, 8), (77, 1000, 32), (5000, 33, 2), (20000, 256, 4),
         (40, 300, 6), (513, 16, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_against_64_bits(cuda_device, T, E, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(T + E)
    for pad, masked in ((0, False), (1, True), (8, True)):
        logits = (2.0 * torch.randn(T, E + pad, device="cuda", generator=gen)).to(dtype)[:, :E]
        ids = torch.randint(-2, E + 2, (T, k), device="cuda", generator=gen).int()
        mask = (torch.rand(T, device="cuda", generator=gen) < 0.7).to(torch.uint8) * 3 if masked else None
        if E > 1 and T > 2:
            logits[1, : E // 2] = float("-inf")  # experts that a token may not have
            logits[2] = float("-inf")            # a token without any
        if masked:
            logits[mask == 0] = float("nan")     # padding is not looked at
            ids[mask == 0] = 2 ** 30
        loss, counts, d = run(logits, ids, mask)
        x = logits.double().requires_grad_()
        want, want_counts = reference(x, ids, mask)
        (grad,) = torch.autograd.grad(0.5 * want, x)
        assert torch.equal(counts.long(), want_counts)
        assert abs(float(loss) - float(want.detach())) <= 2.0 ** -17 * abs(float(want.detach()))
        grad = torch.where(torch.isfinite(logits), grad, 0.0)
        if masked:
            grad[mask == 0] = 0.0
        n = max(1, T if mask is None else int((mask != 0).sum()))
        slopes = E * (want_counts.double() - want_counts.double().mean()).abs().max() / (n * n * k)
        p = torch.softmax(torch.where(torch.isfinite(logits), logits.double(), -1e9), 1)
        bound = 0.5 * p * slopes * 2.0 ** -17 + ROUNDING[dtype] * grad.abs() + 2.0 ** -130
        assert bool(((d.double() - grad).abs() <= bound).all())


def test_against_differences(cuda_device):
    T, E, k = 30, 12, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    logits = torch.randn(T, E, device="cuda", generator=gen)
    ids = torch.randint(0, 4, (T, k), device="cuda", generator=gen).int()  # far from balanced
    _, _, d = run(logits, ids, None, 1.0)
    x = logits.double()
    for t, e in ((0, 0), (7, 3), (29, 11), (15, 5)):
        h = torch.zeros_like(x)
        h[t, e] = 1e-4
        want = (reference(x + h, ids, None)[0] - reference(x - h, ids, None)[0]) / 2e-4
        assert abs(float(d[t, e]) - float(want)) <= 1e-5 * float(d.abs().max())  # 1e-8 of the third derivative, 1e-12 of the difference


def test_nothing_counts_and_bad_numbers(cuda_device):
    logits, ids = torch.randn(9, 5, device="cuda"), torch.zeros(9, 1, dtype=torch.int32, device="cuda")
    loss, counts, d = run(logits, ids, torch.zeros(9, dtype=torch.uint8, device="cuda"))
    assert float(loss) == 0.0 and not bool(counts.any()) and not bool(d.any())
    loss, counts, d = run(logits[:0], ids[:0], None)
    assert float(loss) == 0.0 and not bool(counts.any())
    for bad in (float("nan"), float("inf")):
        x = logits.clone()
        x[4, 2] = bad
        loss, counts, d = run(x, ids, None)
        assert bool(loss.isnan()) and counts.tolist() == [9, 0, 0, 0, 0]
        assert bool(d[4].isnan().all()) and bool(torch.isfinite(d[[0, 1, 2, 3, 5, 6, 7, 8]]).all())


def test_alike_counts_keep_their_digits(cuda_device):
    """999 pairs to one expert, 1001 to another: the gradient's slopes are 1e-3 of the counts, and as exact as any."""
    T, E = 2000, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(T, E, device="cuda", generator=gen)
    ids = (torch.arange(T, device="cuda") >= 999).int()[:, None].contiguous()
    _, _, d = run(logits, ids, None, 1.0)
    x = logits.double().requires_grad_()
    (want,) = torch.autograd.grad(reference(x, ids, None)[0], x)
    assert float((d.double() - want).abs().max()) <= 2.0 ** -19 * float(want.abs().max())
