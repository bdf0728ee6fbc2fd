"""Attention over a cache in 8 bits against 64 bits, each call to the bound of the arithmetic that
serves it."""
import pytest
import torch

import test_gpu_paged_quant as quant
import test_gpu_paged_smaller_many as many
from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, NAN, WEIGHTS, assert_rows, attention64, batch_of, ctx, fused_rows  # noqa: F401
from test_gpu_paged_quant import FEW, QuantPages

pytestmark = pytest.mark.gpu

# Many rows hold weights in bf16, each off by half a step, 2^-8 of it, and not their sum; codes times
# scales that are powers of two are exact in bf16; logits as in 16 bits: WEIGHTS. Few rows hold weights
# times scale as fp16 hi + lo, multiples of a number that is at most the row's largest such product R:
# off by 2^-22 of themselves (in FEW) or 2^-25 R, whichever is more.


def cases(test):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize")


def bound(n, B, g, d, packed):
    """By the rule that chooses the kernel: mean rows of a sequence and KV-head."""
    least = 8 if d == 256 else 16
    if g > 128 or -(-n * g // B) <= least or (not packed and g <= 2 * least):
        return FEW
    return WEIGHTS


def prefill(ctx, p, new, q):  # noqa: F811
    out = torch.full(q.shape, NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, out)
    return out


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta,heads_first",
                         cases(quant.test_prefill_matches_64_bits))
def test_prefill(ctx, d, H, Hq, page, new, past, beta, heads_first):  # noqa: F811
    p = QuantPages(90, [a + b for a, b in zip(new, past)], H, d, page, beta, heads_first)
    q, _ = fused_rows(91, sum(new), [Hq, 1], d)
    assert_rows(prefill(ctx, p, new, q), *attention64(p, q, new),
                bound(sum(new), len(new), Hq // H, d, True))


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta", cases(many.test_prefill_of_long_calls))
def test_prefill_of_long_calls(ctx, d, H, Hq, page, new, past, beta):  # noqa: F811
    p = QuantPages(92, [a + b for a, b in zip(new, past)], H, d, page, beta)
    q, = fused_rows(93, sum(new), [Hq], d)
    assert_rows(prefill(ctx, p, new, q), *attention64(p, q, new),
                bound(sum(new), len(new), Hq // H, d, True))


@pytest.mark.parametrize("d,g", [(64, 33), (64, 160), (128, 32), (128, 33), (128, 129), (256, 16),
                                 (256, 17), (256, 200)])
def test_single_tokens_of_large_groups(ctx, d, g):  # noqa: F811
    p = QuantPages(94, [700, 0, 65], 1, d, 16, beta=True)
    q, = fused_rows(95, 3, [g], d)
    out = torch.full_like(q, NAN)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * 3), bound(3, 3, g, d, False))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 70])
def test_blocks_of_very_different_sizes(ctx, d, new):  # noqa: F811
    sizes = torch.tensor([2.0 ** -40, 2.0 ** -20, 1.0, 3.0, 2.0 ** 18, 2.0 ** 30], device=DEV)
    p = QuantPages(96, [700, 90, 33], 1, d, 32, size=sizes)
    p.scales[0].copy_(torch.where(torch.isnan(p.scales[0]), NAN, 2.0 ** -8))  # keys alike
    p.read()
    counts = [1] * 3 if new == 1 else [new, 70, 20]
    q, = fused_rows(97, sum(counts), [4], d)
    if new > 1:
        assert_rows(prefill(ctx, p, counts, q), *attention64(p, q, counts), WEIGHTS)
        return
    out = torch.full_like(q, NAN)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    ref, size = attention64(p, q, counts)
    tol = 2.0 ** -8 * ref.abs() + FEW * size
    for b, n in enumerate(p.lens):
        w = torch.softmax(q[b].double() @ p.rows(p.K, b)[:, 0].T / d ** 0.5, -1)  # [heads, slots]
        blocks = p.table[b, :-(-n // 32)].long()
        s = p.scales[1][blocks, 0].flatten().double().repeat_interleave(16)[:n]
        largest = (w * s).amax(1)
        tol[b] += 2.0 ** -25 * largest[:, None] * (p.rows(p.V, b)[:, 0].abs() / s[:, None]).sum(0)
    assert torch.isfinite(out).all() and ((out.double() - ref).abs() <= tol).all()
