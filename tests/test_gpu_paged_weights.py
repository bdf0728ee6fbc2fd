"""Attention weights over a paged cache where sequences are very long or rows are no numbers, by both
kernels that add them up."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, NAN, Pages, batch_of, ctx, fused_rows, i32  # noqa: F401
from test_gpu_paged_evict import OFF, scratch_of, slots, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g,page,n_slots", [(128, 65536, 17_100_000), (64, 256, 33_600_001)])
def test_weights_of_very_long_sequences(ctx, g, page, n_slots):  # noqa: F811
    """Slots times query heads beyond 2^31: every slot gets its weight."""
    d, n_pages = 64, -(-n_slots // page)
    gen = torch.Generator(device=DEV).manual_seed(71)
    K = torch.empty(n_pages, page, 1, d, device=DEV, dtype=torch.bfloat16).normal_(generator=gen)
    table = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)[None]
    cache, batch = still.PagedCache(K, K), still.PagedBatch(table, i32([n_slots]))
    q, = fused_rows(72, 1, [g], d)
    weight = torch.full((n_pages, 1, page), 2.0 ** -25, device=DEV)
    size = still.still_paged_weigh_scratch(cache, 1, 1)
    scratch = torch.empty(size, dtype=torch.uint8, device=DEV)
    still.still_paged_weigh(ctx, cache, batch, q, weight, scratch, decay=0.5)
    got = weight[table[0].long()].flatten()[:n_slots]
    step = 1 << 20
    logits = lambda j: q[0].double() @ K[table[0, j // page:-(-(j + step) // page)].long()].view(
        -1, d)[j % page:j % page + step][:n_slots - j].double().T / 8  # slots [j, j + step)
    total = sum(logits(j).exp().sum(1) for j in range(0, n_slots, step))
    for j in range(0, n_slots, step):
        want = (logits(j).exp() / total[:, None]).sum(0) + 2.0 ** -26
        if j + step >= n_slots:
            want[-1] -= 2.0 ** -26  # the new token's own begins at 0
        assert ((got[j:j + step].double() - want).abs() <= OFF * want).all(), j
