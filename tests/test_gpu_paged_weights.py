"""Attention weights over a paged cache where sequences are very long or rows are no numbers, by both
kernels that add them up."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import (DEV, NAN, WEIGHTS, Pages, assert_rows, attention64, batch_of, ctx,  # noqa: F401
                            fused_rows, i32)
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


def row_of_nan(q, kind):
    q = q.clone()
    q[..., 5] = NAN if kind == "nan" else math.inf
    return q


@pytest.mark.parametrize("kind", ["nan", "inf"])
@pytest.mark.parametrize("d,new", [(64, 1), (128, 2), (256, 3), (64, 9), (128, 70)])
def test_rows_of_nan(ctx, d, new, kind):  # noqa: F811
    """What a row's weights are, slots that it sees become, whichever kernel adds them up: NaN, but 0
    for those that are masked; other slots, KV-heads and sequences stay as they were."""
    past = 100
    p = Pages(73, [past + new, 70], 2, d, 16, beta=True)
    masked = [3, 40, 64, past - 1]
    for j in masked:
        p.beta[int(p.table[0, j // 16]), :, j % 16] = -math.inf
    q, = fused_rows(74, 2 * new, [4], d)
    q = q.clone()
    bad = (new - 1) // 2  # a token in the middle, a query head of KV-head 0
    before = weights_of(p, 75)

    def weigh(q):
        w = before.clone()
        still.still_paged_weigh(ctx, p.cache(), batch_of(p, [new] * 2), q, w, scratch_of(p, 2 * new, 4))
        return w
    clean = weigh(q)
    q[bad, 1] = row_of_nan(q[bad, 1], kind)
    w = weigh(q)
    got, ref = slots(p, w, 0), slots(p, clean, 0)
    seen = torch.arange(past + new, device=DEV) <= past + bad
    seen[masked] = False
    assert torch.isnan(got[seen, 0]).all()
    # (the other rows' shares of an unseen or masked slot are what they were)
    assert torch.equal(got[~seen, 0], ref[~seen, 0]) and torch.isfinite(ref).all()
    assert torch.equal(got[:, 1], ref[:, 1]) and torch.equal(slots(p, w, 1), slots(p, clean, 1))


@pytest.mark.parametrize("kind", ["nan", "inf"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("beta", [False, True])
def test_rows_of_nan_beside_a_decode(ctx, d, beta, kind):  # noqa: F811
    p = Pages(76, [300, 70], 2, d, 32, beta=beta)
    masked = [3, 40, 64, 298] if beta else []
    for j in masked:
        p.beta[int(p.table[0, j // 32]), :, j % 32] = -math.inf
    q, = fused_rows(77, 2, [6], d)
    q = q.clone()
    before = weights_of(p, 78)

    def weigh(q):
        w, out = before.clone(), torch.empty_like(q)
        still.still_paged_decode_weigh(ctx, p.cache(), batch_of(p), q, out, w, scratch_of(p, 2, 6))
        return w, out
    clean, o0 = weigh(q)
    q[0, 4] = row_of_nan(q[0, 4], kind)  # KV-head 1
    w, o1 = weigh(q)
    got, ref = slots(p, w, 0), slots(p, clean, 0)
    seen = torch.ones(300, dtype=torch.bool, device=DEV)
    seen[masked] = False
    assert torch.isnan(got[seen, 1]).all() and torch.isnan(o1[0, 4]).all()
    assert torch.equal(got[~seen, 1], ref[~seen, 1]) and torch.isfinite(ref).all()
    assert torch.equal(got[:, 0], ref[:, 0]) and torch.equal(slots(p, w, 1), slots(p, clean, 1))
    assert torch.equal(o0[0, :3], o1[0, :3]) and torch.equal(o0[1], o1[1])
    # (the other rows of the group are formed again with weights in bf16, for the infinite values
    # that a NaN may come from)
    q[0, 4] = 0
    ref, size = attention64(p, q, [1, 1])
    for i in (3, 5):
        assert_rows(o1[0, i], ref[0, i], size[0, i], WEIGHTS)


@pytest.mark.parametrize("d,new", [(64, 1), (128, 2), (64, 40), (256, 70)])
def test_scratch_of_weights_alone(ctx, d, new):  # noqa: F811
    """still_paged_weigh needs 8 bytes for every token and query head, rounded up to 256, and uses no
    more; a decode needs what still_paged_weigh_scratch gives."""
    p = Pages(79, [new + 90, new], 2, d, 16)
    Hq = 6
    q, = fused_rows(80, 2 * new, [Hq], d)
    before = weights_of(p, 81)
    least = -(-2 * new * Hq * 8 // 256) * 256
    pool = p.K.shape[0] * 16 * Hq * 4
    assert still.still_paged_weigh_scratch(p.cache(), 2 * new, Hq) == least + pool

    def weigh(scratch):
        w = before.clone()
        still.still_paged_weigh(ctx, p.cache(), batch_of(p, [new] * 2), q, w, scratch)
        return w
    scratch = torch.full((least + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    w = weigh(scratch[:least])
    assert (scratch[least:] == 0x5a).all()
    assert torch.equal(w.view(torch.int32), weigh(scratch_of(p, 2 * new, Hq)).view(torch.int32))
    for size in (0, least - 1):
        with pytest.raises(still.StillError, match="SHAPE|INVALID_ARG"):
            weigh(scratch[:size])
    one = q[:2].contiguous()
    small = torch.empty(255 + pool, dtype=torch.uint8, device=DEV)
    with pytest.raises(still.StillError, match="SHAPE"):
        still.still_paged_decode_weigh(ctx, p.cache(), batch_of(p), one, torch.empty_like(one),
                                       before.clone(), small)
