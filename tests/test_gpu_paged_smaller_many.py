"""Many rows over a smaller cache: weights added up on the tensor cores and prefill over 8 bits, where
their running maxima move, rows are NaN, ranges of items are cut, and calls are captured."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, NAN, Pages, assert_rows, attention64, batch_of, ctx, fused_rows, i32  # noqa: F401
from test_gpu_paged_evict import OFF, assert_weights, scratch_of, slots, weighed64, weights_of
from test_gpu_paged_quant import MANY, QuantPages

pytestmark = pytest.mark.gpu


def weigh(ctx, p, q, new, before, decay=1.0, scale=0.0, stream=None):  # noqa: F811
    w = before.clone()
    still.still_paged_weigh(ctx, p.cache(), batch_of(p, new), q, w, scratch_of(p, q.shape[0], q.shape[1]),
                            scale=scale, decay=decay, stream=stream)
    return w


def off_of(p, q, new, scale):
    """What fp32 sums of exact products leave: a logit is off by at most 2^-24 x d/16 partial sums of
    the size of sum |q k| scale, here all of d; with a row's sum that is off alike, twice that."""
    most = 0.0
    for b in range(len(new)):
        k = p.rows(p.K, b).abs().double()
        most = max(most, float(q.abs().double().amax(1).amax(0) @ k.amax(1).amax(0)) if len(k) else 0)
    return OFF + 2 * 2.0 ** -24 * (q.shape[2] / 16 + 1) * most * scale


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("beta", [False, True])
def test_maxima_that_move(ctx, d, beta):  # noqa: F811
    """Keys that grow along the sequence: a row's maximum passes the one that it began with many times
    over, and m + log l is large, where it must not be held in one number."""
    p = Pages(31, [900, 300], 2, d, 64, beta)
    for b in range(2):
        n = p.lens[b]
        j = torch.arange(n, device=DEV)
        page = p.table[b].long()[j // 64]
        grow = torch.linspace(0.05, 12, n, device=DEV)[:, None, None]
        p.K[page, j % 64] = (p.K[page, j % 64].float() * grow).bfloat16()
    q, = fused_rows(32, 333, [6], d)
    new = [300, 33]
    before = weights_of(p, 33)
    want = weighed64(p, q, new, before, 1.0)
    assert_weights(p, weigh(ctx, p, q, new, before), before, want, off_of(p, q, new, d ** -0.5))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_first_slots_masked(ctx, d):  # noqa: F811
    """Rows that see nothing in their first tiles of slots, then a few slots of a tile."""
    p = Pages(34, [1000, 200], 1, d, 32, beta=True)
    for j in list(range(0, 700)) + list(range(710, 780)):
        p.beta[int(p.table[0, j // 32]), :, j % 32] = -math.inf
        p.K[int(p.table[0, j // 32]), j % 32] = (NAN, math.inf)[j % 2]
    q, = fused_rows(35, 320, [3], d)
    new = [200, 120]
    before = weights_of(p, 36)
    w = weigh(ctx, p, q, new, before)
    assert_weights(p, w, before, weighed64(p, q, new, before, 1.0))


@pytest.mark.parametrize("d,past", [(64, 0), (128, 200), (256, 60)])
def test_a_row_of_nan_spoils_what_it_sees(ctx, d, past):  # noqa: F811
    """Slots that a NaN query sees become NaN, of its own KV-head; later ones and others do not."""
    p = Pages(37, [past + 150, 70], 2, d, 16)
    q, = fused_rows(38, 220, [8], d)
    q = q.clone()
    q[60, 1, 5] = NAN
    before = weights_of(p, 39)
    w = weigh(ctx, p, q, [150, 70], before)
    got = slots(p, w, 0)
    assert torch.isnan(got[:past + 61, 0]).all()
    q[60, 1] = 0
    clean = weigh(ctx, p, q, [150, 70], before)
    assert torch.equal(got[past + 61:, 0], slots(p, clean, 0)[past + 61:, 0])
    assert torch.equal(got[:, 1], slots(p, clean, 0)[:, 1])
    assert torch.equal(slots(p, w, 1), slots(p, clean, 1))


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta", [
    (128, 4, 28, 64, [3001], [0], False),          # many items, cut into ranges
    (128, 2, 8, 64, [64, 64], [20000, 9000], True),  # few rows of many slots
    (64, 1, 1, 256, [2000], [300], False),
    (256, 1, 2, 32, [700, 1, 90], [4000, 900, 0], True),
    (128, 1, 128, 16, [5], [3000], False),
    (64, 3, 9, 16, [(13 * i) % 61 for i in range(200)], [(29 * i) % 300 for i in range(200)], False),
])
def test_weights_of_long_calls(ctx, d, H, Hq, page, new, past, beta):  # noqa: F811
    p = Pages(40, [a + b for a, b in zip(new, past)], H, d, page, beta)
    q, = fused_rows(41, sum(new), [Hq], d)
    before = weights_of(p, 42)
    w = weigh(ctx, p, q, new, before, decay=0.75)
    assert_weights(p, w, before, weighed64(p, q, new, before, 0.75))
    assert torch.equal(weigh(ctx, p, q, new, before, decay=0.75).view(torch.int32), w.view(torch.int32))


def test_captured_calls_follow_lengths(ctx):  # noqa: F811
    """Weights and a prefill over 8 bits, captured on a side stream with most of the slots idle, then
    replayed at other lengths: both are what a call outside a graph gives."""
    H, d, page = 2, 128, 32
    p = Pages(43, [900, 700], H, d, page)
    e = QuantPages(44, [900, 700], H, d, page)
    q, = fused_rows(45, 120, [8], d)
    q = q.contiguous()
    lens, cu = i32([900, 700]), i32([0, 70, 120])
    batch = still.PagedBatch(p.table, lens, cu)
    batch8 = still.PagedBatch(e.table, lens, cu)
    before = weights_of(p, 46)
    w, out = before.clone(), torch.empty_like(q)
    scratch = scratch_of(p, 120, 8)
    cache, cache8 = p.cache(), e.cache()
    still.still_paged_weigh(ctx, cache, batch, q, w, scratch)  # the workspace, outside the capture
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            still.still_paged_weigh(ctx, cache, batch, q, w, scratch, stream=stream)
            still.still_paged_prefill_quant(ctx, cache8, batch8, q, out, stream=stream)
        for n, c in (([900, 700], [0, 70, 120]), ([130, 0], [0, 119, 120]), ([33, 512], [0, 0, 120])):
            lens.copy_(i32(n))
            cu.copy_(i32(c))
            w.copy_(before)
            graph.replay()
            stream.synchronize()
            w2, out2 = before.clone(), torch.empty_like(out)
            still.still_paged_weigh(ctx, cache, batch, q, w2, scratch, stream=stream)
            still.still_paged_prefill_quant(ctx, cache8, batch8, q, out2, stream=stream)
            stream.synchronize()
            assert torch.equal(w.view(torch.int32), w2.view(torch.int32)) and torch.equal(out, out2)
            p.lens = e.lens = n
            new = [c[1] - c[0], c[2] - c[1]]
            if n[0] >= new[0] and n[1] >= new[1]:
                assert_rows(out, *attention64(e, q, new), MANY)
            p.lens = e.lens = [900, 700]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("beta", [False, True])
def test_scales_that_are_no_powers_of_two(ctx, d, beta):  # noqa: F811
    """Many rows round code times scale to bf16: of K by 2^-9, which moves a logit by at most 2^-9 of
    scale sum |q k| and a weight by twice that (its sum moves too); of V by 2^-9 of a value."""
    p = QuantPages(47, [700, 129], 2, d, 32, beta)
    for s, f in zip(p.scales, (1.37, 0.71)):
        s.mul_(f)
    p.read()
    new = [300, 129]
    q, = fused_rows(48, sum(new), [8], d)
    out = torch.empty_like(q)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, out)
    most = max(float((q[a:b].abs().double().flatten(0, 1) @ p.rows(p.K, i)[:, h].abs().T).max())
               for i, (a, b) in enumerate(((0, 300), (300, 429))) for h in range(2))
    moved = 2.0 ** -9 * most * d ** -0.5
    assert_rows(out, *attention64(p, q, new), MANY + 2.0 ** -9 + math.expm1(2 * moved))
    one = torch.empty(2, 8, d, device=DEV, dtype=torch.bfloat16)  # few rows round nothing
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q[:2], one)
    assert_rows(one, *attention64(p, q[:2], [1, 1]), 2.0 ** -11 + 2.0 ** -20)


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta", [
    (128, 4, 28, 64, [2500], [0], False),
    (128, 2, 8, 16, [40, 64, 3], [20000, 9000, 70], True),
    (256, 2, 4, 16, [900, 200], [0, 3000], False),
    (256, 1, 1, 128, [40], [12000], True),
    (64, 2, 4, 32, [1500], [1000], True),
    (64, 4, 64, 64, [33, 20], [6000, 100], False),
])
def test_prefill_of_long_calls(ctx, d, H, Hq, page, new, past, beta):  # noqa: F811
    p = QuantPages(49, [a + b for a, b in zip(new, past)], H, d, page, beta)
    q, = fused_rows(50, sum(new), [Hq], d)
    out = torch.full_like(q, NAN)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, out)
    assert_rows(out, *attention64(p, q, new), MANY)
    again = torch.full_like(q, NAN)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, again)
    assert torch.equal(out, again)


def test_large_groups_of_single_tokens(ctx):  # noqa: F811
    """Decode in 8 bits of groups that the few rows' kernel reads the pool twice for, and beyond."""
    for d, g in ((64, 32), (128, 32), (128, 33), (256, 16), (256, 17), (128, 128)):
        p = QuantPages(51, [700, 0, 65], 1, d, 16)
        q, = fused_rows(52, 3, [g], d)
        out = torch.full_like(q, NAN)
        still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
        few = g <= (16 if d == 256 else 32)
        assert_rows(out, *attention64(p, q, [1] * 3), 2.0 ** -11 + 2.0 ** -20 if few else MANY)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_scales_beyond_an_exponent_apart(ctx, d):  # noqa: F811
    """A block whose scale is 2^160 of the others' and whose weights are below the smallest float."""
    p = QuantPages(53, [64], 1, d, 16)
    q, = fused_rows(54, 1, [4], d)
    q = q.abs().contiguous()
    far = int(p.table[0, 2])
    p.codes[0].view(torch.uint8)[far] = 0xf8  # keys of -256 each
    for page in p.table[0, :4].tolist():
        p.scales[0][page] = 2.0 ** -8
        p.scales[1][page] = 2.0 ** 100 if page == far else 2.0 ** -60
    p.scales[0][far] = 2.0 ** 8
    p.read()
    out = torch.empty_like(q)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1]), 2.0 ** -11 + 2.0 ** -20)


@pytest.mark.parametrize("B,H,n,keep", [
    (1, 2, 14000, 700),     # a cluster each, keys in its shared memory
    (2, 1, 60001, 30000),
    (8, 8, 60001, 333),     # one CTA each, more keys than it holds
    (20, 8, 9000, 8999),    # one CTA each, and held
])
def test_choices_of_clusters_and_of_single_ctas(ctx, B, H, n, keep):  # noqa: F811
    """Weights of few different sizes, so that the border falls among equals: the lowest slots stay."""
    d, page, sinks, recent = 64, 64, 5, 40
    lens = [n - 37 * b for b in range(B)]
    g = torch.Generator(device=DEV).manual_seed(55)
    need = -(-n // page)
    pools = [torch.randint(-9, 9, (B * need, page, H, d), generator=g, device=DEV).bfloat16()
             for _ in "KV"]
    table = torch.randperm(B * need, generator=g, device=DEV).to(torch.int32).view(B, need)
    w = torch.randint(-3, 50, (B * need, H, page), generator=g, device=DEV).float()
    w = torch.where(w < 0, torch.where(w < -2, NAN, -math.inf), (w - 7) / 8)
    to_need = -(-keep // page)
    to = [torch.zeros(B * to_need, page, H, d, device=DEV, dtype=torch.bfloat16) for _ in "KV"]
    to_table = torch.arange(B * to_need, dtype=torch.int32, device=DEV).view(B, to_need)
    kept = torch.full((B, H, keep), -9, dtype=torch.int32, device=DEV)
    to_lens = torch.full((B,), -9, dtype=torch.int32, device=DEV)
    still.still_paged_evict(ctx, still.PagedCache(*pools), still.PagedBatch(table, i32(lens)), w, keep,
                            sinks, recent, still.PagedCache(*to), to_table, kept, to_lens)
    assert to_lens.tolist() == [min(keep, m) for m in lens]
    j = torch.arange(n, device=DEV)
    for b, m in enumerate(lens):
        x = w[table[b].long()[j // page], :, j % page].T.double()  # [H, n]
        x = torch.where(torch.isnan(x), -1e30, x.clamp_min(-1e20))
        x[:, :sinks] = math.inf
        x[:, m - recent:] = math.inf
        x[:, m:] = -math.inf
        count = min(keep, m)
        idx = x.sort(dim=1, descending=True, stable=True).indices[:, :count].sort(1).values
        assert torch.equal(kept[b, :, :count].long(), idx)
        assert (kept[b, :, count:] == -1).all()
        r = torch.arange(count, device=DEV)
        for h in range(H):
            src, dst = table[b].long()[idx[h] // page], to_table[b].long()[r // page]
            for old, new in zip(pools, to):
                assert torch.equal(new[dst, r % page, h], old[src, idx[h] % page, h])
