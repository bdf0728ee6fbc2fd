"""The kernel of many rows (more than 16 rows, tokens x heads of a group, per sequence and KV-head;
more than 8 with 256 channels, pairs of CTAs above 128) where only it can go wrong: a running maximum
that moves, masks and infinities, a scale, captured and repeated calls, uneven batches."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import (DEV, NAN, WEIGHTS, Pages, assert_rows, attention64, batch_of, fused_rows,
                            i32)

pytestmark = pytest.mark.gpu

# head dims, and for 256 channels rows of a sequence for one CTA (20 tokens of 4 heads) and for a
# pair (40 tokens)
FORMS = [(64, 40), (128, 40), (256, 20), (256, 40)]


@pytest.fixture(scope="module")
def ctx():
    c = still.still_create(0)
    yield c
    code, det = still.still_get_device_status(c)
    still.still_destroy(c)
    assert code == 0, (still.STATUS[code], det)


def prefill(ctx, p, new, q, **kw):
    out = torch.full(q.shape, NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill(ctx, p.cache(), batch_of(p, new), q, out, **kw)
    return out


def staircase(length, tiles):
    """Logits of slots: 6 more from the last slot of each of `tiles` (of 128 slots) on, that slot
    itself 2 above its successors, and 8 less behind the last one. The 128 slots of a tile below the
    last step weigh 128 e^-8 = 0.04 together where that one slot weighs 1."""
    at = torch.tensor([128 * t + 127 for t in tiles if t >= 0], device=DEV)
    slots = torch.arange(length, device=DEV)
    step = (slots[:, None] >= at).sum(1)
    return step * 6.0 - 2.0 * ~torch.isin(slots, at) - 6.0 * (slots > at[-1]), step


def steps(last):
    """Tiles of the steps that rows of the first kind see, of the second."""
    return (last - 5, last - 3, last), (last - 4, last - 2, last - 1)


@pytest.mark.parametrize("H,ends", [
    (1, [2]), (1, [3]), (1, [8]), (1, [13]),               # a few tiles of slots a CTA, joined
    (8, [13, 2, 12, 7, 8, 3]), (8, [1 + i % 13 for i in range(26)])])  # more of them, whole items
@pytest.mark.parametrize("grow", ["keys", "keys beside biases", "biases"])
@pytest.mark.parametrize("d,n", FORMS)
def test_the_running_maximum_moves(ctx, d, n, grow, H, ends):
    """Row maxima rise by 6 (8.7 in units of log 2, beyond the 8 that a tile may lie above the running
    one) several times, the last time in each tile from the first to the 14th: at odd and even ones,
    in a third of a warp's rows at a time or in all, in items that one CTA has whole and in items that
    several share. V changes its sign with every step, so that what is rescaled wrongly shows."""
    B, g = len(ends), 4
    p = Pages(70, [128 * (t + 1) + n for t in ends], H, d, 64, beta=grow != "keys")
    q, = fused_rows(71, n * B, [H * g], d)
    q = q * 0.1
    # rows follow one staircase, the other, or none
    kind = (torch.arange(n * B, device=DEV)[:, None] + torch.arange(H * g, device=DEV)) % 3
    q[..., 0] = 4.0 * (kind == 0)
    q[..., 1] = 4.0 * (kind == 1)
    for b, last in enumerate(ends):
        slots = torch.arange(p.lens[b], device=DEV)
        pages, at = p.table[b].long()[slots // 64], slots % 64
        (first, step), (second, _) = (staircase(p.lens[b], x) for x in steps(last))
        k, v = p.K[pages, at] * 0.1, p.V[pages, at] * 0.1
        k[..., 0] = (first * math.sqrt(d) / 4)[:, None].bfloat16()
        k[..., 1] = (second * math.sqrt(d) / 4)[:, None].bfloat16()
        if grow == "biases":
            k[..., :2] = 0
            p.beta[pages, :, at] = first[:, None].expand(-1, H).float()
        p.K[pages, at] = k
        p.V[pages, at] = v + (1 - 2 * (step & 1))[:, None, None]
    out = prefill(ctx, p, [n] * B, q)
    # (logits below 2^5: their fp32 rounding, 2^-18, is far below the bound that WEIGHTS has for it)
    assert_rows(out, *attention64(p, q, [n] * B), WEIGHTS)


@pytest.mark.parametrize("last", range(1, 14))
def test_a_wrong_rescale_would_show(last):
    """The bound above rejects outputs whose older part is weighed once too often or not at all."""
    logits, step = staircase(128 * (last + 1) + 40, steps(last)[0])
    w, v = torch.softmax(logits.double(), 0), (1 - 2 * (step & 1)).double()
    ref, size = (w * v).sum(), w.sum()
    for factor in (0.0, math.exp(-6), math.exp(6)):
        x = torch.where(step == step.max(), w, w * factor)
        wrong = (x * v).sum() / x.sum()
        assert (wrong - ref).abs() > 4 * (2.0 ** -8 * ref.abs() + WEIGHTS * size)


@pytest.mark.parametrize("past", [0, 30, 2000])
@pytest.mark.parametrize("d,n", FORMS)
def test_biases_of_the_lowest_size(ctx, d, n, past):
    """Slots of the type's lowest bias weigh nothing beside others and evenly among themselves."""
    lens = [past + n, past + n + 77]
    p = Pages(72, lens, 2, d, 32, beta=True)
    low = torch.finfo(torch.float32).min
    for b, kept in enumerate((lens[0] - 1, lens[1] // 2)):
        for x in range(-(-lens[b] // 32)):
            p.beta[int(p.table[b, x])] = low
        p.beta[int(p.table[b, kept // 32]), :, kept % 32] = 0.5
    q, = fused_rows(73, 2 * n, [8], d)
    assert_rows(prefill(ctx, p, [n, n], q), *attention64(p, q, [n, n]), WEIGHTS)


@pytest.mark.parametrize("past", [60, 2000])
@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("d,n", FORMS)
def test_infinities(ctx, d, n, beta, past):
    """An infinite value stays in its channel, two of opposite signs are NaN there; an infinite logit
    makes its row NaN and no other."""
    p = Pages(74, [past + n], 1, d, 16, beta=beta)
    for j, c, x in ((17, 3, math.inf), (past - 1, 5, -math.inf), (3, 9, math.inf), (40, 9, -math.inf)):
        p.V[int(p.table[0, j // 16]), j % 16, 0, c] = x
    q, = fused_rows(75, n, [4], d)
    out = prefill(ctx, p, [n], q)
    assert torch.isposinf(out[..., 3]).all() and torch.isneginf(out[..., 5]).all()
    assert torch.isnan(out[..., 9]).all()
    rest = [c for c in range(d) if c not in (3, 5, 9)]
    assert torch.isfinite(out[..., rest]).all()
    q = q.clone()
    q[7, 2, 5] = math.inf
    two = prefill(ctx, p, [n], q)
    assert torch.isnan(two[7, 2]).all()
    two[7, 2] = out[7, 2]
    assert torch.equal(two[..., rest], out[..., rest])


@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("d,n", FORMS)
def test_scale(ctx, d, n, beta):
    """A scale of the caller's, in whole items and in those that several CTAs share and join."""
    for lens in ([5000], [200] * 30):
        p = Pages(76, lens, 1 if len(lens) == 1 else 8, d, 32, beta=beta)
        new = [n] * len(lens)
        q, = fused_rows(77, sum(new), [4 * p.H], d)
        for scale in (0.03, 0.2):
            out = prefill(ctx, p, new, q, scale=scale)
            # at 0.2 logits are 3.2 times those of 1 / sqrt(256), for which WEIGHTS holds 2^-11
            assert_rows(out, *attention64(p, q, new, scale), WEIGHTS + 2.0 ** -10)


@pytest.mark.parametrize("d,n", FORMS)
def test_captured_call_follows_its_arrays(ctx, d, n):
    """Lengths, offsets of the new tokens and pages are read when a captured call runs."""
    p = Pages(78, [3000, 500, 200], 2, d, 16)
    total = 3 * n
    cache, batch = p.cache(), batch_of(p, [n, n, n])
    q, = fused_rows(79, total, [8], d)
    out = torch.empty(total, 8, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill(ctx, cache, batch, q, out)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        still.still_paged_prefill(ctx, cache, batch, q, out, stream=stream)
    with torch.cuda.stream(stream):
        for new, lens in (([n, n, n], [3000, 500, 200]), ([1, total - 1, 0], [2999, 400, 0]),
                          ([0, 0, total], [7, 0, 180]), ([total, 0, 0], [5, 3, 0])):
            batch.tensors[1].copy_(i32(lens))
            batch.tensors[2].copy_(i32([0] + new).cumsum(0).to(torch.int32))
            p.lens = lens
            out.fill_(NAN)
            graph.replay()
            stream.synchronize()
            assert_rows(out, *attention64(p, q, new), WEIGHTS)
        p.table = p.table.flip(0).contiguous()
        batch.tensors[0].copy_(p.table)
        p.lens = [150, 300, 1000]
        batch.tensors[1].copy_(i32(p.lens))
        batch.tensors[2].copy_(i32([0, n, n, total]))
        graph.replay()
        stream.synchronize()
        assert_rows(out, *attention64(p, q, [n, 0, 2 * n]), WEIGHTS)


@pytest.mark.parametrize("d,n", FORMS)
def test_same_inputs_same_bits_on_two_streams(d, n):
    """Two contexts on streams of their own, calls of several sizes under way at once: each result is
    what the call gives alone, every time."""
    cs = [still.still_create(0) for _ in range(2)]
    try:
        cases = []
        for i, (lens, new) in enumerate([([4000], [n]), ([300] * 40, [n] * 40), ([90, 2500], [5, n])]):
            p = Pages(80 + i, lens, 2, d, 64, beta=i == 2)
            q, = fused_rows(90 + i, sum(new), [8], d)
            alone = prefill(cs[0], p, new, q)
            cases.append((p.cache(), batch_of(p, new), q, alone))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in cs]
        outs = []
        for turn in range(12):
            for c, s in zip(cs, streams):
                cache, batch, q, alone = cases[(turn + (c is cs[1])) % 3]
                out = torch.empty_like(alone)
                s.wait_stream(torch.cuda.current_stream())
                still.still_paged_prefill(c, cache, batch, q, out, stream=s)
                outs.append((out, alone))
        torch.cuda.synchronize()
        for out, alone in outs:
            assert torch.equal(out, alone)
        for c in cs:
            assert still.still_get_device_status(c)[0] == 0
    finally:
        for c in cs:
            still.still_destroy(c)


@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("long,ones,idle", [(700, 60, 40), (300, 120, 9), (33, 3, 0)])
def test_a_prompt_beside_single_tokens_and_idle_places(ctx, d, long, ones, idle, beta):
    """One long prompt, many sequences of one new token, places without tokens and places of one token
    without slots: by the rows that they come to on average, of either kernel."""
    new = [1] * (ones // 2) + [long] + [1] * (ones - ones // 2) + [0, 1] * (idle // 2)
    past = [(53 * i) % 400 for i in range(ones + 1)] + [0] * (2 * (idle // 2))
    p = Pages(82, [a + b for a, b in zip(new, past)], 2, d, 32, beta=beta)
    for b in range(ones + 1, len(new)):
        p.lens[b] = 0
    q, = fused_rows(83, sum(new), [8], d)
    assert_rows(prefill(ctx, p, new, q), *attention64(p, q, new), WEIGHTS)


@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_hundreds_of_sequences_of_one_tile_of_slots(ctx, d, beta):
    """A CTA (or pair) has one short item after another: of 128 slots at most, or a few of two."""
    for least, most, count in ((5, 20, 500), (65, 100, 300)):
        new = [least + (7 * i) % (most - least) for i in range(count)]
        lens = [x + (11 * i) % 30 + (40 if i % 9 == 0 else 0) for i, x in enumerate(new)]
        p = Pages(84, lens, 2, d, 16, beta=beta)
        q, = fused_rows(85, sum(new), [4], d)
        assert_rows(prefill(ctx, p, new, q), *attention64(p, q, new), WEIGHTS)


@pytest.mark.parametrize("d,n", FORMS)
def test_pools_of_one_page_and_one_head(ctx, d, n):
    """Axes of one entry, whose strides the binding replaces."""
    p = Pages(86, [128], 1, d, 128, spare=0)
    p.K = p.K.transpose(1, 2).contiguous().transpose(1, 2)
    q, = fused_rows(87, n, [4], d)
    assert_rows(prefill(ctx, p, [n], q), *attention64(p, q, [n]), WEIGHTS)
