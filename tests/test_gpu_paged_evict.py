"""Eviction from a paged cache by accumulated attention weight, against plain 64-bit restatements:
weights of single tokens and of many, the choice of slots and their move, and a run of them all."""
import ctypes
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import (DEV, NAN, WEIGHTS, Pages, assert_rows, attention64, batch_of, ctx,  # noqa: F401
                            fused_rows, i32)

pytestmark = pytest.mark.gpu

# Logits are fp32 sums of exact products of up to 256 channels of size 1/16 .. 4, off by less than
# 2^-12.7, and so is a row's sum; exponentials 2^-22. A slot's sum over its rows in fp32 adds less than
# 2^-24 for each of their number, at most 2^-11 for 8,192 rows.
OFF = 2.0 ** -11 + 2.0 ** -11


def scratch_of(p, n, Hq):
    size = still.still_paged_weigh_scratch(p.cache(), n, Hq)
    return torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)


def weights_of(p, seed, fill=None):
    """Weights of earlier steps; NaN where no sequence has a slot."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.full((p.K.shape[0], p.H, p.page), NAN, device=DEV)
    for b, n in enumerate(p.lens):
        pages = p.table[b, :-(-n // p.page)].long()
        x = torch.rand(len(pages) * p.page, p.H, generator=g, device=DEV)
        if fill is not None:
            x.fill_(fill)
        x[n:] = NAN
        w[pages] = x.view(len(pages), p.page, p.H).transpose(1, 2)
    return w


def slots(p, x, b):
    """[len, H] of a pool of weights."""
    pages = p.table[b, :-(-p.lens[b] // p.page)].long()
    return x[pages].permute(0, 2, 1).reshape(-1, p.H)[:p.lens[b]]


def weighed64(p, q, new, before, decay, scale=None):
    """Per sequence [len, H]: the weights after the call."""
    Hq, d = q.shape[1:]
    g = Hq // p.H
    got, at = [], 0
    for b, n in enumerate(new):
        L = p.lens[b]
        old = slots(p, before, b).double()
        if n == 0 or L == 0:
            got.append(old)
            at += n
            continue
        fresh = torch.arange(L, device=DEV)[:, None] >= L - n
        old = torch.where(fresh, 0.0, old * decay) if decay else torch.zeros_like(old)
        k = p.rows(p.K, b).double()
        late = torch.arange(L, device=DEV) >= torch.arange(L - n, L, device=DEV)[:, None] + 1
        for h in range(p.H):
            bias = p.rows(p.beta, b)[:, h].double() if p.beta is not None else torch.zeros(
                L, dtype=torch.float64, device=DEV)
            hidden = late | (bias == -math.inf)
            kh = torch.where((bias == -math.inf)[:, None], 0.0, k[:, h])
            for i in range(h * g, (h + 1) * g):
                x = q[at:at + n, i].double() @ kh.T * (scale or 1 / math.sqrt(d)) + bias
                x = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
                old[:, h] += torch.where(hidden.all(-1)[:, None], 0.0, x).sum(0)
        got.append(old)
        at += n
    return got


def assert_weights(p, weight, before, want, off=OFF):
    touched = torch.zeros_like(weight, dtype=torch.bool)
    for b, n in enumerate(p.lens):
        x = slots(p, weight, b).double()
        assert torch.isfinite(x).all()
        assert ((x - want[b]).abs() <= off * want[b] + 1e-30).all()
        pages = p.table[b].long()[torch.arange(n, device=DEV) // p.page]
        touched[pages, :, torch.arange(n, device=DEV) % p.page] = True
    rest = ~touched
    assert torch.equal(weight[rest].view(torch.int32), before[rest].view(torch.int32))


CASES = [
    (64, 1, 1, 16, [1], [0], False, False),
    (64, 2, 6, 16, [1, 0, 3, 40], [0, 5, 16, 100], True, True),
    (64, 1, 20, 64, [65, 64, 2, 1], [0, 1, 300, 62], False, False),
    (128, 2, 14, 16, [37, 75, 1], [129, 0, 700], False, True),
    (128, 1, 16, 256, [33], [1000], True, False),
    (128, 8, 32, 64, [64, 64, 64], [900, 3, 5000], False, False),
    (128, 1, 1, 32, [257, 128, 0, 1], [1, 128, 77, 0], True, False),
    (128, 4, 4, 64, [1500, 90], [0, 700], True, True),
    (256, 1, 3, 16, [129, 1, 20], [0, 31, 1000], True, False),
    (256, 2, 10, 128, [300], [2000], False, True),
    (64, 1, 160, 32, [3, 1], [200, 0], False, False),
    (128, 1, 4, 16, [(7 * i) % 23 for i in range(300)], [(11 * i) % 50 for i in range(300)], True,
     False),
]


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta,heads_first", CASES)
@pytest.mark.parametrize("decay", [1.0, 0.0, 0.9])
def test_weights_of_many_tokens(ctx, d, H, Hq, page, new, past, beta, heads_first, decay):  # noqa: F811
    p = Pages(3, [a + b for a, b in zip(new, past)], H, d, page, beta, heads_first)
    q, _ = fused_rows(4, sum(new), [Hq, 1], d)
    before = weights_of(p, 5, fill=NAN if decay == 0 else None)
    for b, n in enumerate(new):  # the new tokens' own are whatever was there
        j = torch.arange(past[b], p.lens[b], device=DEV)
        before[p.table[b].long()[j // page], :, j % page] = NAN
        if n == 0:
            before.nan_to_num_(nan=3.0)
    w = before.clone()
    still.still_paged_weigh(ctx, p.cache(), batch_of(p, new), q, w, scratch_of(p, sum(new), Hq),
                            decay=decay)
    assert_weights(p, w, before, weighed64(p, q, new, before, decay))


@pytest.mark.parametrize("d,H,Hq,page,lens,beta,heads_first", [
    (64, 1, 1, 16, [1], False, False),
    (64, 2, 6, 16, [0, 15, 16, 17, 33], True, True),
    (64, 1, 20, 64, [63, 64, 65, 300], False, False),
    (128, 2, 2, 16, [1, 2, 31, 127, 129], True, False),
    (128, 4, 28, 32, [777, 0, 1, 64], False, True),
    (128, 1, 16, 256, [255, 257, 1000], True, False),
    (256, 2, 18, 64, [65, 500], False, False),
    (256, 2, 4, 64, [30000], True, False),
    (128, 1, 7, 16, [20000, 40, 12000], False, True),
    (64, 1, 160, 32, [200, 31], True, False),
    (128, 1, 5, 32, [(37 * i) % 90 for i in range(300)], False, False),
])
@pytest.mark.parametrize("decay", [1.0, 0.0, 0.5])
def test_decode_and_weights(ctx, d, H, Hq, page, lens, beta, heads_first, decay):  # noqa: F811
    """still_paged_decode's rows, and the weights that still_paged_weigh gives."""
    p = Pages(1, lens, H, d, page, beta, heads_first)
    q, _ = fused_rows(2, len(lens), [Hq, 3], d)
    out = torch.full((len(lens), Hq, d), NAN, device=DEV, dtype=torch.bfloat16)
    before = weights_of(p, 5, fill=NAN if decay == 0 else None)
    w = before.clone()
    still.still_paged_decode_weigh(ctx, p.cache(), batch_of(p), q, out, w,
                                   scratch_of(p, len(lens), Hq), decay=decay)
    assert_rows(out, *attention64(p, q, [1] * len(lens)), WEIGHTS)
    assert_weights(p, w, before, weighed64(p, q, [1] * len(lens), before, decay))
    two = before.clone()
    still.still_paged_weigh(ctx, p.cache(), batch_of(p), q, two, scratch_of(p, len(lens), Hq),
                            decay=decay)
    assert_weights(p, two, before, weighed64(p, q, [1] * len(lens), before, decay))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_masked_slots_get_nothing(ctx, d):  # noqa: F811
    """Biases of -inf before NaN and infinities: such slots get 0, a token that sees nothing gives
    nothing; biases of the lowest value share evenly."""
    lens = [40, 130, 16, 70, 33]
    p = Pages(5, lens, 2, d, 16, beta=True)
    for b, (lo, hi) in enumerate([(0, 40), (3, 120), (15, 16), (0, 69)]):
        for j in range(lo, hi):
            page, at = int(p.table[b, j // 16]), j % 16
            p.beta[page, :, at] = -math.inf
            p.K[page, at] = (NAN, math.inf, -math.inf)[j % 3]
            p.V[page, at] = (math.inf, NAN, -math.inf)[j % 3]
    for j in range(33):
        p.beta[int(p.table[4, j // 16]), :, j % 16] = torch.finfo(torch.float32).min
        p.K[int(p.table[4, j // 16]), j % 16] = 0
    before = weights_of(p, 6)
    for new in ([1] * 5, [40, 65, 1, 70, 5]):
        q, = fused_rows(6, sum(new), [6], d)
        want = weighed64(p, q, new, before, 1.0)
        w = before.clone()
        still.still_paged_weigh(ctx, p.cache(), batch_of(p, new), q, w, scratch_of(p, sum(new), 6))
        assert_weights(p, w, before, want)
        if sum(new) == 5:
            w, out = before.clone(), torch.empty_like(q)
            still.still_paged_decode_weigh(ctx, p.cache(), batch_of(p), q, out, w,
                                           scratch_of(p, 5, 6))
            assert_weights(p, w, before, want)
            assert (out[0] == 0).all()


def test_more_new_tokens_than_slots_and_scale(ctx):  # noqa: F811
    p = Pages(10, [20, 0, 300], 1, 128, 16)
    q, = fused_rows(11, 77, [5], 128)
    before = weights_of(p, 12)
    w = before.clone()
    new = [32, 5, 40]
    still.still_paged_weigh(ctx, p.cache(), batch_of(p, new), q, w, scratch_of(p, 77, 5), scale=0.03)
    x = q.clone()
    want = []
    for b, (n, at) in enumerate(zip(new, (0, 32, 37))):
        skip = max(0, n - p.lens[b])  # tokens before the first slot
        one = Pages.__new__(Pages)
        one.__dict__.update(p.__dict__)
        one.lens, one.table = [p.lens[b]], p.table[b:b + 1]
        want += weighed64(one, x[at + skip:at + n], [n - skip], before, 1.0, 0.03)
    assert_weights(p, w, before, want)


def test_one_peak_beside_many(ctx):  # noqa: F811
    """Weights of very different sizes: one slot takes nearly all, others 2^-60 of it and less."""
    p = Pages(13, [5000], 1, 128, 32)
    q, = fused_rows(14, 64, [4], 128)
    p.K[int(p.table[0, 40]), 7, 0] = (q[:, 0].float().mean(0) * 40).bfloat16()
    before = weights_of(p, 15, fill=0.0)
    w = before.clone()
    still.still_paged_weigh(ctx, p.cache(), batch_of(p, [64]), q, w, scratch_of(p, 64, 4))
    want = weighed64(p, q, [64], before, 1.0)
    # logits of up to 40 x 128 x 2^-3 / 11: fp32 sums move them by 2^-24 x 128 of that, 2^-9
    assert_weights(p, w, before, want, OFF + 2.0 ** -8)


# ------------------------------------------------------------------------------ eviction

def chosen(w, keep, sinks, recent):
    """w [len]: the slots that stay."""
    n = w.shape[0]
    if n <= keep:
        return torch.arange(n, device=DEV)
    w = torch.where(torch.isnan(w), -math.inf, w.double())
    order = sorted(range(sinks, n - recent), key=lambda j: (-float(w[j]), j))
    # NaN below all others, -inf among them
    stay = list(range(min(sinks, n))) + list(range(n - recent, n))
    return torch.tensor(sorted(stay + order[:keep - len(stay)]), device=DEV)


def evict(ctx, p, w, keep, sinks, recent, page, offset=None, heads_first=False, to_weight=True):  # noqa: F811
    need = -(-min(max(p.lens + [1]), keep) // page)
    need = max(need, -(-keep // page))
    B = len(p.lens)
    n = B * need + 1
    shape = (n, p.H, page, p.d) if heads_first else (n, page, p.H, p.d)
    pool = lambda: torch.full(shape, NAN, device=DEV, dtype=torch.bfloat16)
    r = dict(K=pool(), V=pool(), beta=None if p.beta is None else torch.full(
        (n, p.H, page), NAN, device=DEV))
    if heads_first:
        r["K"], r["V"] = r["K"].transpose(1, 2), r["V"].transpose(1, 2)
    order = torch.randperm(n - 1, device=DEV).to(torch.int32)
    r["table"] = order.view(B, need)
    r["weight"] = torch.full((n, p.H, page), NAN, device=DEV) if to_weight else None
    r["kept"] = torch.full((B, p.H, keep), -9, dtype=torch.int32, device=DEV)
    r["lens"] = torch.full((B,), -9, dtype=torch.int32, device=DEV)
    r["offset"] = torch.full((B,), -9, dtype=torch.int64, device=DEV) if offset else None
    r["page"] = page
    to = still.PagedCache(r["K"], r["V"], r["beta"])
    still.still_paged_evict(ctx, p.cache(), batch_of(p, offset=offset), w, keep, sinks, recent, to,
                            r["table"], r["kept"], r["lens"], to_weight=r["weight"],
                            to_offset=r["offset"])
    return r


def assert_evicted(p, w, keep, sinks, recent, r, offset=None):
    bits = lambda x: x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)
    want = {x: r[x].clone() for x in ("K", "V", "beta", "weight") if r[x] is not None}
    for x in want.values():
        x.fill_(NAN)
    for b, n in enumerate(p.lens):
        m = min(n, keep)
        assert int(r["lens"][b]) == m
        if offset:
            assert int(r["offset"][b]) == offset[b] + n - m
        rank = torch.arange(m, device=DEV)
        to, at = r["table"][b].long()[rank // r["page"]], rank % r["page"]
        for h in range(p.H if n else 0):
            j = chosen(slots(p, w, b)[:, h], keep, sinks, recent)
            assert torch.equal(r["kept"][b, h, :m].long(), j), (b, h)
            assert (r["kept"][b, h, m:] == -1).all()
            src = p.table[b].long()[j // p.page], j % p.page
            want["K"][to, at, h] = p.K[src[0], src[1], h]
            want["V"][to, at, h] = p.V[src[0], src[1], h]
            if "beta" in want:
                want["beta"][to, h, at] = p.beta[src[0], h, src[1]]
            if "weight" in want:
                want["weight"][to, h, at] = w[src[0], h, src[1]]
        if n == 0:
            assert (r["kept"][b] == -1).all()
    for x, y in want.items():  # and nothing else was written
        assert torch.equal(bits(r[x]), bits(y)), x


@pytest.mark.parametrize("d,H,page,lens,keep,sinks,recent,to_page,beta,heads_first", [
    (64, 1, 16, [1, 0, 2], 1, 0, 0, 16, False, False),
    (64, 2, 16, [40, 16, 17, 0, 200], 16, 4, 5, 32, True, True),
    (128, 8, 64, [700, 64, 65], 64, 0, 64, 16, False, False),
    (128, 2, 32, [777, 31, 900], 100, 100, 0, 128, True, False),
    (256, 1, 16, [129, 300], 7, 1, 1, 16, True, True),
    (128, 1, 256, [5000, 255, 4097], 1311, 4, 64, 64, False, True),
    (64, 3, 128, [9000, 20000, 8192], 600, 4, 32, 16, True, False),
    (64, 1, 256, [70001], 9001, 0, 0, 256, False, False),
    (128, 1, 32, [(37 * i) % 90 for i in range(200)], 33, 2, 3, 16, False, False),
])
def test_evict_matches(ctx, d, H, page, lens, keep, sinks, recent, to_page, beta, heads_first):  # noqa: F811
    p = Pages(20, lens, H, d, page, beta, heads_first)
    w = weights_of(p, 21)
    offset = [1000 * b for b in range(len(lens))]
    r = evict(ctx, p, w, keep, sinks, recent, to_page, offset, not heads_first)
    assert_evicted(p, w, keep, sinks, recent, r, offset)


@pytest.mark.parametrize("n", [100, 6000, 9000])
def test_ties_and_odd_weights(ctx, n):  # noqa: F811
    """Equal weights go to the lowest slots; zeros of both signs are equal; NaN is below all,
    infinities where they belong; few distinct bits in any step of the choice."""
    p = Pages(22, [n], 4, 64, 16)
    w = weights_of(p, 23)
    view = slots(p, w, 0)
    x = torch.zeros_like(view)
    x[:, 1] = (torch.arange(n, device=DEV) * 7919 % 13).float()
    x[::3, 0] = -0.0
    x[5::7, 2], x[6::7, 2], x[1::7, 2] = math.inf, NAN, -3.0
    x[:, 3] = 1 + torch.arange(n, device=DEV).remainder(700).float() * 2.0 ** -23
    j = torch.arange(n, device=DEV)
    w[p.table[0].long()[j // 16], :, j % 16] = x
    for keep, sinks, recent in ((16, 0, 0), (50, 3, 4), (n - 1, 0, 0), (n * 6 // 7 + 3, 1, 1)):
        r = evict(ctx, p, w, keep, sinks, recent, 16)
        assert_evicted(p, w, keep, sinks, recent, r)


def test_more_slots_than_a_cluster_holds(ctx):  # noqa: F811
    """Keys of a sequence beyond what its CTAs' shared memory holds are read again."""
    n = 8 * 48 * 1024 + 5000
    p = Pages.__new__(Pages)
    page = 256
    need = -(-n // page)
    p.H, p.d, p.page, p.lens, p.beta = 1, 64, page, [n], None
    p.K = torch.randn(need, page, 1, 64, device=DEV).bfloat16()
    p.V = torch.randn(need, page, 1, 64, device=DEV).bfloat16()
    p.table = torch.randperm(need, device=DEV).to(torch.int32)[None].contiguous()
    w = torch.rand(need, 1, page, device=DEV)
    r = evict(ctx, p, w, 4000, 4, 100, 16)
    x = slots(p, w, 0)[:, 0].clone()
    x[:4], x[-100:] = 2, 2
    want = torch.sort(x, descending=True, stable=True).indices[:4000].sort().values
    assert torch.equal(r["kept"][0, 0].long(), want)
    j = torch.arange(4000, device=DEV)
    assert torch.equal(r["K"][r["table"][0].long()[j // 16], j % 16, 0], p.rows(p.K, 0)[want, 0])


def test_within_one_pool_and_biases_of_none(ctx):  # noqa: F811
    """Into free pages of the same pool; a cache with biases takes 0 from one without."""
    p = Pages(24, [300, 90], 2, 64, 16, spare=12)
    w = weights_of(p, 25)
    used = set(p.table.flatten().tolist())
    free = [x for x in range(p.K.shape[0]) if x not in used][:8]
    table = i32([free[:4], free[4:]])
    K0 = p.K.clone()
    beta = torch.full((p.K.shape[0], 2, 16), NAN, device=DEV)
    kept, lens = torch.empty(2, 2, 50, dtype=torch.int32, device=DEV), i32([0, 0])
    still.still_paged_evict(ctx, p.cache(), batch_of(p), w, 50, 2, 8,
                            still.PagedCache(p.K, p.V, beta), table, kept, lens)
    for b in range(2):
        for h in range(2):
            j = chosen(slots(p, w, b)[:, h], 50, 2, 8)
            assert torch.equal(kept[b, h].long(), j)
            r = torch.arange(50, device=DEV)
            to = table[b].long()[r // 16]
            assert torch.equal(p.K[to, r % 16, h], K0[p.table[b].long()[j // 16], j % 16, h])
            assert (beta[to, h, r % 16] == 0).all()


# ------------------------------------------------------------------------------ together

def test_a_prompt_weighed_evicted_held_in_8_bits_and_decoded(ctx):  # noqa: F811
    """Append, weights of a window, eviction, the rest into a cache of 8 bits, and decoding on: each
    call's result from the one before it, the last against 64 bits, captured and replayed on a side
    stream."""
    H, g, d, page, keep = 2, 4, 128, 32, 96
    lens = [500, 80, 333]
    B = len(lens)
    p = Pages(30, lens, H, d, page)
    cache = p.cache()
    qkv = fused_rows(31, sum(lens), [H * g, H, H], d)
    qo = torch.empty(sum(lens), H * g, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_append(ctx, cache, batch_of(p, lens), *qkv[1:], q=qkv[0], q_out=qo,
                             rope_theta=1e4)
    window = 16
    ends = [sum(lens[:b + 1]) for b in range(B)]
    last = torch.cat([qo[e - window:e] for e in ends])
    w = weights_of(p, 32, fill=NAN)
    before = w.clone()
    still.still_paged_weigh(ctx, cache, batch_of(p, [window] * B), last, w,
                            scratch_of(p, B * window, H * g), decay=0.0)
    assert_weights(p, w, before, weighed64(p, last, [window] * B, before, 0.0))
    r = evict(ctx, p, w, keep, 4, window, page, offset=[0] * B)
    assert_evicted(p, w, keep, 4, window, r, [0] * B)
    # the kept rows of every sequence, as a pool of one page a sequence: packed rows
    kept = [min(x, keep) for x in lens]
    rows = [torch.cat([x[r["table"][b].long()].flatten(0, 1)[:kept[b]] for b in range(B)])
            for x in (r["K"], r["V"])]
    E4M3 = torch.float8_e4m3fn
    codes = [torch.zeros(B * 5, page, H, d, device=DEV, dtype=torch.uint8).view(E4M3) for _ in "KV"]
    scales = [torch.zeros(B * 5, H, page // 16, device=DEV) for _ in "KV"]
    table = torch.arange(B * 5, dtype=torch.int32, device=DEV).view(B, 5)
    held = still.PagedCacheQuant(*codes, *scales)
    cu = i32([0] + kept).cumsum(0).to(torch.int32)
    still.still_paged_append_quant(ctx, held, still.PagedBatch(table, r["lens"], cu), *rows)
    now, off = r["lens"].clone(), r["offset"]
    q, k, v = (x.contiguous() for x in fused_rows(33, B, [H * g, H, H], d))
    q2, out = torch.empty_like(q), torch.empty_like(q)
    batch = still.PagedBatch(table, now, None, off)
    still.still_paged_decode_quant(ctx, held, batch, q, out)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            now.add_(1)
            still.still_paged_append_quant(ctx, held, batch, k, v, q=q, q_out=q2, rope_theta=1e4,
                                           stream=stream)
            still.still_paged_decode_quant(ctx, held, batch, q2, out, stream=stream)
        for _ in range(20):
            graph.replay()
        stream.synchronize()
    assert now.tolist() == [x + 20 for x in kept]
    full = Pages.__new__(Pages)
    full.H, full.d, full.page, full.lens, full.beta, full.table = H, d, page, now.tolist(), None, table
    full.K, full.V = (c.float().double() * s.double().transpose(1, 2).repeat_interleave(16, 1)[
        ..., None] for c, s in zip(codes, scales))
    assert_rows(out, *attention64(full, q2, [1] * B), WEIGHTS)
    # the codes are the kept rows, each off by 2^-4 of itself or 2^-18 of its block's largest; the
    # block that decoding went on in may have been brought to a larger scale
    for b in range(B):
        whole = kept[b] // 16 * 16
        x = rows[0][sum(kept[:b]):][:whole].double()
        y = full.K[table[b].long()].flatten(0, 1)[:whole]
        top = x.abs().view(-1, 16, H, d).amax((1, 3)).repeat_interleave(16, 0)[..., None]
        assert ((x - y).abs() <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -17 * top)).all()


def test_steps_that_keep_count(ctx):  # noqa: F811
    """Decode steps with weights beside them, captured: the sum of the steps; then evicted."""
    lens = [200, 64]
    p = Pages(40, [x + 12 for x in lens], 2, 128, 32)
    now = i32(lens)
    batch = still.PagedBatch(p.table, now)
    cache, sc = p.cache(), scratch_of(p, 2, 8)
    q, = fused_rows(41, 2, [8], 128)
    q = q.contiguous()
    out = torch.empty_like(q)
    p.lens = lens
    start = weights_of(p, 42)
    w = start.clone()
    still.still_paged_decode_weigh(ctx, cache, batch, q, out, w, sc)
    w.copy_(start)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            now.add_(1)
            still.still_paged_decode_weigh(ctx, cache, batch, q, out, w, sc, decay=0.9,
                                           stream=stream)
        want = start
        for step in range(12):
            q.copy_(fused_rows(50 + step, 2, [8], 128)[0])
            graph.replay()
            stream.synchronize()
            p.lens = [x + step + 1 for x in lens]
            after = weighed64(p, q, [1, 1], want, 0.9)
            want = want.clone()
            for b in range(2):
                j = torch.arange(p.lens[b], device=DEV)
                want[p.table[b].long()[j // 32], :, j % 32] = after[b].float()
            assert_rows(out, *attention64(p, q, [1, 1]), WEIGHTS)
    for b in range(2):
        x, y = slots(p, w, b).double(), slots(p, want, b).double()
        assert ((x - y).abs() <= 12 * OFF * y).all()
    r = evict(ctx, p, w, 50, 2, 10, 16)
    assert_evicted(p, w, 50, 2, 10, r)


def test_same_inputs_same_bits(ctx):  # noqa: F811
    p = Pages(60, [3000, 1, 700, 64, 5000], 2, 128, 64)
    new = [300, 1, 90, 64, 500]
    q, = fused_rows(61, sum(new), [8], 128)
    one = q[:5].contiguous()
    start = weights_of(p, 62)
    first = None
    for _ in range(5):
        a, b, out = start.clone(), start.clone(), torch.empty_like(one)
        still.still_paged_weigh(ctx, p.cache(), batch_of(p, new), q, a, scratch_of(p, sum(new), 8))
        still.still_paged_decode_weigh(ctx, p.cache(), batch_of(p), one, out, b, scratch_of(p, 5, 8))
        got = [x.view(torch.int32) for x in (a, b)] + [out]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(got, first))


def test_device_side_faults_are_recorded():
    c = still.still_create(0)
    try:
        def recorded():
            code, det = still.still_get_device_status(c)
            return still.STATUS[code] == "STILL_ERR_CUDA" and det[0] == 2
        p = Pages(70, [40], 1, 64, 16)
        q, = fused_rows(71, 1, [1], 64)
        many, = fused_rows(72, 40, [1], 64)
        out, w = torch.empty_like(q), weights_of(p, 73)
        good = p.table.clone()
        for bad in (-1, p.K.shape[0], 2 ** 31 - 1):
            p.table[0, 2] = bad
            still.still_paged_weigh(c, p.cache(), batch_of(p, [40]), many, w, scratch_of(p, 40, 1))
            assert recorded(), bad
            still.still_paged_decode_weigh(c, p.cache(), batch_of(p), q, out, w, scratch_of(p, 1, 1))
            assert recorded(), bad
            evict(c, p, w, 20, 0, 0, 16)
            assert recorded(), bad
        p.table.copy_(good)
        p.lens = [p.table.shape[1] * 16 + 1]
        p.table[0, 3:] = p.table[0, 0]
        for call in ("weigh", "decode", "evict"):
            if call == "weigh":
                still.still_paged_weigh(c, p.cache(), batch_of(p, [40]), many, w,
                                        scratch_of(p, 40, 1))
            elif call == "decode":
                still.still_paged_decode_weigh(c, p.cache(), batch_of(p), q, out, w,
                                               scratch_of(p, 1, 1))
            else:
                evict(c, p, w, 20, 0, 0, 16)
            assert recorded(), call
        p.lens = [40]
        r = evict(c, p, w, 20, 0, 0, 16)
        assert still.still_get_device_status(c)[0] == 0
        r["table"][0, 1] = -1
        to = still.PagedCache(r["K"], r["V"])
        still.still_paged_evict(c, p.cache(), batch_of(p), w, 20, 0, 0, to, r["table"], r["kept"],
                                r["lens"])
        assert recorded()
    finally:
        still.still_destroy(c)


def test_refusals(ctx):  # noqa: F811
    L = still.lib()
    p = Pages(80, [40], 2, 64, 16, beta=True)
    cache, batch, w = p.cache(), batch_of(p), weights_of(p, 81)
    q, _ = fused_rows(82, 1, [4, 4], 64)
    out = torch.empty(1, 4, 64, device=DEV, dtype=torch.bfloat16)
    sc = scratch_of(p, 1, 4)
    to_K, to_V = (torch.zeros(2, 16, 2, 64, device=DEV, dtype=torch.bfloat16) for _ in "KV")
    to = still.PagedCache(to_K, to_V, torch.zeros(2, 2, 16, device=DEV))
    table, kept = i32([[0, 1]]), torch.zeros(1, 2, 20, dtype=torch.int32, device=DEV)
    lens, off = i32([0]), torch.zeros(1, dtype=torch.int64, device=DEV)
    inv, uns, ali = "STILL_ERR_INVALID_ARG", "STILL_ERR_UNSUPPORTED", "STILL_ERR_ALIGNMENT"
    shape = "STILL_ERR_SHAPE"

    def changed(struct, **over):
        s = type(struct)()
        ctypes.pointer(s)[0] = struct
        for name, value in over.items():
            setattr(s, name, value)
        return ctypes.byref(s)

    def decode(c=ctx, cache=cache.ref, batch=batch.ref, q=q.data_ptr(), Hq=4, scale=0.0,
               out=out.data_ptr(), w=w.data_ptr(), decay=1.0, sc=sc.data_ptr(), n=sc.numel()):
        return still.STATUS[L.still_paged_decode_weigh(c, cache, batch, q, 512, Hq, scale, out, w,
                                                       decay, sc, n, None)]

    def weigh(c=ctx, cache=cache.ref, batch=batch.ref, t=1, q=q.data_ptr(), Hq=4, scale=0.0,
              w=w.data_ptr(), decay=1.0, sc=sc.data_ptr(), n=sc.numel()):
        return still.STATUS[L.still_paged_weigh(c, cache, batch, t, q, 512, Hq, scale, w, decay, sc,
                                                n, None)]

    def evict_(c=ctx, cache=cache.ref, batch=batch.ref, w=w.data_ptr(), keep=20, sinks=1, recent=2,
               to=to.ref, table=table.data_ptr(), s=2, pages=2, tw=None, kept=kept.data_ptr(),
               lens=lens.data_ptr(), off=off.data_ptr()):
        return still.STATUS[L.still_paged_evict(c, cache, batch, w, keep, sinks, recent, to, table,
                                                s, pages, tw, kept, lens, off, None)]

    assert decode() == weigh() == evict_() == "STILL_OK"
    for call in (decode, weigh):
        assert call(c=None) == call(cache=None) == call(batch=None) == call(q=None) == inv
        assert call(w=None) == call(sc=None) == call(Hq=3) == call(scale=-1.0) == inv
        assert call(decay=-0.1) == call(decay=1.5) == call(decay=NAN) == inv
        assert call(w=w.data_ptr() + 2) == call(sc=sc.data_ptr() + 8) == ali
        assert call(n=100) == shape
        assert call(cache=changed(cache.struct, page_size=48)) == uns
    assert decode(out=None) == inv and weigh(t=2) == inv
    assert decode(n=sc.numel() - 1) == shape
    assert decode(batch=changed(batch.struct, cu_new=lens.data_ptr())) == inv
    assert weigh(t=0, batch=changed(batch.struct, cu_new=lens.data_ptr())) == "STILL_OK"
    assert evict_(c=None) == evict_(cache=None) == evict_(batch=None) == evict_(to=None) == inv
    assert evict_(w=None) == evict_(kept=None) == evict_(lens=None) == evict_(table=None) == inv
    assert evict_(keep=0) == evict_(sinks=-1) == evict_(recent=-1) == inv
    assert evict_(sinks=11, recent=10) == evict_(s=1) == evict_(pages=0) == inv
    assert evict_(to=changed(to.struct, beta=None)) == inv
    assert evict_(keep=33) == evict_(to=changed(to.struct, n_kv_heads=1)) == shape
    assert evict_(to=changed(to.struct, head_dim=128)) == shape
    assert evict_(to=changed(to.struct, page_size=24)) == uns
    assert evict_(kept=kept.data_ptr() + 2) == evict_(off=off.data_ptr() + 4) == ali
    assert evict_(w=w.data_ptr() + 1) == evict_(tw=w.data_ptr() + 1) == ali
    assert evict_(off=None, tw=w.data_ptr()) == "STILL_OK"
    with pytest.raises(AssertionError):
        still.still_paged_weigh(ctx, cache, batch, q, w[:, :1], sc)
