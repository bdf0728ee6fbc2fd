"""The paged cache in 8 bits against plain 64-bit restatements: append with its scales, decode and
prefill attention, at the edges of blocks, pages, tiles and masks; refusals, streams, captured graphs
and large pools."""
import ctypes
import math

import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import (DEV, NAN, assert_rows, attention64, batch_of, ctx, fused_rows,  # noqa: F401
                            i32, rotate64)

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
BLOCK = 16


def least_scale(top):
    """The smallest power of two, 2^-126 at least, by which values up to `top` (64 bits) are 448 at
    most."""
    e = torch.ceil(torch.log2(top / 448)).clamp_min(-126)
    return torch.where(top > 0, torch.exp2(e), 2.0 ** -126)


class QuantPages:
    """A pool whose free slots hold NaN codes and whose free blocks have NaN scales, and B sequences
    with `lens` slots; K and V are the values that codes and scales stand for, as Pages has them."""

    def __init__(self, seed, lens, H, d, page, beta=False, heads_first=False, spare=2, size=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.H, self.d, self.page, self.lens = H, d, page, list(lens)
        need = [-(-x // page) for x in lens]
        n = sum(need) + spare
        shape = (n, H, page, d) if heads_first else (n, page, H, d)
        pool = lambda: torch.full(shape, 0x7f, device=DEV, dtype=torch.uint8).view(E4M3)
        self.codes = [pool(), pool()]
        if heads_first:
            self.codes = [x.transpose(1, 2) for x in self.codes]
        self.scales = [torch.full((n, H, page // BLOCK), NAN, device=DEV) for _ in "KV"]
        self.beta = torch.full((n, H, page), NAN, device=DEV) if beta else None
        order = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(lens), max(need + [1]) + 1), -7, dtype=torch.int32, device=DEV)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = order[at:at + k]
            at += k
            if k == 0:
                continue
            pages, m = self.table[b, :k].long(), lens[b]
            blocks = -(-m // BLOCK)
            for codes, scales in zip(self.codes, self.scales):
                x = torch.randn(blocks, BLOCK, H, d, generator=g, device=DEV)
                if size is not None:  # of every block
                    x *= size[torch.randint(0, len(size), (blocks,), generator=g, device=DEV)][
                        :, None, None, None]
                s = least_scale(x.abs().amax((1, 3)).double()).float()  # [blocks, H]
                c = (x / s[:, None, :, None]).to(E4M3).view(torch.uint8).flatten(0, 1)[:m]
                c = torch.cat([c, torch.full((k * page - m, H, d), 0x7f, device=DEV,
                                             dtype=torch.uint8)])
                codes.view(torch.uint8)[pages] = c.view(k, page, H, d)
                s = torch.cat([s, torch.full((k * page // BLOCK - blocks, H), NAN, device=DEV)])
                scales[pages] = s.view(k, -1, H).transpose(1, 2)
            if beta:
                x = torch.randn(k * page, H, generator=g, device=DEV)
                x[m:] = NAN
                self.beta[pages] = x.view(k, page, H).transpose(1, 2)
        self.read()

    def read(self):
        self.K, self.V = (
            c.float().double() * s.double().transpose(1, 2).repeat_interleave(BLOCK, 1)[..., None]
            for c, s in zip(self.codes, self.scales))

    def cache(self):
        return still.PagedCacheQuant(*self.codes, *self.scales, self.beta)

    def rows(self, x, b):
        n = self.lens[b]
        pages = self.table[b, :-(-n // self.page)].long()
        if x is self.beta:
            return x[pages].permute(0, 2, 1).reshape(-1, self.H)[:n]
        return x[pages].reshape(-1, self.H, self.d)[:n]


# Logits are fp32 sums of exact products: WEIGHTS of the 16-bit cache without the rounding of weights
# to bf16, fp32 sums and exponentials (2^-11). Few rows: weights in fp16 hi + lo, 2^-21 of the largest
# weight times scale. Many rows: e4m3 hi (off by 2^-4 at most) + e5m2 lo (off by 2^-3 of that): 2^-7 of
# a weight, and 2^-17 of the largest one times its scale over 256 where lo is subnormal.
FEW = 2.0 ** -11 + 2.0 ** -20
MANY = 2.0 ** -7 + 2.0 ** -11


@pytest.mark.parametrize("d,H,Hq,page,lens,beta,heads_first", [
    (64, 1, 1, 16, [1], False, False),
    (64, 2, 6, 16, [0, 15, 16, 17, 33], True, True),
    (64, 1, 20, 64, [63, 64, 65, 300], False, False),
    (128, 2, 2, 16, [1, 2, 31, 127, 129], True, False),
    (128, 4, 28, 32, [777, 0, 1, 64], False, True),
    (128, 1, 16, 256, [255, 257, 1000], True, False),
    (128, 2, 16, 128, [5000], True, False),
    (256, 1, 3, 16, [1, 16, 47, 129], True, True),
    (256, 2, 16, 64, [65, 500], False, False),
    (256, 2, 4, 64, [30000], True, False),
    (128, 1, 7, 16, [20000, 40, 12000], False, True),
    (64, 1, 1, 256, [70000], False, False),
    (64, 1, 160, 32, [200, 31], True, False),
    (128, 1, 4, 16, [16], False, False),
    (128, 1, 5, 32, [(37 * i) % 90 for i in range(300)], False, False),
])
def test_decode_matches_64_bits(ctx, d, H, Hq, page, lens, beta, heads_first):  # noqa: F811
    p = QuantPages(1, lens, H, d, page, beta, heads_first)
    q, _ = fused_rows(2, len(lens), [Hq, 3], d)
    out = torch.full((len(lens), Hq, d), NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * len(lens)), MANY if Hq // H > 128 else FEW)


@pytest.mark.parametrize("d,H,Hq,page,new,past,beta,heads_first", [
    (64, 1, 1, 16, [1, 0, 3], [0, 5, 16], False, False),
    (64, 2, 6, 16, [40, 17], [0, 100], True, True),
    (128, 1, 4, 32, [130, 1, 64, 0], [0, 300, 63, 0], True, False),
    (128, 2, 14, 64, [37, 75], [129, 0], False, True),
    (128, 1, 1, 128, [257, 128], [1, 128], False, False),
    (128, 1, 16, 256, [33], [700], True, False),
    (256, 1, 2, 16, [129, 65], [0, 31], True, False),
    (256, 2, 10, 32, [30], [99], False, True),
    (128, 1, 4, 16, [3, 70], [2000, 1500], True, False),
    (128, 8, 32, 64, [700, 513, 1], [900, 3, 128], False, False),
    (128, 8, 24, 32, [600, 1, 999], [0, 77, 1500], True, True),
    (128, 1, 4, 256, [64], [9000], True, True),
    (64, 8, 8, 16, [1500, 900], [0, 700], False, True),
    (64, 1, 48, 128, [31, 5], [3000, 0], True, False),
    (256, 8, 16, 16, [700, 90, 350], [0, 1000, 64], False, False),
    (256, 2, 4, 64, [100], [5000], True, False),
    (256, 1, 128, 32, [3], [700], True, False),
    (256, 4, 8, 256, [900, 0, 65], [300, 5, 0], False, False),
    (64, 1, 200, 16, [3, 1], [70, 0], False, False),
    (128, 1, 2, 16, [(7 * i) % 23 for i in range(300)], [(11 * i) % 50 for i in range(300)], True,
     False),
])
def test_prefill_matches_64_bits(ctx, d, H, Hq, page, new, past, beta, heads_first):  # noqa: F811
    p = QuantPages(3, [a + b for a, b in zip(new, past)], H, d, page, beta, heads_first)
    q, _ = fused_rows(4, sum(new), [Hq, 1], d)
    out = torch.full((sum(new), Hq, d), NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, out)
    assert_rows(out, *attention64(p, q, new), MANY)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 70])
def test_blocks_of_very_different_sizes(ctx, d, new):  # noqa: F811
    """Scales from 2^-40 to 2^30 side by side: an error is measured by the row's largest weight times
    scale, of which every code (448 at most) is a multiple."""
    sizes = torch.tensor([2.0 ** -40, 2.0 ** -20, 1.0, 3.0, 2.0 ** 18, 2.0 ** 30], device=DEV)
    p = QuantPages(5, [700, 90, 33], 1, d, 32, size=sizes)
    p.scales[0].copy_(torch.where(torch.isnan(p.scales[0]), NAN, 2.0 ** -8))  # keys alike
    p.read()
    n = new if new == 1 else [new, 70, 20]
    counts = [1] * 3 if new == 1 else n
    q, = fused_rows(6, sum(counts), [4], d)
    out = torch.full_like(q, NAN)
    call = still.still_paged_decode_quant if new == 1 else still.still_paged_prefill_quant
    call(ctx, p.cache(), batch_of(p, None if new == 1 else n), q, out)
    ref, size = attention64(p, q, counts)
    # sum_j p_j |v_j| of all channels together bounds the row's largest weight times scale times 224
    top = size.amax(-1, keepdim=True)
    tol = 2.0 ** -8 * ref.abs() + (FEW if new == 1 else MANY) * size
    tol += (2.0 ** -21 if new == 1 else 2.0 ** -17) * 700 * top
    assert torch.isfinite(out).all() and ((out.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_masked_slots_count_for_nothing(ctx, d):  # noqa: F811
    """Biases of -inf: NaN codes behind them stay there, and NaN scales of blocks that are masked
    whole; a row without a slot is zero."""
    lens = [40, 130, 16, 70]
    p = QuantPages(5, lens, 2, d, 16, beta=True)
    for b, (lo, hi) in enumerate([(0, 40), (3, 120), (15, 16), (0, 69)]):
        for j in range(lo, hi):
            page, at = int(p.table[b, j // 16]), j % 16
            p.beta[page, :, at] = -math.inf
            for x in p.codes:
                x.view(torch.uint8)[page, at] = 0xff if j % 2 else 0x7f
    for b, j in ((0, 0), (0, 32), (1, 64), (3, 48)):
        for s in p.scales:
            s[int(p.table[b, j // 16])] = NAN
    p.read()
    q, = fused_rows(6, 4, [6], d)
    out = torch.empty_like(q)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * 4), FEW)
    assert (out[0] == 0).all()
    new = [40, 65, 1, 70]
    q, = fused_rows(7, sum(new), [6], d)
    out = torch.empty_like(q)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, new), q, out)
    assert_rows(out, *attention64(p, q, new), MANY)
    assert (out[:40] == 0).all() and (out[106:175] == 0).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_biases_of_the_lowest_size_and_nan(ctx, d):  # noqa: F811
    """Biases of the type's lowest value weigh nothing beside others and evenly among themselves; a
    NaN code or query gives NaN where the formula does."""
    p = QuantPages(8, [50, 33, 33], 1, d, 32, beta=True)
    low = torch.finfo(torch.float32).min
    for j in range(49):
        p.beta[int(p.table[0, j // 32]), :, j % 32] = low
    for j in range(33):
        p.beta[int(p.table[1, j // 32]), :, j % 32] = low
        p.codes[0].view(torch.uint8)[int(p.table[1, j // 32]), j % 32] = 0
    p.codes[1].view(torch.uint8)[int(p.table[2, 1]), 0, 0, 11] = 0x7f
    p.read()
    q, = fused_rows(9, 3, [4], d)
    for call, new in ((still.still_paged_decode_quant, None),
                      (still.still_paged_prefill_quant, [1, 1, 1])):
        out = torch.empty_like(q)
        call(ctx, p.cache(), batch_of(p, new), q, out)
        last = p.rows(p.V, 0)[49, 0]
        assert ((out[0].double() - last).abs() <= 2.0 ** -8 * last.abs()).all()
        mean = p.rows(p.V, 1)[:, 0]
        assert_rows(out[1:2], mean.mean(0).expand(1, 4, d), mean.abs().mean(0).expand(1, 4, d), MANY)
        hit = torch.arange(d, device=DEV) == 11
        assert torch.isnan(out[2][:, hit]).all() and torch.isfinite(out[2][:, ~hit]).all()
    q[0, 2, 5] = math.inf
    out = torch.empty_like(q)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    assert torch.isnan(out[0, 2]).all() and torch.isfinite(out[0, [0, 1, 3]]).all()


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -30, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("new", [1, 40])
def test_queries_of_any_size(ctx, size, new):  # noqa: F811
    """Logits of ordinary size from very large or small queries: `scale` makes up for it."""
    p = QuantPages(10, [300, 77], 1, 128, 16)
    q, = fused_rows(11, 2 * new, [4], 128)
    big = (q.float() * size).bfloat16()
    out = torch.empty_like(big)
    batch = batch_of(p, [new] * 2)
    still.still_paged_prefill_quant(ctx, p.cache(), batch, big, out, scale=128 ** -0.5 / size)
    assert_rows(out, *attention64(p, q, [new] * 2), MANY)


def test_more_new_tokens_than_slots(ctx):  # noqa: F811
    p = QuantPages(10, [20, 0], 1, 128, 16)
    q, = fused_rows(11, 37, [5], 128)
    out = torch.full_like(q, NAN)
    still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, [32, 5]), q, out)
    assert_rows(out, *attention64(p, q, [32, 5]), MANY)
    assert (out[:12] == 0).all() and (out[32:] == 0).all()


def test_a_token_alone_and_as_the_last_of_many(ctx):  # noqa: F811
    lens = [3000, 70, 41, 900]
    for d in (64, 128, 256):
        p = QuantPages(102, lens, 2, d, 32, beta=True)
        q, = fused_rows(103, 4 * 33, [8], d)
        many = torch.full_like(q.contiguous(), NAN)
        still.still_paged_prefill_quant(ctx, p.cache(), batch_of(p, [33] * 4), q, many)
        last = q[32::33].contiguous()
        one = torch.full_like(last, NAN)
        still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), last, one)
        ref, size = attention64(p, last, [1] * 4)
        assert ((one.double() - many[32::33].double()).abs()
                <= 2.0 ** -7 * ref.abs() + (FEW + MANY) * size).all()


# ------------------------------------------------------------------------------ append

def put64(codes, scales, x, slots, pages, page):
    """x [n, H, d] (as a 16-bit cache holds it) in consecutive slots, block by block, the codes by
    the type's own rounding."""
    at = 0
    while at < len(slots):
        j = int(slots[at])
        n = min(len(slots) - at, BLOCK - j % BLOCK)
        p, i = int(pages[at]), j % page
        rows = x[at:at + n].double()
        finite = torch.where(torch.isfinite(rows), rows.abs(), 0.0)
        s = least_scale(finite.amax((0, 2)))
        block = slice(i // BLOCK * BLOCK, i)
        if j % BLOCK:
            old = scales[p, :, i // BLOCK].double()
            s = torch.maximum(s, old)
            held = codes[p, block].float().double()
            codes.view(torch.uint8)[p, block] = (held * (old / s)[:, None]).float().to(E4M3).view(
                torch.uint8)
        scales[p, :, i // BLOCK] = s.float()
        c = (rows / s[:, None]).clamp(-448, 448).float().to(E4M3)
        codes.view(torch.uint8)[p, i:i + n] = c.view(torch.uint8)
        at += n


def same(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("d,H,Hq,page,new,past,offset,beta,heads_first,theta", [
    (64, 1, 1, 16, None, [0], None, False, False, 1e4),
    (64, 2, 8, 16, None, [15, 16, 31, 0, 200], [0, 5, 1 << 20, 7, 1], True, True, 1e4),
    (128, 8, 32, 64, [3, 0, 130, 1], [63, 9, 1, 64], [160000, 0, 3, 1], False, False, 1e6),
    (128, 2, 2, 32, [33, 70], [31, 0], None, True, False, 1e6),
    (256, 1, 3, 128, [129, 1], [0, 127], [0, (1 << 31) - 200], True, True, 1e6),
    (128, 1, 0, 16, [2500], [5], None, False, False, 1e6),
    (128, 2, 0, 32, [164, 1, 0, 17], [0, 0, 0, 3], None, True, False, 0.0),
    (256, 3, 0, 16, [40, 1, 0, 17, 2], [0, 15, 0, 3, 31], None, True, True, 0.0),
    (64, 1, 0, 64, [5, 3, 1, 2] * 30, [(5 * i) % 37 for i in range(120)], None, False, False, 0.0),
])
def test_append_matches_64_bits(ctx, d, H, Hq, page, new, past, offset, beta, heads_first,  # noqa: F811
                                theta):
    counts = new or [1] * len(past)
    n = sum(counts)
    p = QuantPages(14, past, H, d, page, beta, heads_first, spare=2 + len(past) + n // page)
    full = QuantPages(15, [a + b for a, b in zip(counts, past)], H, d, page)  # its table
    taken = 0
    spare = [x for x in range(p.codes[0].shape[0]) if not (p.table == x).any()]
    table = torch.full_like(full.table, -7)
    table[:, :p.table.shape[1]] = p.table[:, :table.shape[1]]
    for b, x in enumerate(full.lens):
        for i in range(-(-past[b] // page), -(-x // page)):
            table[b, i] = spare[taken]
            taken += 1
    p.table, p.lens = table, full.lens
    q, k, v = fused_rows(15, n, [Hq, H, H], d)
    new_beta = torch.randn(n, H, device=DEV) if beta and not theta else None
    qo = torch.full((n, Hq, d), NAN, device=DEV, dtype=torch.bfloat16) if Hq else None
    want = [x.clone() for x in p.codes], [x.clone() for x in p.scales]
    b0 = p.beta.clone() if beta else None
    still.still_paged_append_quant(ctx, p.cache(), batch_of(p, new, offset), k, v,
                                   q=q if Hq else None, q_out=qo, beta=new_beta, rope_theta=theta)
    at = 0
    for b, m in enumerate(counts):
        rows = slice(at, at + m)
        at += m
        slots = torch.arange(past[b], past[b] + m, device=DEV)
        pos = slots + (offset[b] if offset else 0)
        pages = p.table[b].long()[slots // page]
        x = k[rows]
        if theta:
            if Hq:
                ref = rotate64(q[rows], pos, theta)
                # as the 16-bit cache's test
                assert ((qo[rows].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18).all()
            x = rotate64(x, pos, theta).bfloat16()
        put64(want[0][0], want[1][0], x, slots, pages, page)
        put64(want[0][1], want[1][1], v[rows], slots, pages, page)
        if beta:
            b0[pages, :, slots % page] = (new_beta[rows] if new_beta is not None
                                          else torch.zeros(m, H, device=DEV))
    assert same(p.codes[1], want[0][1]) and same(p.scales[1], want[1][1])
    if theta:
        # a rotated key may round to the other side, in bf16 and then as a code: one step, 2^-3 of it
        # or 2^-9; the scales follow the same bits unless a largest value lies at a border
        assert same(p.scales[0], want[1][0])
        a, b = p.codes[0].float(), want[0][0].float()
        fine = torch.isnan(a) & torch.isnan(b)
        off = (a - b).abs() > torch.maximum(2.0 ** -3 * b.abs(), torch.tensor(2.0 ** -9))
        assert not (off & ~fine).any()
        assert ((a != b) & ~fine).sum() <= 1e-3 * a.numel() + 1
    else:
        assert same(p.codes[0], want[0][0]) and same(p.scales[0], want[1][0])
    assert not beta or same(p.beta, b0)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_block_that_grows(ctx, d):  # noqa: F811
    """Token by token, rows of sizes up and down: every step's scale and codes."""
    H, page = 2, 32
    p = QuantPages(20, [0], H, d, page, spare=2)
    p.table = i32([[1, 0]])
    codes, scales = [x.clone() for x in p.codes], [x.clone() for x in p.scales]
    sizes = [1, 2.0 ** -30, 2.0 ** 7, 3, 0, 2.0 ** 20, 2.0 ** 19, 1e30, 1, 0, 0, 447, 449, 2.0 ** -120,
             1, 1, 0, 2.0 ** -140, 2.0 ** -9, 1, 1e38]
    for j, size in enumerate(sizes):
        k, v = fused_rows(21 + j, 1, [H, H], d)
        k, v = (k.float() * size).bfloat16(), (v.float() / 7 * size).bfloat16()
        p.lens = [j + 1]
        still.still_paged_append_quant(ctx, p.cache(), batch_of(p), k, v)
        for i, x in enumerate((k, v)):
            put64(codes[i], scales[i], x, [j], [int(p.table[0, j // page])], page)
            assert same(p.codes[i], codes[i]) and same(p.scales[i], scales[i]), (j, size)


def test_append_of_nan_and_infinities(ctx):  # noqa: F811
    """NaN stays NaN, infinities become the block's largest code, neither moves the scale."""
    p = QuantPages(22, [0], 1, 64, 16, spare=3)
    p.table = i32([[1, 2]])
    p.lens = [20]
    k, v = fused_rows(23, 20, [1, 1], 64)
    k, v = k.contiguous(), v.contiguous()
    k[3, 0, 7], k[4, 0, 8], k[5, 0, 9], v[17, 0] = NAN, math.inf, -math.inf, math.inf
    still.still_paged_append_quant(ctx, p.cache(), batch_of(p, [20]), k, v)
    got = p.codes[0].float()
    assert torch.isnan(got[1, 3, 0, 7]) and got[1, 4, 0, 8] == 448 and got[1, 5, 0, 9] == -448
    assert torch.isfinite(p.scales[0][1]).all()
    fine = torch.where(torch.isfinite(k[:16]), k[:16].double().abs(), 0.0)
    assert p.scales[0][1, 0, 0] == least_scale(fine.amax())
    assert (p.codes[1].float()[2, 1] == 448).all()


def test_append_idle_places(ctx):  # noqa: F811
    p = QuantPages(16, [0, 3], 1, 64, 16)
    codes = p.codes[0].clone()
    k, v = fused_rows(18, 6, [1, 1], 64)
    # sequence 0 has no slots and one new token, sequence 1 three slots and five new tokens
    still.still_paged_append_quant(ctx, p.cache(), batch_of(p, [1, 5]), k, v)
    page = int(p.table[1, 0])
    s = p.scales[0][page, 0, 0]
    assert s == least_scale(k[3:6].double().abs().amax())
    want = (k[3:6].float() / s).to(E4M3)
    assert same(p.codes[0][page, :3], want)
    codes.view(torch.uint8)[page, :3] = want.view(torch.uint8)
    assert same(p.codes[0], codes)


# ------------------------------------------------------------------------------ surroundings

def test_append_then_attend_and_captured_lengths(ctx):  # noqa: F811
    """Appends and decodes of a captured step follow the arrays' values when it is replayed, on a
    side stream; the values are what a 16-bit cache would give, up to the codes' rounding."""
    H, d, page = 2, 128, 32
    p = QuantPages(24, [0, 0], H, d, page, spare=12)
    p.table = torch.arange(12, dtype=torch.int32, device=DEV).view(2, 6)
    cache = p.cache()
    lens, off = i32([0, 0]), torch.tensor([1000, 0], device=DEV)
    batch = still.PagedBatch(p.table, lens, None, off)
    q, k, v = (x.contiguous() for x in fused_rows(25, 2, [8, H, H], d))
    qo, out = torch.empty_like(q), torch.empty_like(q)
    still.still_paged_decode_quant(ctx, cache, batch, q, out)  # the workspace, outside the capture
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            still.still_paged_append_quant(ctx, cache, batch, k, v, q=q, q_out=qo, rope_theta=1e4,
                                           stream=stream)
            still.still_paged_decode_quant(ctx, cache, batch, qo, out, stream=stream)
        for step in range(70):
            for x, y in zip((q, k, v), fused_rows(30 + step, 2, [8, H, H], d)):
                x.copy_(y)
            n = [step + 1, max(0, step - 20)]
            lens.copy_(i32(n))
            graph.replay()
            stream.synchronize()
            if step % 23 == 22 or step == 69:
                p.lens = n
                p.read()
                assert_rows(out, *attention64(p, qo, [1, 1]), FEW)


def test_offsets_beyond_32_bits(ctx):  # noqa: F811
    """A page beyond 2^32 elements of its pool."""
    n_pages, page, H, d = 1 << 14, 64, 32, 128
    K = torch.empty(n_pages + 1, page, H, d, device=DEV, dtype=torch.uint8).view(E4M3)
    V = torch.empty(n_pages + 1, page, H, d, device=DEV, dtype=torch.uint8).view(E4M3)
    scales = [torch.empty(n_pages + 1, H, page // BLOCK, device=DEV) for _ in "KV"]
    table = i32([[n_pages, 3]])
    k, v, q = fused_rows(21, 100, [H, H, H], d)
    cache = still.PagedCacheQuant(K, V, *scales)
    batch = still.PagedBatch(table, i32([100]), i32([0, 100]))
    still.still_paged_append_quant(ctx, cache, batch, k, v)
    p = QuantPages.__new__(QuantPages)
    p.H, p.d, p.page, p.lens, p.beta = H, d, page, [100], None
    p.codes = [torch.stack([x[n_pages], x[3]]) for x in (K, V)]
    p.scales = [torch.stack([x[n_pages], x[3]]) for x in scales]
    p.table = i32([[0, 1]])
    p.codes = [x.clone() for x in p.codes]
    for x in p.codes:
        x.view(torch.uint8)[1, 36:] = 0
    for x in p.scales:
        x[1, :, 3:] = 1
    p.read()
    assert ((p.rows(p.K, 0) - k.double()).abs() <= 2.0 ** -4 * k.double().abs() + 2.0 ** -9).all()
    out = torch.empty(100, H, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill_quant(ctx, cache, batch, q, out)
    assert_rows(out, *attention64(p, q, [100]), MANY)
    one = torch.empty(1, H, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode_quant(ctx, cache, still.PagedBatch(table, i32([100])), q[99:], one)
    assert_rows(one, *attention64(p, q[99:], [1]), FEW)


def test_same_inputs_same_bits(ctx):  # noqa: F811
    p = QuantPages(24, [3000, 1, 700, 64, 5000], 2, 128, 64)
    small = QuantPages(26, [20], 1, 64, 16)
    q2, = fused_rows(27, 1, [1], 64)
    for new in (None, [300, 1, 90, 64, 500]):
        q, = fused_rows(25, 5 if new is None else sum(new), [8], 128)
        call = still.still_paged_decode_quant if new is None else still.still_paged_prefill_quant
        first = torch.empty(q.shape, device=DEV, dtype=torch.bfloat16)
        call(ctx, p.cache(), batch_of(p, new), q, first)
        for _ in range(10):
            still.still_paged_decode_quant(ctx, small.cache(), batch_of(small), q2,
                                           torch.empty_like(q2))
            out = torch.empty_like(first)
            call(ctx, p.cache(), batch_of(p, new), q, out)
            assert torch.equal(out, first)


def test_device_side_faults_are_recorded():
    c = still.still_create(0)
    try:
        def recorded():
            code, det = still.still_get_device_status(c)
            return still.STATUS[code] == "STILL_ERR_CUDA" and det[0] == 2
        p = QuantPages(30, [40], 1, 64, 16)
        q, k, v = fused_rows(31, 1, [1, 1, 1], 64)
        many, = fused_rows(34, 40, [1], 64)
        out = torch.empty(1, 1, 64, device=DEV, dtype=torch.bfloat16)
        good = p.table.clone()
        for bad in (-1, p.codes[0].shape[0], 2 ** 31 - 1):
            p.table[0, 2] = bad
            batch = batch_of(p)
            still.still_paged_append_quant(c, p.cache(), batch, k, v)
            assert recorded(), bad
            still.still_paged_decode_quant(c, p.cache(), batch, q, out)
            assert recorded(), bad
            still.still_paged_prefill_quant(c, p.cache(), batch_of(p, [40]), many,
                                            torch.empty_like(many))
            assert recorded(), bad
        p.table.copy_(good)
        cap = p.table.shape[1] * 16
        p.table[0, 3:] = p.table[0, 0]
        for lens, cu in (([cap + 1], None), ([-1], None), ([20], [0, 2]), ([20], [-1, 1]),
                         ([20], [1, 0])):
            b = still.PagedBatch(p.table, i32(lens), None if cu is None else i32(cu))
            still.still_paged_prefill_quant(c, p.cache(), b, q, out)
            assert recorded(), (lens, cu)
            still.still_paged_append_quant(c, p.cache(), b, k, v)
            assert recorded(), (lens, cu)
        still.still_paged_decode_quant(c, p.cache(), batch_of(p), q, out)
        assert still.still_get_device_status(c)[0] == 0
    finally:
        still.still_destroy(c)


def test_refusals(ctx):  # noqa: F811
    L = still.lib()
    p = QuantPages(32, [40], 2, 64, 16, beta=True)
    cache, batch = p.cache(), batch_of(p)
    q, k, v = fused_rows(33, 1, [4, 2, 2], 64)
    beta = torch.zeros(1, 2, device=DEV)
    out = torch.empty(1, 4, 64, device=DEV, dtype=torch.bfloat16)
    pitch = 8 * 64

    def changed(struct, **over):
        s = type(struct)()
        ctypes.pointer(s)[0] = struct
        for name, value in over.items():
            setattr(s, name, value)
        return ctypes.byref(s)

    def decode(cache=cache.ref, batch=batch.ref, q=q.data_ptr(), s=pitch, Hq=4, scale=0.0,
               out=out.data_ptr(), c=ctx):
        return still.STATUS[L.still_paged_decode_quant(c, cache, batch, q, s, Hq, scale, out, None)]

    def prefill(n=1, q=q.data_ptr()):
        return still.STATUS[L.still_paged_prefill_quant(ctx, cache.ref, batch.ref, n, q, pitch, 4,
                                                        0.0, out.data_ptr(), None)]

    def append(cache=cache.ref, n=1, k=k.data_ptr(), ks=pitch, q=q.data_ptr(), Hq=4,
               beta=beta.data_ptr(), theta=1e4, qo=out.data_ptr()):
        return still.STATUS[L.still_paged_append_quant(ctx, cache, batch.ref, n, k, ks,
                                                       v.data_ptr(), pitch, q, pitch, Hq, beta,
                                                       theta, qo, None)]

    cs = cache.struct
    assert decode() == prefill() == append() == "STILL_OK"
    inv, uns, ali = "STILL_ERR_INVALID_ARG", "STILL_ERR_UNSUPPORTED", "STILL_ERR_ALIGNMENT"
    for over, want in [
            (dict(K=None), inv), (dict(V=None), inv), (dict(k_scale=None), inv),
            (dict(v_scale=None), inv), (dict(n_pages=0), inv), (dict(s_page=0), inv),
            (dict(page_size=8), uns), (dict(page_size=48), uns), (dict(head_dim=96), uns),
            (dict(s_slot=cs.s_slot + 8), ali), (dict(s_head=72), ali), (dict(K=cs.K + 8), ali),
            (dict(k_scale=cs.k_scale + 2), ali), (dict(v_scale=cs.v_scale + 1), ali),
            (dict(beta=cs.beta + 2), ali)]:
        assert decode(cache=changed(cs, **over)) == want, over
        assert append(cache=changed(cs, **over)) == want, over
    assert decode(c=None) == decode(cache=None) == decode(batch=None) == inv
    assert decode(q=None) == decode(out=None) == decode(Hq=3) == decode(s=128) == inv
    assert decode(scale=-1.0) == decode(scale=NAN) == inv and decode(s=pitch + 4) == ali
    assert prefill(n=2) == prefill(n=-1) == prefill(q=None) == inv
    assert append(n=2) == append(k=None) == append(q=None) == append(qo=None) == inv
    assert append(theta=-1.0) == append(theta=0.0) == append(ks=64) == inv
    assert append(cache=changed(cs, beta=None)) == inv and append(k=k.data_ptr() + 2) == ali
    with pytest.raises(AssertionError):
        still.PagedCacheQuant(p.codes[0].view(torch.uint8), p.codes[1].view(torch.uint8), *p.scales)
    with pytest.raises(AssertionError):
        still.PagedCacheQuant(*p.codes, p.scales[0][:, :1], p.scales[1])
