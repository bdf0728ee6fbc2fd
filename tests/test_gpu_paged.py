"""The paged cache (App. B: compact caches installed in a serving engine's pages) against plain
64-bit restatements: append with rotation, decode and prefill attention, at the edges of pages,
tiles, groups of query heads and masks; refusals; streams, captured graphs and large pools."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import still

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NAN = float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = still.still_create(0)
    yield c
    code, det = still.still_get_device_status(c)
    still.still_destroy(c)
    assert code == 0, (still.STATUS[code], det)


class Pages:
    """A pool whose free slots hold NaN, and B sequences with `lens` slots of normal values."""

    def __init__(self, seed, lens, H, d, page, beta=False, heads_first=False, spare=2):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.H, self.d, self.page, self.lens = H, d, page, list(lens)
        need = [-(-x // page) for x in lens]
        n = sum(need) + spare
        shape = (n, H, page, d) if heads_first else (n, page, H, d)
        pool = lambda: torch.full(shape, NAN, device=DEV, dtype=torch.bfloat16)
        self.K, self.V = pool(), pool()
        if heads_first:
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        self.beta = torch.full((n, H, page), NAN, device=DEV) if beta else None
        order = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        # unused entries of the table name no page
        self.table = torch.full((len(lens), max(need + [1]) + 1), -7, dtype=torch.int32, device=DEV)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = order[at:at + k]
            at += k
            for j0 in range(0, lens[b], page):
                m = min(page, lens[b] - j0)
                p = int(self.table[b, j0 // page])
                rnd = lambda *s: torch.randn(s, generator=g, device=DEV)
                self.K[p, :m] = rnd(m, H, d).bfloat16()
                self.V[p, :m] = rnd(m, H, d).bfloat16()
                if beta:
                    self.beta[p, :, :m] = rnd(H, m)

    def cache(self):
        return still.PagedCache(self.K, self.V, self.beta)

    def rows(self, x, b):
        """The slots of sequence b: [len, H, ...] of K or V, or biases [len, H]."""
        n = self.lens[b]
        pages = self.table[b, :-(-n // self.page)].long()
        if x is self.beta:
            return x[pages].permute(0, 2, 1).reshape(-1, self.H)[:n]
        return x[pages].reshape(-1, self.H, self.d)[:n]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def batch_of(p, new=None, offset=None, lens=None):
    cu = None
    if new is not None:
        cu = i32([0] + new).cumsum(0).to(torch.int32)
    off = None if offset is None else torch.tensor(offset, dtype=torch.int64, device=DEV)
    return still.PagedBatch(p.table, i32(p.lens if lens is None else lens), cu, off)


def fused_rows(seed, n, heads, d):
    """Slices of a fused projection: [n, h, d] for every h of heads, one pitch."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, sum(heads) * d, generator=g, device=DEV).bfloat16()
    return [y.unflatten(1, (h, d)) for h, y in zip(heads, x.split([h * d for h in heads], 1))]


def attention64(p, q, new, scale=None):
    """Rows [n, Hq, d] and, per output, sum_j p_j |v_j| (the size that weights' errors act on)."""
    Hq, d = q.shape[1:]
    g = Hq // p.H
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    size = torch.zeros_like(out)
    at = 0
    for b, n in enumerate(new):
        L = p.lens[b]
        k, v = p.rows(p.K, b).double(), p.rows(p.V, b).double()
        see = torch.arange(L - n, L, device=DEV) + 1  # slots that each new token sees
        late = torch.arange(L, device=DEV) >= see[:, None]
        for h in range(p.H if n and L else 0):
            bias = p.rows(p.beta, b)[:, h].double() if p.beta is not None else torch.zeros(
                L, dtype=torch.float64, device=DEV)
            hidden = late | (bias == -math.inf)
            kh = torch.where((bias == -math.inf)[:, None], 0.0, k[:, h])
            vh = torch.where((bias == -math.inf)[:, None], 0.0, v[:, h])
            x = torch.einsum("nid,jd->nij", q[at:at + n, h * g:(h + 1) * g].double(), kh)
            x = (x * (scale or 1 / math.sqrt(d)) + bias).masked_fill(hidden[:, None], -math.inf)
            w = torch.softmax(x, -1)
            w = torch.where(hidden.all(-1)[:, None, None], 0.0, w)
            out[at:at + n, h * g:(h + 1) * g] = w @ vh
            size[at:at + n, h * g:(h + 1) * g] = w @ vh.abs()
        at += n
    return out, size


def assert_rows(got, ref, size, weights):
    # rounding to bf16 moves a value by at most 2^-9 of itself, taken twice; `weights`: relative
    # error of a softmax weight, which moves an output by that share of sum_j p_j |v_j|
    err = (got.double() - ref).abs()
    tol = 2.0 ** -8 * ref.abs() + weights * size
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), float((err / tol.clamp_min(1e-30)).max())


# A weight e^s may be rounded to bf16 (half an ulp, 2^-9, of it) if the sum of the weights takes it
# as rounded: an output moves by at most 2^-9 (sum_j p_j |v_j| + |o|) <= 2^-8 sum_j p_j |v_j|. fp32
# sums of up to 256 products of size about 1/16 .. 4 move s by less than 256 * 2^-24 * 10 = 2^-12.7,
# and the weight and the sum by as much.
WEIGHTS = 2.0 ** -8 + 2.0 ** -11


@pytest.mark.parametrize("d,H,Hq,page,lens,beta,heads_first", [
    (64, 1, 1, 16, [1], False, False),
    (64, 2, 6, 16, [0, 15, 16, 17, 33], True, True),
    (64, 1, 20, 64, [63, 64, 65, 300], False, False),
    (128, 2, 2, 16, [1, 2, 31, 127, 129], True, False),
    (128, 4, 28, 32, [777, 0, 1, 64], False, True),
    (128, 1, 16, 256, [255, 257, 1000], True, False),
    (128, 2, 16, 128, [5000], True, False),
    (256, 1, 3, 16, [1, 16, 47, 129], True, True),
    (256, 2, 18, 64, [65, 500], False, False),
    (256, 1, 33, 32, [100], False, False),
    # slots of one set in many warps, groups that fit no tile, ranges shorter than a CTA
    (256, 2, 4, 64, [30000], True, False),
    (128, 1, 7, 16, [20000, 40, 12000], False, True),
    (64, 1, 1, 256, [70000], False, False),
    (64, 1, 160, 32, [200, 31], True, False),
    (128, 1, 4, 16, [16], False, False),
])
def test_decode_matches_64_bits(ctx, d, H, Hq, page, lens, beta, heads_first):
    p = Pages(1, lens, H, d, page, beta, heads_first)
    q, _ = fused_rows(2, len(lens), [Hq, 3], d)
    out = torch.full((len(lens), Hq, d), NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * len(lens)), WEIGHTS)


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
    # several items per CTA, slots split over CTAs, every table of pages
    (128, 8, 32, 64, [700, 513, 1], [900, 3, 128], False, False),
    (128, 8, 24, 32, [600, 1, 999], [0, 77, 1500], True, True),
    (128, 1, 4, 64, [40], [9000], False, False),
    (128, 1, 4, 256, [64], [9000], True, True),
    (64, 8, 8, 16, [1500, 900], [0, 700], False, True),
    (64, 1, 48, 128, [31, 5], [3000, 0], True, False),
    (256, 8, 16, 16, [700, 90, 350], [0, 1000, 64], False, False),
    (256, 2, 4, 64, [100], [5000], True, False),
    (256, 1, 128, 32, [3], [700], True, False),
    (256, 2, 4, 128, [400, 30], [0, 1000], True, True),
    (256, 4, 8, 256, [900, 0, 65], [300, 5, 0], False, False),
    (256, 1, 1, 16, [130, 257, 1], [0, 128, 77], True, False),
    (256, 8, 24, 32, [333, 40, 700, 2], [0, 1500, 77, 0], True, True),
    # items in more ranges than a block of the join looks through alone
    (64, 1, 40, 16, [2], [9000], False, True),
    (128, 1, 24, 64, [1, 30], [20, 11000], True, False),
    (256, 1, 12, 16, [3], [9000], True, False),
    (256, 1, 16, 64, [20], [12000], True, False),
    (64, 1, 200, 16, [3, 1], [70, 0], False, False),
    (128, 1, 2, 16, [(7 * i) % 23 for i in range(500)], [(11 * i) % 50 for i in range(500)], True,
     False),
])
def test_prefill_matches_64_bits(ctx, d, H, Hq, page, new, past, beta, heads_first):
    p = Pages(3, [a + b for a, b in zip(new, past)], H, d, page, beta, heads_first)
    q, _ = fused_rows(4, sum(new), [Hq, 1], d)
    out = torch.full((sum(new), Hq, d), NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill(ctx, p.cache(), batch_of(p, new), q, out)
    assert_rows(out, *attention64(p, q, new), WEIGHTS)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_masked_slots_count_for_nothing(ctx, d):
    """Biases of -inf: NaN and infinities behind them stay there; a row without a slot is zero."""
    lens = [40, 130, 16, 70]
    p = Pages(5, lens, 2, d, 16, beta=True)
    for b, (lo, hi) in enumerate([(0, 40), (3, 120), (15, 16), (0, 69)]):
        for j in range(lo, hi):
            page, at = int(p.table[b, j // 16]), j % 16
            p.beta[page, :, at] = -math.inf
            p.K[page, at] = (NAN, math.inf, -math.inf)[j % 3]
            p.V[page, at] = (math.inf, NAN, -math.inf)[j % 3]
    q, = fused_rows(6, 4, [6], d)
    out = torch.empty_like(q)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * 4), WEIGHTS)
    assert (out[0] == 0).all()
    q, = fused_rows(7, 40 + 65 + 1 + 70, [6], d)
    out = torch.empty_like(q)
    new = [40, 65, 1, 70]
    still.still_paged_prefill(ctx, p.cache(), batch_of(p, new), q, out)
    assert_rows(out, *attention64(p, q, new), WEIGHTS)
    assert (out[:40] == 0).all() and (out[106:175] == 0).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_of_the_lowest_size_and_infinities(ctx, d):
    """Biases of the type's lowest value weigh nothing beside others and evenly among themselves;
    an infinite value stays in its channel; an infinite logit gives NaN, as the formula does."""
    lens = [50, 33, 33]
    p = Pages(8, lens, 1, d, 32, beta=True)
    low = torch.finfo(torch.float32).min
    for j in range(49):
        p.beta[int(p.table[0, j // 32]), :, j % 32] = low
    for j in range(33):
        p.beta[int(p.table[1, j // 32]), :, j % 32] = low
        p.K[int(p.table[1, j // 32]), j % 32] = 0
    p.V[int(p.table[2, 1]), 0, 0, 11] = math.inf
    q, = fused_rows(9, 3, [4], d)
    for call, new in ((still.still_paged_decode, None), (still.still_paged_prefill, [1, 1, 1])):
        out = torch.empty_like(q)
        call(ctx, p.cache(), batch_of(p, new), q, out)
        last = p.rows(p.V, 0)[49, 0].double()
        assert ((out[0].double() - last).abs() <= 2.0 ** -8 * last.abs()).all()
        mean = p.rows(p.V, 1)[:, 0].double()
        assert_rows(out[1:2], mean.mean(0).expand(1, 4, d), mean.abs().mean(0).expand(1, 4, d),
                    WEIGHTS)
        inf = torch.arange(d, device=DEV) == 11
        assert torch.isposinf(out[2][:, inf]).all() and torch.isfinite(out[2][:, ~inf]).all()
    q[0, 2, 5] = math.inf
    out = torch.empty_like(q)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    assert torch.isnan(out[0, 2]).all() and torch.isfinite(out[0, [0, 1, 3]]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_infinite_values_of_a_long_sequence(ctx, d):
    """Infinite values among slots that many warps share stay in their channels; two of opposite
    signs in one channel are NaN there."""
    p = Pages(40, [4000, 300], 1, d, 16)
    for j, c, x in ((17, 3, math.inf), (2500, 5, -math.inf), (3999, 9, math.inf),
                    (100, 9, -math.inf)):
        p.V[int(p.table[0, j // 16]), j % 16, 0, c] = x
    q, = fused_rows(41, 2, [4], d)
    out = torch.empty_like(q)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    assert torch.isposinf(out[0, :, 3]).all() and torch.isneginf(out[0, :, 5]).all()
    assert torch.isnan(out[0, :, 9]).all()
    rest = [c for c in range(d) if c not in (3, 5, 9)]
    assert torch.isfinite(out[0][:, rest]).all() and torch.isfinite(out[1]).all()


def test_more_new_tokens_than_slots(ctx):
    """Tokens before the first slot see nothing: zeros."""
    p = Pages(10, [20, 0], 1, 128, 16)
    q, = fused_rows(11, 37, [5], 128)
    out = torch.full_like(q, NAN)
    still.still_paged_prefill(ctx, p.cache(), batch_of(p, [32, 5]), q, out)
    ref, size = attention64(p, q, [32, 5])
    assert_rows(out, ref, size, WEIGHTS)
    assert (out[:12] == 0).all() and (out[32:] == 0).all()


def test_scale(ctx):
    p = Pages(12, [300], 1, 64, 16)
    q, = fused_rows(13, 1, [3], 64)
    out = torch.empty_like(q)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out, scale=0.03)
    assert_rows(out, *attention64(p, q, [1], 0.03), WEIGHTS)


# ------------------------------------------------------------------------------ append

def rotate64(x, pos, theta):
    half = x.shape[-1] // 2
    w = theta ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    a = (pos.double()[:, None] * w)[:, None]
    lo, hi = x[..., :half].double(), x[..., half:].double()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


@pytest.mark.parametrize("d,H,Hq,page,new,past,offset,beta,heads_first,theta", [
    (64, 1, 1, 16, None, [0], None, False, False, 1e4),
    (64, 2, 8, 16, None, [15, 16, 31, 0, 200], [0, 5, 1 << 20, 7, 1], True, True, 1e4),
    (128, 8, 32, 64, [3, 0, 130, 1], [63, 9, 1, 64], [160000, 0, 3, 1], False, False, 1e6),
    (128, 2, 2, 32, [33, 70], [31, 0], None, True, False, 1e6),
    (256, 1, 3, 128, [129, 1], [0, 127], [0, (1 << 31) - 200], True, True, 1e6),
    (128, 1, 0, 16, [2500], [5], None, False, False, 1e6),
    (128, 2, 0, 32, [164, 1, 0, 17], [0, 0, 0, 3], None, True, False, 0.0),
])
def test_append_matches_64_bits(ctx, d, H, Hq, page, new, past, offset, beta, heads_first, theta):
    counts = new or [1] * len(past)
    n = sum(counts)
    p = Pages(14, [a + b for a, b in zip(counts, past)], H, d, page, beta, heads_first)
    K0, V0 = p.K.clone(), p.V.clone()
    b0 = p.beta.clone() if beta else None
    q, k, v = fused_rows(15, n, [Hq, H, H], d)
    new_beta = torch.randn(n, H, device=DEV) if beta and not theta else None
    qo = torch.full((n, Hq, d), NAN, device=DEV, dtype=torch.bfloat16) if Hq else None
    still.still_paged_append(ctx, p.cache(), batch_of(p, new, offset), k, v,
                             q=q if Hq else None, q_out=qo, beta=new_beta, rope_theta=theta)
    at = 0
    for b, m in enumerate(counts):
        rows = slice(at, at + m)
        at += m
        slots = torch.arange(past[b], past[b] + m, device=DEV)
        pos = slots + (offset[b] if offset else 0)
        pages = p.table[b].long()[slots // page]
        for x, y in [(k, p.K[pages, slots % page])] + ([(q, qo[rows])] if Hq else []):
            if not theta:
                assert torch.equal(y, x[rows])
                continue
            ref = rotate64(x[rows], pos, theta)
            # bf16 rounding, and angles: 2^-32 turns, their fp32 form 2^-25, positions below 2^31
            # times a frequency of 53 bits 2^-22 rad; |x| < 8
            assert ((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18).all()
        assert torch.equal(p.V[pages, slots % page], v[rows])
        K0[pages, slots % page] = p.K[pages, slots % page]
        V0[pages, slots % page] = v[rows]
        if beta:
            want = new_beta[rows] if new_beta is not None else torch.zeros(m, H, device=DEV)
            assert torch.equal(p.beta[pages, :, slots % page], want)
            b0[pages, :, slots % page] = want
    # nothing else moved
    same = lambda x, y: torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16
                                    else x.view(torch.int32),
                                    y.view(torch.int16) if y.dtype == torch.bfloat16
                                    else y.view(torch.int32))
    assert same(p.K.contiguous(), K0.contiguous()) and same(p.V.contiguous(), V0.contiguous())
    assert not beta or same(p.beta, b0)


def test_append_idle_places_and_in_place_queries(ctx):
    p = Pages(16, [0, 3], 1, 64, 16)
    K0 = p.K.clone()
    q, = fused_rows(17, 9, [2], 64)
    k, v = fused_rows(18, 9, [1, 1], 64)
    q = q.contiguous()
    ref = rotate64(q[:6], i32([-1, -2, -1, 0, 1, 2]), 1e4)
    # sequence 0 has no slots and one new token, sequence 1 three slots and five new tokens
    still.still_paged_append(ctx, p.cache(), batch_of(p, [1, 5]), k[:6], v[:6], q=q[:6],
                             q_out=q[:6], rope_theta=1e4)
    assert ((q[:6].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18).all()
    page = int(p.table[1, 0])
    K0[page, :3] = p.K[page, :3]
    assert torch.isfinite(p.K[page, :3]).all() and torch.equal(p.V[page, :3], v[3:6])
    assert torch.equal(p.K.view(torch.int16), K0.view(torch.int16))


def test_append_then_attend(ctx):
    """Slots written by append are what the attention reads; decode equals prefill of one token."""
    p = Pages(19, [77, 130], 2, 128, 16, beta=True)
    cache, batch = p.cache(), batch_of(p, offset=[1000, 0])
    q, k, v = fused_rows(20, 2, [8, 2, 2], 128)
    qo, out = torch.empty(2, 8, 128, device=DEV, dtype=torch.bfloat16), None
    still.still_paged_append(ctx, cache, batch, k, v, q=q, q_out=qo, rope_theta=1e6)
    out = torch.empty_like(qo)
    still.still_paged_decode(ctx, cache, batch, qo, out)
    assert_rows(out, *attention64(p, qo, [1, 1]), WEIGHTS)
    two = torch.empty_like(qo)
    still.still_paged_prefill(ctx, cache, batch, qo, two)
    assert torch.equal(out, two)


# ------------------------------------------------------------------------------ surroundings

def test_offsets_beyond_32_bits(ctx):
    """A page beyond 2^32 elements of its pool."""
    n_pages, page, H, d = 1 << 14, 64, 32, 128  # 2^32 elements
    K = torch.empty(n_pages + 1, page, H, d, device=DEV, dtype=torch.bfloat16)
    V = torch.empty_like(K)
    lens = i32([100])
    table = i32([[n_pages, 3]])
    k, v, q = fused_rows(21, 100, [H, H, H], d)
    cache = still.PagedCache(K, V)
    batch = still.PagedBatch(table, lens, i32([0, 100]))
    qo = torch.empty(100, H, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_append(ctx, cache, batch, k, v, q=q, q_out=qo, rope_theta=1e6)
    assert torch.equal(V[n_pages], v[:64]) and torch.equal(V[3, :36], v[64:])
    p = Pages.__new__(Pages)
    p.H, p.d, p.page, p.lens, p.K, p.V, p.beta, p.table = H, d, page, [100], K, V, None, table
    one = still.PagedBatch(table, lens)
    out = torch.empty(1, H, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode(ctx, cache, one, qo[99:], out)
    assert_rows(out, *attention64(p, qo[99:], [1]), WEIGHTS)
    out = torch.empty(100, H, d, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill(ctx, cache, batch, qo, out)
    assert_rows(out, *attention64(p, qo, [100]), WEIGHTS)


def test_side_stream_and_captured_lengths(ctx):
    """Calls on a side stream; a captured step follows the arrays' values when replayed."""
    p = Pages(22, [200, 64], 2, 128, 32)
    batch = batch_of(p, lens=[150, 30])
    cache = p.cache()
    q, = fused_rows(23, 2, [8], 128)
    out = torch.empty(2, 8, 128, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode(ctx, cache, batch, q, out)  # the workspace grows outside the capture
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            still.still_paged_decode(ctx, cache, batch, q, out, stream=stream)
        for lens in ([150, 30], [200, 64], [0, 1]):
            batch.tensors[1].copy_(i32(lens))
            out.fill_(NAN)
            graph.replay()
            stream.synchronize()
            p.lens = lens
            assert_rows(out, *attention64(p, q, [1, 1]), WEIGHTS)


def test_same_inputs_same_bits(ctx):
    """Results do not depend on what ran before or on the order in which CTAs end."""
    p = Pages(24, [3000, 1, 700, 64, 5000], 2, 128, 64)
    q, = fused_rows(25, 5, [8], 128)
    first = torch.empty(5, 8, 128, device=DEV, dtype=torch.bfloat16)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, first)
    small = Pages(26, [20], 1, 64, 16)
    q2, = fused_rows(27, 1, [1], 64)
    for _ in range(20):
        still.still_paged_decode(ctx, small.cache(), batch_of(small), q2, torch.empty_like(q2))
        out = torch.empty_like(first)
        still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
        assert torch.equal(out, first)


def test_many_short_sequences(ctx):
    lens = [(37 * i) % 90 for i in range(700)]
    p = Pages(28, lens, 1, 64, 16)
    q, = fused_rows(29, 700, [2], 64)
    out = torch.full_like(q, NAN)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    assert_rows(out, *attention64(p, q, [1] * 700), WEIGHTS)


# ------------------------------------------------------------------------------ refusals

def test_device_side_faults_are_recorded():
    """Pages outside the pool, lengths beyond the table and bad offsets end in the error record;
    nothing outside the pool is read or written."""
    c = still.still_create(0)
    try:
        def recorded():
            code, det = still.still_get_device_status(c)
            return still.STATUS[code] == "STILL_ERR_CUDA" and det[0] == 2
        p = Pages(30, [40], 1, 64, 16)
        q, k, v = fused_rows(31, 1, [1, 1, 1], 64)
        out = torch.empty(1, 1, 64, device=DEV, dtype=torch.bfloat16)
        good = p.table.clone()
        for bad in (-1, p.K.shape[0], 2 ** 31 - 1):
            for call in ("append", "decode", "prefill", "prefill of many"):
                p.table[0, 2] = bad
                batch = batch_of(p)
                if call == "append":
                    still.still_paged_append(c, p.cache(), batch, k, v)
                elif call == "decode":
                    still.still_paged_decode(c, p.cache(), batch, q, out)
                elif call == "prefill of many":
                    many, = fused_rows(34, 40, [1], 64)
                    still.still_paged_prefill(c, p.cache(), batch_of(p, [40]), many,
                                              torch.empty_like(many))
                else:
                    still.still_paged_prefill(c, p.cache(), batch, q, out)
                assert recorded(), (bad, call)
        p.table.copy_(good)
        cap = p.table.shape[1] * 16
        p.table[0, 3:] = p.table[0, 0]
        for lens, cu in (([cap + 1], None), ([-1], None), ([20], [0, 2]), ([20], [-1, 1]),
                         ([20], [1, 0])):
            b = still.PagedBatch(p.table, i32(lens), None if cu is None else i32(cu))
            still.still_paged_prefill(c, p.cache(), b, q, out)
            assert recorded(), (lens, cu)
            still.still_paged_append(c, p.cache(), b, k, v)
            assert recorded(), (lens, cu)
        # the context stays usable
        still.still_paged_decode(c, p.cache(), batch_of(p), q, out)
        assert still.still_get_device_status(c)[0] == 0
    finally:
        still.still_destroy(c)


def test_refusals(ctx):
    import ctypes
    L = still.lib()
    p = Pages(32, [40], 2, 64, 16, beta=True)
    cache, batch = p.cache(), batch_of(p)
    q, k, v = fused_rows(33, 1, [4, 2, 2], 64)
    beta = torch.zeros(1, 2, device=DEV)
    out = torch.empty(1, 4, 64, device=DEV, dtype=torch.bfloat16)
    pitch = 8 * 64  # of the fused rows (a tensor of one row may report another)

    def changed(struct, **over):
        s = type(struct)()
        ctypes.pointer(s)[0] = struct
        for name, value in over.items():
            setattr(s, name, value)
        return ctypes.byref(s)

    def decode(cache=cache.ref, batch=batch.ref, q=q.data_ptr(), s=pitch, Hq=4, scale=0.0,
               out=out.data_ptr(), c=ctx):
        return still.STATUS[L.still_paged_decode(c, cache, batch, q, s, Hq, scale, out, None)]

    def prefill(n=1, batch=batch.ref, q=q.data_ptr()):
        return still.STATUS[L.still_paged_prefill(ctx, cache.ref, batch, n, q, pitch, 4, 0.0,
                                                  out.data_ptr(), None)]

    def append(cache=cache.ref, n=1, k=k.data_ptr(), ks=pitch, q=q.data_ptr(), Hq=4,
               beta=beta.data_ptr(), theta=1e4, qo=out.data_ptr(), qs=pitch):
        return still.STATUS[L.still_paged_append(ctx, cache, batch.ref, n, k, ks, v.data_ptr(),
                                                 pitch, q, qs, Hq, beta, theta, qo, None)]

    cs, bs = cache.struct, batch.struct
    assert decode() == prefill() == append() == "STILL_OK"
    inv, uns, ali = "STILL_ERR_INVALID_ARG", "STILL_ERR_UNSUPPORTED", "STILL_ERR_ALIGNMENT"
    for over, want in [
            (dict(K=None), inv), (dict(V=None), inv), (dict(n_pages=0), inv),
            (dict(n_kv_heads=0), inv), (dict(s_page=0), inv), (dict(s_slot=-64), inv),
            (dict(page_size=8), uns), (dict(page_size=48), uns), (dict(page_size=1 << 17), uns),
            (dict(head_dim=96), uns), (dict(n_kv_heads=2000), uns), (dict(s_slot=68), ali),
            (dict(K=cs.K + 2), ali), (dict(V=cs.V + 8), ali), (dict(beta=cs.beta + 2), ali)]:
        assert decode(cache=changed(cs, **over)) == want, over
        assert append(cache=changed(cs, **over)) == want, over
    for over, want in [
            (dict(table=None), inv), (dict(len=None), inv), (dict(B=0), inv),
            (dict(table_pages=0), inv), (dict(s_table=1), inv), (dict(cu_new=bs.len), inv),
            (dict(table=bs.table + 2), ali), (dict(len=bs.len + 1), ali),
            (dict(pos_offset=bs.len + 4), ali)]:
        assert decode(batch=changed(bs, **over)) == want, over
    assert decode(c=None) == decode(cache=None) == decode(batch=None) == inv
    assert decode(q=None) == decode(out=None) == decode(Hq=3) == decode(Hq=1) == inv
    assert decode(s=pitch + 4) == ali and decode(s=128) == inv
    assert decode(scale=-1.0) == decode(scale=NAN) == decode(scale=math.inf) == inv
    assert decode(q=q.data_ptr() + 2) == decode(out=out.data_ptr() + 8) == ali
    assert prefill(n=2) == prefill(n=-1) == prefill(q=None) == inv
    assert prefill(n=0, batch=changed(bs, cu_new=bs.len)) == "STILL_OK"
    assert append(n=2) == append(k=None) == append(q=None) == append(Hq=0) == append(qo=None) == inv
    assert append(theta=-1.0) == append(theta=NAN) == append(theta=0.0) == append(ks=64) == inv
    assert append(cache=changed(cs, beta=None)) == inv and append(qo=q.data_ptr()) == inv
    assert append(k=k.data_ptr() + 2) == append(beta=beta.data_ptr() + 1) == ali
    with pytest.raises(AssertionError):
        still.still_paged_decode(ctx, cache, batch, q.float(), out)
    with pytest.raises(still.StillError):
        still.still_paged_decode(ctx, cache, batch_of(p, [1]), q, out)
