"""The paged cache in 8 bits where its scales are far apart: values before and behind a maximum that
jumps, blocks of zeros."""
import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, NAN, assert_rows, attention64, batch_of, ctx, fused_rows  # noqa: F401
from test_gpu_paged_quant import FEW, QuantPages

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.float32).min


def blocks(p, b):
    """Pages of sequence b, of 16 slots: a block each."""
    assert p.page == 16
    return p.table[b, :-(-p.lens[b] // 16)].tolist()


def decode(ctx, p, q):  # noqa: F811
    out = torch.full_like(q, NAN)
    still.still_paged_decode_quant(ctx, p.cache(), batch_of(p), q, out)
    return out


def assert_small_rows(out, ref, size, weights):
    """assert_rows where outputs may be subnormal: their rounding is 2^-134 at most there."""
    assert torch.isfinite(out).all()
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + weights * size + 2.0 ** -134).all()


@pytest.mark.parametrize("d,Hq", [(64, 4), (128, 4), (128, 16), (256, 5)])
@pytest.mark.parametrize("apart", [8, 16, 24, 40, 90])
def test_values_behind_a_maximum_that_jumps(ctx, d, Hq, apart):  # noqa: F811
    """Every other block has biases of the lowest float and values 2^apart times the others': they
    weigh nothing, and what they were multiples of must not stay the unit of those that do."""
    p = QuantPages(61, [240, 3000], 1, d, 16, beta=True)
    for b in range(2):
        for page in blocks(p, b)[::2]:
            p.beta[page] = LOWEST
            p.scales[1][page] *= 2.0 ** apart
    p.read()
    q, = fused_rows(62, 2, [Hq], d)
    assert_rows(decode(ctx, p, q), *attention64(p, q, [1, 1]), FEW)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("old,new", [(-12, -120), (-20, -124), (40, -60), (100, -14)])
def test_both_sides_of_a_jump_count(ctx, d, old, new):  # noqa: F811
    """Weights of e^-80 = 2^-115.4 on values of 448 2^old beside weights of 1 on values of 2^new: sums
    of either side are of the same size, though 2^old 2^-115.4 may lie below the normal floats."""
    p = QuantPages(63, [240], 1, d, 16, beta=True)
    for i, page in enumerate(blocks(p, 0)):
        p.beta[page] = 0.0 if i % 2 else -80.0
        p.scales[1][page] = 2.0 ** (new if i % 2 else old)
        p.codes[1].view(torch.uint8)[page] = 0x38 if i % 2 else 0x7e  # 1, 448
    p.read()
    q, = fused_rows(64, 1, [4], d)
    q = (q.float() / 16).bfloat16()  # logits within 1 of their bias
    assert_small_rows(decode(ctx, p, q), *attention64(p, q, [1]), FEW)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scale", [2, 5, 8, 30])
@pytest.mark.parametrize("gap", [83, 85, 86.5])
def test_a_block_of_zeros_has_the_maximum(ctx, d, scale, gap):  # noqa: F811
    """Values of zero have the smallest scale, 2^-126; others 2^128 times that and more, whose weights
    are among the smallest normal floats (e^-86.5 = 2^-124.8)."""
    p = QuantPages(65, [240], 1, d, 16, beta=True)
    for i, page in enumerate(blocks(p, 0)):
        p.beta[page] = 0.0 if i % 4 == 0 else -gap
        p.scales[1][page] = 2.0 ** (-126 if i % 4 == 0 else scale)
        if i % 4 == 0:
            p.codes[1].view(torch.uint8)[page] = 0
    p.read()
    q, = fused_rows(66, 1, [4], d)
    q = (q.float() / 32).bfloat16()  # logits within 0.5 of their bias: no weight below 2^-126
    assert_small_rows(decode(ctx, p, q), *attention64(p, q, [1]), FEW)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_keys_whose_logits_are_large(ctx, d):  # noqa: F811
    """Logits up to 2^120 or so: finite, so that one slot has all the weight."""
    p = QuantPages(67, [240], 1, d, 16)
    p.scales[0].mul_(2.0 ** 112)
    p.read()
    q, = fused_rows(68, 1, [4], d)
    assert_rows(decode(ctx, p, q), *attention64(p, q, [1]), FEW)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_a_code_is_off_by(ctx, d):  # noqa: F811
    """2^-4 of a value or 2^-10 of the scale, whichever is more, and 2^-10 of the new scale more where
    a block's scale grew: both are met by what lies halfway between two subnormal codes."""
    p = QuantPages(69, [0], 1, d, 16, spare=40)
    p.table = torch.arange(40, dtype=torch.int32, device=DEV)[None]
    g = torch.Generator(device=DEV).manual_seed(70)
    n = 40 * 16 - 1  # the last block is filled up behind it
    x = torch.randn(n + 1, 1, d, generator=g, device=DEV)
    x *= torch.exp2(20 * torch.rand(n + 1, 1, d, generator=g, device=DEV) - 20)
    x[::16, :, 0], x[::16, :, 1] = 225.0, 2.0 ** -10  # 225 is 1 as a scale, 2^-10 half a step
    x[n] = 0
    x[n, :, 0] = 900.0  # 4
    x = x.bfloat16()
    half = torch.maximum(2.0 ** -4 * x.double().abs(), torch.tensor(2.0 ** -10))

    def append(lo, hi):
        p.lens = [hi]
        still.still_paged_append_quant(ctx, p.cache(), batch_of(p, [hi - lo]), x[lo:hi], x[lo:hi])
        p.read()
        return [(p.rows(y, 0) - x[:hi].double()).abs() for y in (p.K, p.V)]
    for off in append(0, n):
        assert (off <= half[:n]).all() and (off[::16, :, 1] == 2.0 ** -10).all()
    assert (p.scales[0] == 1).all() and (p.scales[1] == 1).all()
    last = slice(n - 15, n)
    for scales, off in zip(p.scales, append(n, n + 1)):
        assert scales[-1] == 4 and (scales[:-1] == 1).all()
        assert (off[:n - 15] <= half[:n - 15]).all() and (off[n] == 900 - 896).any()
        assert (off[last] <= half[last] + 2.0 ** -8).all() and (off[last] > half[last]).any()
