"""The kernel of few rows (decode): weights to 2^-17, and the same rows from the kernel of many."""
import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, NAN, WEIGHTS, Pages, attention64, batch_of, fused_rows

pytestmark = pytest.mark.gpu

# P goes into its product as bf16 hi + lo: hi leaves less than 2^-8 of the power of two below a weight,
# lo half a unit of its last place, 2^-17. The sum takes weights before any rounding. fp32 sums of up
# to 256 products of size about 1/16 .. 4 move a logit by less than 2^-12.7, and a weight and the sum
# by as much (exponentials: 2^-22).
FEW = 2.0 ** -17 + 2.0 ** -11


def bound(ref, size, weights):
    return 2.0 ** -8 * ref.abs() + (1 + 2.0 ** -8) * weights * size  # a bf16 output, its weights


@pytest.fixture(scope="module")
def ctx():
    c = still.still_create(0)
    yield c
    code, det = still.still_get_device_status(c)
    still.still_destroy(c)
    assert code == 0, (still.STATUS[code], det)


def alternating(p):
    """Values whose sign alternates with the slot: outputs near zero beside sum_j p_j |v_j|, so that
    the error of the weights is not covered by the rounding of the outputs."""
    sign = 1 - 2 * (torch.arange(p.page, device=DEV) % 2)
    p.V.copy_((1 + p.V.float().abs() / 8).bfloat16() * sign[:, None, None])


def rounded_weights(p, q):
    """The outputs with every weight e^(s - max) rounded to bf16, and the sum of the unrounded."""
    d, g = q.shape[2], q.shape[1] // p.H
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(p.lens):
        k, v = p.rows(p.K, b).double(), p.rows(p.V, b).double()
        for h in range(p.H if n else 0):
            s = q[b, h * g:(h + 1) * g].double() @ k[:, h].T / d ** 0.5
            if p.beta is not None:
                s = s + p.rows(p.beta, b)[:, h].double()
            w = (s - s.amax(-1, keepdim=True)).exp()
            out[b, h * g:(h + 1) * g] = w.bfloat16().double() @ v[:, h] / w.sum(-1, keepdim=True)
    return out


@pytest.mark.parametrize("d,g", [(64, 1), (64, 8), (64, 16), (128, 4), (128, 12), (256, 8)])
@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("lens", [[2, 3, 4, 6, 8, 16, 20, 33] * 4, [700, 2, 5000, 64]])
def test_weights_keep_the_rest_of_their_rounding(ctx, d, g, beta, lens):
    p = Pages(100, lens, 4, d, 16, beta=beta)
    alternating(p)
    q, = fused_rows(101, len(lens), [4 * g], d)
    out = torch.full_like(q, NAN)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), q, out)
    ref, size = attention64(p, q, [1] * len(lens))
    assert torch.isfinite(out).all()
    assert ((out.double() - ref).abs() <= bound(ref, size, FEW)).all()
    if len(lens) > 4:  # weights of 8 bits would not pass
        planted = rounded_weights(p, q).bfloat16().double()
        assert ((planted - ref).abs() > bound(ref, size, FEW)).any()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("beta", [False, True])
def test_a_token_alone_and_as_the_last_of_many(ctx, d, beta):
    """Decode, and the same tokens as the last ones of longer calls that take the other kernel."""
    lens = [3000, 70, 41, 900]
    p = Pages(102, lens, 2, d, 32, beta=beta)
    new = [9] * 4
    q, = fused_rows(103, 36, [8], d)
    many = torch.full((36, 8, d), NAN, device=DEV, dtype=torch.bfloat16)
    still.still_paged_prefill(ctx, p.cache(), batch_of(p, new), q, many)  # 36 rows a KV-head
    last = q[8::9].contiguous()
    one = torch.full_like(last, NAN)
    still.still_paged_decode(ctx, p.cache(), batch_of(p), last, one)
    ref, size = attention64(p, last, [1] * 4)
    assert ((one.double() - ref).abs() <= bound(ref, size, FEW)).all()
    apart = (one.double() - many[8::9].double()).abs()
    assert (apart <= bound(ref, size, FEW) + bound(ref, size, WEIGHTS)).all()
