"""Eviction from sequences as long as a table can name."""
import pytest
import torch

from paper_2606_07878_gb300 import still
from test_gpu_paged import DEV, ctx, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [1, 5])  # short ones beside it
@pytest.mark.parametrize("n", [0x7fffff00, 0x7fffff00 - 4097])
def test_slots_up_to_2_31(ctx, n, B):  # noqa: F811
    """One page, listed 32,768 times, is a sequence of 2^31 slots: the heaviest slot of the page is the
    heaviest of them all as often as it is listed, and the lowest ones stay."""
    page, keep, sinks, recent, d = 65536, 24, 2, 3, 64
    gen = torch.Generator(device=DEV).manual_seed(1)
    K, V = (torch.randn(1, page, 1, d, generator=gen, device=DEV).bfloat16() for _ in "KV")
    weight = torch.rand(1, 1, page, generator=gen, device=DEV)
    top = page // 2 + 77
    weight[0, 0, top] = 2.0
    lens = [n] + [700] * (B - 1)
    table = torch.zeros(B, 32768, dtype=torch.int32, device=DEV)
    to = [torch.zeros(2 * B, 16, 1, d, device=DEV, dtype=torch.bfloat16) for _ in "KV"]
    to_table = torch.arange(2 * B, dtype=torch.int32, device=DEV).view(B, 2)
    kept, to_lens = torch.zeros(B, 1, keep, dtype=torch.int32, device=DEV), i32([0] * B)
    still.still_paged_evict(ctx, still.PagedCache(K, V), still.PagedBatch(table, i32(lens)), weight,
                            keep, sinks, recent, still.PagedCache(*to), to_table, kept, to_lens)
    want = [0, 1] + [top + page * i for i in range(keep - 5)] + [n - 3, n - 2, n - 1]
    assert kept[0, 0].tolist() == want and to_lens.tolist() == [keep] * B
    at = torch.tensor(want, device=DEV) % page
    for x, y in zip(to, (K, V)):
        assert torch.equal(x[:2].view(-1, d)[:keep], y[0, at, 0])
    for b in range(1, B):
        w = weight[0, 0, :700].clone()
        w[:sinks] = w[700 - recent:] = float("inf")
        idx = w.sort(descending=True, stable=True).indices[:keep].sort().values
        assert kept[b, 0].tolist() == idx.tolist()


def test_more_kept_than_there_are(ctx):  # noqa: F811
    """`keep` of 2^31 - 1 slots over a sequence of 40: they move, and all others are -1."""
    page, d, keep = 65536, 64, 2 ** 31 - 1
    K = torch.randn(1, page, 1, d, device=DEV).bfloat16()
    to = [torch.zeros(1, page, 1, d, device=DEV, dtype=torch.bfloat16) for _ in "KV"]
    to_table = torch.full((1, 32768), -1, dtype=torch.int32, device=DEV)
    to_table[0, 0] = 0
    kept, lens = torch.full((1, 1, keep), 5, dtype=torch.int32, device=DEV), i32([0])
    still.still_paged_evict(ctx, still.PagedCache(K, K), still.PagedBatch(i32([[0]]), i32([40])),
                            torch.zeros(1, 1, page, device=DEV), keep, 0, 0, still.PagedCache(*to),
                            to_table, kept, lens)
    assert kept[0, 0, :40].tolist() == list(range(40)) and (kept[0, 0, 40:] == -1).all()
    assert lens.tolist() == [40] and torch.equal(to[0][0, :40], K[0, :40])
    assert not to[0][0, 40:].any() and not to[1][0, 40:].any()
