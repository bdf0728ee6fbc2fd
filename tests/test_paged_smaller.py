"""CPU checks of the calls that make a paged cache smaller: handles, scratch sizes and refusals that
need no device."""
import pytest
import torch

from paper_2606_07878_gb300 import still

E4M3 = torch.float8_e4m3fn


def pools(n, page, H, d, first=False, dtype=E4M3):
    x = [torch.zeros((n, H, page, d) if first else (n, page, H, d), dtype=torch.uint8 if
                     dtype == E4M3 else dtype) for _ in "KV"]
    x = [y.view(E4M3) if dtype == E4M3 else y for y in x]
    return [y.transpose(1, 2) for y in x] if first else x


def scales(n, H, page):
    return [torch.zeros(n, H, page // 16) for _ in "KV"]


@pytest.mark.parametrize("first", [False, True])
def test_layout_of_a_cache_in_8_bits(first):
    s = still.PagedCacheQuant(*pools(5, 32, 2, 64, first), *scales(5, 2, 32)).struct
    want = (4096, 64, 2048) if first else (4096, 128, 64)
    assert (s.s_page, s.s_slot, s.s_head) == want
    assert (s.n_pages, s.page_size, s.n_kv_heads, s.head_dim) == (5, 32, 2, 64) and not s.beta


def test_handles_that_are_refused():
    K, V = pools(5, 32, 2, 64)
    k, v = scales(5, 2, 32)
    for bad in [(K, V, k, v.double()), (K, V, k[:, :1], v), (K, V, k, None), (K, V[:4], k, v),
                (K, pools(5, 32, 2, 64, True)[1], k, v), (K.view(torch.uint8), V, k, v),
                (K, V, k, torch.zeros(5, 2, 4)[..., ::2]), (K, V, k, v, torch.zeros(5, 32, 2))]:
        with pytest.raises(AssertionError):
            still.PagedCacheQuant(*bad)


def test_scratch_of_weights():
    cache = still.PagedCache(*pools(5, 32, 2, 64, dtype=torch.bfloat16))
    logits = 5 * 32 * 8 * 4
    assert still.still_paged_weigh_scratch(cache, 0, 8) == logits
    assert still.still_paged_weigh_scratch(cache, 3, 8) == 256 + logits
    big = still.still_paged_weigh_scratch(cache, 1 << 20, 64)
    assert big == (1 << 20) * 64 * 8 + logits * 8
    assert still.lib().still_paged_weigh_scratch(None, 1, 1) == 0


def test_calls_without_a_context_are_refused():
    L = still.lib()
    cache = still.PagedCache(*pools(5, 32, 2, 64, dtype=torch.bfloat16))
    quant = still.PagedCacheQuant(*pools(5, 32, 2, 64), *scales(5, 2, 32))
    batch = still.PagedBatch(torch.zeros(1, 2, dtype=torch.int32),
                             torch.zeros(1, dtype=torch.int32))
    c, q, b = cache.ref, quant.ref, batch.ref
    assert still.STATUS[1] == "STILL_ERR_INVALID_ARG"
    assert L.still_paged_append_quant(None, q, b, 1, 16, 128, 16, 128, None, 0, 0, None, 0.0, None,
                                      None) == 1
    assert L.still_paged_decode_quant(None, q, b, 16, 128, 2, 0.0, 16, None) == 1
    assert L.still_paged_prefill_quant(None, q, b, 1, 16, 128, 2, 0.0, 16, None) == 1
    assert L.still_paged_decode_weigh(None, c, b, 16, 128, 2, 0.0, 16, 16, 1.0, 16, 1 << 20, None) == 1
    assert L.still_paged_weigh(None, c, b, 1, 16, 128, 2, 0.0, 16, 1.0, 16, 1 << 20, None) == 1
    assert L.still_paged_evict(None, c, b, 16, 1, 0, 0, c, 16, 2, 2, None, 16, 16, None, None) == 1
