"""CPU checks that a call over a paged cache takes no handle of another kind: the two caches' structs
differ in size and layout, so that one read as the other is read beyond its end."""
import ctypes

import pytest
import torch

from paper_2606_07878_gb300 import still


def handles():
    K = torch.zeros(3, 16, 1, 64, dtype=torch.bfloat16)
    codes = torch.zeros(3, 16, 1, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales, beta = torch.ones(3, 1, 1), torch.zeros(3, 1, 16)
    batch = still.PagedBatch(torch.zeros(1, 2, dtype=torch.int32), torch.ones(1, dtype=torch.int32))
    return still.PagedCache(K, K, beta), still.PagedCacheQuant(codes, codes, scales, scales, beta), batch


def calls(L, c16, c8, b):
    """Every call, without a context, over a cache in 16 bits or in 8 as it wants one."""
    return [
        lambda: L.still_paged_append(None, c16, b, 1, 16, 64, 16, 64, None, 0, 0, None, 0.0, None, None),
        lambda: L.still_paged_decode(None, c16, b, 16, 64, 1, 0.0, 16, None),
        lambda: L.still_paged_prefill(None, c16, b, 1, 16, 64, 1, 0.0, 16, None),
        lambda: L.still_paged_append_quant(None, c8, b, 1, 16, 64, 16, 64, None, 0, 0, None, 0.0, None,
                                           None),
        lambda: L.still_paged_decode_quant(None, c8, b, 16, 64, 1, 0.0, 16, None),
        lambda: L.still_paged_prefill_quant(None, c8, b, 1, 16, 64, 1, 0.0, 16, None),
        lambda: L.still_paged_decode_weigh(None, c16, b, 16, 64, 1, 0.0, 16, 16, 1.0, 16, 4096, None),
        lambda: L.still_paged_weigh(None, c16, b, 1, 16, 64, 1, 0.0, 16, 1.0, 16, 4096, None),
        lambda: L.still_paged_evict(None, c16, b, 16, 1, 0, 0, c16, 16, 2, 2, None, 16, 16, None, None)]


def test_a_handle_of_the_other_kind_is_none():
    L = still.lib()
    c16, c8, b = (x.ref for x in handles())
    for call in calls(L, c16, c8, b):
        assert still.STATUS[call()] == "STILL_ERR_INVALID_ARG"  # there is no context
    for call in calls(L, c8, c16, b) + calls(L, c16, c8, c16) + [
            lambda: L.still_paged_weigh_scratch(c8, 1, 1),
            lambda: L.still_paged_evict(None, c16, b, 16, 1, 0, 0, c8, 16, 2, 2, None, 16, 16, None,
                                        None)]:
        with pytest.raises(ctypes.ArgumentError):
            call()
    assert L.still_paged_weigh_scratch(c16, 1, 1) == 256 + 3 * 16 * 4
