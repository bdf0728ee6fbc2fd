"""CPU checks of the cost by which a prefill over a paged cache is cut into ranges."""
import ctypes

import numpy as np
import pytest

from paper_2606_07878_gb300 import still


def cost(count, slots, tokens, q0, q1):
    f = still.lib().still_internal_paged_cost
    f.restype = ctypes.c_int64
    return f(count, slots, tokens, q0, q1)


def expected(count, slots, tokens, q0, q1):
    seen = slots - count + np.minimum(count, (np.arange(q0, q1, dtype=np.int64) + 1) * tokens)
    return int((np.maximum(0, -(-seen // 128)) + 2).sum())


@pytest.mark.parametrize("count,slots,tokens", [
    (1, 1, 256), (300, 300, 64), (300, 100, 64), (5, 0, 2), (8192, 8192, 36), (777, 9000, 1)])
def test_cost_of_a_sequence_and_of_its_parts(count, slots, tokens):
    nq = -(-count // tokens)
    assert cost(count, slots, tokens, 0, nq) == expected(count, slots, tokens, 0, nq)
    cut = nq // 3
    assert (cost(count, slots, tokens, 0, cut) + cost(count, slots, tokens, cut, nq)
            == cost(count, slots, tokens, 0, nq))


def test_a_prompt_of_a_million_tokens_passes_32_bits():
    """Two tokens an item (128 query heads to a KV-head), added up by one thread where a call has more
    sequences than half its threads."""
    n = 1 << 20
    assert cost(n, n, 2, 0, n // 2) == expected(n, n, 2, 0, n // 2) > 1 << 31
