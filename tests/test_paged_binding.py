"""CPU checks of the handles of the paged cache: what they pass on of their tensors' layouts."""
import pytest
import torch

from paper_2606_07878_gb300 import still


def batch(table):
    return still.PagedBatch(table, torch.zeros(table.shape[0], dtype=torch.int32))


def pages(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


@pytest.mark.parametrize("table,pitch", [
    (pages(3, 5), 5), (pages(3, 8)[:, :5], 8), (pages(6, 5)[::2], 10), (pages(1, 5), 5),
    (pages(9, 5)[2:3], 5), (pages(1, 5).expand(1, 5), 5),
    (torch.as_strided(pages(40), (1, 5), (0, 1)), 5), (pages(4, 1), 1)])
def test_pitch_of_a_table(table, pitch):
    s = batch(table).struct
    assert (s.s_table, s.table_pages, s.B) == (pitch, table.shape[1], table.shape[0])
    rows = [pitch * b + i for b in range(s.B) for i in range(s.table_pages)]
    assert max(rows) * 4 < table.untyped_storage().nbytes() - 4 * table.storage_offset()


@pytest.mark.parametrize("table", [
    pages(1, 5).expand(3, 5),                         # one row for all
    torch.as_strided(pages(40), (3, 5), (2, 1)),      # rows that overlap
    pages(5, 3).t()])                                 # entries apart
def test_tables_that_would_be_read_beyond_their_end(table):
    with pytest.raises(AssertionError):
        batch(table)


def strided(shape, strides):
    x = torch.zeros(sum((n - 1) * s for n, s in zip(shape, strides)) + 1, dtype=torch.bfloat16)
    return torch.as_strided(x, shape, strides)


def test_strides_of_one_page_or_one_head_do_not_count():
    """A pool of one KV-head in two orders, or of one page cut out of larger pools, is one layout."""
    for shape, of_k, of_v, want in [
            ((4, 16, 1, 64), (1024, 64, 64, 1), (1024, 64, 1024, 1), (1024, 64, 64)),
            ((4, 16, 1, 64), (1024, 64, 3, 1), (1024, 64, 64, 1), (1024, 64, 64)),
            ((1, 16, 2, 64), (2048, 128, 64, 1), (1, 128, 64, 1), (64, 128, 64)),
            ((1, 16, 1, 64), (0, 64, 0, 1), (5, 64, 7, 1), (64, 64, 64))]:
        s = still.PagedCache(strided(shape, of_k), strided(shape, of_v)).struct
        assert (s.s_page, s.s_slot, s.s_head) == want
    for of_v in [(2048, 128, 128, 1), (2048, 64, 64, 1), (4096, 128, 64, 1), (4096, 256, 128, 2)]:
        with pytest.raises(AssertionError):
            still.PagedCache(strided((4, 16, 2, 64), (2048, 128, 64, 1)),
                             strided((4, 16, 2, 64), of_v))
