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
