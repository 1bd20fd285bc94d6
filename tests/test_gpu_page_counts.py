"""Counts of a page pool that do not cover its table's entries: kv_release flags
what it finds and leaves no count below zero, so that the page is free again."""
import numpy as np
import pytest
import torch

from test_gpu_pages import Pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dreams():
    import paper_2606_00535_gb300 as d
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    d._lib()
    return d


def test_release_of_a_page_with_count_zero(dreams):
    p = Pool(dreams, 2, 3, 6, table=[[0, 1, -1], [2, -1, -1]], ref=[1, 0, 1, 0, 0, 0])
    assert p.release([0, 0], [192, 0]) == dreams.DATA_BAD_PAGE
    assert p.ref.tolist() == [0, 0, 1, 0, 0, 0] and (p.table[0] == -1).all()
    assert p.reserve([0, 10], [129, 100]) == 0  # page 1 goes out like any free one
    assert p.table.tolist() == [[0, 1, 3], [2, 4, -1]]


@pytest.mark.parametrize("holders,count", [(1, 0), (7, 3), (400, 399), (400, 1), (3000, 2990)])
def test_more_entries_than_counted(dreams, holders, count):
    """All sequences give the same page back at once; those beyond its count are flagged. Twice, the counts being right
    for another page of each."""
    table = np.full((holders, 3), -1, np.int32)
    table[:, 0], table[:, 2] = 5, 9
    ref = np.zeros(12, np.int32)
    ref[5], ref[9] = count, holders
    p = Pool(dreams, holders, 3, 12, table=table, ref=ref)
    assert p.release(np.zeros(holders), np.full(holders, 64)) == dreams.DATA_BAD_PAGE
    assert p.ref.tolist() == [0] * 9 + [holders, 0, 0]
    assert p.release(np.zeros(holders), np.full(holders, 192)) == 0
    assert not p.ref.any()
