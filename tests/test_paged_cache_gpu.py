"""PagedCache: what its methods leave to the caller and what not."""
import pytest
import torch

from paper_2509_21354_amd import binding as kb
from tests.test_pages_gpu import ints, normal, shape_of

pytestmark = pytest.mark.gpu


def test_append_without_counts_writes_what_was_reserved():
    """Rows that reserved fewer than Tn, or none: the rest of what append() is given goes nowhere, least of all into a page that a fork shares."""
    sh = shape_of(L=2, B=3, H=2, d=64)
    K, V = normal(1, 2, 3, 2, 20, 64), normal(2, 2, 3, 2, 20, 64)

    def started():
        c = kb.PagedCache(sh, 16, 12, 4, 20)
        c.pool.zero_()
        c.reserve(ints([20, 0, 0]))
        c.append(K, V, 20)
        assert c.start.tolist() == [0, 0, 0]
        c.fork(ints([0]), ints([1]), 1)
        c.trim(ints([1]), 1, None, ints([17]))           # (both hold the second page)
        return c
    c = started()
    before = c.pool.clone()
    k, v = torch.zeros_like(K), torch.zeros_like(V)
    c.read(ints([0] * 3), c.length, 20, k, v)
    assert not k[:, 2].any() and k[:, 0].any() and torch.equal(k[:, 0, :, :17], k[:, 1, :, :17])
    c.reserve(ints([0, 0, 0]))
    c.append(K, V, 20)
    assert torch.equal(c.pool, before)
    # fewer than Tn in one row, a copy of the shared page in another: as with the counts
    new, old = ints([0, 3, 5]), []
    for counts in (new, None):
        c = started()
        c.reserve(new)
        c.append(K.flip(3).contiguous(), V, 20, *([] if counts is None else [counts]))
        old.append([c.pool, c.table, c.length, c.refs])
        assert c.length.tolist() == [20, 20, 5]
    assert all(torch.equal(x, y) for x, y in zip(*old))
