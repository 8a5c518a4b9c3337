"""What an append costs the host: it looks at the pages of its own histories, not at all that the cache has.  None of it touches a GPU."""
import numpy as np
import pytest

from tests.test_history_pages_host import append, consistent, history, store  # noqa: F401


class Pages(np.ndarray):
    """Counts of pages that may not be read or copied as a whole."""

    def copy(self, *args, **kw):
        raise AssertionError("all pages are copied")

    def __array_ufunc__(self, ufunc, method, *inputs, **kw):
        for x in inputs:
            assert not (isinstance(x, Pages) and x.base is None), "all pages are gone over"
        return getattr(ufunc, method)(*(np.asarray(x) for x in inputs), **kw)


def test_an_append_looks_at_its_own_pages(store):  # noqa: F811
    append(store, [0, 1], [130, 64])
    store.fork([0, 0, 1], [2, 3, 4])
    plain = store.shares
    store.shares = np.ndarray.__new__(Pages, plain.shape, plain.dtype)
    store.shares[:] = plain
    with pytest.raises(AssertionError, match="all pages"):
        store.shares.copy()
    with pytest.raises(AssertionError, match="all pages"):
        store.shares > 1
    before = history(store, 0)
    append(store, [0, 2, 3, 4], [1, 2, 3, 1])
    append(store, [0, 2, 1], [1, 70, 1])
    store.shares = np.asarray(store.shares)
    assert consistent(store) and store.copies == [2] and [history(store, u)[:130] == before for u in (0, 2, 3)] == [True] * 3
