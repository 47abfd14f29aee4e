"""Pages that a PagedCache has ahead of its requests' rows, on the host."""
import pytest
import torch

import paper_2608_06690_amd as P
from tests.test_paged_cache_columns_host import owned
from tests.test_paged_cache_host import cache, grow


def refuse(*args):
    raise P.PmpeError(-5, "pmpe_kv_write")


def test_a_refused_write_keeps_the_pages_that_were_there(monkeypatch):
    # (pages reserved ahead may hold rows of replayed steps that the host has not counted)
    monkeypatch.setattr("paper_2608_06690_amd._native.pmpe_kv_write", refuse)
    c = cache()
    for r in range(3):
        c.open(r, None)
    grow(c, [4, 0, 16])
    c._reserve([40, 20, 0])
    mine, free = [list(p) for p in c._pages], list(c._free)
    assert [len(p) for p in mine] == [3, 2, 1]
    for counts in ([3, 3, 3], [1, 0, 0], [45, 0, 1]):
        k = torch.zeros(sum(counts), 2, 64, dtype=torch.bfloat16)
        with pytest.raises(P.PmpeError):
            c.write(k, k, counts)
        assert c._pages == mine and sorted(c._free) == sorted(free) and c.block_table.tolist() == owned(c)
        assert c.lengths == [4, 0, 16] and all(int(c.page_tag[p]) == 0 for p in sum(mine, []))


class Broken:
    """A tensor that cannot be written (as in a capture that allows no copies)."""

    def __init__(self, t):
        self.t, self.device = t, t.device

    def __setitem__(self, at, value):
        raise RuntimeError("not now")


@pytest.mark.parametrize("name", ["block_table", "page_tag"])
def test_pages_that_the_device_does_not_learn_of_are_not_taken(name):
    c = cache()
    for r in range(3):
        c.open(r, None)
    grow(c, [20, 0, 1])
    mine, free, users = [list(p) for p in c._pages], list(c._free), list(c._users)
    whole = getattr(c, name)
    setattr(c, name, Broken(whole))
    k = torch.zeros(40, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        c.write(k, k, [20, 20, 0])
    assert c._pages == mine and c._free == free and c._users == users and c.lengths == [20, 0, 1]
    setattr(c, name, whole)
    grow(c, [20, 20, 0])
    assert [len(p) for p in c._pages] == [3, 2, 1] and c.block_table.tolist() == owned(c)
    assert all(int(c.page_tag[p]) == 0 for p in sum(c._pages, []))


def replay(c, counts):
    """What replays of a captured write do to the device's lengths."""
    c.seq_len += torch.tensor(counts, dtype=torch.int32)


def test_reserved_pages_and_rows_of_replays():
    c = cache()
    for r in range(3):
        c.open(r, {"allow_private": r == 1})
    grow(c, [4, 0, 16])
    replay(c, [4, 0, 16])
    c.reserve([13, 16, 0])
    assert [len(p) for p in c._pages] == [2, 1, 1] and c.lengths == [4, 0, 16] and c.block_table.tolist() == owned(c)
    c.reserve([28, 3, 0])         # inside what it has
    assert [len(p) for p in c._pages] == [2, 1, 1]
    for counts in ([64, 0, 0], [0, 0, 64], [0, 65, 0], [1, 0], [0, 0, -1], [44, 64, 33]):
        with pytest.raises(ValueError):
            c.reserve(counts)
    assert c.advance() == [0, 0, 0] and c.lengths == [4, 0, 16] and [len(p) for p in c._pages] == [2, 1, 1]
    replay(c, [28, 5, 0])
    assert c.advance() == [28, 5, 0] and c.lengths == [32, 5, 16] == c.seq_len.tolist()
    c.close(0)
    replay(c, [3, 0, 0])          # not open
    assert c.advance() == [0, 0, 0] and c.lengths == [0, 5, 16] == c.seq_len.tolist()
    with pytest.raises(ValueError):
        c.reserve([1, 0, 0])


@pytest.mark.parametrize("late", [False, True])
def test_refused_rows_of_replays_are_counted_nowhere(late):
    # (a page that is reserved after them holds what another request left in it)
    c = cache()
    for r in range(3):
        c.open(r, None)
    grow(c, [14, 3, 0])
    replay(c, [14, 3, 0])
    replay(c, [5, 5, 0])          # request 0 has a page for two of its five
    if not late:
        assert c.advance() == [2, 5, 0] and c.seq_len.tolist() == [16, 8, 0]
    c.reserve([20, 0, 0])
    assert c.seq_len.tolist() == [16, 8, 0] and len(c._pages[0]) >= 2
    replay(c, [1, 1, 0])
    assert c.advance() == ([3, 6, 0] if late else [1, 1, 0]) and c.lengths == [17, 9, 0] == c.seq_len.tolist()


def test_a_request_with_reserved_pages_does_not_share():
    c = cache()
    for r in range(3):
        c.open(r, None)
    grow(c, [40, 0, 0])
    c.reserve([0, 20, 0])
    with pytest.raises(ValueError):
        c.share(1, 0, 40)         # its own two pages would be lost
    assert sum(map(len, c._pages)) + len(c._free) == 8
    assert c.share(2, 0, 40) == 32
