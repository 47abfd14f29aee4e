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
