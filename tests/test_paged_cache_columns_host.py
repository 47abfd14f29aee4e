"""The block table of a PagedCache on the host: a column that a request has no page for names none."""
import torch

from tests.test_paged_cache_host import cache, grow


def owned(c):
    """What the table should hold: each request's pages, then -1."""
    return [p + [-1] * (c.desc.max_pages - len(p)) for p in c._pages]


def test_columns_without_a_page_name_none():
    c = cache()
    assert c.block_table.tolist() == [[-1] * 4] * 3
    for r in range(3):
        c.open(r, None)
    grow(c, [40, 17, 0])
    assert c.block_table.tolist() == owned(c)
    c.close(0)
    assert c.block_table.tolist() == owned(c) and c.block_table[0].tolist() == [-1] * 4
    grow(c, [0, 0, 50])           # (its pages were request 0's)
    assert c.block_table.tolist() == owned(c)
    c.open(1, {"allow_private": True})
    assert c.block_table.tolist() == owned(c)
    c.open(0, None)
    assert c.share(0, 2, 40) == 32
    assert c.block_table.tolist() == owned(c)
    c.close(2)
    c.close(0)
    assert c.block_table.tolist() == [[-1] * 4] * 3 and sorted(c._free) == list(range(8))


def test_columns_of_a_refused_write_name_none(monkeypatch):
    def refuse(*args):
        raise ValueError("refused")

    monkeypatch.setattr("paper_2608_06690_amd._native.pmpe_kv_write", refuse)
    c = cache()
    for r in range(3):
        c.open(r, None)
    grow(c, [16, 0, 5])
    k = torch.zeros(60, 2, 64, dtype=torch.bfloat16)
    try:
        c.write(k, k, [40, 20, 0])
    except ValueError:
        pass
    assert c.block_table.tolist() == owned(c) and [len(p) for p in c._pages] == [1, 0, 1]
