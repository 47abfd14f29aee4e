"""The books of PagedCache on the host: pages, decisions and what may be shared."""
import pytest
import torch

import paper_2608_06690_amd as P

ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)
REV, FP = bytes(range(32)), bytes(range(32, 64))


def cache(**kw):
    args = dict(requests=3, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, max_pages=4, model_revision=REV,
                checkpoint_fingerprint=FP, device="cpu")
    args.update(kw)
    return P.PagedCache(**args)


def grow(c, counts):
    c._reserve(counts)
    c.lengths = [a + b for a, b in zip(c.lengths, counts)]


def test_pages_carry_the_decision_and_come_back():
    c = cache()
    assert c.page_tag.tolist() == [-1] * 8
    c.open(0, {"allow_private": True})
    c.open(1, {"allow_private": "yes"})  # malformed: denies
    assert c.words.tolist() == [ALLOW, 0, 0] and c.decision == [1, 0, None]
    grow(c, [20, 1, 0])
    assert [len(p) for p in c._pages] == [2, 1, 0] and len(c._free) == 5
    for r, want in ((0, ALLOW), (1, 0)):
        for i, p in enumerate(c._pages[r]):
            assert int(c.page_tag[p]) == want and int(c.block_table[r, i]) == p
    grow(c, [12, 15, 0])  # inside the pages they have
    assert [len(p) for p in c._pages] == [2, 1, 0]
    mine = list(c._pages[0])
    c.close(0)
    assert all(int(c.page_tag[p]) == -1 for p in mine) and len(c._free) == 7 and c.decision[0] is None
    assert sorted(c._free + c._pages[1]) == list(range(8))


def test_no_page_is_taken_where_not_all_can_be():
    c = cache()
    for r in range(3):
        c.open(r, None)
    with pytest.raises(ValueError):
        grow(c, [64, 64, 1])      # nine pages
    with pytest.raises(ValueError):
        grow(c, [65, 0, 0])       # more than max_pages
    assert len(c._free) == 8 and c._pages == [[], [], []]
    c.close(2)
    with pytest.raises(ValueError):
        grow(c, [0, 0, 1])        # not open
    with pytest.raises(ValueError):
        grow(c, [-1, 0, 0])


def test_sharing_needs_equal_tags():
    c = cache()
    c.open(0, {"allow_private": True})
    c.open(1, {"allow_private": False})
    c.open(2, {"allow_private": True})
    grow(c, [40, 0, 0])
    with pytest.raises(P.PmpeError):
        c.share(1, 0, 40)
    for other in (P.make_cache_tag(1, FP, FP), P.make_cache_tag(1, REV, REV), P.make_cache_tag(0, REV, FP)):
        with pytest.raises(P.PmpeError):
            c.share(2, 0, 40, other)
    with pytest.raises(P.PmpeError):  # a tag of the request's own does not make the pages its own
        c.share(1, 0, 40, P.make_cache_tag(0, REV, FP))
    assert c.share(2, 0, 40) == 32 and c._pages[2] == c._pages[0][:2]
    assert c.block_table[2, :2].tolist() == c._pages[0][:2]
    with pytest.raises(ValueError):
        c.share(2, 0, 40)         # not empty
    with pytest.raises(ValueError):
        c.share(0, 0, 16)
    shared, own = c._pages[0][:2], c._pages[0][2]
    c.close(0)
    assert all(int(c.page_tag[p]) == ALLOW for p in shared) and int(c.page_tag[own]) == -1
    grow(c, [0, 0, 5])
    assert len(c._pages[2]) == 3 and c._pages[2][2] not in shared
    c.close(2)
    assert sorted(c._free) == list(range(8)) and c.page_tag.tolist() == [-1] * 8


def test_open_begins_anew():
    c = cache()
    c.open(0, {"allow_private": True})
    grow(c, [30, 0, 0])
    c.open(0, {})
    assert c.lengths[0] == 0 and c.decision[0] == 0 and len(c._free) == 8 and int(c.words[0]) == 0


def test_closed_requests_have_no_tag_and_digests_have_32_bytes():
    c = cache()
    with pytest.raises(ValueError):
        c.tag(0)
    with pytest.raises(ValueError):
        cache(model_revision=b"x")


def test_a_refused_write_leaves_the_books_as_they_were(monkeypatch):
    # (the pages' memory may hold another decision's rows: a length without a write would show them)
    def refuse(*args):
        raise P.PmpeError(-5, "pmpe_kv_write")

    monkeypatch.setattr("paper_2608_06690_amd._native.pmpe_kv_write", refuse)
    for counts in ([3, 3, 3], [17, 0, 1]):
        c = cache()
        for r in range(3):
            c.open(r, None)
        grow(c, [4, 0, 0])
        c.seq_len[0] = 4
        mine = [list(p) for p in c._pages]
        k = torch.zeros(sum(counts), 2, 64, dtype=torch.bfloat16)
        with pytest.raises(P.PmpeError):
            c.write(k, k, counts)
        assert c.lengths == [4, 0, 0] and c.seq_len.tolist() == [4, 0, 0]
        assert c._pages == mine and len(c._free) == 7
        assert all(int(c.page_tag[p]) == -1 for p in c._free)
        assert sorted(c._free + mine[0]) == list(range(8))


def test_offsets_that_do_not_fit_the_counts_are_refused():
    c = cache()
    for r in range(3):
        c.open(r, None)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for offset in (torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 1, dtype=torch.int32)):
        with pytest.raises(ValueError):
            c.write(k, k, [1, 1, 2], offset)
        assert c.lengths == [0, 0, 0] and c.seq_len.tolist() == [0, 0, 0] and len(c._free) == 8


@pytest.mark.parametrize("rows", [-1, -16, -17])
def test_sharing_a_negative_number_of_rows_is_refused(rows):
    c = cache()
    for r in range(2):
        c.open(r, None)
    grow(c, [40, 0, 0])
    users = list(c._users)
    with pytest.raises(ValueError):
        c.share(1, 0, rows)
    assert c._users == users and c._pages[1] == [] and c.lengths == [40, 0, 0]


def test_shared_pages_come_back_once():
    c = cache()
    for r in range(2):
        c.open(r, None)
    grow(c, [40, 0, 0])
    assert c.share(1, 0, 40) == 32
    c.close(0)
    assert len(c._free) == 6 and all(int(c.page_tag[p]) == 0 for p in c._pages[1])
    c.close(1)
    assert sorted(c._free) == list(range(8)) and c.page_tag.tolist() == [-1] * 8
