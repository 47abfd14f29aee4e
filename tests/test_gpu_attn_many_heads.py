"""Attention of more heads than one launch has threads for, and of as many as make no head be cut."""
import pytest
import torch

import paper_2608_06690_amd as P
from tests import decode_cases as D
from tests.decode_cases import Cache, log, randn
from tests.test_gpu_attn_decode import check

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)


@pytest.mark.parametrize("R", [65536, 16385])
def test_the_largest_batches_of_many_heads(R):
    log(f"many heads, {R} requests of 256")
    kv, dim, page, pages = 256, 32, 16, 7
    desc = P.make_cache_desc(pages, page, kv, dim, 1)
    k, v = (randn((pages, kv, page, dim), s, 1.0, BF16).cuda() for s in (1, 2))
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    pick = lambda n: torch.randint(0, n, (R,), generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    at, words, length, first = pick(pages), pick(2) * ALLOW, (pick(8) > 0).int(), (pick(8) == 0).int()
    tag = torch.tensor([0, ALLOW, 0, ALLOW, ALLOW, 0, 5], dtype=torch.int32, device="cuda")
    q = torch.empty(R, kv, dim, dtype=BF16, device="cuda").normal_(generator=g)
    out, lse = torch.full_like(q, 9.0), torch.full((R, kv), 9.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert P.pmpe_attn_decode_workspace_bytes(desc, R, kv) == 0
    P.pmpe_attn_decode(desc, q, first, length, at.view(R, 1), tag, words, k, v, None, None, 0.25, out, lse, st, None)
    torch.cuda.synchronize()
    seen = (length > first) & (tag[at.long()] == words)
    assert int(st) == P.PMPE_DEV_CACHE_REFUSED and 0 < int(seen.sum()) < R
    for r0 in range(0, R, 4096):        # one row: the output is that row
        rows = slice(r0, min(R, r0 + 4096))
        page_of, ok = at[rows].long(), seen[rows]
        want = torch.where(ok[:, None, None], v[page_of, :, 0], 0.0)
        assert torch.equal(out[rows], want), r0
        s = 0.25 * (q[rows].float() * k[page_of, :, 0].float()).sum(dim=2)
        assert torch.equal(torch.isinf(lse[rows]), ~ok[:, None].expand(-1, kv)), r0
        # fp32 sums of 32 products, in two orders
        most = 0.25 * (q[rows].float() * k[page_of, :, 0].float()).abs().sum(dim=2)
        assert bool(((lse[rows] - s).abs()[ok] <= 80 * 2.0 ** -24 * most[ok] + 2.0 ** -22).all()), r0


@pytest.mark.parametrize("dt,q8", [(BF16, False), (BF16, True), (torch.float32, False)])
def test_heads_of_long_tables_that_are_not_cut(dt, q8):
    """32 requests of 256 virtual heads: as many as fill the card without parts, over tables of more than 1024 rows."""
    log(f"no cut by the number of heads {dt} {q8}")
    lens = [(37 * r) % 90 for r in range(32)]
    lens[5], lens[17] = 1100, 1057
    c = Cache(lens, 256, 32, 16, dt, q8)
    assert c.cols * 16 > 1024 and P.pmpe_attn_decode_workspace_bytes(c.desc, 32, 256) == 0
    first = [max(0, n - 1030) if n > 1000 else n // 3 for n in lens]
    check(c, D.randn((32, 256, 32), 5, 1.0, dt), first, lens, 0.2)
