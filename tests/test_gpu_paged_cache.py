"""PagedCache on the GPU: captured steps, their pages and lengths, and what they may not touch."""
import pytest
import torch

import paper_2608_06690_amd as P
from tests.decode_cases import log, randn

pytestmark = pytest.mark.gpu
REV, FP = bytes(32), bytes(range(32))
KV, DIM, HEADS = 2, 64, 8
BF16 = torch.bfloat16


def rows(n, seed):
    return randn((n, KV, DIM), seed, 1.0, BF16).cuda()


@pytest.mark.parametrize("fp8", [False, True])
def test_replays_past_the_pages_leave_other_requests_alone(fp8):
    log(f"replays past the pages fp8 {fp8}")
    cache = P.PagedCache(3, 8, 16, KV, DIM, 4, REV, FP, fp8=fp8)
    for r in range(3):
        cache.open(r, None)             # of one decision: no tag keeps their pages apart
    cache.write(rows(16, 1), rows(16, 2), [0, 16, 0])  # (page 0 is request 1's)
    cache.write(rows(26, 7), rows(26, 8), [14, 0, 12])
    cache.close(2)
    cache.open(2, None)
    cache.write(rows(20, 3), rows(20, 4), [0, 20, 0])  # (with the page that was request 2's)
    k, v, off = rows(1, 5), rows(1, 6), torch.tensor([0, 1, 1, 1], dtype=torch.int32, device="cuda")
    cache.write(k, v, [1, 0, 0], off)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.write(k, v, [1, 0, 0], off)
    mine = int(cache.block_table[0, 0])
    others = [p for p in range(8) if p != mine]
    before = [x[others].clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale) if x is not None]
    g.replay()                          # row 15, the last of its page
    torch.cuda.synchronize()
    assert int(cache.dev_status) == 0 and int(cache.seq_len[0]) == 16
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert int(cache.dev_status) == P.PMPE_DEV_CACHE_RANGE
    after = [x[others] for x in (cache.k, cache.v, cache.k_scale, cache.v_scale) if x is not None]
    assert all(torch.equal(a, b) for a, b in zip(before, after))


def test_a_captured_write_that_needs_pages_is_refused():
    log("captured write without pages")
    cache = P.PagedCache(2, 8, 16, KV, DIM, 4, REV, FP)
    for r in range(2):
        cache.open(r, None)
    cache.write(rows(20, 1), rows(20, 2), [16, 4])
    k, v, off = rows(2, 3), rows(2, 4), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    books = [list(p) for p in cache._pages], list(cache._free), list(cache.lengths)
    x, g = torch.zeros(4, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(ValueError):
            cache.write(k, v, [1, 1], off)
        x.add_(1)                       # (the capture goes on)
    assert books == (cache._pages, cache._free, cache.lengths) and cache.seq_len.tolist() == [16, 4]
    g.replay()
    cache.write(k, v, [1, 1], off)
    got, _ = cache.read([17, 5])
    assert torch.equal(got[16], k[0]) and torch.equal(got[21], k[1]) and x.tolist() == [1.0] * 4 and int(cache.dev_status) == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_captured_steps_through_the_public_calls(fp8):
    log(f"captured steps fp8 {fp8}")
    cache, eager = (P.PagedCache(3, 16, 16, KV, DIM, 5, REV, FP, fp8=fp8) for _ in range(2))
    k0, v0 = rows(60, 1), rows(60, 2)
    for c in (cache, eager):
        for r in range(3):
            c.open(r, {"allow_private": r == 1})
        c.write(k0, v0, [30, 10, 20])
    off = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    k, v, q = rows(3, 3), rows(3, 4), randn((3, HEADS, DIM), 5, 1.0, BF16).cuda()
    cache.reserve([20, 20, 20])
    cache.attend(q, 0.125)              # (its workspace)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.write(k, v, [1, 1, 1], off)
        out = cache.attend(q, 0.125)
    assert cache.lengths == [30, 10, 20] and cache.seq_len.tolist() == [30, 10, 20]
    for i in range(6):
        for n, t in enumerate((k, v)):
            t.copy_(rows(3, 10 + 2 * i + n))
        q.copy_(randn(q.shape, 40 + i, 1.0, BF16))
        g.replay()
        eager.write(k, v, [1, 1, 1], off)
        assert torch.equal(out, eager.attend(q, 0.125))
    assert cache.advance() == [6, 6, 6]
    assert cache.lengths == eager.lengths == cache.seq_len.tolist() == [36, 16, 26]
    more = rows(5, 60), rows(5, 61)     # eager rows go on from the replays'
    for c in (cache, eager):
        c.write(*more, [0, 5, 0])
    for a, b in zip(cache.read([36, 21, 26]), eager.read([36, 21, 26])):
        assert torch.equal(a, b)
    assert int(cache.dev_status) == 0 and cache.lengths == [36, 21, 26]


def serve(cache, q, stream, reads):
    """Requests that come, share, end and come again, with the kernels' outputs after every change."""
    out, at = [], 0

    def put(counts):
        nonlocal at
        n = sum(counts)
        cache.write(reads[0][at:at + n], reads[1][at:at + n], counts, stream=stream)
        out.append(cache.attend(q, 0.125, stream=stream))
        at += n
    for r in range(4):
        cache.open(r, {"allow_private": r % 2 == 1}, stream=stream)
    put([20, 33, 5, 1])
    for turn in range(6):
        cache.close(turn % 3, stream=stream)
        cache.open(turn % 3, {"allow_private": turn % 2 == 0}, stream=stream)
        put([3 + 5 * (turn % 3 == r) for r in range(4)])
        cache.open(3, {"allow_private": cache.decision[1] == 1}, stream=stream)
        got = cache.share(3, 1, 40, stream=stream)
        assert got == min(40, cache.lengths[1]) // 16 * 16
        cache.reserve([17, 0, 17, 2], stream=stream)
        put([1, 1, 1, 1])
        out += cache.read([1, 2, 3, 1], stream=stream)
    return out


def test_every_call_on_a_side_stream_with_the_current_one_busy():
    log("all calls on a side stream")
    kv, q = (rows(300, 1), rows(300, 2)), randn((4, HEADS, DIM), 3, 1.0, BF16).cuda()
    results = []
    busy = torch.randn(4096, 4096, device="cuda")
    for side in (False, True):
        cache = P.PagedCache(4, 24, 16, KV, DIM, 6, REV, FP)
        torch.cuda.synchronize()
        s = torch.cuda.Stream() if side else None
        if side:
            for _ in range(40):         # what is put on the current stream comes tens of milliseconds later
                busy = torch.mm(busy, busy).clamp_(-1.0, 1.0)
        out = serve(cache, q, s, kv)
        if side:
            s.synchronize()
        results.append([x.cpu() for x in out] + [cache.seq_len.cpu(), cache.dev_status.cpu()])
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and int(results[1][-1]) == 0


def test_replays_past_the_pages_go_on_once_more_are_reserved():
    log("replays past the pages, then more pages")
    cache = P.PagedCache(2, 8, 16, KV, DIM, 4, REV, FP)
    cache.open(0, {"allow_private": True})
    cache.write(rows(60, 1), rows(60, 2), [60, 0])
    cache.close(0)                      # the pages to come hold rows of an allowed request
    for r in range(2):
        cache.open(r, None)
    k0, v0 = rows(14, 3), rows(14, 4)
    cache.write(k0, v0, [14, 0])
    k, v, q = rows(1, 5), rows(1, 6), randn((2, HEADS, DIM), 7, 1.0, BF16).cuda()
    off = torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.write(k, v, [1, 0], off)
    ks, vs = [k0], [v0]
    for i in range(9):
        k.copy_(rows(1, 20 + i))
        v.copy_(rows(1, 40 + i))
        if i < 2 or i >= 5:             # the third to fifth meet no page
            ks.append(k.clone())
            vs.append(v.clone())
        if i == 5:
            assert int(cache.dev_status) == P.PMPE_DEV_CACHE_RANGE
            cache.reserve([10, 0])
        g.replay()
    assert cache.advance() == [6, 0] and cache.lengths == [20, 0] == cache.seq_len.tolist()
    got = cache.read([20, 0])
    assert torch.equal(got[0], torch.cat(ks)) and torch.equal(got[1], torch.cat(vs))
    fresh = P.PagedCache(2, 8, 16, KV, DIM, 4, REV, FP)
    fresh.open(0, None)
    fresh.write(torch.cat(ks), torch.cat(vs), [20, 0])
    assert torch.equal(cache.attend(q, 0.125), fresh.attend(q, 0.125))
