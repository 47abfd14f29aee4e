"""Attention of one new token per request over a paged cache, against a plain form in 64 bits on the host."""
import math

import pytest
import torch

import paper_2608_06690_amd as P
from tests import decode_cases as D
from tests.decode_cases import Cache, log, randn

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(BF16, False), (BF16, True), (F32, False)]


def i32(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32).cuda()


def call(c, q, first, lens, scale, lse=True, dev=None, stream=None):
    (table, tag, words), cache = dev or c.cuda()
    R, heads, _ = q.shape
    out = torch.full((R, heads, c.dim), 9.0, dtype=c.dt, device="cuda")
    ls = torch.full((R, heads), 9.0, device="cuda") if lse else None
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = P.pmpe_attn_decode_workspace_bytes(c.desc, R, heads)
    ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN everywhere
    P.pmpe_attn_decode(c.desc, q, i32(first), i32(lens), table, tag, words, *cache, scale, out, ls, st, ws, stream)
    torch.cuda.synchronize()
    return out, ls, int(st)


def check(c, q, first, lens, scale, status=0):
    out, lse, st = call(c, q.cuda(), first, lens, scale)
    want, wlse, spread, most = D.attend(c, q, first, lens, scale)
    n = max(lens)
    err = (out.cpu().double() - want).abs()
    tol = D.tolerance(c.dt, c.dim, n, spread, most, want)
    ratio = float((err / tol).max())  # (NaN where either is)
    assert ratio <= 1.0, ratio
    got = lse.cpu().double()
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(got), empty)
    assert bool(((got - wlse).abs()[~empty] <= D.lse_tolerance(c.dim, n, most, wlse)[~empty]).all())
    assert st == status
    return out, lse


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 300]


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,group,dim,page", [
    (1, 1, 32, 16), (2, 8, 128, 16), (4, 4, 64, 32), (1, 16, 128, 48), (3, 5, 96, 16), (1, 24, 128, 64), (2, 9, 256, 16),
    (2, 7, 160, 80), (1, 40, 192, 256), (1, 3, 224, 112)])
def test_lengths_heads_and_pages(dt, q8, kv, group, dim, page):
    log(f"attend {dt} {q8} kv {kv} group {group} dim {dim} page {page}")
    c = Cache(LENS, kv, dim, page, dt, q8)
    check(c, randn((len(LENS), kv * group, dim), 5, 1.0, dt), None, LENS, dim ** -0.5)


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("lens", [[5000], [3000, 1, 700, 0, 2049], [1024] * 40])
def test_long_and_ragged(dt, q8, lens):
    log(f"long {dt} {q8} {lens[:5]}")
    c = Cache(lens, 2, 128, 16, dt, q8)
    check(c, randn((len(lens), 8, 128), 5, 2.0, dt), None, lens, 128 ** -0.5)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_windows(dt, q8):
    log(f"windows {dt} {q8}")
    lens = [100, 100, 100, 100, 100, 100, 700, 700, 700]
    first = [0, 1, 15, 16, 99, 100, 690, 512, 333]
    c = Cache(lens, 2, 64, 16, dt, q8)
    q = randn((9, 6, 64), 5, 1.0, dt)
    check(c, q, first, lens, 0.125)
    # windows past the end or before the start
    check(c, q, [200, -4, 2 ** 30, 99, 98, 97, 0, 700, 701], lens, 0.125)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_rows_out_of_the_window_may_hold_anything(dt, q8):
    log(f"anything outside {dt} {q8}")
    lens, first = [70, 33, 500, 17, 48], [20, 0, 130, 16, 5]
    c = Cache(lens, 2, 64, 32, dt, q8)
    q = randn((5, 6, 64), 5, 1.0, dt)
    used = torch.zeros(c.n_pages, 32, dtype=torch.bool)
    for r in range(5):
        for p in range(first[r], lens[r]):
            used[int(c.table[r, p // 32]), p % 32] = True
    for name, x in (("k", math.nan), ("v", math.inf)):
        for j, y in enumerate((x, -x, torch.finfo(dt).min if not q8 else x)):
            m = ~used
            m[:, j::3] &= True
            if q8:
                getattr(c, name).masked_fill_(m[:, None, :, None], 0x7F)
                getattr(c, name + "s").masked_fill_(m[:, None, None, :], 255)
            else:
                m[:, [i for i in range(32) if i % 3 != j]] = False
                getattr(c, name).masked_fill_(m[:, None, :, None], y)
    check(c, q, first, lens, 0.125)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_refused_pages_take_no_part(dt, q8):
    log(f"refused {dt} {q8}")
    lens = [100, 100, 100, 100, 100, 300]
    c = Cache(lens, 2, 64, 16, dt, q8)
    bad = c.table[1, 1:3].clone()
    c.table[0, 2], c.table[0, 6] = bad[0], bad[1]  # an allow request meets pages of deny
    for name in ("k", "v"):  # whose rows must not be seen, not even through 0 * inf
        getattr(c, name)[bad.long()] = 0x7F if q8 else math.inf
    c.tag[c.table[2].long()[:7]] = 5               # all pages of request 2 malformed
    lens2 = [100, 0, 100, 100, 100, 300]
    out, lse = check(c, randn((6, 4, 64), 5, 1.0, dt), None, lens2, 0.125, P.PMPE_DEV_CACHE_REFUSED)
    assert float(out[2].abs().max()) == 0 and bool(torch.isinf(lse[2]).all())
    c.table[5, 3], c.table[5, 18] = c.n_pages, -1  # the last one a page of its own
    check(c, randn((6, 4, 64), 6, 1.0, dt), None, lens2, 0.125, P.PMPE_DEV_CACHE_REFUSED | P.PMPE_DEV_CACHE_RANGE)
    c.words = None                                 # every request denies, and request 0 may read its deny pages
    for name in ("k", "v"):
        getattr(c, name)[bad.long()] = 0
    check(c, randn((6, 4, 64), 6, 1.0, dt), None, lens2, 0.125, P.PMPE_DEV_CACHE_REFUSED | P.PMPE_DEV_CACHE_RANGE)


def test_lengths_outside_the_table():
    log("lengths outside")
    c = Cache([64, 64, 64], 2, 64, 16, extra_cols=0)
    q = randn((3, 4, 64), 5, 1.0, BF16)
    (table, tag, words), cache = c.cuda()
    got, lse, st = call(c, q.cuda(), None, [64, 2 ** 31 - 1, -2 ** 31], 0.125)
    want, wlse, spread, most = D.attend(c, q, None, [64, 64, 0], 0.125)
    tol = D.tolerance(BF16, 64, 64, spread, most, want)
    assert bool(((got.cpu().double() - want).abs() <= tol).all()) and st == P.PMPE_DEV_CACHE_RANGE
    assert float(got[2].abs().max()) == 0


@pytest.mark.parametrize("dt,q8", TYPES)
def test_large_scores_and_equal_ones(dt, q8):
    log(f"large scores {dt} {q8}")
    lens = [400, 64, 1]
    c = Cache(lens, 2, 64, 16, dt, q8)
    q = randn((3, 8, 64), 5, 1.0, dt)
    check(c, q, None, lens, 30.0)     # one weight near 1, the rest far below
    check(c, q, None, lens, -30.0)
    check(c, q, None, lens, 0.0)      # the mean
    c = Cache(lens, 2, 64, 16, dt, q8, std=0.0)
    check(c, q, None, lens, 1.0)
    # rising and falling maxima: each row's score is above, then below, all before
    for up in (1.0, -1.0):
        c = Cache([256], 1, 64, 16, F32 if dt == F32 else dt, False)
        for p in range(256):
            c.k[int(c.table[0, p // 16]), 0, p % 16] = up * (p - 128) / 8
        check(c, torch.ones(1, 2, 64, dtype=c.dt), None, [256], 0.25)


def test_a_row_that_is_not_finite_shows():
    log("not finite")
    for dt, q8 in TYPES:
        c = Cache([40, 40], 2, 64, 16, dt, q8)
        p = int(c.table[0, 1])
        if q8:
            c.vs[p, 1, 0, 3] = 255
        else:
            c.v[p, 1, 3, :32] = math.nan
        out, lse, _ = call(c, randn((2, 4, 64), 5, 1.0, dt).cuda(), None, [40, 40], 0.125)
        assert bool(torch.isnan(out[0, 2:, :32]).all()) and bool(torch.isfinite(out[0, :2]).all())
        assert bool(torch.isfinite(out[0, 2:, 32:]).all()) and bool(torch.isfinite(out[1]).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dt,q8", TYPES)
def test_strides_and_no_lse(dt, q8):
    log(f"strides {dt} {q8}")
    lens = [77, 130, 1]
    c = Cache(lens, 2, 64, 16, dt, q8, tags=False)
    q = randn((3, 8, 64), 5, 1.0, dt)
    wide = torch.full((3, 12, 64), math.nan, dtype=dt)
    wide[:, :8] = q
    a, _, _ = call(c, q.cuda(), None, lens, 0.125)
    b, _, _ = call(c, wide.cuda()[:, :8], None, lens, 0.125, lse=False)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_equal_calls_have_equal_bits(dt, q8):
    log(f"equal bits {dt} {q8}")
    lens = [3000, 17, 900, 0, 5000]
    c = Cache(lens, 4, 128, 16, dt, q8)
    q = randn((5, 32, 128), 5, 1.0, dt).cuda()
    dev = c.cuda()
    a = call(c, q, None, lens, 0.09, dev=dev)
    for _ in range(5):
        b = call(c, q, None, lens, 0.09, dev=dev)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_past_32_bits():
    log("offsets past 32 bits")
    n, kv, page, dim = 16400, 8, 256, 128  # 4.3e9 bytes of values each
    desc = P.make_cache_desc(n, page, kv, dim, 3, fp8=True)
    cache = [torch.zeros(n, kv, page, dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.full((n, kv, dim // 32, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    small = Cache([600], kv, dim, page, BF16, True, spare=0, extra_cols=0, tags=False)
    big = torch.tensor([16399, 2, 16390])
    at = small.table[0].long()
    for t, s in zip((*cache, *scale), (small.k, small.v, small.ks, small.vs)):
        t[big.cuda()] = s[at].cuda()
    q = randn((1, 32, dim), 5, 1.0, BF16)
    out = torch.empty_like(q, device="cuda")
    ws = torch.empty(max(16, P.pmpe_attn_decode_workspace_bytes(desc, 1, 32)), dtype=torch.uint8, device="cuda")
    P.pmpe_attn_decode(desc, q.cuda(), None, i32([600]), big.int().view(1, 3).cuda(), None, None, *cache, *scale, 0.09, out, None, None, ws)
    want, _, spread, most = D.attend(small, q, None, [600], 0.09)
    assert bool(((out.cpu().double() - want).abs() <= D.tolerance(BF16, dim, 600, spread, most, want)).all())


def test_captured_steps_over_a_growing_cache():
    log("captured steps")
    lens = [30, 700, 2000, 5]
    c = Cache([n + 8 for n in lens], 2, 128, 16, BF16, True)
    (table, tag, words), cache = c.cuda()
    q, ln = randn((4, 16, 128), 5, 1.0, BF16).cuda(), i32(lens)
    out, st = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.empty(4, 16, device="cuda")
    ws = torch.empty(max(16, P.pmpe_attn_decode_workspace_bytes(c.desc, 4, 16)), dtype=torch.uint8, device="cuda")

    def step():
        P.pmpe_attn_decode(c.desc, q, None, ln, table, tag, words, *cache, 0.09, out, lse, st, ws)
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
        ln.add_(1)
    for i in range(5):
        q.copy_(randn((4, 16, 128), 50 + i, 1.0, BF16))
        g.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), lse.clone()
        eager = call(c, q, None, [n + i for n in lens], 0.09, dev=((table, tag, words), cache))
        assert torch.equal(a, eager[0]) and torch.equal(b, eager[1])
    assert int(st) == 0


def test_two_streams_with_workspaces_of_their_own():
    log("two streams")
    lens = [900, 3000, 64, 0, 1500]
    c = Cache(lens, 4, 128, 16, BF16, False)
    dev, qs = c.cuda(), [randn((5, 32, 128), s, 1.0, BF16).cuda() for s in (1, 2)]
    want = [call(c, q, None, lens, 0.09, dev=dev)[0] for q in qs]
    streams, ln = [torch.cuda.Stream() for _ in qs], i32(lens)
    ws = [torch.empty(max(16, P.pmpe_attn_decode_workspace_bytes(c.desc, 5, 32)), dtype=torch.uint8, device="cuda") for _ in qs]
    outs = [torch.empty_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for q, s, w, o in zip(qs, streams, ws, outs):
            P.pmpe_attn_decode(c.desc, q, None, ln, *dev[0], *dev[1], 0.09, o, None, None, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("heads", [2, 18, 24])
def test_scales_at_their_ends(heads):
    log(f"scales at their ends {heads}")
    # one row: the output is that row, whatever its scales; NaN scales show in their block of 32 only
    ends = [1, 2, 60, 127, 200, 245, 246, 255]
    c = Cache([1], 2, 256, 16, BF16, True, tags=False)
    p = int(c.table[0, 0])
    c.vs[p, 0, :, 0] = torch.tensor(ends, dtype=torch.uint8)
    c.vs[p, 1, :, 0] = 127
    out, _, _ = call(c, randn((1, heads, 256), 5, 0.01, BF16).cuda(), None, [1], 0.01)
    want = c.rows("v", 0, 0, 1)[0].repeat_interleave(heads // 2, dim=0).to(BF16)
    got = out[0].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    small = want.double().abs() < 2.0 ** -120
    assert torch.equal(torch.nan_to_num(got)[~small], torch.nan_to_num(want)[~small])
    assert bool(((got.double() - want.double()).abs()[small] <= 2.0 ** -126).all())
    # a key of NaN spoils the heads that read it
    c.ks[p, 1, 3, 0] = 255
    out, lse, _ = call(c, randn((1, heads, 256), 5, 0.01, BF16).cuda(), None, [1], 0.01)
    assert bool(torch.isnan(out[0, heads // 2:]).all()) and bool(torch.isnan(lse[0, heads // 2:]).all())
    assert bool(torch.isfinite(lse[0, :heads // 2]).all())
