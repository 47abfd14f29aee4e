"""Attention whose heads are cut into parts (tables of more than 1024 rows): head sizes, groups, windows, refused pages
and parts that have no row, on both ways of joining parts."""
import math

import pytest
import torch

import paper_2608_06690_amd as P
from tests.decode_cases import Cache, log, randn
from tests.test_gpu_attn_decode import call, check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(BF16, False), (BF16, True), (F32, False)]
LENS = [1500, 0, 1100, 17, 1283]


def virtual_heads(R, kv, group):
    return R * kv * -(-group // 16)


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,group,dim,page", [
    (1, 1, 32, 16), (1, 9, 32, 16), (2, 24, 32, 32), (2, 16, 64, 48), (1, 40, 96, 16), (3, 5, 96, 64), (1, 12, 128, 16), (2, 3, 160, 16),
    (1, 17, 160, 80), (1, 9, 192, 16), (2, 8, 224, 112), (1, 24, 224, 16), (1, 1, 256, 256), (1, 40, 256, 16),
    (16, 1, 32, 16), (14, 9, 64, 16), (8, 24, 96, 16), (13, 2, 160, 16), (7, 17, 224, 16), (13, 1, 256, 16)])
def test_head_sizes_and_groups(dt, q8, kv, group, dim, page):
    n = virtual_heads(len(LENS), kv, group)
    log(f"cut heads {dt} {q8} kv {kv} group {group} dim {dim} page {page}: {n} virtual heads")
    c = Cache(LENS, kv, dim, page, dt, q8)
    assert c.cols * page > 1024 and P.pmpe_attn_decode_workspace_bytes(c.desc, len(LENS), kv * group) > 0
    check(c, randn((len(LENS), kv * group, dim), 5, 1.0, dt), None, LENS, dim ** -0.5)


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,group", [(2, 3), (1, 11), (14, 1), (5, 18)])
def test_windows(dt, q8, kv, group):
    log(f"windows of cut heads {dt} {q8} kv {kv} group {group}")
    lens = [1400] * 8
    q = randn((8, kv * group, 64), 5, 1.0, dt)
    c = Cache(lens, kv, 64, 16, dt, q8)
    check(c, q, [0, 1, 15, 33, 777, 1000, 1399, 1400], lens, 0.125)
    check(c, q, [500, 31, 32, 1383, 1384, 2 ** 30, -7, 640], [1400, 1399, 1345, 1400, 1385, 1400, 1, 641], 0.125)


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,group,dim", [(2, 3, 64), (1, 12, 96), (14, 1, 32), (5, 18, 64)])
def test_refused_pages_and_parts_without_a_row(dt, q8, kv, group, dim):
    log(f"refused pages of cut heads {dt} {q8} kv {kv} group {group} dim {dim}")
    lens = [1500, 1500, 1500, 1500, 1100]
    c = Cache(lens, kv, dim, 16, dt, q8)
    c.tag[c.table[0, 10:60].long()] = 5             # rows 160 to 960: whole parts of every way to cut
    c.tag[c.table[1].long()[:94]] = 5               # all of it
    c.tag[c.table[2, 1::2].long()[:46]] = 5         # every other half tile
    bad = torch.cat([c.table[0, 10:60], c.table[1, :94], c.table[2, 1::2][:46]]).long()
    for name in ("k", "v"):                         # whose rows must not be seen, not even through 0 * inf
        getattr(c, name)[bad] = 0x7F if q8 else math.inf
    c.table[3, 0], c.table[3, 50], c.table[3, 93] = c.n_pages, -1, -2 ** 31
    q = randn((5, kv * group, dim), 5, 1.0, dt)
    bits = P.PMPE_DEV_CACHE_REFUSED | P.PMPE_DEV_CACHE_RANGE
    out, lse = check(c, q, None, lens, dim ** -0.5, bits)
    assert float(out[1].abs().max()) == 0 and bool(torch.isinf(lse[1]).all())
    check(c, q, [200, 0, 777, 30, 1090], [900, 1500, 1490, 1500, 1100], dim ** -0.5, bits)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_rows_out_of_the_window_may_hold_anything(dt, q8):
    log(f"anything outside {dt} {q8}")
    lens, first = [1270, 1500, 1100], [40, 611, 1050]
    c = Cache(lens, 2, 64, 32, dt, q8)
    used = torch.zeros(c.n_pages, 32, dtype=torch.bool)
    for r in range(3):
        for p in range(first[r], lens[r]):
            used[int(c.table[r, p // 32]), p % 32] = True
    for name in ("k", "v"):
        for j, x in enumerate((math.nan, math.inf, -math.inf)):
            m = ~used
            m[:, [i for i in range(32) if i % 3 != j]] = False
            if q8:
                getattr(c, name).masked_fill_(m[:, None, :, None], 0x7F)
                getattr(c, name + "s").masked_fill_(m[:, None, None, :], 255)
            else:
                getattr(c, name).masked_fill_(m[:, None, :, None], x)
    check(c, randn((3, 6, 64), 5, 1.0, dt), first, lens, 0.125)


@pytest.mark.parametrize("group", [3, 12, 24])
def test_equal_calls_have_equal_bits(group):
    log(f"equal bits, group {group}")
    lens = [3000, 17, 900, 0, 5000]
    c = Cache(lens, 2, 96, 16, BF16, True)
    q = randn((5, 2 * group, 96), 5, 1.0, BF16).cuda()
    dev = c.cuda()
    a = call(c, q, None, lens, 0.1, dev=dev)
    for _ in range(4):
        b = call(c, q, None, lens, 0.1, dev=dev)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
