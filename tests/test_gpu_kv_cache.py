"""Keys and values written into a paged cache and read back, against a plain form on the host: both are exact."""
import pytest
import torch

import paper_2608_06690_amd as P
from tests.decode_cases import Cache, log, quantise, randn, values

pytestmark = pytest.mark.gpu
TYPES = [(torch.bfloat16, True), (torch.bfloat16, False), (torch.float32, False)]


def i32(v):
    return torch.tensor(v, dtype=torch.int32)


def wanted(c, k, v, off, lens):
    """The cache's arrays after the write, and the status word."""
    out = {n: None if getattr(c, n) is None else getattr(c, n).clone() for n in ("k", "v", "ks", "vs")}
    status = 0
    for r in range(c.R):
        for t in range(off[r], off[r + 1]):
            pos = lens[r] - (off[r + 1] - t)
            p = c.usable(r, pos)
            if p is None:
                inside = 0 <= pos < c.cols * c.page and 0 <= int(c.table[r, pos // c.page]) < c.n_pages
                status |= P.PMPE_DEV_CACHE_REFUSED if inside else P.PMPE_DEV_CACHE_RANGE
                continue
            for name, x in (("k", k), ("v", v)):
                if c.q8:
                    q, e = quantise(x[t].float())
                    out[name][p, :, pos % c.page] = q
                    out[name + "s"][p, :, :, pos % c.page] = e
                else:
                    out[name][p, :, pos % c.page] = x[t]
    return out, status


def same(a, b):
    """Equal bits, NaN as any NaN."""
    if a is None:
        return b is None
    b = b.cpu()
    if a.dtype == torch.uint8:
        return torch.equal(a, b)
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def write(c, k, v, off, lens, seed=0):
    (table, tag, words), cache = c.cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    qkv = torch.cat([randn((k.shape[0], 3, c.dim), 99, 1.0, c.dt), k, v], dim=1).cuda()  # parts of one projection
    P.pmpe_kv_write(c.desc, qkv[:, 3:3 + c.kv], qkv[:, 3 + c.kv:], i32(off).cuda(), i32(lens).cuda(), table, tag, words, *cache, st)
    torch.cuda.synchronize()
    return cache, int(st)


def check_write(c, k, v, off, lens):
    cache, status = write(c, k, v, off, lens)
    want, bits = wanted(c, k, v, off, lens)
    for name, got in zip(("k", "v", "ks", "vs"), cache):
        assert same(want[name], got), name
    assert status == bits


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,dim,page,new,before", [
    (1, 32, 16, [1], [0]), (2, 64, 16, [1, 1, 1, 1, 1], [0, 15, 16, 17, 100]), (5, 96, 48, [47, 0, 49, 1], [0, 3, 48, 95]),
    (4, 128, 64, [130, 1, 63], [5, 64, 0]), (3, 256, 32, [33, 0, 0, 7], [31, 0, 9, 32]), (16, 160, 16, [3, 20], [0, 1])])
def test_write(dt, q8, kv, dim, page, new, before):
    log(f"write {dt} {q8} kv {kv} dim {dim} page {page} {new} {before}")
    lens = [a + b for a, b in zip(new, before)]
    c = Cache(lens, kv, dim, page, dt, q8)
    off = [sum(new[:r]) for r in range(len(new) + 1)]
    k, v = randn((off[-1], kv, dim), 7, 1.0, dt), randn((off[-1], kv, dim), 8, 3.0, dt)
    check_write(c, k, v, off, lens)


@pytest.mark.parametrize("q8", [True, False])
def test_write_of_a_padded_batch_leaves_the_rest(q8):
    log(f"padded batch {q8}")
    # tokens ahead of the first request, behind the last, and none at all
    c = Cache([20, 30], q8=q8)
    k, v = randn((40, 2, 64), 1, 1.0, torch.bfloat16), randn((40, 2, 64), 2, 1.0, torch.bfloat16)
    check_write(c, k, v, [4, 10, 29], [20, 30])
    check_write(c, k, v, [0, 0, 0], [20, 30])
    check_write(c, k, v, [40, 40, 40], [20, 30])


@pytest.mark.parametrize("q8", [True, False])
def test_write_refuses_pages_of_another_decision(q8):
    log(f"refused pages {q8}")
    c = Cache([40, 40, 40, 40, 40], q8=q8)
    c.table[0, 1] = c.table[1, 1]     # allow meets a page of deny
    c.table[2, 0] = c.table[0, 0]     # two allow requests, one page: one of them writes it
    c.tag[int(c.table[3, 2])] = 12345  # a malformed tag
    c.table[4, 0], c.table[4, 1] = c.n_pages, -1
    off = [0, 40, 40, 62, 102, 142]
    k, v = randn((142, 2, 64), 1, 1.0, torch.bfloat16), randn((142, 2, 64), 2, 1.0, torch.bfloat16)
    check_write(c, k, v, off, [40, 40, 40, 40, 40])
    # without words every request denies; without tags none is refused
    c.words = None
    check_write(c, k, v, off, [40, 40, 40, 40, 40])
    c = Cache([40, 40], q8=q8, tags=False)
    check_write(c, k[:80], v[:80], [0, 40, 80], [40, 40])


@pytest.mark.parametrize("lens", [[5, 20], [-3, 20], [32, 60], [2 ** 31 - 1, -2 ** 31]])
def test_write_of_positions_outside_the_table(lens):
    log(f"positions outside {lens}")
    c = Cache([32, 32], extra_cols=0)
    k, v = randn((20, 2, 64), 1, 1.0, torch.bfloat16), randn((20, 2, 64), 2, 1.0, torch.bfloat16)
    check_write(c, k, v, [0, 10, 20], lens)


def test_write_of_values_at_the_ends_of_the_range():
    log("ends of the range")
    for dt in (torch.bfloat16,):
        c = Cache([40], 1, 64, 16, dt, True)
        k = randn((40, 1, 64), 1, 1.0, dt)
        for t, x in enumerate([0.0, -0.0, 1e-38, 1e-40, 3e38, 448.0, 449.0, 464.0, 1.75, 1.7578125, 0.875, 2.0 ** -126]):
            k[t] = x
            k[t, 0, 5] = -x / 4
        k[20, 0, 3], k[21, 0, 40], k[22, 0, 63] = float("nan"), float("inf"), -float("inf")
        check_write(c, k, k.flip(0), [0, 40], [40])


@pytest.mark.parametrize("dt,q8", TYPES)
@pytest.mark.parametrize("kv,dim,page,n,first", [
    (1, 32, 16, [1], None), (2, 64, 16, [0, 5, 16, 33], [3, 0, 16, 15]), (5, 96, 48, [60, 100], [0, 47]), (4, 128, 64, [130, 1], None),
    (2, 256, 32, [31, 2, 64], [1, 31, 32])])
def test_read(dt, q8, kv, dim, page, n, first):
    log(f"read {dt} {q8} kv {kv} dim {dim} page {page} {n} {first}")
    at = first or [0] * len(n)
    c = Cache([a + b for a, b in zip(n, at)], kv, dim, page, dt, q8)
    off = [3 + sum(n[:r]) for r in range(len(n) + 1)]
    check_read(c, off, first, off[-1] + 5)


def check_read(c, off, first, T):
    (table, tag, words), cache = c.cuda()
    k, v = (torch.full((T, c.kv, c.dim), 7.0, dtype=c.dt, device="cuda") for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.pmpe_kv_read(c.desc, k, v, i32(off).cuda(), None if first is None else i32(first).cuda(), table, tag, words, *cache, st)
    torch.cuda.synchronize()
    for name, got in (("k", k), ("v", v)):
        want = torch.full((T, c.kv, c.dim), 7.0, dtype=c.dt)
        for r in range(c.R):
            for t in range(off[r], off[r + 1]):
                pos = (first[r] if first else 0) + t - off[r]
                p = c.usable(r, pos)
                want[t] = 0 if p is None else c.row(name, p, pos % c.page).to(c.dt)
        assert same(want, got), name
    return int(st)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_read_gives_zeros_for_pages_of_another_decision(dt, q8):
    log(f"read refused {dt} {q8}")
    c = Cache([40, 40, 40], dt=dt, q8=q8)
    assert check_read(c, [0, 40, 80, 120], None, 120) == 0
    c.table[0, 1] = c.table[1, 1]
    assert check_read(c, [0, 40, 80, 120], None, 120) == P.PMPE_DEV_CACHE_REFUSED
    c.table[2, 2] = c.n_pages + 7
    assert check_read(c, [0, 40, 80, 120], None, 120) == P.PMPE_DEV_CACHE_REFUSED | P.PMPE_DEV_CACHE_RANGE


def test_read_of_exponents_at_their_ends():
    log("exponents at their ends")
    c = Cache([32], 1, 32, 32, torch.bfloat16, True)
    c.ks[int(c.table[0, 0]), 0, 0, :5] = torch.tensor([0, 1, 254, 255, 127], dtype=torch.uint8)
    c.k[int(c.table[0, 0]), 0, 2] = 0x38  # 1.0: 2^127 is finite
    check_read(c, [0, 32], None, 32)


@pytest.mark.parametrize("dt,q8", TYPES)
def test_written_rows_come_back(dt, q8):
    log(f"round trip {dt} {q8}")
    c = Cache([70, 3], 3, 96, 16, dt, q8)
    k, v = randn((73, 3, 96), 1, 1.0, dt), randn((73, 3, 96), 2, 1.0, dt)
    (table, tag, words), _ = c.cuda()
    cache, status = write(c, k, v, [0, 70, 73], [70, 3])
    assert status == 0
    for n, t in zip(("k", "v", "ks", "vs"), cache):
        setattr(c, n, None if t is None else t.cpu())
    assert check_read(c, [0, 70, 73], None, 73) == 0
    if not q8:
        assert torch.equal(c.rows("k", 0, 0, 70).to(dt), k[:70])


def test_offsets_past_32_bits():
    log("offsets past 32 bits")
    # 2^32 bytes lie behind page 16384 of the 8-bit cache
    kv, dim, page, n = 8, 128, 256, 16400
    desc = P.make_cache_desc(n, page, kv, dim, 2, fp8=True)
    cache = [torch.zeros(n, kv, page, dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(n, kv, dim // 32, page, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = i32([[16399, 3]]).cuda()
    k, v = randn((300, kv, dim), 1, 1.0, torch.bfloat16).cuda(), randn((300, kv, dim), 2, 1.0, torch.bfloat16).cuda()
    P.pmpe_kv_write(desc, k, v, i32([0, 300]).cuda(), i32([300]).cuda(), table, None, None, *cache, *scale, None)
    back = [torch.empty_like(k), torch.empty_like(v)]
    P.pmpe_kv_read(desc, *back, i32([0, 300]).cuda(), None, table, None, None, *cache, *scale, None)
    for x, y in ((k, back[0]), (v, back[1])):
        q, e = quantise(x.cpu().float())
        assert torch.equal(values(q, e).to(torch.bfloat16), y.cpu())
    q, _ = quantise(k.cpu().float())
    assert torch.equal(cache[0][16399].cpu(), q[:256].transpose(0, 1)) and int(cache[0][:3].max()) == 0


def test_a_step_on_another_stream_and_captured():
    log("stream and capture")
    c = Cache([50, 50, 50], q8=True)
    (table, tag, words), cache = c.cuda()
    off, lens = i32([0, 1, 2, 3]).cuda(), i32([10, 20, 30]).cuda()
    k, v = randn((3, 2, 64), 1, 1.0, torch.bfloat16).cuda(), randn((3, 2, 64), 2, 1.0, torch.bfloat16).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        P.pmpe_kv_write(c.desc, k, v, off, lens, table, tag, words, *cache, None)
        lens.add_(1)
    host = [10, 20, 30]
    for step in range(4):
        k.copy_(randn((3, 2, 64), 10 + step, 1.0, torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        want, _ = wanted(c, k.cpu(), v.cpu(), [0, 1, 2, 3], host)
        for name, got in zip(("k", "v", "ks", "vs"), cache):
            assert same(want[name], got), name
            setattr(c, name, want[name])
        host = [n + 1 for n in host]
    # the same call on a stream that is given
    cache2 = [t.cuda() for t in (c.k, c.v, c.ks, c.vs)]
    lens2 = i32(host).cuda()
    s.wait_stream(torch.cuda.current_stream())
    P.pmpe_kv_write(c.desc, k, v, off, lens2, table, tag, words, *cache2, None, stream=s)
    s.synchronize()
    want, _ = wanted(c, k.cpu(), v.cpu(), [0, 1, 2, 3], host)
    assert all(same(want[n], got) for n, got in zip(("k", "v", "ks", "vs"), cache2))

