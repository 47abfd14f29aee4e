"""Sampling a token per row, against the definition in 64 bits on the host (sorted rows, cumulated masses).

A choice may go either way only where a cumulated mass comes within 2^-40 of its threshold: the tests accept
what the definition gives with the threshold moved by that much to either side."""
import math

import numpy as np
import pytest
import torch

import paper_2608_06690_amd as P
from tests.decode_cases import gen, log

pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -40


def choices(z, t, k, p, least, u):
    """[(token, prob, kept)] that the definition allows for one row (numpy float32 logits)."""
    z = np.where(z > -np.inf, np.minimum(z, np.finfo(np.float32).max), -np.inf).astype(np.float64)
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if len(order) == 0:
        return [(-1, 0.0, 0)]
    if not t > 0:
        return [(int(order[0]), 1.0, 1)]
    z = z[order]
    m = np.exp((z - z[0]) / np.float64(t))
    n = min(k, len(m)) if k > 0 else len(m)
    out = []
    for e in (0.0, -NEAR, NEAR):
        cut = n
        if p < 1:
            c = np.cumsum(m[:n])
            cut = min(n, max(1, int(np.searchsorted(c, max(p, 0.0) * c[-1] * (1 + e))) + 1))
        if least > 0:
            cut = min(cut, max(1, int((m[:cut] >= min(least, 1.0) * (1 + e)).sum())))
        c = np.cumsum(m[:cut])
        x = u if u > 0 else 0.0
        for f in (0.0, -NEAR, NEAR):
            j = min(cut - 1, int(np.searchsorted(c, x * c[-1] * (1 + f), side="right")))
            out.append((int(order[j]), m[j] / c[-1], cut))
    return out


def call(logits, par, u, prob=True, ws_fill=0xFF):
    B, V = logits.shape
    dev = {n: None if x is None else torch.tensor(x, dtype=torch.int32 if n == "top_k" else torch.float32).cuda() for n, x in par.items()}
    token = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    pr, kept = (torch.full((B,), 9.0, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda")) if prob else (None, None)
    ws = torch.full((max(16, P.pmpe_sample_workspace_bytes(B, V)),), ws_fill, dtype=torch.uint8, device="cuda")
    P.pmpe_sample(logits, *(dev.get(n) for n in ("temperature", "top_k", "top_p", "min_p")),
                  torch.tensor(u, dtype=torch.float32).cuda(), token, pr, kept, ws)
    torch.cuda.synchronize()
    return token.cpu(), None if pr is None else pr.cpu(), None if kept is None else kept.cpu()


DEFAULT = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


def check(z, par, u):
    """z [B, V] on the host; par: lists of B values, or missing."""
    token, prob, kept = call(z.cuda(), par, u)
    f = z.float().numpy()
    u = np.asarray(u, dtype=np.float32)
    for b in range(z.shape[0]):
        v = [np.float32(par[n][b]) if n != "top_k" and par.get(n) is not None else par[n][b] if par.get(n) is not None else d
             for n, d in DEFAULT.items()]
        fits = choices(f[b], float(v[0]), int(v[1]), float(v[2]), float(v[3]), float(u[b]))
        got = (int(token[b]), int(kept[b]))
        near = [x for x in fits if (x[0], x[2]) == got]
        assert near, (b, v, float(u[b]), got, fits[0])
        # masses and sums in 64 bits, the quotient rounded once
        assert abs(float(prob[b]) - near[0][1]) <= 2.0 ** -23 * near[0][1] + 1e-40, (b, float(prob[b]), near[0][1])
    return token, prob, kept


def logits(B, V, seed, dt=torch.float32, std=2.5):
    z = torch.randn(B, V, generator=gen(seed)) * std
    z.scatter_add_(1, torch.randint(0, V, (B, min(V, 20)), generator=gen(seed + 1)),
                   torch.empty(B, min(V, 20)).exponential_(0.25, generator=gen(seed + 2)))
    return z.to(dt)


def uniform(B, seed):
    u = torch.rand(B, generator=gen(seed)).tolist()
    u[0] = 0.0
    u[-1] = 1.0 - 2.0 ** -24
    return u


MODES = {
    "free": {}, "cold": dict(temperature=0.3), "hot": dict(temperature=3.0), "greedy": dict(temperature=0.0),
    "top_k": dict(temperature=0.8, top_k=50), "one": dict(top_k=1), "many": dict(top_k=3000), "top_p": dict(temperature=0.8, top_p=0.9),
    "most": dict(top_p=0.999), "least": dict(top_p=0.0), "min_p": dict(min_p=0.05), "all": dict(temperature=0.9, top_k=200, top_p=0.95, min_p=0.01),
    "wide": dict(temperature=1.5, top_k=5000, top_p=0.99, min_p=1e-5)}
SIZES = [1, 2, 3, 63, 64, 65, 511, 512, 513, 1000, 4095, 4097, 8191, 16385, 50001, 131071]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", SIZES)
def test_modes(V, dt):
    log(f"sample V {V} {dt}")
    rows = [m for m in MODES for _ in range(3)]
    par = {n: [MODES[m].get(n, d) for m in rows] for n, d in DEFAULT.items()}
    check(logits(len(rows), V, V, dt), par, uniform(len(rows), V + 1))


@pytest.mark.parametrize("B,V", [(1, 262144), (1, 524288), (2, 200003), (200, 5003), (600, 129)])
def test_rows_and_sizes(B, V):
    log(f"sample {B} x {V}")
    rows = [list(MODES)[(b * 5 + 3) % len(MODES)] for b in range(B)]
    par = {n: [MODES[m].get(n, d) for m in rows] for n, d in DEFAULT.items()}
    check(logits(B, V, B + V), par, uniform(B, 3))


@pytest.mark.parametrize("V", [40, 5000, 70001])
def test_ties(V):
    log(f"ties {V}")
    names = list(MODES)
    par = {n: [MODES[m].get(n, d) for m in names] for n, d in DEFAULT.items()}
    B = len(names)
    u = torch.rand(B, generator=gen(5)).tolist()
    check(torch.zeros(B, V), par, u)                                   # all equal
    check(torch.full((B, V), -3.25, dtype=torch.bfloat16), par, u)
    check(torch.round(logits(B, V, 1)), par, u)                        # few values
    z = torch.zeros(B, V)
    z[:, ::2] = -0.0                                                   # -0 is 0
    check(z, par, u)
    z = torch.full((B, V), 1.0)
    z[:, V // 3] = 30.0                                                # one above a plain
    check(z, par, u)
    check(-z, par, u)


def test_thresholds_that_are_met():
    log("thresholds that are met")
    z = torch.zeros(8, 8)
    # four of eight equal tokens hold a half; u of a quarter of four is the second's start
    check(z, dict(top_p=[0.5] * 8), [0.0, 0.25, 0.5, 0.75, 0.125, 0.999, 0.25, 0.5])
    token, prob, kept = call(z.cuda(), dict(top_p=[0.5] * 8), [0.0, 0.25, 0.5, 0.75, 0.125, 0.999, 0.25, 0.5])
    assert kept.tolist() == [4] * 8 and token.tolist() == [0, 1, 2, 3, 0, 3, 1, 2] and prob.tolist() == [0.25] * 8
    z = torch.tensor([[0.0, 1.0, 1.0, -2.0]] * 3)
    _, _, kept = check(z, dict(min_p=[1.0, 1.5, 0.9]), [0.9] * 3)
    assert kept.tolist() == [2, 2, 2]


@pytest.mark.parametrize("V", [7, 3000, 40000])
def test_masked_and_infinite_logits(V):
    log(f"masked {V}")
    inf, nan = math.inf, math.nan
    low = torch.finfo(torch.float32).min
    for fill in (-inf, nan, low):
        z = torch.full((6, V), fill)
        z[1, V - 1] = -5.0
        z[2, [1, 3]] = 2.0
        z[3, 2], z[3, 5] = inf, 3e38
        z[4, 1:5] = inf
        z[5, ::2] = torch.randn(len(range(0, V, 2)), generator=gen(1))
        for par in ({}, dict(top_k=[3] * 6), dict(top_p=[0.7] * 6), dict(min_p=[0.1] * 6), dict(temperature=[0.0] * 6),
                    dict(temperature=[0.5] * 6, top_k=[V] * 6, top_p=[0.5] * 6)):
            token, prob, kept = check(z, par, [0.3, 0.9, 0.6, 0.2, 0.7, 0.5])
            if fill != low:
                assert int(token[0]) == -1 and int(kept[0]) == 0 and float(prob[0]) == 0


def test_parameters_at_their_ends():
    log("parameters at their ends")
    nan, inf = math.nan, math.inf
    B, V = 12, 3001
    z = logits(B, V, 9)
    base = dict(temperature=[0.7] * B, top_k=[0] * B, top_p=[1.0] * B, min_p=[0.0] * B)
    u = torch.rand(B, generator=gen(2)).tolist()
    check(z, dict(base, temperature=[0.0, -1.0, nan, 1e-30, 1e-45, 1e30, inf, 1e-3, 0.01, 100.0, 1e5, 1.0]), u)
    check(z, dict(base, top_k=[-1, -2 ** 31, 2 ** 31 - 1, V, V - 1, V + 1, 1, 2, 64, 2048, 2049, 1024]), u)
    check(z, dict(base, top_p=[nan, 2.0, 1.0, -1.0, 0.0, 1e-30, 1 - 2.0 ** -24, 0.5, inf, -inf, 1e-7, 0.99]), u)
    check(z, dict(base, min_p=[nan, -1.0, 0.0, 1e-30, 1.0, 2.0, inf, -inf, 1e-10, 0.5, 0.999, 1e-3]), u)
    check(z, base, [0.0, -1.0, nan, 1.0, 2.0, inf, 1 - 2.0 ** -24, 1e-30, -inf, 0.5, 0.25, 0.75])


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_spread_logits(dt):
    log(f"spread {dt}")
    # masses over hundreds of orders of magnitude, a plain with a spike, a crowd at the far end
    V = 20011
    rows = [torch.linspace(-300, 300, V), torch.linspace(300, -300, V), torch.randn(V, generator=gen(1)) * 1e-4,
            torch.randn(V, generator=gen(2)) * 100, torch.cat([torch.tensor([80.0]), torch.randn(V - 1, generator=gen(3))]),
            torch.cat([torch.randn(V - 1, generator=gen(3)) * 0.01 + 40, torch.tensor([41.0])]), torch.randn(V, generator=gen(4)) * 3e37,
            torch.arange(V) * 1e-6]
    z = torch.stack(rows).to(dt)
    for par in ({}, dict(top_p=[0.9] * 8), dict(top_k=[7000] * 8, top_p=[0.8] * 8), dict(min_p=[0.3] * 8), dict(temperature=[20.0] * 8),
                dict(temperature=[0.05] * 8, top_p=[0.99] * 8), dict(temperature=[1e3] * 8, top_k=[15000] * 8)):
        check(z, par, [0.5, 0.999, 0.3, 0.7, 0.99, 0.9, 0.1, 0.8])


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_strided_rows_and_optional_outputs(dt):
    log(f"strides {dt}")
    z = logits(5, 4099, 3, dt)
    wide = torch.full((5, 4111), math.inf, dtype=dt)
    wide[:, 3:4102] = z
    par, u = dict(top_p=[0.9] * 5), [0.1, 0.3, 0.5, 0.7, 0.9]
    a = call(z.cuda(), par, u)
    b = call(wide.cuda()[:, 3:4102], par, u, prob=False)
    assert torch.equal(a[0], b[0])
    c = call(z.cuda(), par, u, ws_fill=0)
    assert all(torch.equal(x, y) for x, y in zip(a, c))


def test_frequencies():
    log("frequencies")
    # 4096 numbers over one row: each token's share is its mass, to one number's weight
    z = logits(1, 37, 4)
    n = 4096
    u = ((torch.arange(n) + 0.5) / n).tolist()
    token, _, _ = call(z.expand(n, 37).contiguous().cuda(), {}, u)
    w = torch.softmax(z[0].double(), dim=0)
    share = torch.bincount(token.long(), minlength=37).double() / n
    assert float((share - w).abs().max()) <= 1.0 / n + 1e-9


def test_captured_draws():
    log("captured draws")
    B, V = 6, 33333
    z, u = logits(B, V, 1).cuda(), torch.rand(B).cuda()
    par = dict(temperature=[0.8] * B, top_k=[0, 50, 0, 4000, 0, 1], top_p=[0.9, 1, 0.5, 0.9, 1, 1], min_p=[0, 0, 0, 0, 0.1, 0])
    dev = [torch.tensor(par[n], dtype=torch.int32 if n == "top_k" else torch.float32).cuda() for n in DEFAULT]
    token, prob, kept = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, P.pmpe_sample_workspace_bytes(B, V)), dtype=torch.uint8, device="cuda")
    P.pmpe_sample(z, *dev, u, token, prob, kept, ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.pmpe_sample(z, *dev, u, token, prob, kept, ws)
    for i in range(4):
        z.copy_(logits(B, V, 20 + i))
        u.copy_(torch.rand(B, generator=gen(i)))
        g.replay()
        torch.cuda.synchronize()
        a = token.cpu(), prob.cpu(), kept.cpu()
        b = check(z.cpu(), par, u.tolist())
        assert all(torch.equal(x, y) for x, y in zip(a, b))
