"""Routing by scores on the GPU against a token-by-token selection in 64 bits: score kinds, groups,
balance bias, pools from one expert to the largest, ties, masked and non-finite logits, both logit
types, the soft control; the gradient against the formula and against differences; the layer's
forward and training step with a score rule.

Tolerances: selections are equal. Gates are 64-bit values rounded to fp32 (2^-24, and 2^-40 for
the exponentials). The gradient is fp32: expf of an argument z - top of up to 32 is off by
2^-24 * 32 + 2 steps, s / sum and the products by a few steps: 2^-18 of the sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

import paper_2608_06690_amd as P
import workloads as W
from oracle import pmpe_oracle as O
from tests import pmpe_cases as C

pytestmark = pytest.mark.gpu
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)
BIG = float(np.finfo(np.float32).max)


def log(msg):
    print(msg, flush=True)


def scores(z, kind):
    """Scores of one pool's logits (fp64 list); masked ones 0."""
    live = [v > -math.inf for v in z]
    z = [min(v, BIG) if a else v for v, a in zip(z, live)]
    if kind == P.PMPE_SCORE_SIGMOID:
        return [0.0 if not a else 1.0 / (1.0 + math.exp(-v)) if v >= 0 else math.exp(v) / (1.0 + math.exp(v))
                for v, a in zip(z, live)], live
    top = max([v for v, a in zip(z, live) if a], default=0.0)
    e = [math.exp(v - top) if a else 0.0 for v, a in zip(z, live)]
    total = math.fsum(e)
    return [v / total if total else 0.0 for v in e], live


def choose(z, bias, k, rule, groups, keep, renorm):
    """Ids (ascending), gates and margin of one token over one pool."""
    s, live = scores(z, rule.score)
    u = [-math.inf] * len(z)
    for i, a in enumerate(live):
        if a and s[i] + bias[i] > -math.inf:
            u[i] = s[i] + bias[i]
    cand = range(len(z))
    if keep < groups:
        gs = len(z) // groups

        def rank(g):
            best = sorted((v for v in u[g * gs:(g + 1) * gs] if v > -math.inf), reverse=True)[:rule.group_top]
            if len(best) < 2 or math.isinf(sum(best)):
                return sum(best) if best else -math.inf
            m, e = math.frexp(sum(best))
            return math.ldexp(round(math.ldexp(m, 45)), e - 45)  # a sum of two ranks by 45 bits
        kept = sorted(sorted(range(groups), key=lambda g: (-rank(g), g))[:keep])
        cand = [i for g in kept for i in range(g * gs, (g + 1) * gs)]
    order = sorted(cand, key=lambda i: (-u[i], i))
    idx = sorted(order[:k])
    margin = math.inf
    if len(order) > k and u[order[k]] > -math.inf:
        margin = u[order[k - 1]] - u[order[k]] if u[order[k - 1]] != u[order[k]] else 0.0
    elif len(order) > k and u[order[k - 1]] == -math.inf:
        margin = 0.0
    if not renorm:
        gate = [s[i] for i in idx]
    elif rule.score == P.PMPE_SCORE_SIGMOID:
        total = sum(s[i] for i in idx) + 1e-20
        gate = [s[i] / total for i in idx]
    else:
        gate = scores([z[i] for i in idx], rule.score)[0]
    return idx, [g * rule.scale for g in gate], margin


def run(d, rule, logits, bias, words, margin=True):
    T, k = logits.shape[0], d.top_k
    out = dict(idx=torch.full((T, k), -7, dtype=torch.int32, device="cuda"), gate=torch.empty(T, k, device="cuda"),
               logit=torch.empty(T, k, device="cuda"), allow=torch.empty(T, dtype=torch.uint8, device="cuda"),
               margin=torch.empty(T, device="cuda") if margin else None)
    P.pmpe_select(d, rule, T, logits, bias, words, out["idx"], out["gate"], out["logit"], out["allow"], out["margin"])
    torch.cuda.synchronize()
    return out


def check(d, rule, logits, bias, words, soft=False):
    got = run(d, rule, logits, bias, words)
    T, k, n = logits.shape[0], d.top_k, d.n_pub
    renorm = d.gate_mode == P.PMPE_GATE_RENORM_TOPK
    z, b = logits.double().cpu().tolist(), (bias.double().cpu().tolist() if bias is not None else [0.0] * logits.shape[1])
    allow = (words.cpu() == ALLOW).tolist() if words is not None else [False] * T
    for t in range(T):
        first, last, g, keep = (0, n, rule.n_group_pub, rule.topk_group_pub)
        if allow[t]:
            first, last, g, keep = n, n + d.n_priv, rule.n_group_priv, rule.topk_group_priv
        if soft:
            first, last, g, keep = 0, n + d.n_priv, 1, 1
        idx, gate, margin = choose(z[t][first:last], b[first:last], k, rule, g, keep, renorm)
        assert got["idx"][t].tolist() == [first + i for i in idx], t
        assert got["allow"][t].item() == int(allow[t])
        zs = [z[t][first + i] for i in idx]
        np.testing.assert_array_equal(got["logit"][t].double().cpu().numpy(), zs)
        for a, e in zip(got["gate"][t].tolist(), gate):
            assert abs(a - e) <= (2.0 ** -24 + 2.0 ** -40) * abs(e) + 2.0 ** -149, (t, a, e)
        m = got["margin"][t].item()
        if math.isfinite(margin):
            size = max([1.0] + [abs(v) for v in b[first:last] if math.isfinite(v)])
            assert abs(m - margin) <= 2.0 ** -24 * margin + 2.0 ** -49 * size, (t, m, margin)
        else:
            assert m == margin, (t, m, margin)
    return got


def words_of(T, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.zeros(T, dtype=torch.int32)
    w[torch.rand(T, generator=g) < 0.5] = ALLOW
    w[::7] = 99  # malformed: denies
    return w.cuda()


def rand(shape, seed, std=1.0, dt=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=g)


# pub, priv, k, groups (of, stay), private groups, best of a group
POOLS = [(1, 1, 1, (1, 1), (1, 1), 1), (8, 4, 2, (1, 1), (1, 1), 2), (64, 16, 6, (8, 3), (4, 2), 2),
         (60, 20, 4, (5, 2), (4, 3), 1), (128, 32, 8, (1, 1), (2, 2), 1), (128, 32, 16, (4, 2), (2, 1), 2),
         (160, 24, 8, (8, 3), (3, 2), 2), (256, 256, 8, (8, 4), (64, 5), 2), (256, 64, 16, (64, 4), (64, 16), 2),
         (65, 63, 3, (13, 1), (9, 9), 2), (256, 16, 16, (2, 1), (1, 1), 1)]


@pytest.mark.parametrize("pools", POOLS, ids=str)
@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_selection(pools, score, renorm, dt):
    log(f"select {pools} score={score} renorm={renorm} {dt}")
    pub, priv, k, g, pg, top = pools
    d = P.make_desc(128, 64, pub, priv, k, gate_mode=P.PMPE_GATE_RENORM_TOPK if renorm else P.PMPE_GATE_POOL_SOFTMAX)
    rule = P.make_score_rule(score, g, pg, top, 2.5)
    z = rand((37, pub + priv), 1, 2.0, dt)
    bias = rand((pub + priv,), 2, 0.1)
    check(d, rule, z, bias, words_of(37, 3))
    check(d, rule, z[:5].contiguous(), None, None)  # no bias; every token denies


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("groups", [((1, 1), (1, 1)), ((8, 2), (4, 3))])
@pytest.mark.parametrize("renorm", [True, False])
def test_ties_masks_and_values_that_are_not_finite(score, groups, renorm):
    d = P.make_desc(128, 64, 64, 16, 6, gate_mode=P.PMPE_GATE_RENORM_TOPK if renorm else P.PMPE_GATE_POOL_SOFTMAX)
    rule = P.make_score_rule(score, *groups, 2, 1.0)
    z = torch.randint(-2, 3, (24, 80)).float().cuda()  # equal logits everywhere
    inf = math.inf
    z[0] = 0.0                       # nothing but ties
    z[1, 3:] = -inf                  # fewer live experts than top-k, in the public pool
    z[2] = -inf                      # a row that the mask leaves empty
    z[3] = float("nan")
    z[4, :60] = -inf                 # live experts in the last group only
    z[5, 10] = inf
    z[6, [7, 9]] = inf
    z[7] = torch.finfo(torch.float32).min   # a mask written as the type's lowest value
    z[8, :] = -300.0                 # every sigmoid underflows fp32
    z[9] = 200.0                     # every sigmoid is 1
    z[10, ::2] = float("nan")
    z[11] = 1e30
    z[12, 64:] = -inf
    z[13, 64:76] = -inf
    words = torch.zeros(24, dtype=torch.int32)
    words[12:] = ALLOW
    words = words.cuda()
    check(d, rule, z, None, words)
    bias = torch.zeros(80)
    bias[::3] = 0.25
    bias[5] = -inf
    bias[6] = float("nan")
    bias[70] = 1e30
    check(d, rule, z, bias.cuda(), words)


def test_groups_whose_sums_agree_but_for_rounding_tie():
    """s(z) + s(-z) is 1 for every z, up to the rounding of the two: the lower group stays."""
    d = P.make_desc(128, 64, 64, 16, 2)
    rule = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (32, 1), (8, 1), 2)
    half = rand((500, 40), 11, 2.0)
    z = torch.stack([half, -half], dim=2).reshape(500, 80).contiguous()
    words = torch.zeros(500, dtype=torch.int32)
    words[250:] = ALLOW
    got = check(d, rule, z, None, words.cuda())
    assert (got["idx"][:250].cpu() == torch.tensor([0, 1])).all() and (got["idx"][250:].cpu() == torch.tensor([64, 65])).all()


def test_near_ties_are_those_of_64_bits():
    """Logits and biases whose order fp32 scores cannot tell."""
    d = P.make_desc(128, 64, 128, 8, 8)
    z = 3.0 + torch.arange(128).double() * 2.0 ** -22
    perm = torch.randperm(128, generator=torch.Generator().manual_seed(5))
    z = torch.cat([z[perm], torch.zeros(8).double()]).float().repeat(5, 1).cuda()
    for score in (P.PMPE_SCORE_SIGMOID, P.PMPE_SCORE_SOFTMAX):
        rule = P.make_score_rule(score, (16, 6), (1, 1), 2)
        check(d, rule, z, None, None)
        bias = rand((136,), 6, 1e-9)
        check(d, rule, z, bias, None)


def test_soft_control_ranks_the_concatenated_pool():
    d = P.make_desc(128, 64, 200, 150, 16, route_mode=P.PMPE_ROUTE_SOFT)
    check(d, P.make_score_rule(P.PMPE_SCORE_SIGMOID), rand((20, 350), 8), rand((350,), 9, 0.1), words_of(20, 4), soft=True)


def test_outputs_end_with_the_batch_and_any_stream():
    d, rule = P.make_desc(128, 64, 64, 16, 6), P.make_score_rule(P.PMPE_SCORE_SIGMOID, (8, 4), (2, 1))
    z, words = rand((9, 80), 11), words_of(9, 5)
    want = run(d, rule, z, None, words)
    idx, gate = torch.full((11, 6), -7, dtype=torch.int32, device="cuda"), torch.full((11, 6), 9.0, device="cuda")
    allow = torch.full((11,), 77, dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    P.pmpe_select(d, rule, 9, z, None, words, idx[1:10], gate[1:10], None, allow[1:10], None, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(idx[1:10], want["idx"]) and torch.equal(gate[1:10], want["gate"])
    assert torch.all(idx[[0, 10]] == -7) and torch.all(gate[[0, 10]] == 9.0) and torch.all(allow[[0, 10]] == 77)
    # no tokens: nothing is written
    P.pmpe_select(d, rule, 0, z[:0], None, words[:0], idx[:0], gate[:0], None, allow[:0], None)


def gradient64(z, idx, dg, rule, renorm):
    """dz of one pool [T, N] and the sum of the magnitudes it is made of."""
    live = z > -math.inf
    zc = torch.where(live, z.clamp(max=BIG), -1e308)
    sel = torch.zeros_like(z).scatter_(1, idx, 1.0).bool()
    up = torch.zeros_like(z).scatter_(1, idx, dg)
    c = rule.scale
    if rule.score == P.PMPE_SCORE_SIGMOID:
        e = torch.exp(-zc.abs())
        s = torch.where(live, torch.where(zc < 0, e, 1.0) / (1 + e), 0.0)
        slope = torch.where(live, e / (1 + e) ** 2, 0.0)
        if not renorm:
            return c * up * slope, c * up.abs() * slope
        total = (s * sel).sum(1, keepdim=True) + 1e-20
        mean = (s * up).sum(1, keepdim=True) / total
        size = (s * up.abs()).sum(1, keepdim=True) / total
        return c / total * (up - mean) * slope * sel, c / total * (up.abs() + size) * slope * sel
    pool = live & sel if renorm else live
    p = torch.where(pool, zc, -1e308)
    p = torch.where(pool, torch.exp(p - p.amax(1, keepdim=True)), 0.0)
    p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    return c * p * (up - (p * up).sum(1, keepdim=True)), c * p * (up.abs() + (p * up.abs()).sum(1, keepdim=True))


@pytest.mark.parametrize("pools", POOLS, ids=str)
@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gradient(pools, score, renorm, dt):
    log(f"select backward {pools} score={score} renorm={renorm} {dt}")
    pub, priv, k, g, pg, top = pools
    d = P.make_desc(128, 64, pub, priv, k, gate_mode=P.PMPE_GATE_RENORM_TOPK if renorm else P.PMPE_GATE_POOL_SOFTMAX)
    rule = P.make_score_rule(score, g, pg, top, 2.5)
    T = 53
    z, words = rand((T, pub + priv), 21, 3.0, dt), words_of(T, 6)
    z[4] = -math.inf
    z[5, ::2] = float("nan")
    z[6, 1::2] = -math.inf
    got = run(d, rule, z, rand((pub + priv,), 22, 0.1), words)
    dg = rand((T, k), 23)
    dz = torch.full((T, pub + priv), 5.0, device="cuda")
    P.pmpe_select_backward(d, rule, T, z, got["idx"], dg, dz)
    torch.cuda.synchronize()
    for pool, (first, n) in enumerate(((0, pub), (pub, priv))):
        mine = (got["allow"] == pool)
        idx = got["idx"][mine].long() - first
        want, size = gradient64(z[mine][:, first:first + n].double(), idx, dg[mine].double(), rule, renorm)
        part = dz[mine][:, first:first + n].double()
        assert torch.all((part - want).abs() <= 2.0 ** -18 * size + 1e-30)
        rest = torch.ones(pub + priv, dtype=torch.bool, device="cuda")
        rest[first:first + n] = False
        assert torch.all(dz[mine][:, rest] == 0)
    dz2 = torch.empty_like(dz)
    P.pmpe_select_backward(d, rule, T, z, got["idx"], dg, dz2)
    assert torch.equal(dz, dz2)


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm):
    d = P.make_desc(128, 64, 16, 4, 3, gate_mode=P.PMPE_GATE_RENORM_TOPK if renorm else P.PMPE_GATE_POOL_SOFTMAX)
    rule = P.make_score_rule(score, (1, 1), (1, 1), 1, 1.0)
    z = (torch.arange(20).float() * 0.25 - 2.0)[torch.randperm(20, generator=torch.Generator().manual_seed(1))].view(1, 20).cuda()
    dg = rand((1, 3), 31)
    h = 2.0 ** -5  # smaller than half the gap of any two logits: the selection stays
    base = run(d, rule, z, None, None)
    dz = torch.empty_like(z)
    P.pmpe_select_backward(d, rule, 1, z, base["idx"], dg, dz)
    for i in range(20):
        val = []
        for sgn in (1, -1):
            zz = z.clone()
            zz[0, i] += sgn * h
            r = run(d, rule, zz, None, None)
            assert torch.equal(r["idx"], base["idx"])
            val.append(float((r["gate"].double() * dg.double()).sum()))
        # third derivatives of gates are below 1 in magnitude: h^2 / 6 per unit of dg; gates are rounded
        tol = float(dg.abs().sum()) * (h * h / 6 + 2.0 ** -24 / h)
        assert abs((val[0] - val[1]) / (2 * h) - float(dz[0, i])) <= tol


def test_graph_replays():
    d, rule = P.make_desc(128, 64, 128, 32, 8), P.make_score_rule(P.PMPE_SCORE_SIGMOID, (8, 4), (4, 2))
    T = 65
    z, words, dg, dz = rand((T, 160), 41), words_of(T, 7), rand((T, 8), 42), torch.empty(T, 160, device="cuda")
    idx, gate = torch.empty(T, 8, dtype=torch.int32, device="cuda"), torch.empty(T, 8, device="cuda")
    allow = torch.empty(T, dtype=torch.uint8, device="cuda")

    def both():
        P.pmpe_select(d, rule, T, z, None, words, idx, gate, None, allow, None)
        P.pmpe_select_backward(d, rule, T, z, idx, dg, dz)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (51, 52, 53):
        z.copy_(rand((T, 160), seed))
        graph.replay()
        got = [v.clone() for v in (idx, gate, dz)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (idx, gate, dz)))


# ------------------------------------------------------------------ the layer with a score rule


def scored_layer(cfg, rule, bias):
    layer, Lw = C.device_layer(cfg)
    layer.rule, layer.select_bias = rule, bias
    return layer, Lw


@pytest.mark.parametrize("tokens", [5, 2304])  # both router kernels
@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
def test_layer_forward(tokens, score):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=tokens, requests=1 if tokens == 5 else 9, hidden=256, inter=128,
                          n_pub=64, n_priv=16, top_k=4)
    rule, bias = P.make_score_rule(score, (8, 4), (2, 1), 2, 1.5), rand((80,), 61, 0.02)
    layer, Lw = scored_layer(cfg, rule, bias)
    x, T = W.make_x(cfg, "cuda"), tokens
    words = words_of(T, 8)
    offs = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    audit = layer.audit_buffers(T, 1)
    b = layer.forward(x, words, audit, offs)
    torch.cuda.synchronize()
    z = x.double() @ torch.cat([Lw.wr_pub, Lw.wr_priv]).double().t()
    # the selection is that of the layer's own fp32 logits: tokens with a margin above their error
    # (256 fp32 additions of products of size 0.02 |x|) route like the exact logits
    got = run(layer.desc, rule, z.float(), bias, words)
    idx = b.topk_idx.view(T, 4)
    sure = (got["margin"] > 1e-4) & (b.kgap > 1e-4)
    differ = (idx != got["idx"]).any(dim=1)
    assert int((differ & sure).sum()) <= int(0.002 * T)  # a near tie of groups does not show in the margin
    assert int(sure.sum()) > 0.9 * T
    zsel = z.gather(1, idx.long())
    size = (x.double().abs() @ torch.cat([Lw.wr_pub, Lw.wr_priv]).double().abs().t()).gather(1, idx.long())
    assert torch.all((b.topk_logit.view(T, 4).double() - zsel).abs() <= 256 * 2.0 ** -24 * size)
    same = ~differ
    assert torch.all((b.topk_gate.view(T, 4) - got["gate"])[same].abs() <= 1e-4)
    assert torch.equal(b.allow, (words == ALLOW).to(torch.uint8))
    assert int(audit.violations) == 0 and int(audit.total) == 4 * int(b.allow.sum())


@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
def test_layer_training_step(score, renorm):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=300, requests=3, hidden=256, inter=128, n_pub=16, n_priv=8, top_k=4,
                          gate_mode="renorm" if renorm else "pool_softmax")
    rule = P.make_score_rule(score, (4, 2), (2, 1), 2, 2.5)
    layer, Lw = scored_layer(cfg, rule, rand((24,), 71, 0.05))
    T, k, n = 300, 4, 16
    x, words, dout = W.make_x(cfg, "cuda"), words_of(T, 9), rand((T, 256), 72, 1.0, torch.bfloat16)
    offs = torch.tensor([0, 100, 200, 300], dtype=torch.int32, device="cuda")
    b = layer.forward(x, words, layer.audit_buffers(T, 3), offs, train=True)
    g = layer.backward(x, dout, b)
    torch.cuda.synchronize()
    idx, y = b.topk_idx.view(T, k).long(), b.y_perm.double()[b.token_row.long()].view(T, k, 256)
    xd, w = x.double(), torch.cat([Lw.wr_pub, Lw.wr_priv]).double()
    z = xd @ w.t()
    dg = (dout.double().unsqueeze(1) * y).sum(dim=2)
    # the router's own gradient, from the layer's outputs: fp32 sums of 256 products and of T rows
    dz, size = torch.zeros_like(z), torch.zeros_like(z)
    for pool, (first, cnt) in enumerate(((0, n), (n, 8))):
        mine = (b.allow == pool).nonzero().view(-1)
        v, s = gradient64(z[mine][:, first:first + cnt], idx[mine] - first, dg[mine], rule, renorm)
        dz[mine, first:first + cnt], size[mine, first:first + cnt] = v, s
    want = (dz.t() @ xd)[n:]
    room = (size.t() @ xd.abs())[n:]
    assert torch.all((g.dwr_priv.double() - want).abs() <= 2.0 ** -14 * room + 1e-12)
    # the input gradient as a whole, against autograd of the layer in 64 bits
    xa = xd.clone().requires_grad_()
    za = xa @ w.t()
    gate = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    for pool, (first, cnt) in enumerate(((0, n), (n, 8))):
        mine = (b.allow == pool).nonzero().view(-1)
        zp, ip = za[mine][:, first:first + cnt], idx[mine] - first
        sc = torch.sigmoid(zp) if score else torch.softmax(zp, dim=1)
        sel = sc.gather(1, ip)
        gate = gate.index_add(0, mine, rule.scale * (sel / sel.sum(1, keepdim=True) if renorm else sel))
    w13, w2 = torch.cat([Lw.w13_pub, Lw.w13_priv]).double(), torch.cat([Lw.w2_pub, Lw.w2_priv]).double()
    ab = torch.stack([xa @ w13[e].t() for e in range(24)], 1).gather(1, idx.unsqueeze(2).expand(T, k, 256))
    h = torch.nn.functional.silu(ab[:, :, :128]) * ab[:, :, 128:]
    ya = torch.stack([(w2[idx[:, j]] @ h[:, j].unsqueeze(2)).squeeze(2) for j in range(k)], 1)
    ((gate.unsqueeze(2) * ya).sum(1) * dout.double()).sum().backward()
    err = float((g.dx.double() - xa.grad).norm() / xa.grad.norm())
    log(f"dx rel {err:.2e}")
    assert err <= C.RTOL_BF16
    assert np.all(np.abs(b.topk_gate.view(T, k).double().cpu().numpy() - gate.detach().cpu().numpy()) <= 1e-5 * rule.scale)


def test_layer_keeps_other_layers_results():
    """A layer without a rule routes as before, also next to one with a rule on the same weights."""
    cfg = W.scaled_config(W.get_config("qwen"), tokens=64, requests=4, hidden=256, inter=128, n_pub=16, n_priv=8, top_k=4)
    layer, Lw = C.device_layer(cfg)
    x, words = W.make_x(cfg, "cuda"), words_of(64, 10)
    a = layer.forward(x, words, layer.audit_buffers(64, 1))
    want = [t.clone() for t in (a.topk_idx, a.topk_gate, a.out)]
    layer.rule = P.make_score_rule(P.PMPE_SCORE_SOFTMAX)
    s = layer.forward(x, words, layer.audit_buffers(64, 1))
    assert torch.equal(s.topk_idx, want[0])  # softmax is monotone, and no bias
    assert torch.all((s.topk_gate - want[1]).abs() <= 2e-6)
    layer.rule = None
    a = layer.forward(x, words, layer.audit_buffers(64, 1))
    assert all(torch.equal(u, v) for u, v in zip(want, (a.topk_idx, a.topk_gate, a.out)))
