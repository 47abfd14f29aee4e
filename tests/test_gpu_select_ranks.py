"""Ranks of groups in routing by scores: a rank that is a sum of two is (s + s) + (bias + bias), with
s(z) = 1 - s(-z), in 64 bits. Sums that are equal in the mathematics (one bias on either of two
experts, the sigmoids of z and -z) are then equal in their bits, and the lower group stays; any other
difference that 64 bits hold decides."""
import math

import pytest
import torch

import paper_2608_06690_amd as P
from tests.test_gpu_select import run, words_of

pytestmark = pytest.mark.gpu


def log(msg):
    print(msg, flush=True)


def sigmoid(z):
    q = math.exp(-abs(z)) / (1.0 + math.exp(-abs(z)))
    return q if z < 0 else 1.0 - q


def softmax(z):
    top = max(z)
    e = [math.exp(v - top) for v in z]
    inv = 1.0 / math.fsum(e)
    return [v * inv for v in e]


def choose(z, bias, k, score, groups, keep):
    s = [sigmoid(v) for v in z] if score == P.PMPE_SCORE_SIGMOID else softmax(z)
    u = [a + b for a, b in zip(s, bias)]
    gs = len(z) // groups

    def rank(g):
        best = sorted(range(g * gs, g * gs + gs), key=lambda e: (-u[e], e))[:2]
        return sum(s[e] for e in best) + sum(bias[e] for e in best) if len(best) == 2 else u[best[0]]
    kept = sorted(range(groups), key=lambda g: (-rank(g), g))[:keep]
    cand = [e for g in kept for e in range(g * gs, g * gs + gs)]
    return sorted(sorted(cand, key=lambda e: (-u[e], e))[:k])


def check(d, rule, z, bias, words=None):
    got = run(d, rule, z, bias, words)
    allow = (words.cpu() != 0).logical_and(words.cpu() == P.PMPE_POLICY_ALLOW - (1 << 32)) if words is not None else None
    zs, b = z.double().cpu().tolist(), [0.0] * z.shape[1] if bias is None else bias.double().cpu().tolist()
    for t in range(z.shape[0]):
        first, n, g, keep = 0, d.n_pub, rule.n_group_pub, rule.topk_group_pub
        if allow is not None and allow[t]:
            first, n, g, keep = d.n_pub, d.n_priv, rule.n_group_priv, rule.topk_group_priv
        want = [first + i for i in choose(zs[t][first:first + n], b[first:first + n], d.top_k, rule.score, g, keep)]
        assert got["idx"][t].tolist() == want, t
    return got


@pytest.mark.parametrize("bias", [None, 0.0, 0.25])
@pytest.mark.parametrize("lower,higher", [(20.0, 20.001), (33.0, 35.0), (34.0, 34.5), (-33.0, -32.999)])
def test_saturated_scores_are_told_apart(bias, lower, higher):
    """Sums that differ by a few steps of 64 bits: the higher one stays, whatever its place."""
    log(f"ranks {lower} {higher} bias={bias}")
    d = P.make_desc(128, 64, 32, 8, 2)
    rule = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (16, 1), (4, 1), 2)
    z = torch.full((19, 40), lower)
    for t in range(16):
        z[t, 2 * t:2 * t + 2] = higher
    z[16, 34:36] = z[17, 38:40] = z[18, 32:34] = higher
    words = torch.zeros(19, dtype=torch.int32)
    words[16:] = P.PMPE_POLICY_ALLOW - (1 << 32)
    b = None if bias is None else torch.full((40,), bias, device="cuda")
    if bias == 0.25 and lower < 0:
        b = b * 2.0 ** -40  # (scores of 5e-15: a bias of their size keeps their difference in 64 bits)
    got = check(d, rule, z.cuda(), b, words.cuda())
    want = [[2 * t, 2 * t + 1] for t in range(16)] + [[34, 35], [38, 39], [32, 33]]
    assert got["idx"].tolist() == want


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("pools", [(64, 16, 6, (8, 3), (4, 3)), (128, 64, 8, (32, 7), (64, 9)), (256, 32, 4, (4, 2), (2, 1)),
                                   (60, 20, 4, (5, 2), (4, 3))], ids=str)
def test_equal_sums_tie_wherever_the_bias_lies(score, pools):
    """Few values of logits and biases: many groups whose best two add up to the same."""
    pub, priv, k, g, pg = pools
    d, rule = P.make_desc(128, 64, pub, priv, k), P.make_score_rule(score, g, pg, 2)
    gen = torch.Generator().manual_seed(pub + score)
    z = torch.randint(-2, 3, (400, pub + priv), generator=gen).float().cuda()
    bias = (torch.randint(0, 3, (pub + priv,), generator=gen).float() * 0.3).cuda()
    words = words_of(400, 1)
    check(d, rule, z, bias, words)
    check(d, rule, z, None, words)
    check(d, rule, z.bfloat16(), torch.zeros_like(bias), words)


@pytest.mark.parametrize("value", [0.05, -0.7, 3.0])
def test_pairs_of_opposite_logits_tie_under_an_equal_bias(value):
    d = P.make_desc(128, 64, 64, 16, 2)
    rule = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (32, 1), (8, 1), 2)
    g = torch.Generator(device="cuda").manual_seed(7)
    half = torch.empty(500, 40, device="cuda").normal_(0, 2.0, generator=g)
    z = torch.stack([half, -half], dim=2).reshape(500, 80).contiguous()
    words = torch.zeros(500, dtype=torch.int32)
    words[250:] = P.PMPE_POLICY_ALLOW - (1 << 32)
    got = check(d, rule, z, torch.full((80,), value, device="cuda"), words.cuda())
    assert (got["idx"][:250].cpu() == torch.tensor([0, 1])).all() and (got["idx"][250:].cpu() == torch.tensor([64, 65])).all()


def test_biases_that_mask_or_are_huge():
    d = P.make_desc(128, 64, 16, 8, 2)
    rule = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (4, 1), (2, 1), 2)
    z = torch.ones(1, 24, device="cuda")
    inf = math.inf
    for bias, want in (([-inf, -inf, -inf, 0.5] + [0.0] * 12, [4, 5]),           # one live expert against two
                       ([-inf] * 4 + [-inf, -inf, 0.0, -inf] + [-inf] * 8, [6, 0]),  # masked groups rank behind
                       ([0.0] * 8 + [1e30, -1e30, 0.0, 0.0] + [0.0] * 4, [8, 10]),
                       ([0.0] * 12 + [inf, inf, 0.0, 0.0], [12, 13]),
                       ([inf, 0.0, 0.0, 0.0] * 4, [0, 1]),                       # infinite ranks tie
                       ([float("nan")] * 16, [0, 1])):
        b = torch.tensor(bias + [0.0] * 8, device="cuda")
        got = run(d, rule, z, b, None)
        if want == [6, 0]:  # the group that stays has one live expert; the other place goes to its lowest masked one
            want = [4, 6]
        assert got["idx"][0].tolist() == want, bias


@pytest.mark.parametrize("T", [5, 300, 2304])  # logits in partial sums, and whole
@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
def test_a_layer_whose_experts_have_one_router_row(T, score):
    """Logits that are equal, or nearly so (their sums have an order of their own in each lane of the router):
    the selection is that of the layer's own fp32 logits, read one expert at a time through a bias that
    nothing else reaches."""
    pub, priv, k, H = 64, 16, 4, 256
    d = P.make_desc(H, 128, pub, priv, k)
    rule = P.make_score_rule(score, (8, 3), (4, 2), 2)
    gen = torch.Generator().manual_seed(T)
    bias = torch.randint(0, 4, (pub + priv,), generator=gen).float() * 0.3
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.empty(T, H, device="cuda").normal_(0, 1, generator=g).bfloat16()
    row = torch.empty(1, H, device="cuda").normal_(0, 0.06, generator=g)
    ws = torch.empty(P.pmpe_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
    words, allow = words_of(T, 2), torch.empty(T, dtype=torch.uint8, device="cuda")

    def route(d, rule, bias, words):
        idx = torch.full((T, d.top_k), -7, dtype=torch.int32, device="cuda")
        gate, logit = torch.empty(T, d.top_k, device="cuda"), torch.empty(T, d.top_k, device="cuda")
        P.pmpe_route_scored(d, rule, T, x, row.repeat(pub, 1), row.repeat(priv, 1), None, bias.cuda(), words, idx, gate, logit,
                            allow, None, None, ws)
        torch.cuda.synchronize()
        return idx, gate, logit

    z = torch.empty(T, pub + priv)
    one, any_rule = P.make_desc(H, 128, pub, priv, 1), P.make_score_rule(score)
    for e in range(pub + priv):
        b = torch.zeros(pub + priv)
        b[e] = 100.0
        idx, _, logit = route(one, any_rule, b, torch.full_like(words, P.PMPE_POLICY_ALLOW - (1 << 32)) if e >= pub else None)
        assert torch.all(idx == e)
        z[:, e] = logit.view(-1).cpu()
    idx, gate, logit = route(d, rule, bias, words)
    zs, b, al = z.double().tolist(), bias.double().tolist(), allow.tolist()
    for t in range(T):
        first, n, groups, keep = (pub, priv, 4, 2) if al[t] else (0, pub, 8, 3)
        pool = zs[t][first:first + n]
        want = choose(pool, b[first:first + n], k, score, groups, keep)
        assert idx[t].tolist() == [first + i for i in want], t
        assert logit[t].tolist() == [pool[i] for i in want]
        s = [sigmoid(pool[i]) for i in want] if score == P.PMPE_SCORE_SIGMOID else softmax([pool[i] for i in want])
        for got, e in zip(gate[t].tolist(), s):
            assert abs(got - e / sum(s)) <= (2.0 ** -24 + 2.0 ** -40) * e / sum(s)
