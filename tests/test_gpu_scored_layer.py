"""A layer that routes by scores, with what a router's logit bias can mask and the layer's other options:
forward and backward against 64-bit arithmetic on the selection that the layer made.

Masking rule: a logit of -inf or NaN has score and gate 0 and no gradient, +inf counts as the largest
finite value. Tolerances: logits are fp32 sums of H products (2^-24 H of their sum of magnitudes, 1e-5 here
as in the other layer tests); bf16 y, dh and [da; db] as in the other backward tests."""
import math

import pytest
import torch

import paper_2608_06690_amd as P
from tests import pmpe_cases as C
from tests.test_gpu_select import gradient64, scores

pytestmark = pytest.mark.gpu
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)
PUB, PRIV, K, H, I = 16, 8, 4, 256, 128
E = PUB + PRIV
INF, NAN = math.inf, math.nan


def log(msg):
    print(msg, flush=True)


class Case:
    def __init__(self, T, score, renorm, bias, shared=0, soft=False, drop_router=False, groups=True):
        g = torch.Generator(device="cuda").manual_seed(T + 8 * score + renorm)

        def rand(*shape, std=1.0, dtype=torch.bfloat16):
            return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0, std, generator=g)

        self.T, self.soft, self.renorm = T, soft, renorm
        self.rule = P.make_score_rule(score, (4, 2), (2, 1), 2, 2.5) if groups and not soft else P.make_score_rule(score, scale=2.5)
        d = P.make_desc(H, I, PUB, PRIV, K, shared, 128 if shared else 0,
                        gate_mode=P.PMPE_GATE_RENORM_TOPK if renorm else P.PMPE_GATE_POOL_SOFTMAX,
                        route_mode=P.PMPE_ROUTE_SOFT if soft else P.PMPE_ROUTE_MASKED)
        self.wr, self.bias = rand(E, H, std=H ** -0.5, dtype=torch.float32), rand(E, dtype=torch.float32)
        for e, v in bias.items():
            self.bias[e] = v
        self.w13, self.w2 = rand(E, 2 * I, H, std=H ** -0.5), rand(E, H, I, std=I ** -0.5)
        s = shared * 128
        self.w13s, self.w2s = (rand(2 * s, H, std=H ** -0.5), rand(H, s, std=s ** -0.5)) if shared else (None, None)
        self.layer = P.PolicyMaskedMoE(d, self.wr[:PUB], None if drop_router else self.wr[PUB:], self.bias, self.w13[:PUB],
                                       self.w2[:PUB], self.w13[PUB:], self.w2[PUB:], self.w13s, self.w2s, rule=self.rule,
                                       select_bias=rand(E, std=0.05, dtype=torch.float32))
        self.x, self.dout = rand(T, H), rand(T, H)
        allow = torch.rand(T, generator=g, device="cuda") < 0.5
        self.words = torch.where(allow, ALLOW, 0).to(torch.int32)
        self.allow = allow & (not drop_router)
        self.offs = torch.tensor([0, T], dtype=torch.int32, device="cuda")

    def pools(self):
        if self.soft:
            return [(torch.arange(self.T, device="cuda"), 0, E)]
        return [((~self.allow).nonzero().view(-1), 0, PUB), (self.allow.nonzero().view(-1), PUB, PRIV)]

    def gates(self, idx):
        """Gates of the selection idx in 64 bits."""
        z = (self.x.double() @ self.wr.double().t() + self.bias.double()).cpu().tolist()
        out, sel = torch.zeros(self.T, K, dtype=torch.float64), idx.cpu().tolist()
        for rows, first, n in self.pools():
            for t in rows.tolist():
                mine = [z[t][e] for e in sel[t]]
                if self.renorm and self.rule.score == P.PMPE_SCORE_SOFTMAX:
                    s = scores(mine, self.rule.score)[0]
                else:
                    pool = scores(z[t][first:first + n], self.rule.score)[0]
                    s = [pool[e - first] for e in sel[t]]
                    if self.renorm:
                        total = sum(s) + 1e-20
                        s = [v / total for v in s]
                out[t] = torch.tensor(s) * self.rule.scale
        return out.cuda()

    def experts(self, xd, idx):
        """Outputs [T, K, H] of the selected experts."""
        w13, w2 = self.w13.double(), self.w2.double()
        y = []
        for j in range(K):
            o = torch.zeros(self.T, H, dtype=torch.float64, device="cuda")
            for e in range(E):
                rows = (idx[:, j] == e).nonzero().view(-1)
                ab = xd[rows] @ w13[e].t()
                o = o.index_add(0, rows, (torch.nn.functional.silu(ab[:, :I]) * ab[:, I:]) @ w2[e].t())
            y.append(o)
        return torch.stack(y, 1)

    def shared(self, xd):
        if self.w13s is None:
            return 0.0
        ab, s = xd @ self.w13s.double().t(), self.w2s.shape[1]
        return (torch.nn.functional.silu(ab[:, :s]) * ab[:, s:]) @ self.w2s.double().t()

    def check(self):
        lay, T = self.layer, self.T
        audit = lay.audit_buffers(T, 1)
        b = lay.forward(self.x, self.words, audit, self.offs, train=True)
        g = lay.backward(self.x, self.dout, b)
        torch.cuda.synchronize()
        idx = b.topk_idx.view(T, K).long()
        for rows, first, n in self.pools():
            assert torch.all((idx[rows] >= first) & (idx[rows] < first + n))
        want = self.gates(idx)
        assert torch.all((b.topk_gate.view(T, K).double() - want).abs() <= 1e-5 * self.rule.scale)
        xa = self.x.double().requires_grad_()
        y = self.experts(xa, idx)
        out = (want.unsqueeze(2) * y).sum(1) + self.shared(xa)
        (out * self.dout.double()).sum().backward()
        assert C.rel_l2(b.out.double().cpu().numpy(), out.detach().cpu().numpy()) <= C.RTOL_BF16
        # the router's part: from the layer's own expert outputs
        xd = self.x.double()
        z = xd @ self.wr.double().t() + self.bias.double()
        dg = (self.dout.double().unsqueeze(1) * b.y_perm.double()[b.token_row.long()].view(T, K, H)).sum(2)
        dz, size = torch.zeros_like(z), torch.zeros_like(z)
        for rows, first, n in self.pools():
            dz[rows, first:first + n], size[rows, first:first + n] = gradient64(
                z[rows][:, first:first + n], idx[rows] - first, dg[rows], self.rule, self.renorm)
        finite = [bool(torch.isfinite(t).all()) for t in (g.dx, g.dw13_priv, g.dw2_priv, g.dwr_priv)]
        assert all(finite), finite
        dwr, room = (dz.t() @ xd)[PUB:], (size.t() @ xd.abs())[PUB:]
        assert torch.all((g.dwr_priv.double() - dwr).abs() <= 2.0 ** -14 * room + 1e-12)
        dx = xa.grad + dz @ self.wr.double()
        err = C.rel_l2(g.dx.double().cpu().numpy(), dx.cpu().numpy())
        log(f"dx rel {err:.2e}")
        assert err <= C.RTOL_BF16
        assert int(audit.total) == int((idx >= PUB).sum())
        assert int(audit.violations) == int(((idx >= PUB).any(1) & (self.words != ALLOW)).sum())
        return b


BIASES = {
    "finite": {},
    "single experts": {0: -INF, 5: -INF, PUB + 1: -INF},
    "one not a number": {3: NAN, PUB + 2: NAN},
    "plus infinity": {2: INF, PUB + 3: INF},
    "fewer than top-k": {**{e: -INF for e in range(2, PUB)}, **{PUB + e: NAN for e in range(1, PRIV)}},
    "the private pool": {PUB + e: -INF for e in range(PRIV)},
    "both pools": {e: NAN if e % 2 else -INF for e in range(E)},
}


# (logits of the softmax backward recomputed inside its kernel, and by the router's)
@pytest.mark.parametrize("T", [9, 4200])
@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("bias", list(BIASES))
def test_logit_bias_that_masks(T, score, renorm, bias):
    log(f"scored layer T={T} score={score} renorm={renorm} {bias}")
    c = Case(T, score, renorm, BIASES[bias])
    b = c.check()
    if bias == "the private pool":
        assert torch.all(b.topk_gate.view(T, K)[c.allow] == 0) and torch.all(b.out[c.allow] == 0)


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T", [40, 4200])
def test_shared_experts(T, score, renorm):
    log(f"scored layer with shared experts T={T} score={score} renorm={renorm}")
    Case(T, score, renorm, {}, shared=2).check()


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T", [40, 4200])
def test_soft_control(T, score, renorm):
    """One pool of all experts, without a mask: deny tokens reach private experts, and the audit says so."""
    log(f"scored soft control T={T} score={score} renorm={renorm}")
    Case(T, score, renorm, {1: -INF, PUB: NAN}, soft=True).check()


@pytest.mark.parametrize("score", [P.PMPE_SCORE_SOFTMAX, P.PMPE_SCORE_SIGMOID])
@pytest.mark.parametrize("T", [40, 4200])
def test_absent_private_router(T, score):
    """Every token routes in the public pool then, and the status word says why."""
    c = Case(T, score, True, {}, drop_router=True)
    audit = c.layer.audit_buffers(T, 1)
    b = c.layer.forward(c.x, c.words, audit, c.offs)
    torch.cuda.synchronize()
    idx = b.topk_idx.view(T, K).long()
    assert torch.all(idx < PUB) and not b.allow.any() and int(b.dev_status) == 1  # PMPE_DEV_PRIV_ROUTER_MISSING
    assert torch.all((b.topk_gate.view(T, K).double() - c.gates(idx)).abs() <= 1e-5 * c.rule.scale)
    assert int(audit.total) == 0 and int(audit.violations) == 0
