"""Host-side bookkeeping of the operators around the layer (no GPU): buffers that outlive the calls that
use them."""
import gc
import types
import weakref

import torch

import paper_2608_06690_amd as P
from paper_2608_06690_amd import _native as N
from paper_2608_06690_amd import layer as Lmod

H, I, PUB, PRIV, K = 256, 128, 8, 4, 2


def make_layer(rule=None, select_bias=None):
    desc = P.make_desc(H, I, PUB, PRIV, K)
    w = lambda *s: torch.randn(*s, dtype=torch.float32)  # noqa: E731
    b = lambda *s: torch.randn(*s).bfloat16()  # noqa: E731
    return P.PolicyMaskedMoE(desc, w(PUB, H), w(PRIV, H), None, b(PUB, 2 * I, H), b(PUB, H, I), b(PRIV, 2 * I, H),
                             b(PRIV, H, I), rule=rule, select_bias=select_bias)


def test_the_workspace_of_a_backward_outlives_it(monkeypatch):
    """The kernels of a backward on another stream run on after the call has returned: its workspace may not
    go back to the allocator then, nor be another one while a captured pass holds the first."""
    seen = []
    monkeypatch.setattr(N, "pmpe_rmsnorm_backward", lambda dy, dres, r, w, rstd, dx, dw, ws, stream: seen.append(
        (None, 0, dw) if ws is None else (weakref.ref(ws), ws.data_ptr(), dw)))
    blk = P.NormedMoE(make_layer(), torch.ones(H))
    monkeypatch.setattr(blk.layer, "backward", lambda x, dout, b, g, stream: types.SimpleNamespace(dx=torch.zeros(x.shape)))
    b = blk.buffers(8)
    b.residual = torch.zeros(8, H).bfloat16()
    dx, dw = torch.zeros(8, H).bfloat16(), torch.zeros(H)
    blk.backward(None, dx, b, dx, dweight=dw)
    blk.backward(None, dx, b, dx)
    blk.backward(None, dx, b, dx, dweight=dw)
    gc.collect()
    (first, at, _), (none, _, no_dw), (again, at2, _) = seen
    assert none is None and no_dw is None  # a frozen norm needs none
    assert first() is not None and again() is first() and at2 == at
    assert first().numel() >= P.pmpe_rmsnorm_backward_workspace_bytes(8, H)


def grads_of(lay, value):
    like = lambda p: torch.full(p.shape, value, dtype=torch.float32)  # noqa: E731
    return Lmod.GradBuffers(None, like(lay.w13_priv), like(lay.w2_priv), like(lay.wr_priv), None, None)


def total_of(*grads):
    return sum(float(t.double().square().sum()) for g in grads for t in (g.dwr_priv, g.dw13_priv, g.dw2_priv)) ** 0.5


def test_every_optimizer_shows_the_norm_of_its_own_last_step(monkeypatch):
    """Joint steps of several optimizers, in changing company, and single ones: `norm` is that of the
    optimizer's last step, and the factor that a step reads is written by that step only."""
    used = []

    def grad_norm(grads, max_norm, norm, ws, stream):
        n = sum(float(t.double().square().sum()) for t in grads.tensors) ** 0.5
        norm.copy_(torch.tensor([n, min(1.0, max_norm / (n + 1e-6))]))

    monkeypatch.setattr(N, "pmpe_grad_norm", grad_norm)
    monkeypatch.setattr(N, "pmpe_adamw_clipped", lambda *a: used.append(a[-2]))
    lays = [make_layer() for _ in range(3)]
    a, b, c = [P.PrivateAdamW(lay, max_norm=0.5) for lay in lays]
    ga, gb, gc_ = [grads_of(lay, v) for lay, v in zip(lays, (1.0, 2.0, 4.0))]
    expected = {}

    def check():
        for opt, n in expected.items():
            assert abs(float(opt.norm[0]) - n) <= 2.0 ** -22 * n

    def joint(*pairs):
        norm = P.step_clipped(pairs, 0.5)
        n = total_of(*[g for _, g in pairs])
        assert abs(float(norm[0]) - n) <= 2.0 ** -22 * n and all(u is norm for u in used[-3 * len(pairs):])
        expected.update({opt: n for opt, _ in pairs})
        check()
        return norm

    def single(opt, g):
        opt.step(g)
        assert all(u is opt.norm for u in used[-3:])
        expected[opt] = total_of(g)
        check()

    first = joint((a, ga), (b, gb))
    single(b, gb)   # leaves the joint step's norm to a
    single(a, ga)
    assert joint((a, ga), (b, gb)) is first  # the same tensors each time: a captured step may hold them
    joint((a, ga), (c, gc_))                 # a steps with others: b's last step stays b's
    joint((b, gb), (a, ga))
    single(c, gc_)
    single(a, ga)
