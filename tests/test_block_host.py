"""Host-side bookkeeping of the operators around the layer (no GPU): buffers that outlive the calls that
use them."""
import gc
import types
import weakref

import pytest
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


def scored_route_args(T=6):
    """pmpe_route_scored's tensors by name, in order, as a layer with a score rule gives them."""
    d = P.make_desc(H, I, PUB, PRIV, K)
    E = PUB + PRIV
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return d, P.make_score_rule(), T, dict(
        x=f(T, H).bfloat16(), wr_pub=f(PUB, H), wr_priv=f(PRIV, H), logit_bias=f(E), select_bias=f(E), policy_word=i(T),
        topk_idx=i(T * K), topk_gate=f(T * K), topk_logit=f(T * K), allow=torch.zeros(T, dtype=torch.uint8), margin=f(T),
        dev_status=i(1), ws=torch.zeros(P.pmpe_workspace_bytes(d, T), dtype=torch.uint8))


def scored_backward_args(T=6):
    d = P.make_desc(H, I, PUB, PRIV, K, 1, 128)
    E, R = PUB + PRIV, T * K
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    b = lambda *s: torch.zeros(*s).bfloat16()  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return d, P.make_score_rule(), T, dict(
        topk_logit=f(R), x=b(T, H), dout=b(T, H), topk_idx=i(R), topk_gate=f(R), expert_count=i(E), expert_offset=i(E + 1),
        row_token=i(R), token_row=i(R), y_perm=b(R, H), wr_pub=f(PUB, H), wr_priv=f(PRIV, H), w13_pub=b(PUB, 2 * I, H),
        w2_pub=b(PUB, H, I), w13_priv=b(PRIV, 2 * I, H), w2_priv=b(PRIV, H, I), logit_bias=f(E), w13_sh=b(2 * 128, H),
        w2_sh=b(H, 128), w2t_pub=b(PUB, I, H), w13t_pub=b(PUB, H, 2 * I), w2t_priv=b(PRIV, I, H), w13t_priv=b(PRIV, H, 2 * I),
        ab=f(R, 2 * I), dx=f(T, H), dw13_priv=f(PRIV, 2 * I, H), dw2_priv=f(PRIV, H, I), dwr_priv=f(PRIV, H),
        grad_rows=i(PRIV), ws=torch.zeros(P.pmpe_backward_workspace_bytes(d, T), dtype=torch.uint8))


@pytest.mark.parametrize("call,make", [("pmpe_route_scored", scored_route_args), ("pmpe_backward_scored", scored_backward_args)])
def test_calls_of_a_scored_layer_check_their_tensors(monkeypatch, call, make):
    """Every tensor has to have its elements, type, device and order: a short one would be read or written
    past its end."""
    d, rule, T, good = make()
    calls, here = [], []
    monkeypatch.setattr(N, "_lib", types.SimpleNamespace(**{call: lambda *a: calls.append(a) or 0}))
    monkeypatch.setattr(N, "_here", lambda t, name: here.append(name) or -1)  # the device of these tensors
    monkeypatch.setattr(N, "_stream", lambda stream: 0)
    f = lambda v: getattr(P, call)(d, rule, T, *v.values())  # noqa: E731
    f(good)
    assert len(calls) == 1 and here == ["x"]
    for name, t in good.items():
        if name in ("x", "ws"):  # (the library checks a workspace's size)
            continue
        other = torch.float64 if t.dtype != torch.float64 else torch.float32
        longer = torch.cat([t.flatten(), t.flatten()[:1]])
        for bad in (t.flatten()[:-1], longer, t.to(other), torch.stack([t, t], dim=-1)[..., 0]):
            if bad.dtype == t.dtype and bad.numel() == t.numel() and bad.is_contiguous():
                continue  # one element is contiguous at any stride
            with pytest.raises(ValueError, match=name):
                f({**good, name: bad})
    for bad in (good["x"][:-1], good["x"].double(), good["x"].t().contiguous().t()):
        with pytest.raises(ValueError, match="x must"):
            f({**good, "x": bad})
    with pytest.raises(ValueError, match="workspace"):
        f({**good, "ws": torch.zeros(64, 64, dtype=torch.uint8)[:, 0]})
    monkeypatch.setattr(N, "_here", lambda t, name: 0)  # x on a device, the others on the host
    with pytest.raises(ValueError, match="device"):
        f({**good, "x": types.SimpleNamespace(dtype=good["x"].dtype, get_device=lambda: 0, numel=good["x"].numel,
                                              is_contiguous=lambda: True, data_ptr=lambda: 0)})
    monkeypatch.setattr(N, "_here", lambda t, name: -1)
    assert len(calls) == 1
    # what may be absent
    may = {"pmpe_route_scored": ("wr_priv", "logit_bias", "select_bias", "policy_word", "topk_logit", "margin", "dev_status"),
           "pmpe_backward_scored": ("logit_bias", "w2t_pub", "w13t_pub", "w2t_priv", "w13t_priv", "ab", "grad_rows")}[call]
    f({**good, **dict.fromkeys(may)})
    assert len(calls) == 2


def test_a_layer_checks_its_balance_bias():
    rule = P.make_score_rule()
    make_layer(rule, torch.zeros(PUB + PRIV))
    for bad in (torch.zeros(PUB), torch.zeros(PUB + PRIV).bfloat16(), torch.zeros(2 * (PUB + PRIV))[::2],
                torch.zeros(PUB + PRIV, device="meta")):
        with pytest.raises(ValueError, match="select_bias"):
            make_layer(rule, bad)


def test_a_plain_forward_after_one_in_8_bits_writes_no_bytes(monkeypatch):
    outs = []
    monkeypatch.setattr(N, "pmpe_rmsnorm", lambda x, res, w, eps, total, out, q, s, rstd, stream: outs.append((q, s)))
    blk = P.NormedMoE(make_layer(), torch.ones(H))
    monkeypatch.setattr(blk.layer, "forward", lambda *a: None)
    monkeypatch.setattr(blk.layer, "forward_mx", lambda *a: None)
    h = torch.zeros(4, H).bfloat16()
    blk.forward(h, None, None, None)
    b = blk.forward_mx(h, None, None, None, None)
    kept = b.norm_q, b.norm_scale
    blk.forward(h, None, None, None)
    blk.forward_mx(h, None, None, None, None)
    assert outs[0] == outs[2] == (None, None)
    assert all(t is k for i in (1, 3) for t, k in zip(outs[i], kept))


def test_the_norm_of_a_clipped_step_is_aligned():
    f, hp = N.lib().pmpe_adamw_clipped, (1e-3, 0.9, 0.99, 1e-8, 0.0)
    a, b, c, d, e = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000
    for norm in (e + 1, e + 2, e + 3):
        assert f(a, N.PMPE_F32, None, b, c, d, 4, 1, *hp, norm, None) == -5  # PMPE_ERR_ALIGN
    assert f(a, N.PMPE_F32, None, b, c, d, 0, 1, *hp, e, None) == 0
