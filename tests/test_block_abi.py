"""Refusals of the operators around the layer, on the host: each status comes before any launch,
so the pointers here are never read."""
import ctypes

import pytest
import torch

import paper_2608_06690_amd as P
from paper_2608_06690_amd import _native as N

A, B, C, D, E = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000
F32, BF16 = N.PMPE_F32, N.PMPE_BF16
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = -1, -2, -4, -5, -6


def rmsnorm(T=4, H=64, dt=BF16, x=A, res=None, w=B, wdt=F32, eps=1e-6, total=None, out=C, q=None, s=None, rstd=None):
    return N.lib().pmpe_rmsnorm(T, H, dt, x, res, w, wdt, eps, total, out, q, s, rstd, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(out=None), NULL), (dict(q=D), NULL), (dict(s=D), NULL),
    (dict(res=D), NULL), (dict(total=D), NULL),
    (dict(T=-1), SHAPE), (dict(H=0), SHAPE), (dict(H=16385), SHAPE), (dict(H=65, q=D, s=E), SHAPE),
    (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(dt=2), DTYPE), (dict(wdt=7), DTYPE),
    (dict(x=A + 4), ALIGN), (dict(w=B + 8), ALIGN), (dict(out=C + 2), ALIGN), (dict(q=D + 1, s=E), ALIGN),
    (dict(res=D, total=E + 8), ALIGN), (dict(T=0), 0)])
def test_rmsnorm(kw, status):
    assert rmsnorm(**kw) == status


def rmsnorm_bwd(T=4, H=64, dt=BF16, dy=A, dyt=F32, dres=None, r=B, w=C, wdt=F32, rstd=D, dx=E, dw=None, ws=None, n=0):
    return N.lib().pmpe_rmsnorm_backward(T, H, dt, dy, dyt, dres, r, w, wdt, rstd, dx, dw, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), NULL), (dict(r=None), NULL), (dict(w=None), NULL), (dict(rstd=None), NULL), (dict(dx=None), NULL),
    (dict(T=-1), SHAPE), (dict(H=0), SHAPE), (dict(H=20000), SHAPE), (dict(dt=3), DTYPE), (dict(wdt=2), DTYPE),
    (dict(dt=F32, dyt=BF16), DTYPE), (dict(dy=A + 8), ALIGN), (dict(dres=A + 8), ALIGN), (dict(dx=E + 4), ALIGN),
    (dict(dw=A), WORKSPACE), (dict(dw=A, ws=B, n=64 * 4 - 1), WORKSPACE), (dict(dw=A, ws=B + 8, n=1 << 20), ALIGN),
    (dict(T=0), 0)])
def test_rmsnorm_backward(kw, status):
    assert rmsnorm_bwd(**kw) == status


def test_rmsnorm_workspace():
    assert P.pmpe_rmsnorm_backward_workspace_bytes(0, 64) == 0
    assert P.pmpe_rmsnorm_backward_workspace_bytes(-1, 64) == 0 and P.pmpe_rmsnorm_backward_workspace_bytes(4, 0) == 0
    assert P.pmpe_rmsnorm_backward_workspace_bytes(1, 64) == 64 * 4


def test_binding_refuses_tensors_of_the_host():
    x, w = torch.zeros(2, 64), torch.ones(64)
    with pytest.raises(ValueError):
        P.pmpe_rmsnorm(x, None, w, 1e-6, None, x, None, None, None)
    with pytest.raises(ValueError):
        P.pmpe_rmsnorm_backward(x, None, x, w, torch.ones(2), x, None, None)


def rule(**kw):
    r = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (8, 4), (4, 2), 2, 1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def select(d=None, r=None, T=4, z=A, dt=F32, bias=None, words=None, idx=B, gate=C, logit=None, allow=D, margin=None):
    d, r = d or P.make_desc(2048, 768, 128, 32, 8), r or rule()
    return N.lib().pmpe_select(ctypes.byref(d), ctypes.byref(r), T, z, dt, bias, words, idx, gate, logit, allow, margin, None)


@pytest.mark.parametrize("kw", [
    dict(score=2), dict(score=-1), dict(group_top=0), dict(group_top=3), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(n_group_pub=0), dict(n_group_pub=3), dict(n_group_pub=128, topk_group_pub=64), dict(topk_group_pub=0), dict(topk_group_pub=9),
    dict(n_group_pub=64, topk_group_pub=3), dict(n_group_priv=5), dict(n_group_priv=16, topk_group_priv=3),
    dict(topk_group_priv=5)])
def test_rules_that_do_not_fit(kw):
    r = rule(**kw)
    assert select(r=r) == SHAPE
    d = P.make_desc(2048, 768, 128, 32, 8)
    assert N.lib().pmpe_select_backward(ctypes.byref(d), ctypes.byref(r), 4, A, F32, B, C, D, None) == SHAPE
    assert N.lib().pmpe_route_scored(ctypes.byref(d), ctypes.byref(r), 4, A, A, None, None, None, None, B, C, None, D, None,
                                     None, E, 1 << 30, None) == SHAPE


def test_rules_under_the_soft_control():
    d = P.make_desc(2048, 768, 128, 32, 8, route_mode=P.PMPE_ROUTE_SOFT)
    assert select(d=d) == SHAPE  # groups
    assert select(d=d, r=rule(n_group_pub=1, topk_group_pub=1, n_group_priv=1, topk_group_priv=1), z=None) == NULL


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), NULL), (dict(idx=None), NULL), (dict(gate=None), NULL), (dict(allow=None), NULL), (dict(dt=2), DTYPE),
    (dict(T=-1), SHAPE), (dict(T=0, z=None, idx=None, gate=None, allow=None), 0),
    (dict(d=P.make_desc(2048, 768, 128, 4, 8)), -3)])
def test_select(kw, status):
    assert select(**kw) == status


def test_select_without_a_rule_or_descriptor():
    d, r = P.make_desc(2048, 768, 128, 32, 8), rule()
    lib = N.lib()
    assert lib.pmpe_select(None, ctypes.byref(r), 4, A, F32, None, None, B, C, None, D, None, None) == NULL
    assert lib.pmpe_select(ctypes.byref(d), None, 4, A, F32, None, None, B, C, None, D, None, None) == NULL
    assert lib.pmpe_select_backward(ctypes.byref(d), ctypes.byref(r), 4, A, F32, B, None, D, None) == NULL
    assert lib.pmpe_select_backward(ctypes.byref(d), ctypes.byref(r), 4, A, 5, B, C, D, None) == DTYPE


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), NULL), (dict(wp=None), NULL), (dict(ws=None, n=0), WORKSPACE), (dict(n=64), WORKSPACE), (dict(x=A + 4), ALIGN),
    (dict(wp=A + 8), ALIGN), (dict(ws=E + 8), ALIGN), (dict(T=0, x=None), 0)])
def test_route_scored(kw, status):
    v = dict(T=4, x=A, wp=B, ws=E, n=1 << 20)
    v.update(kw)
    d, r = P.make_desc(2048, 768, 128, 32, 8), rule()
    assert N.lib().pmpe_route_scored(ctypes.byref(d), ctypes.byref(r), v["T"], v["x"], v["wp"], None, None, None, None, B, C,
                                     None, D, None, None, v["ws"], v["n"], None) == status


def test_backward_scored_needs_its_rule():
    d = P.make_desc(256, 128, 16, 8, 4)
    n = len(N.lib().pmpe_backward_scored.argtypes)
    args = lambda r, z: [ctypes.byref(d), r, 4, z] + [A] * (n - 7) + [E, 0, None]  # noqa: E731
    ok = rule(n_group_pub=4, topk_group_pub=2, n_group_priv=2, topk_group_priv=1)
    assert N.lib().pmpe_backward_scored(*args(None, A)) == NULL
    assert N.lib().pmpe_backward_scored(*args(ctypes.byref(rule(topk_group_priv=1)), A)) == SHAPE  # 2 experts for 4 slots
    assert N.lib().pmpe_backward_scored(*args(ctypes.byref(ok), None)) == NULL  # sigmoid without the logits
    assert N.lib().pmpe_backward_scored(*args(ctypes.byref(ok), A)) == WORKSPACE
    ok.scale = 0.0
    assert N.lib().pmpe_backward_scored(*args(ctypes.byref(ok), A)) == SHAPE


def test_a_balance_bias_needs_a_rule():
    w = torch.zeros(1)
    with pytest.raises(ValueError):
        P.PolicyMaskedMoE(P.make_desc(256, 128, 16, 8, 4), w, w, None, w, w, w, w, select_bias=w)


def arrays(ptrs=(A, B), sizes=(10, 20), types=(F32, BF16)):
    n = len(ptrs)
    return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_uint64 * n)(*sizes), (ctypes.c_int32 * n)(*types), n


def grad_norm(a=None, max_norm=1.0, norm=C, ws=D, n=1 << 20):
    p, s, t, c = a or arrays()
    return N.lib().pmpe_grad_norm(p, s, t, c, max_norm, norm, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(a=arrays((A, None))), NULL), (dict(norm=None), NULL), (dict(a=(None, None, None, 1)), NULL),
    (dict(a=arrays(types=(F32, 2))), DTYPE), (dict(a=arrays(sizes=(1 << 43, 1))), SHAPE), (dict(a=(None, None, None, -1)), SHAPE),
    (dict(a=(None, None, None, (1 << 20) + 1)), SHAPE), (dict(max_norm=0.0), SHAPE), (dict(max_norm=-1.0), SHAPE),
    (dict(max_norm=float("nan")), SHAPE), (dict(a=arrays((A + 2, B))), ALIGN), (dict(a=arrays((A, B + 1))), ALIGN),
    (dict(norm=C + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(n=16), WORKSPACE), (dict(ws=D + 8), ALIGN)])
def test_grad_norm(kw, status):
    assert grad_norm(**kw) == status


def clip_grads(a=None, outs=None, norm=C):
    p, s, t, c = a or arrays()
    o = None if outs is None else (ctypes.c_void_p * len(outs))(*outs)
    return N.lib().pmpe_clip_grads(p, o, s, t, c, norm, None)


@pytest.mark.parametrize("kw,status", [
    (dict(a=arrays((None, B))), NULL), (dict(norm=None), NULL), (dict(outs=(A, None)), NULL), (dict(outs=(D, E + 1)), ALIGN),
    (dict(outs=(D + 2, E)), ALIGN), (dict(norm=C + 1), ALIGN), (dict(outs=(A + 4, B)), SHAPE), (dict(outs=(A, B - 2)), SHAPE),
    (dict(a=(None, None, None, 0)), 0), (dict(a=arrays((None,), (0,), (F32,)), outs=(None,)), 0)])
def test_clip_grads(kw, status):
    assert clip_grads(**kw) == status


def test_grad_norm_workspace():
    size = lambda *n: N.lib().pmpe_grad_norm_workspace_bytes((ctypes.c_uint64 * len(n))(*n), len(n))  # noqa: E731
    assert size() > 0 and size(5) == size(1 << 31) < size(1 << 42) and size(5) < size(*[1] * 500) == size(*[1, 0] * 500)
    assert size(1 << 43) == 0 and N.lib().pmpe_grad_norm_workspace_bytes(None, 1) == 0
    assert N.lib().pmpe_grad_norm_workspace_bytes(None, -1) == 0


@pytest.mark.parametrize("ptrs,sizes,outs", [
    ((A, A), (10, 5), None), ((A + 16, A), (10, 5), None), ((A, A + 36), (10, 5), None),   # a tensor twice; one inside the other
    ((B, A, B + 4), (4, 4, 1), None), ((A, B), (10, 5), (D, D)), ((A, B), (10, 5), (D, D + 36)),
    ((A, B), (10, 5), (E, E - 16)), ((A, B), (10, 5), (B, D)), ((A, B), (10, 5), (B + 16, D)),  # an output on another gradient
    ((A, B), (10, 5), (D, A + 36)), ((B, A), (5, 10), (B, A + 4)), ((A, B, C), (9, 0, 9), (B, None, C - 4))])
def test_clip_grads_refuses_outputs_that_overlap(ptrs, sizes, outs):
    assert clip_grads(arrays(ptrs, sizes, (F32,) * len(ptrs)), outs) == SHAPE


def test_a_clipped_step_takes_each_optimizer_once():
    opt = object()
    for steps in ([], [(opt, None), (opt, None)]):
        with pytest.raises(ValueError):
            P.step_clipped(steps, 1.0)


def test_adamw_clipped():
    f = N.lib().pmpe_adamw_clipped
    hp = (1e-3, 0.9, 0.99, 1e-8, 0.0)
    assert f(A, F32, None, B, C, D, 4, 1, *hp, None, None) == NULL
    assert f(A, BF16, None, B, C, D, 4, 1, *hp, E, None) == DTYPE
    assert f(A, F32, None, B, C, D, 4, 0, *hp, E, None) == SHAPE
    assert f(A + 4, F32, None, B, C, D, 4, 1, *hp, E, None) == ALIGN
    assert f(None, F32, None, B, C, D, 0, 1, *hp, E, None) == 0


def mx(d=None, T=4, xq=A, xs=B, cnt=C, off=C, rt=C, w=(A, A, A, A), s=(B, B, B, B), y=D, rows=C, ws=E, n=1 << 30):
    if d is None:
        d = P.make_desc(2048, 768, 128, 32, 8)
        d.w_dtype = N.PMPE_FP8_E4M3
    return N.lib().pmpe_expert_ffn_mx(ctypes.byref(d), T, xq, xs, cnt, off, rt, *w, *s, y, rows, None, None, ws, n, None)


def mx_desc(**kw):
    v = dict(hidden=2048, inter=768, n_pub=128, n_priv=32, top_k=8)
    v.update(kw)
    d = P.make_desc(**v)
    d.w_dtype = N.PMPE_FP8_E4M3
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(d=P.make_desc(2048, 768, 128, 32, 8)), DTYPE), (dict(d=mx_desc(inter=704)), SHAPE), (dict(d=mx_desc(hidden=192)), SHAPE),
    (dict(d=mx_desc(n_shared=1, shared_inter=128)), SHAPE), (dict(d=mx_desc(top_k=33)), SHAPE), (dict(T=-1), SHAPE),
    (dict(xq=None), NULL), (dict(xs=None), NULL), (dict(cnt=None), NULL), (dict(off=None), NULL), (dict(rt=None), NULL),
    (dict(y=None), NULL), (dict(rows=None), NULL), (dict(w=(None, A, A, A)), NULL), (dict(s=(B, None, B, B)), NULL),
    (dict(w=(A, A, None, A)), NULL), (dict(s=(B, B, B, None)), NULL), (dict(xq=A + 8), ALIGN), (dict(y=D + 2), ALIGN),
    (dict(w=(A + 4, A, A, A)), ALIGN), (dict(ws=None), WORKSPACE), (dict(n=4 * 8 * 768), WORKSPACE), (dict(ws=E + 4), ALIGN),
    (dict(T=0, xq=None), 0)])
def test_expert_ffn_mx(kw, status):
    assert mx(**kw) == status


def test_expert_ffn_mx_workspace():
    assert P.pmpe_expert_ffn_mx_workspace_bytes(mx_desc(), 4) >= 4 * 8 * 768 * 33 // 32
    assert P.pmpe_expert_ffn_mx_workspace_bytes(mx_desc(inter=704), 4) == 0
    assert N.lib().pmpe_expert_ffn_mx_workspace_bytes(None, 4) == 0
