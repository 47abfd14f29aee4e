"""Global gradient norm and clipping on the GPU against 64-bit sums: lists of one to many tensors,
both types, odd lengths and starts, empty tensors, values whose squares leave fp32, values that are
not finite, in place and out of place; the clipped AdamW step; the optimizer object.

Tolerances: the sum is 64-bit (relative error below 2^-40 for these lengths) and rounded to fp32 once,
as is the factor: 2^-24 each. A clipped value carries the factor's rounding and its own: 2^-23 in fp32,
2^-8 + 2^-23 in bf16."""
import math

import numpy as np
import pytest
import torch

import paper_2608_06690_amd as P
import workloads as W
from oracle import pmpe_oracle as O
from tests import pmpe_cases as C

pytestmark = pytest.mark.gpu
U = 2.0 ** -24 * (1 + 2.0 ** -10)


def log(msg):
    print(msg, flush=True)


def grads_of(lengths, dt, seed, std=0.02, shift=0):
    """Gradients side by side in one buffer, the first `shift` elements in."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    flat = torch.empty(sum(lengths) + shift, dtype=dt, device="cuda").normal_(0.0, std, generator=g)
    return list(flat[shift:].split(list(lengths)))


def norm_of(grads, max_norm, norm=None):
    norm = torch.empty(2, device="cuda") if norm is None else norm
    ws = torch.empty(P.pmpe_grad_norm_workspace_bytes(grads), dtype=torch.uint8, device="cuda")
    P.pmpe_grad_norm(grads, max_norm, norm, ws)
    torch.cuda.synchronize()
    return norm


def exact(grads, max_norm):
    n = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return n, min(1.0, max_norm / (n + 1e-6))


LISTS = [[1], [7], [8192], [8193], [24576 + 5], [1 << 20], [3, 0, 5], [1, 8192, 17, 100000, 0, 2], [5] * 96, [33] * 97, [11] * 400,
         [40000] * 250, [3_000_001, 70]]


@pytest.mark.parametrize("lengths", LISTS, ids=lambda v: f"{len(v)}x{v[0]}")
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("max_norm", [0.01, 1e6])
def test_norm_and_clip(lengths, dt, shift, max_norm):
    log(f"clip {len(lengths)} x {lengths[0]} {dt} shift={shift} max={max_norm}")
    grads = grads_of(lengths, dt, 1, shift=shift)
    norm = norm_of(grads, max_norm)
    n, coef = exact(grads, max_norm)
    assert abs(float(norm[0]) - n) <= U * n and abs(float(norm[1]) - coef) <= U * coef
    step = (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24) + U
    out = torch.full((sum(lengths) + 4,), 9.0, dtype=dt, device="cuda")
    outs = list(out[2:-2].split(lengths))
    want = [g.double() * coef for g in grads]
    P.pmpe_clip_grads(grads, outs, norm)
    assert torch.all(out[:2] == 9.0) and torch.all(out[-2:] == 9.0)
    for o, w in zip(outs, want):
        assert torch.all((o.double() - w).abs() <= step * w.abs())
    before = [g.clone() for g in grads]
    P.pmpe_clip_grads(grads, None, norm)  # in place
    for g, o, b in zip(grads, outs, before):
        assert torch.equal(g, o)
        assert coef < 1.0 or torch.equal(g, b)


def test_types_of_one_list_and_handles():
    grads = grads_of([100, 9000], torch.float32, 2) + grads_of([50, 20000], torch.bfloat16, 3)
    handle = P.GradList(grads)
    a, b = norm_of(grads, 0.5), norm_of(handle, 0.5)
    assert torch.equal(a, b) and len(handle) == 4
    n, coef = exact(grads, 0.5)
    assert abs(float(a[0]) - n) <= U * n
    assert torch.equal(norm_of(handle, 0.5), b)  # the same bits each time
    grads[1].mul_(2.0)  # the handle names the tensors: their values are read at each call
    n, _ = exact(grads, 0.5)
    assert abs(float(norm_of(handle, 0.5)[0]) - n) <= U * n


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e30, 1e-30])
def test_values_whose_squares_leave_fp32(dt, size):
    grads = grads_of([5000, 12345], dt, 4, std=size)
    n, coef = exact(grads, 1.0)
    got = norm_of(grads, 1.0)
    assert abs(float(got[0]) - n) <= U * n and abs(float(got[1]) - coef) <= U * coef + 2.0 ** -149
    assert coef == 1.0 or coef < 1e-29


def test_empty_lists_and_values_that_are_not_finite():
    assert norm_of([], 1.0).tolist() == [0.0, 1.0]
    e = torch.empty(0, device="cuda")
    assert norm_of([e, e], 1.0).tolist() == [0.0, 1.0]
    P.pmpe_clip_grads([], None, torch.ones(2, device="cuda"))
    z = [torch.zeros(1000, device="cuda")]
    assert norm_of(z, 1.0).tolist() == [0.0, 1.0]
    g = grads_of([300, 9000], torch.float32, 5)
    assert norm_of(g, math.inf)[1] == 1.0
    g[1][8500] = math.inf
    got = norm_of(g, 1.0)
    assert got.tolist() == [math.inf, 0.0]
    P.pmpe_clip_grads(g, None, got)
    assert g[1][8500].isnan() and torch.all(g[0] == 0)
    g[0][0] = float("nan")
    assert norm_of(g, 1.0).isnan().all()


@pytest.mark.parametrize("count", [160, 161, 700])
def test_many_outputs_in_another_order(count):
    grads = grads_of([1 + (37 * i) % 9001 for i in range(count)], torch.bfloat16, 10)
    back = torch.empty(sum(t.numel() for t in grads), dtype=torch.bfloat16, device="cuda")
    outs = list(back.split([t.numel() for t in grads[::-1]]))[::-1]
    norm = norm_of(grads, 0.1)
    n, coef = exact(grads, 0.1)
    assert abs(float(norm[0]) - n) <= U * n
    P.pmpe_clip_grads(grads, outs, norm)
    for o, t in zip(outs, grads):
        w = t.double() * coef
        assert torch.all((o.double() - w).abs() <= (2.0 ** -8 + U) * w.abs())


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_tensors_of_more_than_2_31_elements(dt):
    n = (1 << 31) + 8195
    g = torch.zeros(n, dtype=dt, device="cuda")
    at = torch.tensor([0, 4095, (1 << 31) - 1, 1 << 31, (1 << 31) + 4096, n - 1], device="cuda")
    g[at] = torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0, 32.0], dtype=dt, device="cuda")
    g = [torch.ones(3, dtype=dt, device="cuda"), g]
    norm = norm_of(g, 0.5)
    total = math.sqrt(3 + 1365)
    assert abs(float(norm[0]) - total) <= U * total
    P.pmpe_clip_grads(g, None, norm)
    want = torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0, 32.0], device="cuda").double() * (0.5 / (total + 1e-6))
    step = (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24) + U
    assert torch.all((g[1][at].double() - want).abs() <= step * want)
    g[1][at] = 0
    assert not g[1].any()


def test_refusals_of_the_binding():
    g, norm = grads_of([10, 20], torch.float32, 6), torch.ones(2, device="cuda")
    for outs in (g[:1], [g[0], g[1][:19]], [g[0], g[1].bfloat16()]):
        with pytest.raises(ValueError):
            P.pmpe_clip_grads(g, outs, norm)
    with pytest.raises(ValueError):
        P.pmpe_clip_grads([g[0], g[1].cpu()], None, norm)
    with pytest.raises(ValueError):
        P.pmpe_clip_grads(g, None, norm[:1])
    with pytest.raises(ValueError):
        P.GradList([g[0].double()])
    flat = torch.zeros(100, device="cuda")
    with pytest.raises(P.PmpeError):  # overlapping, not equal
        P.pmpe_clip_grads([flat[:50]], [flat[10:60]], norm)
    with pytest.raises(P.PmpeError):
        P.pmpe_grad_norm(g, 0.0, norm, torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))


def test_outputs_in_any_order_and_partly_in_place():
    g = grads_of([1000, 0, 70, 9000, 5], torch.float32, 8)
    g = [g[3], g[1], g[0], g[4], g[2]]
    norm = norm_of(g, 0.1)
    want = [t.double() * float(norm[1]) for t in g]
    to = torch.full((10020,), 9.0, device="cuda")
    outs = [to[10:9010], to[:0], g[2], to[9010:9015], to[9015:9085]]
    P.pmpe_clip_grads(g, outs, norm)
    for o, w in zip(outs, want):
        assert torch.all((o.double() - w).abs() <= 2.0 ** -23 * w.abs())
    assert torch.all(to[:10] == 9.0) and torch.all(to[9085:] == 9.0)


HP = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("n", [1, 7, 1021, 65536 + 5])
@pytest.mark.parametrize("bf16", [False, True])
def test_clipped_adamw(n, bf16):
    g = torch.Generator().manual_seed(n)
    p0 = torch.randn(n, generator=g, dtype=torch.float64)
    if bf16:
        p0 = p0.to(torch.bfloat16).double()
    param = p0.to(torch.bfloat16 if bf16 else torch.float32).cuda()
    master = p0.float().cuda() if bf16 else None
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    rp, rm, rv = p0.numpy(), np.zeros(n), np.zeros(n)
    for step in (1, 2, 3):
        grad = torch.randn(n, generator=g).float().cuda()
        norm = norm_of([grad], 0.1 if step < 3 else 1e9)
        _, coef = exact([grad], 0.1 if step < 3 else 1e9)
        P.pmpe_adamw_clipped(param, master, grad, m, v, step, *HP.values(), norm)
        rp, rm, rv = O.adamw_step(rp, grad.double().cpu().numpy() * coef, rm, rv, step, **HP)
    torch.cuda.synchronize()
    # fp32 steps of O(10) roundings each
    assert C.rel_l2((master if bf16 else param).double().cpu().numpy(), rp) <= 1e-6
    assert C.rel_l2(m.double().cpu().numpy(), rm) <= 1e-6 and C.rel_l2(v.double().cpu().numpy(), rv) <= 1e-6
    if bf16:
        assert torch.equal(param, master.to(torch.bfloat16))
    # a factor of 1 is the plain step to the bit; a norm that is not finite changes nothing
    state = [t.clone() for t in (param, m, v)]
    ref = [t.clone() for t in state]
    refm, mas = (master.clone(), master.clone()) if bf16 else (None, None)
    P.pmpe_adamw(ref[0], refm, grad, ref[1], ref[2], 4, *HP.values())
    P.pmpe_adamw_clipped(state[0], mas, grad, state[1], state[2], 4, *HP.values(), norm)
    assert all(torch.equal(a, b) for a, b in zip(state, ref))
    for bad in (math.inf, float("nan")):
        norm.fill_(bad)
        P.pmpe_adamw_clipped(state[0], mas, grad, state[1], state[2], 5, *HP.values(), norm)
    assert all(torch.equal(a, b) for a, b in zip(state, ref)) and (not bf16 or torch.equal(mas, refm))


def training_layer(seed):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=128, requests=2, hidden=256, inter=128, n_pub=16, n_priv=8, top_k=4)
    layer, _ = C.device_layer(cfg, layer=seed)
    x = W.make_x(cfg, "cuda")
    words = torch.full((128,), P.PMPE_POLICY_ALLOW - (1 << 32), dtype=torch.int32, device="cuda")
    b = layer.forward(x, words, layer.audit_buffers(128, 1), train=True)
    return layer, layer.backward(x, torch.randn(128, 256, device="cuda").bfloat16(), b)


def test_optimizer_of_one_layer_and_of_several():
    (la, ga), (lb, gb) = training_layer(0), training_layer(1)
    want_p, grads = [], []
    for lay, g in ((la, ga), (lb, gb)):
        grads.append([g.dwr_priv, g.dw13_priv, g.dw2_priv])
    n, coef = exact(grads[0] + grads[1], 0.5)
    assert coef < 1.0
    for lay, gs in ((la, grads[0]), (lb, grads[1])):
        for p, g in zip((lay.wr_priv, lay.w13_priv, lay.w2_priv), gs):
            want_p.append(O.adamw_step(p.double().cpu().numpy(), g.double().cpu().numpy() * coef, np.zeros(p.shape),
                                       np.zeros(p.shape), 1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)[0])
    opts = [P.PrivateAdamW(lay, lr=1e-3) for lay in (la, lb)]
    norm = P.step_clipped(zip(opts, (ga, gb)), 0.5)
    torch.cuda.synchronize()
    assert abs(float(norm[0]) - n) <= U * n and opts[1].norm is norm
    got = [t for o in opts for t in (o.params[0], o.master[1], o.master[2])]
    for a, e in zip(got, want_p):
        assert C.rel_l2(a.double().cpu().numpy(), e) <= 1e-6
    # the transposed copies that a backward keeps follow the clipped step
    assert torch.equal(la._wt_priv[0], la.w2_priv.transpose(1, 2))
    # one layer with max_norm
    lc, gc = training_layer(2)
    n, coef = exact([gc.dwr_priv, gc.dw13_priv, gc.dw2_priv], 0.25)
    w = O.adamw_step(lc.wr_priv.double().cpu().numpy(), gc.dwr_priv.double().cpu().numpy() * coef, np.zeros(lc.wr_priv.shape),
                     np.zeros(lc.wr_priv.shape), 1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)[0]
    opt = P.PrivateAdamW(lc, lr=1e-3, max_norm=0.25)
    opt.step(gc)
    torch.cuda.synchronize()
    assert abs(float(opt.norm[0]) - n) <= U * n and abs(float(opt.norm[1]) - coef) <= U * coef
    assert C.rel_l2(lc.wr_priv.double().cpu().numpy(), w) <= 1e-6
    with pytest.raises(ValueError):
        P.PrivateAdamW(lc, max_norm=0.0)


def test_graph_replays():
    grads = grads_of([33] * 120 + [70000], torch.float32, 8)
    outs = [torch.empty_like(g) for g in grads]
    src, to = P.GradList(grads), P.GradList(outs)
    norm = torch.empty(2, device="cuda")
    ws = torch.empty(P.pmpe_grad_norm_workspace_bytes(src), dtype=torch.uint8, device="cuda")

    def both():
        P.pmpe_grad_norm(src, 0.5, norm, ws)
        P.pmpe_clip_grads(src, to, norm)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (11, 12, 13):
        for g, n in zip(grads, grads_of([33] * 120 + [70000], torch.float32, seed)):
            g.copy_(n)
        graph.replay()
        got = [norm.clone()] + [o.clone() for o in outs]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [norm] + outs))
