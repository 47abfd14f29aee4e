"""The block of norm, layer and residual on other streams than the current one, with the options that a
layer with a score rule has."""
import pytest
import torch

import paper_2608_06690_amd as P
import workloads as W
from tests import pmpe_cases as C

pytestmark = pytest.mark.gpu
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)


def log(msg):
    print(msg, flush=True)


def randn(shape, seed, std=1.0, dt=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=g)


def words_of(T):
    words = torch.zeros(T, dtype=torch.int32)
    words[::2] = ALLOW
    return words.cuda()


def block(T, rule=None):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=T, requests=1, hidden=256, inter=128, n_pub=16, n_priv=8, top_k=4)
    layer, _ = C.device_layer(cfg)
    layer.rule = rule
    if rule is not None:
        layer.select_bias = randn((24,), 3, 0.02, torch.float32)
    return P.NormedMoE(layer, randn((256,), 4, 0.1, torch.float32) + 1.0), torch.tensor([0, T], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("T", [7, 1500])
def test_a_backward_on_another_stream_keeps_its_workspace(T):
    log(f"backward on another stream {T}")
    blk, offs = block(T)
    h, delta, dres, dout = [randn((T, 256), s) for s in (5, 6, 7, 8)]
    b = blk.forward(h, delta, words_of(T), blk.layer.audit_buffers(T, 1), offs, train=True)
    dx, dw = torch.empty_like(h), torch.empty(256, device="cuda")
    blk.backward(dres, dout, b, dx, dweight=dw)
    torch.cuda.synchronize()
    want = dx.clone(), dw.clone()
    b.ws = None  # a first call on the other stream
    g, st = blk.layer.grad_buffers(T), torch.cuda.Stream()
    for _ in range(3):
        dx.zero_(), dw.zero_()
        st.wait_stream(torch.cuda.current_stream())
        blk.backward(dres, dout, b, dx, g=g, dweight=dw, stream=st)
        # the current stream goes on with memory of that size
        n = P.pmpe_rmsnorm_backward_workspace_bytes(T, 256)
        other = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
        assert all(bool((t == 7).all()) for t in other)


def fp8_of(layer):
    """The layer's expert weights as e4m3 bytes with a power-of-two scale per row."""
    q, s = [], []
    for w in (layer.w13_pub, layer.w2_pub, layer.w13_priv, layer.w2_priv):
        e = torch.ceil(torch.log2(w.float().abs().amax(2).clamp(min=1e-30) / 448.0))
        q.append(torch.ldexp(w.float(), -e.unsqueeze(2)).to(torch.float8_e4m3fn).view(torch.uint8))
        s.append(torch.exp2(e).contiguous())
    return tuple(q + s)


SIGMOID = dict(score=P.PMPE_SCORE_SIGMOID, groups=(4, 2), groups_priv=(2, 1), group_top=2, scale=2.0)


def outputs(b, *more):
    """What a forward of the block has written."""
    b8 = [b.norm_q, b.norm_scale] if b.norm_q is not None else []
    return [b.total, b.norm, b.rstd, *b8, b.layer.topk_idx, b.layer.topk_gate, b.layer.allow, b.layer.y_perm, b.layer.out, *more]


def spoil(tensors):
    for t in tensors:
        t.fill_(77)


@pytest.mark.parametrize("T", [1, 37, 1200])
@pytest.mark.parametrize("rule", [False, True])
def test_passes_on_another_stream(T, rule):
    """Forward, 8-bit forward and training step on a side stream give the current stream's results."""
    log(f"passes on another stream {T} {rule}")
    blk, offs = block(T, P.make_score_rule(**SIGMOID) if rule else None)
    w8, words, audit = fp8_of(blk.layer), words_of(T), blk.layer.audit_buffers(T, 1)
    h, delta, dres, dout = [randn((T, 256), s) for s in (15, 16, 17, 18)]
    dx, dw, g = torch.empty_like(h), torch.empty(256, device="cuda"), blk.layer.grad_buffers(T)
    grads = [g.dx, g.dw13_priv, g.dw2_priv, g.dwr_priv]
    st = torch.cuda.Stream()

    def passes(stream):
        got = []
        b = blk.forward_mx(h, delta, words, w8, audit.zero_(), offs, stream=stream)
        torch.cuda.synchronize()
        got += [t.clone() for t in outputs(b)]
        spoil(outputs(b))
        torch.cuda.synchronize()
        b = blk.forward(h, delta, words, audit.zero_(), offs, stream=stream, train=True)
        blk.backward(dres, dout, b, dx, g=g, dweight=dw, stream=stream)
        torch.cuda.synchronize()
        b8 = (b.norm_q, b.norm_scale)
        assert all(bool((t == 77).all()) for t in b8)  # a plain forward leaves them
        got += [t.clone() for t in outputs(b, dx, dw, *grads) if all(t is not q for q in b8)]
        spoil(outputs(b, dx, dw, *grads))
        torch.cuda.synchronize()
        return got

    want = passes(None)
    got = passes(st)
    assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("T", [19, 1000])
@pytest.mark.parametrize("rule", [False, True])
def test_captured_passes_follow_their_inputs(T, rule):
    """Every replay on new inputs, with all outputs overwritten in between, against the eager pass."""
    log(f"captured passes {T} {rule}")
    blk, offs = block(T, P.make_score_rule(**SIGMOID) if rule else None)
    w8, words, audit = fp8_of(blk.layer), words_of(T), blk.layer.audit_buffers(T, 1)
    h, delta, dres, dout = [randn((T, 256), s) for s in (25, 26, 27, 28)]
    dx, dw, g = torch.empty_like(h), torch.empty(256, device="cuda"), blk.layer.grad_buffers(T)
    grads = [dx, dw, g.dx, g.dw13_priv, g.dw2_priv, g.dwr_priv]

    def mx():
        return outputs(blk.forward_mx(h, delta, words, w8, audit, offs))

    def train():
        b = blk.forward(h, delta, words, audit, offs, train=True)
        blk.backward(dres, dout, b, dx, g=g, dweight=dw)
        return [t for t in outputs(b, *grads) if t is not b.norm_q and t is not b.norm_scale]

    for step in (mx, train):
        outs = step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in (31, 41, 51):
            for i, t in enumerate((h, delta, dres, dout)):
                t.copy_(randn((T, 256), seed + i))
            words.copy_(words.flip(0))
            spoil(outs)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in outs]
            spoil(outs)
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, outs))
            assert not any(bool((t == 77).all()) for t in got)


def test_joint_and_single_steps_on_two_streams():
    """After a joint step the optimizers step on their own, on streams of their own: each clips by its own
    norm and shows it."""
    T = 64
    opts, grads = [], []
    for i in range(2):
        blk, offs = block(T)
        b = blk.forward(randn((T, 256), 60 + i), None, words_of(T), blk.layer.audit_buffers(T, 1), offs, train=True)
        grads.append(blk.layer.backward(b.norm, randn((T, 256), 70 + i, 1.0 + 4 * i), b.layer))
        opts.append(P.PrivateAdamW(blk.layer, lr=1e-3, max_norm=0.25))
    torch.cuda.synchronize()
    norms = [sum(float(t.double().square().sum()) for t in (g.dwr_priv, g.dw13_priv, g.dw2_priv)) ** 0.5 for g in grads]
    assert norms[0] < 0.9 * norms[1]

    def shows(opt, n):
        return (abs(float(opt.norm[0]) - n) <= 2.0 ** -23 * n and
                abs(float(opt.norm[1]) - min(1.0, 0.25 / (n + 1e-6))) <= 2.0 ** -23 * min(1.0, 0.25 / n))

    joint = (norms[0] ** 2 + norms[1] ** 2) ** 0.5
    P.step_clipped(zip(opts, grads), 0.25)
    torch.cuda.synchronize()
    assert all(shows(opt, joint) for opt in opts)
    streams = [torch.cuda.Stream() for _ in opts]
    m = [[t.clone() for t in opt.m] for opt in opts]
    torch.cuda.synchronize()
    for _ in range(4):
        for opt, g, st in zip(opts, grads, streams):
            opt.step(g, stream=st)
    torch.cuda.synchronize()
    for opt, g, n, m0 in zip(opts, grads, norms, m):
        assert shows(opt, n)
        # m after four steps of one clipped gradient: 0.9^4 m + (1 - 0.9^4) coef g. fp32: 0.9 and the factor are off
        # by 2^-24, which is 2^-21 of 1 - 0.9, and each step rounds three times
        coef = min(1.0, 0.25 / (n + 1e-6))
        for t, before, gr in zip(opt.m, m0, (g.dwr_priv, g.dw13_priv, g.dw2_priv)):
            want = 0.9 ** 4 * before.double() + (1 - 0.9 ** 4) * coef * gr.double()
            size = before.double().abs() + coef * gr.double().abs()
            assert torch.all((t.double() - want).abs() <= 2.0 ** -19 * size + 1e-30)
    P.step_clipped([(opts[1], grads[1]), (opts[0], grads[0])], 0.25)
    torch.cuda.synchronize()
    assert all(shows(opt, joint) for opt in opts)
