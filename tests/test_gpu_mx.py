"""Expert products on 8-bit activations and weights, on the GPU, against the same definition in 64
bits (h rounded to e4m3 with block scales in between), element by element.

Tolerance of an output: half a bf16 step of it, the errors of the two sums, and where the error of h
reaches a rounding border of e4m3 (or of a block's scale), the whole change that the other rounding of
that value of h makes. fp32 silu and products: 16 steps of 2^-24 of h.

Error of a sum over K. The fp8 instruction aligns the products of 8 consecutive k to the largest of
them and drops what lies below 2^-13 of its power of two (measured on the instruction: next to a product
of 2^16, 2^3 is kept and 2^2 is not; products of other groups of 8 keep down to 2^-23). A product p of a
group is so off by d <= 2^-13 max|p| towards zero, its sign random as the inputs' signs are: by Hoeffding's
inequality the sum of such errors passes t = 7 sqrt(sum d^2) with probability 2 exp(-49 / 2) = 5e-11. At
most 7 products of a group are cut and max p^2 <= sum p^2, so sum d^2 <= 7 * 2^-26 * sum p^2, and
t <= 18.6 * 2^-13 * sqrt(sum p^2). The groups and steps are added in fp32: K / 128 + 16 roundings of the sum
of magnitudes."""
import numpy as np
import pytest
import torch

import paper_2608_06690_amd as P
import workloads as W
from tests import pmpe_cases as C

pytestmark = pytest.mark.gpu
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)


def log(msg):
    print(msg, flush=True)


def exponent(a):
    """log2 of the block scale of a block's largest magnitude (fp64)."""
    m, e = torch.frexp(a)
    return torch.where(a > 0, e - 9 + (m > 0.875).to(e.dtype), 0).clamp(min=-126)


def to_e4m3(v):
    """fp64 magnitudes up to 448 to the nearest e4m3 value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def quantise(h, e=None):
    """Values of h [.., n] with blocks of 32, the exponents given or its own."""
    b = h.unflatten(-1, (-1, 32))
    e = exponent(b.abs().amax(-1)) if e is None else e
    s = torch.exp2(e.double()).unsqueeze(-1)
    return (to_e4m3((b / s).clamp(-448, 448)) * s).flatten(-2), e


def fp8(x, block):
    """e4m3 bytes and exponents of blocks of the last dimension."""
    v = x.double().unflatten(-1, (-1, block))
    e = exponent(v.abs().amax(-1))
    q = to_e4m3(v / torch.exp2(e.double()).unsqueeze(-1)).flatten(-2)
    return q.to(torch.float8_e4m3fn).view(torch.uint8), e


def cut(x, w):
    """Error of the sums x w^T as above."""
    return 18.6 * 2.0 ** -13 * torch.sqrt(x.square() @ w.square().t()) + (x.shape[1] / 128 + 16) * 2.0 ** -24 * (x.abs() @ w.abs().t())


def weights(gen, n, rows, cols):
    w = torch.empty(n, rows, cols, device="cuda").normal_(0.0, 0.05, generator=gen)
    q, e = fp8(w, cols)
    return q, torch.exp2(e.double()).float().view(n, rows).contiguous()


class Case:
    def __init__(self, T, H, I, n, p, k, seed, allow=0.5, hot=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.T, self.H, self.I, self.n, self.p, self.k = T, H, I, n, p, k
        self.d = P.make_desc(H, I, n, p, k)
        self.d.w_dtype = P.PMPE_FP8_E4M3
        x = torch.empty(T, H, device="cuda").normal_(0.0, 1.0, generator=g)
        x *= torch.exp2(torch.randint(-6, 7, (T, 1), generator=g, device="cuda").float())  # rows of different sizes
        x[:, :32] *= 64.0  # and a block of other scale
        self.xq, xe = fp8(x, 32)
        self.xs = (xe + 127).to(torch.uint8)
        self.w = {}
        for pool, c in (("pub", n), ("priv", p)):
            self.w["13" + pool], self.w["13s" + pool] = weights(g, c, 2 * I, H)
            self.w["2" + pool], self.w["2s" + pool] = weights(g, c, H, I)
        z = torch.randn(T, n + p, generator=g, device="cuda")
        if hot is not None:
            z[:, hot] += 9.0  # an expert that most tokens select
        tau = torch.rand(T, generator=g, device="cuda") < allow
        z[:, :n].masked_fill_(tau.unsqueeze(1), -1e9)
        z[:, n:].masked_fill_(~tau.unsqueeze(1), -1e9)
        self.idx = z.topk(k, dim=1).indices.sort(dim=1).values.int().contiguous()
        i32 = dict(dtype=torch.int32, device="cuda")
        self.count, self.off = torch.empty(n + p, **i32), torch.empty(n + p + 1, **i32)
        self.rt, self.tr = torch.empty(T * k, **i32), torch.empty(T * k, **i32)
        d = P.make_desc(H, I, n, p, k)
        ws = torch.empty(P.pmpe_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
        P.pmpe_dispatch(d, T, self.idx, None, self.count, self.off, self.rt, self.tr, None, ws)
        self.ws = torch.empty(P.pmpe_expert_ffn_mx_workspace_bytes(self.d, T), dtype=torch.uint8, device="cuda")

    def run(self, private=True, y=None, stream=None):
        w = self.w
        y = torch.full((self.T * self.k, self.H), 3.0, dtype=torch.bfloat16, device="cuda") if y is None else y
        rows, calls = torch.zeros(self.T, dtype=torch.int32, device="cuda"), torch.zeros(self.p, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pr = (lambda t: t) if private else (lambda t: None)
        P.pmpe_expert_ffn_mx(self.d, self.T, self.xq, self.xs, self.count, self.off, self.rt, w["13pub"], w["2pub"],
                             pr(w["13priv"]), pr(w["2priv"]), w["13spub"], w["2spub"], pr(w["13spriv"]), pr(w["2spriv"]),
                             y, rows, calls, status, self.ws, stream)
        torch.cuda.synchronize()
        return y, rows, calls, int(status)

    def expert(self, j):
        pool, at = ("pub", j) if j < self.n else ("priv", j - self.n)
        deq = lambda a: self.w[a + pool][at].view(torch.float8_e4m3fn).double() * self.w[a + "s" + pool][at].double().unsqueeze(1)  # noqa: E731
        return deq("13"), deq("2")

    def exact(self):
        """Output rows in 64 bits and how far fp32 may be from them."""
        x = self.xq.view(torch.float8_e4m3fn).double().unflatten(1, (-1, 32))
        x = (x * torch.exp2(self.xs.double() - 127).unsqueeze(2)).flatten(1)
        y = torch.zeros(self.T * self.k, self.H, dtype=torch.float64, device="cuda")
        room = torch.zeros_like(y)
        u, off, I = 2.0 ** -24, self.off.tolist(), self.I
        for j in range(self.n + self.p):
            if off[j] == off[j + 1]:
                continue
            w13, w2 = self.expert(j)
            xr = x[self.rt[off[j]:off[j + 1]].long()]
            ab, size = xr @ w13.t(), cut(xr, w13)
            a, b = ab[:, :I], ab[:, I:]
            ea, eb = size[:, :I], size[:, I:]
            sil = torch.nn.functional.silu(a)
            h = sil * b
            eh = 1.1 * ea * b.abs() + sil.abs() * eb + 2 * ea * eb + 16 * u * h.abs()  # |silu'| <= 1.1
            q, e = quantise(h)
            amax, em = [v.unflatten(-1, (-1, 32)).abs().amax(-1) for v in (h, eh)]
            lo_e, hi_e = exponent((amax - em).clamp(min=0)), exponent(amax + em)
            change = torch.zeros_like(h)
            for ee in (e, lo_e, hi_e):
                for v in (h - eh, h + eh):
                    change = torch.maximum(change, (quantise(v, ee)[0] - q).abs())
            y[off[j]:off[j + 1]] = q @ w2.t()
            room[off[j]:off[j + 1]] = change @ w2.abs().t() + cut(q, w2)
        return y, room


def check(c, got, y, room):
    off = (got.double() - y).abs()
    bad = off > 2.0 ** -8 * y.abs() + (1 + 2.0 ** -8) * room + 1e-38
    assert not bad.any(), (int(bad.sum()), float((off / (y.abs() + 1e-30))[bad].max()))
    rel = float((got.double() - y).norm() / y.norm())
    # as a whole: roundings to bf16 (2^-8 / sqrt(3) at most in the root mean square) and few other roundings of h
    assert rel <= 2.0 ** -8
    log(f"  rel {rel:.2e}, mean room {float((room / (y.abs() + 1e-30)).median()):.1e}")


# tokens, H, I, public, private, k: single tokens; 64-row tiles; tiles of one K step; 128-row tiles, ragged, odd widths
CASES = [(1, 128, 128, 4, 4, 2), (3, 256, 128, 8, 4, 2), (64, 384, 256, 16, 8, 4), (33, 128, 128, 200, 56, 16),
         (200, 2048, 768, 128, 32, 8), (700, 256, 128, 8, 4, 4), (1111, 1664, 640, 40, 12, 4), (900, 128, 128, 6, 3, 3),
         (2500, 512, 1408, 64, 16, 6), (4096, 256, 256, 4, 2, 2), (5000, 128, 128, 1, 1, 1)]


@pytest.mark.parametrize("shape", CASES, ids=str)
@pytest.mark.parametrize("allow", [0.5, 0.0, 1.0])
def test_rows_against_64_bits(shape, allow):
    log(f"mx {shape} allow={allow}")
    c = Case(*shape, seed=1, allow=allow)
    got, rows, calls, status = c.run()
    check(c, got, *c.exact())
    priv = torch.zeros_like(rows)
    at = int(c.off[c.n])
    priv.index_add_(0, c.rt[at:].long(), torch.ones_like(c.rt[at:]))
    assert torch.equal(rows, priv) and torch.equal(calls, (c.count[c.n:] > 0).int()) and status == 0
    again = c.run()[0]
    assert torch.equal(got, again)


@pytest.mark.parametrize("T", [90, 3000])
def test_an_expert_with_most_rows_and_others_with_none(T):
    c = Case(T, 256, 256, 24, 8, 2, seed=2, hot=3, allow=0.1)
    log(f"mx hot {T}: {c.count.tolist()}")
    assert int(c.count.max()) > 0.8 * T
    got = c.run()[0]
    check(c, got, *c.exact())


@pytest.mark.parametrize("T", [20, 2000])
def test_missing_private_weights(T):
    c = Case(T, 256, 128, 8, 4, 2, seed=3)
    full = c.run()[0]
    y, rows, calls, status = c.run(private=False)
    at = int(c.off[c.n])
    assert torch.equal(y[:at], full[:at]) and torch.all(y[at:] == 0)
    assert torch.all(rows == 0) and torch.all(calls == 0) and status == P._native.PMPE_DEV_PRIV_WEIGHTS_MISSING


# Batches of the 256 x 256 kernel (768 of its tiles and more, 120 rows per expert): tiles of every number of
# rows, two K steps, a last tile of half the width, three steps, experts of many tiles
LARGE = [(2900, 256, 256, 256, 128, 16), (2900, 384, 256, 256, 128, 16), (4800, 1280, 384, 128, 128, 16), (9000, 256, 2048, 8, 4, 4)]


@pytest.mark.parametrize("shape", LARGE, ids=str)
@pytest.mark.parametrize("allow,hot", [(0.5, None), (0.05, None), (1.0, None), (0.4, 3)])
def test_large_batches(shape, allow, hot):
    log(f"mx {shape} allow={allow} hot={hot}")
    c = Case(*shape, seed=5, allow=allow, hot=hot)
    got, rows, calls, status = c.run()
    check(c, got, *c.exact())
    priv = torch.zeros_like(rows)
    at = int(c.off[c.n])
    priv.index_add_(0, c.rt[at:].long(), torch.ones_like(c.rt[at:]))
    assert torch.equal(rows, priv) and torch.equal(calls, (c.count[c.n:] > 0).int()) and status == 0
    for _ in range(3):
        assert torch.equal(got, c.run()[0])


@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_large_batches_without_private_weights(shape):
    log(f"mx {shape} without private weights")
    c = Case(*shape, seed=6)
    full = c.run()[0]
    y, rows, calls, status = c.run(private=False)
    at = int(c.off[c.n])
    assert torch.equal(y[:at], full[:at]) and torch.all(y[at:] == 0)
    assert torch.all(rows == 0) and torch.all(calls == 0) and status == P._native.PMPE_DEV_PRIV_WEIGHTS_MISSING


def test_values_that_are_not_finite():
    c = Case(600, 256, 128, 8, 4, 2, seed=4)
    want = c.run()[0]
    c.xs[5, 3] = 255  # a block that is not a number
    c.xq[9, 40] = 0x7F
    got = c.run()[0]
    hit = ((c.rt == 5) | (c.rt == 9))
    assert torch.all(got[hit].isnan()) and torch.equal(got[~hit], want[~hit])
    # a hidden value beyond every e4m3 block: an infinite h makes its block, and the row, NaN
    c = Case(40, 128, 128, 4, 4, 1, seed=5)
    want = c.run()[0]
    c.xs[7] = 253
    got = c.run()[0]
    assert torch.all(got[c.rt == 7].isnan() | got[c.rt == 7].isinf()) and torch.equal(got[c.rt != 7], want[c.rt != 7])


def test_rows_behind_the_last_and_streams():
    c = Case(300, 256, 128, 8, 4, 3, seed=6)
    want = c.run()[0]
    buf = torch.full((902, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    c.run(y=buf[1:901], stream=st)
    assert torch.equal(buf[1:901], want) and torch.all(buf[0] == 5.0) and torch.all(buf[901] == 5.0)


def test_refusals_of_the_binding():
    c = Case(8, 256, 128, 8, 4, 2, seed=7)
    for name, bad in (("xq", c.xq[:7]), ("xs", c.xs[:, :7].contiguous()), ("xq", c.xq.view(torch.int8))):
        keep = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises(ValueError):
            c.run()
        setattr(c, name, keep)
    with pytest.raises(ValueError):
        c.run(y=torch.empty(15, 256, dtype=torch.bfloat16, device="cuda"))
    c.ws = c.ws[:-1]
    with pytest.raises(P.PmpeError):
        c.run()


# ------------------------------------------------------------------ the operators together


def block(T, score, H=256, I=128):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=T, requests=1, hidden=H, inter=I, n_pub=16, n_priv=8, top_k=4)
    layer, Lw = C.device_layer(cfg)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    if score:
        layer.rule, layer.select_bias = P.make_score_rule(P.PMPE_SCORE_SIGMOID, (4, 2), (2, 1), 2, 2.0), torch.empty(24, device="cuda").normal_(0, 0.02, generator=g)
    weight = torch.empty(H, device="cuda").normal_(1.0, 0.1, generator=g)
    h, delta = [torch.empty(T, H, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(2)]
    words = torch.zeros(T, dtype=torch.int32)
    words[::2] = ALLOW
    return P.NormedMoE(layer, weight), Lw, h, delta, words.cuda(), torch.tensor([0, T], dtype=torch.int32, device="cuda")


def fp8_of(Lw):
    out = []
    for w in (Lw.w13_pub, Lw.w2_pub, Lw.w13_priv, Lw.w2_priv):
        q, e = fp8(w, w.shape[2])
        out.append((q, torch.exp2(e.double()).float().view(w.shape[:2]).contiguous()))
    return tuple(q for q, _ in out) + tuple(s for _, s in out)


@pytest.mark.parametrize("T", [1, 19, 1000])
@pytest.mark.parametrize("score", [False, True])
def test_block_in_8_bits_is_its_operators(T, score):
    log(f"block {T} {score}")
    blk, Lw, h, delta, words, offs = block(T, score)
    w8 = fp8_of(Lw)
    audit = blk.layer.audit_buffers(T, 1)
    b = blk.forward_mx(h, delta, words, w8, audit, offs)
    torch.cuda.synchronize()
    res, out = b.residual.clone(), b.layer.out.clone()
    assert torch.equal(res, (h.double() + delta.double()).bfloat16())
    assert int(audit.violations) == 0 and int(audit.total) == 4 * int(b.layer.allow.sum())
    # against the bf16 experts on what the bytes stand for: h in 8 bits is 2^-4 off at most per value, and
    # a sum of many such errors of random sign stays below it (h alone differs: x and the weights are the same)
    deq = lambda q, s: (q.view(torch.float8_e4m3fn).double() * s.double().unsqueeze(2)).bfloat16()  # noqa: E731
    x8 = (b.norm_q.view(torch.float8_e4m3fn).double().unflatten(1, (-1, 32)) * torch.exp2(b.norm_scale.double() - 127).unsqueeze(2)).flatten(1).bfloat16()
    y = torch.empty_like(b.layer.y_perm)
    P.pmpe_expert_ffn(blk.layer.desc, T, None, x8, b.layer.expert_count, b.layer.expert_offset, b.layer.row_token,
                      *[deq(w8[i], w8[4 + i]) for i in range(4)], None, None, None, y, torch.zeros_like(audit.token_rows), None,
                      None, b.layer.ws)
    torch.cuda.synchronize()
    assert float((b.layer.y_perm.double() - y.double()).norm() / y.double().norm()) <= 2.0 ** -4
    # the same again, and replayed from a graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.forward_mx(h, delta, words, w8, audit, offs)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.layer.out, out) and torch.equal(b.residual, res)
        blk.forward_mx(h, delta, words, w8, audit, offs)
        torch.cuda.synchronize()
        assert torch.equal(b.layer.out, out)


def test_block_training_step():
    """Norm, scored route, experts, their backward, clipping and AdamW in a row."""
    T = 200
    blk, Lw, h, delta, words, offs = block(T, True)
    audit = blk.layer.audit_buffers(T, 1)
    b = blk.forward(h, delta, words, audit, offs, train=True)
    dres, dout = [torch.randn(T, 256, device="cuda").bfloat16() for _ in range(2)]
    dx, dw = torch.empty_like(h), torch.empty(256, device="cuda")
    g = blk.backward(dres, dout, b, dx, dweight=dw)
    torch.cuda.synchronize()
    r, dy, w = b.residual.double(), g.dx.double(), blk.weight.double()
    rstd = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + blk.eps)
    xh, gg = r * rstd, dy * w
    want = rstd * (gg - xh * (gg * xh).mean(1, keepdim=True)) + dres.double()
    size = rstd * (gg.abs() + xh.abs() * (gg * xh).abs().mean(1, keepdim=True)) + dres.double().abs()
    assert torch.all((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17 * size)
    assert torch.all((dw.double() - (dy * xh).sum(0)).abs() <= 2.0 ** -16 * (dy * xh).abs().sum(0))
    before = [p.clone() for p in (blk.layer.wr_priv, blk.layer.w13_priv, blk.layer.w2_priv)]
    opt = P.PrivateAdamW(blk.layer, lr=1e-2, max_norm=0.5)
    opt.step(g)
    torch.cuda.synchronize()
    total = sum(float(t.double().square().sum()) for t in (g.dwr_priv, g.dw13_priv, g.dw2_priv)) ** 0.5
    assert abs(float(opt.norm[0]) - total) <= 2.0 ** -23 * total
    assert all(not torch.equal(a, p) for a, p in zip(before, (blk.layer.wr_priv, blk.layer.w13_priv, blk.layer.w2_priv)))
    # without a residual's gradient, and with h alone as the stream
    h0 = h.clone()
    b = blk.forward(h, None, words, audit.zero_(), offs, train=True)
    g = blk.backward(None, dout, b, dx)
    b2 = blk.forward(h, delta, words, audit.zero_(), offs)
    torch.cuda.synchronize()
    assert torch.equal(h, h0) and b2.residual is not h
    h2 = h.clone()
    blk.forward(h2, None, words, audit.zero_(), offs)
    blk.forward(h, delta, words, audit.zero_(), offs)
    torch.cuda.synchronize()
    assert torch.equal(h2, h0)  # a stream handed in is never written
