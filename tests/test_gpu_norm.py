"""Residual add and RMS norm on the GPU against 64-bit arithmetic: every type, rows from one
value to the longest, odd lengths, the 8-bit output with its block scales, values that are not
finite, aliased outputs, streams, and the backward against the formula and against differences.

Tolerances, relative to the exact value of the rounded r: the sum of squares of at most 64
fp32 terms per lane and eight tree levels is off by at most 72 * 2^-24, so rstd by 36 * 2^-24,
and y by that and three more roundings: 2^-18 covers it. An output in bf16 is off by half a step
(2^-8) more, one in e4m3 by 2^-4 (or half a step of 2^-9 below the normal range)."""
import pytest
import torch

import paper_2608_06690_amd as P

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -18


def log(msg):
    print(msg, flush=True)


def make(T, H, dt, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(T, H, dtype=dt, device="cuda").normal_(0.0, std, generator=g)


def norm64(r, w, eps):
    r = r.double()
    rstd = 1.0 / torch.sqrt((r * r).mean(dim=1, keepdim=True) + eps)
    return r * rstd * w.double(), rstd.squeeze(1)


def check_q8(q, s, y):
    """8-bit values and scales of y (fp64), whose blocks are finite."""
    v = q.view(torch.float8_e4m3fn).double().unflatten(1, (-1, 32))
    scale = torch.exp2(s.double() - 127.0).unsqueeze(2)
    y = y.unflatten(1, (-1, 32))
    amax = y.abs().amax(dim=2, keepdim=True)
    zero = amax == 0
    assert torch.all(scale[zero] == 1.0)
    assert torch.all((amax <= 448.0 * scale * (1 + F32)) | zero)
    assert torch.all((amax > 224.0 * scale * (1 - F32)) | zero | (s.unsqueeze(2) == 1))
    off = (v * scale - y).abs()
    assert torch.all(off <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * scale) * (1 + F32) + F32 * y.abs())


SIZES = [(1, 1), (3, 7), (5, 31), (1, 32), (130, 96), (7, 513), (1111, 1601), (2049, 1000), (2051, 2048), (9, 2047), (3, 4100),
         (5, 8191), (2, 12345), (3, 16384), (8, 2048)]


@pytest.mark.parametrize("T,H", SIZES)
@pytest.mark.parametrize("dt,wdt", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                    (torch.float32, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("res", [False, True])
def test_forward(T, H, dt, wdt, res):
    log(f"norm {T}x{H} {dt} {wdt} {res}")
    x, residual = make(T, H, dt, 1), make(T, H, dt, 2, 3.0) if res else None
    w = (make(1, H, wdt, 3)[0] * 0.1 + 1.0).to(wdt)
    total = torch.empty_like(x) if res else None
    out = torch.empty_like(x)
    q8 = H % 32 == 0
    q = torch.empty(T, H, dtype=torch.uint8, device="cuda") if q8 else None
    s = torch.empty(T, H // 32, dtype=torch.uint8, device="cuda") if q8 else None
    rstd = torch.empty(T, dtype=torch.float32, device="cuda")
    P.pmpe_rmsnorm(x, residual, w, 1e-6, total, out, q, s, rstd)
    r = x
    if res:
        r = (x.double() + residual.double()).to(dt)
        assert torch.equal(total, r)  # the sum is rounded once
    y, rs = norm64(r, w, 1e-6)
    step = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24
    assert torch.all((out.double() - y).abs() <= (step + F32) * y.abs())
    assert torch.all((rstd.double() - rs).abs() <= F32 * rs)
    if q8:
        check_q8(q, s, y)
        # the 8-bit output alone is the same
        q2, s2 = torch.empty_like(q), torch.empty_like(s)
        P.pmpe_rmsnorm(x, residual, w, 1e-6, total, None, q2, s2, None)
        assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("T,H", [(3, 64), (2050, 64)])
def test_blocks_that_are_empty_or_not_finite(T, H):
    log(f"norm special {T}x{H}")
    x = make(T, H, torch.float32, 4)
    x[0, :32] = 0.0
    x[1] = 0.0
    w = torch.ones(H, device="cuda")
    w[40] = float("nan")
    q, s = torch.empty(T, H, dtype=torch.uint8, device="cuda"), torch.empty(T, H // 32, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    P.pmpe_rmsnorm(x, None, w, 1e-6, None, out, q, s, None)
    assert torch.all(q[0, :32] == 0) and s[0, 0] == 127
    assert torch.all(q[:, 32:] & 0x7F == 0x7F) and torch.all(s[:, 1] == 127)  # the NaN poisons its block alone
    assert torch.all(out[1, :40] == 0) and torch.all(out[:, 40].isnan())
    x[2, 3] = float("inf")
    P.pmpe_rmsnorm(x, None, torch.ones(H, device="cuda"), 1e-6, None, out, q, s, None)
    assert out[2, 3].isnan() and torch.all(out[2, 32:] == 0)  # inf / inf, and finite values over inf
    assert torch.all(q[2, :32] & 0x7F == 0x7F) and torch.all(q[2, 32:] & 0x7F == 0) and torch.all(s[2] == 127)
    # a tiny block: the scale stops at 2^-126
    P.pmpe_rmsnorm(make(T, H, torch.float32, 5), None, torch.full((H,), 1e-38, device="cuda"), 0.0, None, out, q, s, None)
    assert torch.all(s == 1)


def test_aliases_and_streams():
    T, H = 300, 384
    x, res, w = make(T, H, torch.bfloat16, 6), make(T, H, torch.bfloat16, 7), torch.ones(H, device="cuda")
    total, out = torch.empty_like(x), torch.empty_like(x)
    P.pmpe_rmsnorm(x, res, w, 1e-5, total, out, None, None, None)
    res2, out2 = res.clone(), torch.empty_like(x)
    P.pmpe_rmsnorm(x, res2, w, 1e-5, res2, out2, None, None, None)  # the residual stream in place
    assert torch.equal(res2, total) and torch.equal(out2, out)
    x2 = x.clone()
    P.pmpe_rmsnorm(x2, None, w, 1e-5, None, x2, None, None, None)
    P.pmpe_rmsnorm(x, None, w, 1e-5, None, out2, None, None, None)
    assert torch.equal(x2, out2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        out3 = torch.empty_like(x)
        P.pmpe_rmsnorm(x, res, w, 1e-5, total, out3, None, None, None)
    torch.cuda.synchronize()
    assert torch.equal(out3, out)
    # more than one batch behind the other keep their rows apart (rows past T stay as they were)
    big = torch.full((T + 2, H), 7.0, dtype=torch.bfloat16, device="cuda")
    P.pmpe_rmsnorm(x, None, w, 1e-5, None, big[1:T + 1], None, None, None)
    assert torch.all(big[0] == 7.0) and torch.all(big[T + 1] == 7.0) and torch.equal(big[1:T + 1], out2)


def backward64(dy, dres, r, w, rstd):
    r, g, rstd = r.double(), dy.double() * w.double(), rstd.double().unsqueeze(1)
    xh = r * rstd
    gx = g * xh
    dx = rstd * (g - xh * gx.mean(dim=1, keepdim=True))
    size = rstd * (g.abs() + xh.abs() * gx.abs().mean(dim=1, keepdim=True))
    if dres is not None:
        dx, size = dx + dres.double(), size + dres.double().abs()
    t = dy.double() * xh
    return dx, size, t.sum(dim=0), t.abs().sum(dim=0)


@pytest.mark.parametrize("T,H", SIZES + [(5000, 96), (700, 16384)])
@pytest.mark.parametrize("dt,dyt", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                    (torch.float32, torch.float32)])
@pytest.mark.parametrize("res", [False, True])
def test_backward(T, H, dt, dyt, res):
    log(f"norm backward {T}x{H} {dt} {dyt} {res}")
    r, dy, dres = make(T, H, dt, 11, 2.0), make(T, H, dyt, 12), make(T, H, dt, 13) if res else None
    w = make(1, H, torch.float32, 14)[0] + 1.0
    rstd = norm64(r, w, 1e-6)[1].float()
    dx, dw = torch.empty_like(r), torch.empty(H, device="cuda")
    ws = torch.empty(P.pmpe_rmsnorm_backward_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    P.pmpe_rmsnorm_backward(dy, dres, r, w, rstd, dx, dw, ws)
    ex, size, ew, wsize = backward64(dy, dres, r, w, rstd)
    step = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -24
    assert torch.all((dx.double() - ex).abs() <= step * ex.abs() + (1 + step) * F32 * size)
    # a chain of at most T / 512 + 100 fp32 additions
    assert torch.all((dw.double() - ew).abs() <= (T / 256 + 100) * 2.0 ** -24 * wsize)
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    P.pmpe_rmsnorm_backward(dy, dres, r, w, rstd, dx2, dw2, ws)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    P.pmpe_rmsnorm_backward(dy, dres, r, w, rstd, dx2.zero_(), None, None)  # a frozen norm
    assert torch.equal(dx, dx2)
    if res:  # in place of the residual stream's gradient
        P.pmpe_rmsnorm_backward(dy, dres, r, w, rstd, dres, None, None)
        assert torch.equal(dx, dres)


def test_backward_against_differences():
    """d/dh of sum(dy * y) along a direction, by central differences of the forward in fp32."""
    T, H = 4, 192
    x, d, dy = make(T, H, torch.float32, 21), make(T, H, torch.float32, 22), make(T, H, torch.float32, 23)
    w = make(1, H, torch.float32, 24)[0] + 1.0
    dx, dw, rstd = torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(T, device="cuda")
    out = torch.empty_like(x)

    def value(xx, ww):
        P.pmpe_rmsnorm(xx, None, ww, 1e-6, None, out, None, None, rstd)
        return float((out.double() * dy.double()).sum())

    value(x, w)
    ws = torch.empty(P.pmpe_rmsnorm_backward_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    P.pmpe_rmsnorm_backward(dy, None, x, w, rstd, dx, dw, ws)
    h = 2.0 ** -6
    got = (value(x + h * d, w) - value(x - h * d, w)) / (2 * h)
    want = float((dx.double() * d.double()).sum())
    # third derivative times h^2 / 6 (values of order 1 over T * H terms), and the roundings of two sums
    # of |out dy| at 2^-20 each over 2 h
    size = float((dy.double().abs() * (w.double().abs())).sum())
    assert abs(got - want) <= 4 * size * h * h + size * 2.0 ** -20 / h
    e = make(1, H, torch.float32, 25)[0]
    got = (value(x, w + h * e) - value(x, w - h * e)) / (2 * h)
    assert abs(got - float((dw.double() * e.double()).sum())) <= size * 2.0 ** -18 / h  # linear in w


def test_rows_beyond_2_31_elements():
    """The last rows of a batch whose offsets pass 32 bits: the bits that the rows alone give."""
    T, H, n = 131080, 16384, 3
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.empty(T, H, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
    w = torch.empty(H, device="cuda").normal_(1.0, 0.1, generator=g)

    def forward(x, out):
        q = torch.zeros(x.shape, dtype=torch.uint8, device="cuda")
        s = torch.zeros(x.shape[0], H // 32, dtype=torch.uint8, device="cuda")
        rstd = torch.zeros(x.shape[0], device="cuda")
        P.pmpe_rmsnorm(x, None, w, 1e-6, None, out, q, s, rstd)
        return q, s, rstd

    last = x[-n:].clone()
    y = torch.empty_like(last)
    q, s, rstd = forward(last, y)
    dx = torch.empty_like(last)
    P.pmpe_rmsnorm_backward(y, None, last, w, rstd, dx, None, None)
    out = torch.empty_like(x)
    all_q, all_s, all_rstd = forward(x, out)
    assert torch.equal(out[-n:], y) and torch.equal(all_q[-n:], q) and torch.equal(all_s[-n:], s)
    assert torch.equal(all_rstd[-n:], rstd)
    P.pmpe_rmsnorm_backward(out, None, x, w, all_rstd, out, None, None)
    assert torch.equal(out[-n:], dx)


def test_empty_batch_and_graph():
    w, dw = torch.ones(64, device="cuda"), torch.full((64,), 3.0, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    P.pmpe_rmsnorm(e, None, w, 1e-6, None, e, None, None, None)
    P.pmpe_rmsnorm_backward(e, None, e, w, torch.empty(0, device="cuda"), e, dw, None)
    assert torch.all(dw == 0)
    T, H = 33, 640
    x, dy = make(T, H, torch.bfloat16, 31), make(T, H, torch.float32, 32)
    w = torch.ones(H, device="cuda")
    out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(H, device="cuda")
    rstd = torch.empty(T, device="cuda")
    ws = torch.empty(P.pmpe_rmsnorm_backward_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")

    def both():
        P.pmpe_rmsnorm(x, None, w, 1e-6, None, out, None, None, rstd)
        P.pmpe_rmsnorm_backward(dy, None, x, w, rstd, dx, dw, ws)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (41, 42, 43):
        x.copy_(make(T, H, torch.bfloat16, seed))
        graph.replay()
        got = [t.clone() for t in (out, dx, dw)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, dx, dw)))
