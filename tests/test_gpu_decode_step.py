"""A decoding step as a program makes it: projections, the cache written, attention over it, a block of norm and
policy-masked layer, logits, a token drawn; against plain forms of the cache, the attention and the draw."""
import math

import numpy as np
import pytest
import torch

import paper_2608_06690_amd as P
import workloads as W
from tests import decode_cases as D
from tests import pmpe_cases as C
from tests.decode_cases import log, quantise, randn, values
from tests.test_gpu_sample import choices

pytestmark = pytest.mark.gpu
REV, FP = bytes(32), bytes(range(32))
ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)
H, HEADS, KV, DIM, VOCAB = 256, 8, 2, 64, 1003


def model(R):
    cfg = W.scaled_config(W.get_config("qwen"), tokens=R, requests=R, hidden=H, inter=128, n_pub=16, n_priv=8, top_k=4)
    layer, _ = C.device_layer(cfg)
    blk = P.NormedMoE(layer, torch.ones(H, device="cuda"))
    w = [randn(s, i, 0.05, torch.bfloat16).cuda() for i, s in enumerate(((H, (HEADS + 2 * KV) * DIM), (HEADS * DIM, H), (H, VOCAB)))]
    return blk, w


class Rows:
    """What the cache should hold, on the host in 64 bits."""

    def __init__(self, R, fp8):
        self.k, self.v, self.fp8 = [[] for _ in range(R)], [[] for _ in range(R)], fp8

    def add(self, r, k, v):
        for to, x in ((self.k, k), (self.v, v)):
            to[r] += list(values(*quantise(x.float())) if self.fp8 else x.double())

    def attend(self, q, scale):
        class Fake:
            kv = KV
            rows = lambda _, n, r, a, b: torch.stack(getattr(self, n)[r][a:b]) if getattr(self, n)[r] else torch.zeros(0, KV, DIM)  # noqa: E731
        return D.attend(Fake(), q, None, [len(x) for x in self.k], scale)


@pytest.mark.parametrize("fp8", [False, True])
def test_steps(fp8):
    log(f"decoding steps fp8 {fp8}")
    R, scale = 5, DIM ** -0.5
    blk, (wqkv, wo, wv) = model(R)
    cache = P.PagedCache(R, 64, 16, KV, DIM, 12, REV, FP, fp8=fp8)
    metas = [{"allow_private": True}, None, {"allow_private": False}, {"allow_private": True}, {"allow_private": 1}]
    for r, m in enumerate(metas):
        cache.open(r, m)
    words = torch.tensor([P.policy_word(m) for m in metas], dtype=torch.int64).to(torch.int32).cuda()
    assert torch.equal(words, cache.words)
    mine = Rows(R, fp8)
    sample = P.Sampler(R, VOCAB, torch.tensor([0.0, 0.8, 1.0, 0.7, 1.2]).cuda(), torch.tensor([0, 40, 0, 0, 7], dtype=torch.int32).cuda(),
                       torch.tensor([1.0, 0.9, 0.8, 1.0, 1.0]).cuda(), torch.tensor([0.0, 0.0, 0.0, 0.1, 0.0]).cuda())
    audit, offs = blk.layer.audit_buffers(R, R), torch.arange(R + 1, dtype=torch.int32, device="cuda")

    def put(x, counts):
        qkv = (x @ wqkv).view(x.shape[0], HEADS + 2 * KV, DIM)
        k, v = qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        cache.write(k, v, counts)
        at = 0
        for r, n in enumerate(counts):
            mine.add(r, k[at:at + n].cpu(), v[at:at + n].cpu())
            at += n
        return qkv[:, :HEADS]

    prompts = [20, 1, 47, 16, 33]
    put(randn((sum(prompts), H), 1, 1.0, torch.bfloat16).cuda(), prompts)
    h = randn((R, H), 2, 1.0, torch.bfloat16).cuda()
    for step in range(4):
        q = put(h, [1] * R)
        out = cache.attend(q, scale)
        want, _, spread, most = mine.attend(q.cpu(), scale)
        n = max(len(x) for x in mine.k)
        assert bool(((out.cpu().double() - want).abs() <= D.tolerance(torch.bfloat16, DIM, n, spread, most, want)).all())
        delta = out.view(R, HEADS * DIM) @ wo
        b = blk.forward(h, delta, words, audit.zero_(), offs)
        h = (b.residual + b.layer.out).clone()
        logits = h @ wv
        u = torch.rand(R, generator=D.gen(step))
        token = sample(logits, u.cuda()).cpu()
        par = [t.cpu().numpy() for t in (sample.temperature, sample.top_k, sample.top_p, sample.min_p)]
        for r in range(R):
            fits = choices(logits[r].float().cpu().numpy(), float(par[0][r]), int(par[1][r]), float(par[2][r]), float(par[3][r]), float(np.float32(u[r])))
            assert any((int(token[r]), int(sample.kept[r])) == (x[0], x[2]) for x in fits)
        assert int(audit.violations) == 0
    assert int(cache.dev_status) == 0 and cache.seq_len.tolist() == [p + 4 for p in prompts] == cache.lengths
    # what went in comes back
    counts, first = [3, 1, 50, 0, 17], [5, 4, 1, 0, 20]
    k, v = cache.read(counts, first)
    at = 0
    for r, n in enumerate(counts):
        for got, rows in ((k, mine.k), (v, mine.v)):
            if n:
                assert torch.equal(got[at:at + n].cpu().double(), torch.stack(rows[r][first[r]:first[r] + n]).to(torch.bfloat16).double())
        at += n


def test_a_request_that_goes_on_from_anothers_pages():
    log("shared pages")
    cache = P.PagedCache(3, 32, 16, KV, DIM, 8, REV, FP)
    for r, m in enumerate(({"allow_private": True}, {"allow_private": True}, None)):
        cache.open(r, m)
    k, v = randn((60, KV, DIM), 1, 1.0, torch.bfloat16).cuda(), randn((60, KV, DIM), 2, 1.0, torch.bfloat16).cuda()
    cache.write(k[:40], v[:40], [40, 0, 0])
    assert cache.share(1, 0, 40) == 32
    with pytest.raises(P.PmpeError):
        cache.share(2, 0, 40)
    cache.write(k[40:], v[40:], [5, 10, 5])
    q = randn((3, HEADS, DIM), 3, 1.0, torch.bfloat16)
    got = cache.attend(q.cuda(), 0.125).cpu().double()
    mine = Rows(3, False)
    kc, vc = k.cpu(), v.cpu()
    mine.add(0, torch.cat([kc[:40], kc[40:45]]), torch.cat([vc[:40], vc[40:45]]))
    mine.add(1, torch.cat([kc[:32], kc[45:55]]), torch.cat([vc[:32], vc[45:55]]))
    mine.add(2, kc[55:], vc[55:])
    want, _, spread, most = mine.attend(q, 0.125)
    tol = D.tolerance(torch.bfloat16, DIM, 45, spread, most, want)
    assert bool(((got - want).abs() <= tol).all()) and int(cache.dev_status) == 0
    # a table that names the other decision's pages after all: the kernels refuse them
    cache.block_table[2, :2] = cache.block_table[0, :2]
    cache.seq_len[2] = 32
    out = cache.attend(q.cuda(), 0.125)
    assert float(out[2].abs().max()) == 0 and int(cache.dev_status) == P.PMPE_DEV_CACHE_REFUSED


def test_a_step_on_another_stream():
    log("another stream")
    s = torch.cuda.Stream()
    outs = []
    for stream in (None, s):
        cache = P.PagedCache(2, 16, 16, KV, DIM, 4, REV, FP, fp8=True)
        for r in range(2):
            cache.open(r, None)
        k, v = (randn((30, KV, DIM), i, 1.0, torch.bfloat16).cuda() for i in (1, 2))
        q = randn((2, HEADS, DIM), 3, 1.0, torch.bfloat16).cuda()
        s.wait_stream(torch.cuda.current_stream())
        cache.write(k[:28], v[:28], [11, 17], stream=stream)
        cache.write(k[28:], v[28:], [1, 1], stream=stream)
        out = torch.empty_like(q)
        cache.attend(q, 0.125, out=out, stream=stream)
        torch.cuda.synchronize()
        outs.append(out.clone())
    assert torch.equal(*outs)


def test_new_output_belongs_to_the_stream_that_writes_it(monkeypatch):
    # (memory of another stream may be given away while the call still writes it)
    log("output on another stream")
    s = torch.cuda.Stream()
    cache = P.PagedCache(2, 16, 16, KV, DIM, 4, REV, FP)
    for r in range(2):
        cache.open(r, None)
    k, v = (randn((30, KV, DIM), i, 1.0, torch.bfloat16).cuda() for i in (1, 2))
    q = randn((2, HEADS, DIM), 3, 1.0, torch.bfloat16).cuda()
    cache.write(k, v, [12, 18])
    want = cache.attend(q, 0.125)
    torch.cuda.synchronize()
    made, empty = [], torch.empty

    def spy(*args, **kw):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    cache._ws.clear()
    monkeypatch.setattr(torch, "empty", spy)
    got = cache.attend(q, 0.125, stream=s)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert made == [s.cuda_stream] * 2 and torch.equal(got, want)


def test_captured_step():
    log("captured step")
    R = 3
    cache = P.PagedCache(R, 32, 16, KV, DIM, 8, REV, FP, fp8=True)
    for r in range(R):
        cache.open(r, {"allow_private": r == 1})
    k, v = (randn((60, KV, DIM), i, 1.0, torch.bfloat16).cuda() for i in (1, 2))
    cache.write(k[:45], v[:45], [20, 15, 10])
    cache._reserve([5] * R)  # the pages of the steps to come
    qkv = torch.empty(R, HEADS + 2 * KV, DIM, dtype=torch.bfloat16, device="cuda")
    logits, u = torch.empty(R, VOCAB, device="cuda"), torch.empty(R, device="cuda")
    out = torch.empty(R, HEADS, DIM, dtype=torch.bfloat16, device="cuda")
    off = torch.arange(R + 1, dtype=torch.int32, device="cuda")
    sample = P.Sampler(R, VOCAB, top_p=torch.full((R,), 0.9, device="cuda"))
    w = randn((HEADS * DIM, VOCAB), 9, 0.3, torch.bfloat16).cuda()

    def step():
        cache.write(qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:], [1] * R, off)
        cache.attend(qkv[:, :HEADS], 0.125, out=out)
        torch.mm(out.view(R, -1), w, out=mm)
        logits.copy_(mm)
        sample(logits, u)
    mm = torch.empty(R, VOCAB, dtype=torch.bfloat16, device="cuda")
    qkv.copy_(randn(qkv.shape, 50, 1.0, torch.bfloat16))
    u.fill_(0.5)
    # one eager step on a copy's books: the same rows are written again by the first replay
    step()
    cache.seq_len.sub_(1)
    cache.lengths = [n - 1 for n in cache.lengths]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    cache.lengths = [n - 1 for n in cache.lengths]
    mine = Rows(R, True)
    at = 0
    for r, n in enumerate((20, 15, 10)):
        mine.add(r, k[at:at + n].cpu(), v[at:at + n].cpu())
        at += n
    for i in range(4):
        qkv.copy_(randn(qkv.shape, 60 + i, 1.0, torch.bfloat16))
        u.copy_(torch.rand(R, generator=D.gen(i)))
        g.replay()
        torch.cuda.synchronize()
        x = qkv.cpu()
        for r in range(R):
            mine.add(r, x[r:r + 1, HEADS:HEADS + KV], x[r:r + 1, HEADS + KV:])
        want, _, spread, most = mine.attend(x[:, :HEADS], 0.125)
        assert bool(((out.cpu().double() - want).abs() <= D.tolerance(torch.bfloat16, DIM, 30, spread, most, want)).all())
        for r in range(R):
            fits = choices(logits[r].cpu().numpy(), 1.0, 0, float(np.float32(0.9)), 0.0, float(u[r]))
            assert any((int(sample.token[r]), int(sample.kept[r])) == (c[0], c[2]) for c in fits)
    assert int(cache.dev_status) == 0 and cache.seq_len.tolist() == [24, 19, 14]
    assert math.isfinite(float(sample.prob.sum()))
