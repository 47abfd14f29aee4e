"""Paged caches for the tests of a decoding step's operators, and their plain forms in 64 bits."""
import math

import torch

import paper_2608_06690_amd as P

ALLOW = P.PMPE_POLICY_ALLOW - (1 << 32)


def log(msg):
    print(msg, flush=True)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(shape, seed, std=1.0, dt=torch.float32):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float32) * std).to(dt)


def quantise(x):
    """e4m3 bytes and biased exponents of blocks of 32 of the last dimension; x fp32."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(dim=-1)
    fine = torch.isfinite(b).all(dim=-1)
    m, e = torch.frexp(torch.where(fine & (amax > 0), amax, 1.0))
    e = torch.where(fine & (amax > 0), e - 9 + (m > 0.875).int(), 0).clamp(min=-126)
    v = torch.ldexp(b.double(), -e.unsqueeze(-1)).float()
    q = torch.where(fine.unsqueeze(-1), v, 0.0).to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.where(fine.unsqueeze(-1), q, torch.tensor(0x7F, dtype=torch.uint8))
    return q.flatten(-2), (e + 127).to(torch.uint8)


def values(q, s):
    """What e4m3 bytes [.., dim] and exponents [.., dim / 32] stand for, in 64 bits."""
    v = q.view(torch.float8_e4m3fn).double().unflatten(-1, (-1, 32))
    f = torch.where(s == 255, math.nan, torch.exp2(s.double() - 127.0))
    return (v * f.unsqueeze(-1)).flatten(-2)


class Cache:
    """A pool of pages, host copies of its arrays, and block tables of `rows` rows per request."""

    def __init__(self, rows, kv=2, dim=64, page=16, dt=torch.bfloat16, q8=False, tags=True, spare=3, extra_cols=1, seed=0, std=1.0):
        self.kv, self.dim, self.page, self.dt, self.q8, self.R = kv, dim, page, dt, q8, len(rows)
        need = [-(-max(n, 0) // page) for n in rows]
        self.n_pages, self.cols = sum(need) + spare, max(need + [0]) + extra_cols
        order = torch.randperm(self.n_pages, generator=gen(seed + 1)).int()
        self.words = torch.zeros(self.R, dtype=torch.int32)
        self.words[::2] = ALLOW
        self.words[3::4] = 77  # malformed: denies
        self.tag = torch.full((self.n_pages,), -1, dtype=torch.int32)
        # entries past a request's rows are never read: they name no page
        self.table = torch.full((self.R, self.cols), -5, dtype=torch.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = order[at:at + n]
            self.tag[order[at:at + n].long()] = ALLOW if self.words[r] == ALLOW else 0
            at += n
        if not tags:
            self.tag = self.words = None
        shape = (self.n_pages, kv, page, dim)
        self.k, self.v, self.ks, self.vs = [None] * 4
        for name, s in (("k", seed + 2), ("v", seed + 3)):
            x = randn(shape, s, std, dt)
            if q8:
                x, e = quantise(x.float())
                setattr(self, name + "s", e.transpose(2, 3).contiguous())
            setattr(self, name, x)
        self.desc = P.make_cache_desc(self.n_pages, page, kv, dim, self.cols, bf16=dt == torch.bfloat16, fp8=q8)

    def cuda(self):
        """Device copies: (table, tag, words), (k, v, ks, vs)."""
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        return tuple(map(dev, (self.table, self.tag, self.words))), tuple(map(dev, (self.k, self.v, self.ks, self.vs)))

    def usable(self, r, pos):
        """Page of a position that the request may use, else None."""
        if pos < 0 or pos >= self.cols * self.page:
            return None
        p = int(self.table[r, pos // self.page])
        if p < 0 or p >= self.n_pages:
            return None
        if self.tag is not None:
            want = ALLOW if self.words is not None and int(self.words[r]) == ALLOW else 0
            if int(self.tag[p]) != want:
                return None
        return p

    def row(self, name, p, i):
        """Row i of page p in 64 bits: [kv, dim]."""
        x = getattr(self, name)[p, :, i]
        return values(x, getattr(self, name + "s")[p, :, :, i]) if self.q8 else x.double()

    def rows(self, name, r, first, end):
        """Usable rows [n, kv, dim] of positions first .. end - 1 of request r, in 64 bits."""
        at = [(self.usable(r, p), p % self.page) for p in range(max(first, 0), end)]
        at = [(p, i) for p, i in at if p is not None]
        if not at:
            return torch.zeros(0, self.kv, self.dim, dtype=torch.float64)
        p, i = torch.tensor([a[0] for a in at]), torch.tensor([a[1] for a in at])
        x = getattr(self, name)[p, :, i]
        return values(x, getattr(self, name + "s")[p, :, :, i]) if self.q8 else x.double()


def attend(c, q, first, lens, scale):
    """Outputs, lse and, for tolerances, sum of p |v| and the largest scale sum |q k|, in 64 bits."""
    R, heads, dim = q.shape
    g = heads // c.kv
    out, lse = torch.zeros(R, heads, dim, dtype=torch.float64), torch.full((R, heads), -math.inf, dtype=torch.float64)
    spread, most = torch.zeros_like(out), torch.zeros(R, heads, dtype=torch.float64)
    for r in range(R):
        k, v = (c.rows(n, r, first[r] if first is not None else 0, lens[r]) for n in ("k", "v"))
        if len(k) == 0:
            continue
        k, v = k.repeat_interleave(g, dim=1), v.repeat_interleave(g, dim=1)
        x = q[r].double()
        s = torch.einsum("hd,nhd->hn", x, k) * scale
        w = torch.softmax(s, dim=1)
        out[r] = torch.einsum("hn,nhd->hd", w, v)
        spread[r] = torch.einsum("hn,nhd->hd", w, v.abs())
        lse[r] = torch.logsumexp(s, dim=1)
        most[r] = (torch.einsum("hd,nhd->hn", x.abs(), k.abs()) * abs(scale)).amax(dim=1)
    return out, lse, spread, most


def tolerance(dt, dim, n, spread, most, out):
    """Bound of |kernel - exact|. A score is a sum of dim fp32 products: off by (dim + 2) 2^-24 of the sum of
    their magnitudes, and so, in all, is the logarithm of a weight; the exponential, the factors of later maxima (one per
    tile at most) and the sums of n terms add (n + 64) 2^-24. bf16: a weight is stored as two bf16 values, off by
    2^-16 of it, and the output rounded once, by 2^-8 of it."""
    w = 2 * ((dim + 2) * 2.0 ** -24 * most.unsqueeze(-1) + (n + 64) * 2.0 ** -24)
    if dt == torch.bfloat16:
        return (w + 2.0 ** -16) * spread * 1.01 + 2.0 ** -8 * out.abs() * 1.01 + 1e-30
    return w * spread * 1.01 + 2.0 ** -23 * out.abs() + 1e-30


def lse_tolerance(dim, n, most, lse):
    return (dim + 2) * 2.0 ** -24 * most + (n + 64) * 2.0 ** -24 + 4 * 2.0 ** -24 * torch.where(torch.isfinite(lse), lse.abs(), 0.0)
