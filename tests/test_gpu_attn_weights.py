"""Attention whose weighted rows cancel: what is left shows how exactly each weight enters the second product."""
import math

import pytest
import torch

import paper_2608_06690_amd as P
from tests.decode_cases import Cache, gen, log, quantise, values

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def cancelling(R, kv, n, q8, seed):
    """A cache of n rows per request: scores in [-2, 0], values of each row what brings the weighted sum of the rows
    before it nearest to 0. Returns it with the exact weights [R, kv, n] and sums [R, kv, dim]."""
    c = Cache([n] * R, kv, 32, 16, BF16, q8, tags=False)
    s = -2.0 * torch.rand(R, kv, n, generator=gen(seed)).to(BF16).float()
    k = torch.zeros(R, kv, n, 32)
    k[..., 0] = s
    v = torch.zeros(R, kv, n, 32, dtype=torch.float64)
    if q8:
        kq, ke = quantise(k)
        s = values(kq, ke)[..., 0].float()
    w = torch.softmax(s.double(), dim=2)
    total = torch.zeros(R, kv, 32, dtype=torch.float64)
    first = 1.0 + torch.rand(R, kv, 32, generator=gen(seed + 1)).to(BF16).double()
    arrays = {}
    for j in range(n):
        x = first if j == 0 else -total / w[..., j:j + 1]
        if q8:
            q, e = quantise(x.float())
            arrays[j] = (q, e)
            x = values(q, e)
        else:
            x = x.float().to(BF16).double()
        v[..., j, :] = x
        total += w[..., j:j + 1] * x
    for r in range(R):
        p = int(c.table[r, 0])
        if q8:
            c.k[p, :, :n], c.ks[p, :, :, :n] = kq[r], ke[r].transpose(1, 2)
            for j, (q, e) in arrays.items():
                c.v[p, :, j], c.vs[p, :, :, j] = q[r], e[r]
        else:
            c.k[p, :, :n], c.v[p, :, :n] = k[r].to(BF16), v[r].to(BF16)
    return c, w, v, total


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("group", [1, 8, 9, 16, 24])
def test_weights_enter_as_fp32_values(q8, group):
    """The exponent of a weight is off by at most 4 roundings of |s log2 e| <= 3 (6 steps of 2^-24 after the factor
    ln 2 x 3), the exponential by 2 steps, a sum of n terms by 2 n: at most 32 steps of 2^-24 in all, of the sum of
    the magnitudes, and the output by half a step of bf16. Two bf16 parts of a weight would be off by 64 steps of it."""
    log(f"cancelling rows q8 {q8} group {group}")
    R, kv, n = 40, 3, 8 if q8 else 3
    c, w, v, total = cancelling(R, kv, n, q8, 3)
    q = torch.zeros(R, kv * group, 32, dtype=BF16)
    q[..., 0] = 1.0
    (table, _, _), cache = c.cuda()
    out = torch.empty_like(q, device="cuda")
    ws = torch.empty(max(16, P.pmpe_attn_decode_workspace_bytes(c.desc, R, kv * group)), dtype=torch.uint8, device="cuda")
    P.pmpe_attn_decode(c.desc, q.cuda(), None, torch.full((R,), n, dtype=torch.int32).cuda(), table, None, None, *cache, 1.0, out,
                       None, None, ws)
    got = out.cpu().double().view(R, kv, group, 32)
    spread = (w.unsqueeze(-1) * v.abs()).sum(dim=2)
    tol = (32 * 2.0 ** -24 * spread + 2.0 ** -9 * total.abs() * 1.01).unsqueeze(2)
    ratio = float(((got - total.unsqueeze(2)).abs() / tol).max())
    log(f"  largest error over its bound {ratio:.3f}")
    assert ratio <= 1.0 and math.isfinite(ratio)
