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
