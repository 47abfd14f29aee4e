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
