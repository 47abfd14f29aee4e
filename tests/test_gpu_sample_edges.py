"""Sampling where the bins' arithmetic changes and at the ends of parameters, against the definition in 64 bits."""
import pytest
import torch

from tests.decode_cases import gen, log
from tests.test_gpu_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [8192, 20011, 70001])
@pytest.mark.parametrize("t", [1.0, 0.01, 1e-4, 1e-5, 37.5])
def test_largest_logits_next_to_the_border_of_fp32_bins(V, t):
    """8 z / T of about -2^20: parts of a row lie on both sides of the border where bins are made in fp64."""
    log(f"border of fp32 bins V {V} t {t}")
    rows, at = [], torch.arange(V)
    for off in (-60.0, -3.0, -0.2, 0.2, 3.0, 20.0, 63.0):
        for step in (0.5, 5.0, 30.0, -0.5):  # the second half of the row below (above) the first
            x = -131072.0 + off + 3.0 * torch.randn(V, generator=gen(len(rows)), dtype=torch.float64) - step * (at >= V // 2)
            rows.append((x * t).float())
    two = torch.full((V,), -131071.5, dtype=torch.float64)
    two[V // 2:] = -131072.0
    rows.append((two * t).float())
    z = torch.stack(rows)
    B = len(rows)
    u = torch.rand(B, generator=gen(7)).tolist()
    u[-1] = 0.95
    for par in ({}, dict(top_k=[V // 3] * B), dict(top_p=[0.9] * B), dict(min_p=[0.02] * B), dict(top_k=[50] * B),
                dict(top_k=[V - 5] * B, top_p=[0.97] * B, min_p=[0.001] * B)):
        check(z, dict(par, temperature=[t] * B), u)
