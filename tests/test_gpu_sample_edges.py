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


# (largest logit, temperature, min_p) with top + T ln(min_p) between -1e-10 and 0, 5e-11 of the two terms or less
CANCEL = [(1.2379502058029175, 2.248124122619629, 0.5765696167945862), (1.7185120582580566, 1.4391342401504517, 0.30296769738197327),
          (2.1257972717285156, 0.9267536997795105, 0.10088133066892624), (2.1620967388153076, 1.1297087669372559, 0.14751090109348297)]


def test_least_mass_next_to_a_logit_of_zero():
    """The smallest logit that min-p leaves lies many numbers of fp32 below where the logarithm puts it."""
    log("least mass at a logit of zero")
    z = torch.full((len(CANCEL), 300), -1.0)
    z[:, 5] = torch.tensor([c[0] for c in CANCEL])
    z[:, 7:107] = -torch.linspace(1.3e-10, 5.5e-10, 100)  # below the least mass by 2^-33 to 2^-30 of it
    z[:, 200] = 0.0
    par = dict(temperature=[c[1] for c in CANCEL], min_p=[c[2] for c in CANCEL])
    _, _, kept = check(z, par, [0.1, 0.99, 0.5, 0.9])
    assert kept.tolist() == [2] * 4


@pytest.mark.parametrize("t", [100793200.0, 105422080.0, 118912304.0, 1e8, 1e30])
def test_bins_that_meet_at_zero(t):
    """8 z / T of logits next to 0 is 0 in fp32: a bin's edge lies many numbers below it."""
    log(f"bins that meet at zero t {t}")
    B, V = 8, 9000
    z = torch.empty(B, V)
    z[:, :100] = torch.rand(B, 100, generator=gen(1))
    z[:, 100:8000] = -torch.logspace(-39, -37, 7900)
    z[:, 8000:] = -1.0 - torch.rand(B, 1000, generator=gen(2))
    u = [0.0, 0.01, 0.02, 0.3, 0.5, 0.8, 0.95, 1.0 - 2.0 ** -24]
    for par in ({}, dict(top_k=[6000] * B), dict(top_p=[0.6] * B), dict(top_k=[60] * B), dict(min_p=[0.9999999] * B)):
        check(z, dict(par, temperature=[t] * B), u)


@pytest.mark.parametrize("V", [300, 8193, 20011, 70001])
def test_uniform_numbers_of_one_and_more_take_the_last_token(V):
    """The last token before the cut, also where its mass is less than e^-64 of the largest's."""
    log(f"u of one and more V {V}")
    rows = [torch.linspace(-300, 300, V), torch.linspace(40, -60, V), torch.randn(V, generator=gen(1)),
            torch.cat([torch.tensor([80.0]), torch.randn(V - 1, generator=gen(2))]), torch.randn(V, generator=gen(3)) * 100,
            torch.randn(V, generator=gen(4)) * 3e37, torch.cat([torch.tensor([200.0]), torch.full((V - 1,), -1.0)]),
            torch.where(torch.arange(V) % 3 == 0, float("-inf"), torch.linspace(0, -500, V))]
    for u in (1.0, 2.0, float("inf"), 1.0 - 2.0 ** -24):
        for dt in (torch.float32, torch.bfloat16):
            z = torch.stack(rows).to(dt)
            for par in ({}, dict(top_k=[V - 30] * 8), dict(min_p=[1e-35] * 8), dict(top_p=[0.9] * 8), dict(top_k=[5] * 8),
                        dict(temperature=[0.3] * 8, top_k=[V // 2] * 8, min_p=[1e-38] * 8)):
                check(z, par, [u] * 8)


@pytest.mark.parametrize("V", [8192, 30011])
@pytest.mark.parametrize("top", [131072.0, -131200.0, 5e5, -5e5, 1e7])
def test_rows_of_several_pieces_at_and_beyond_the_border(V, top):
    log(f"several pieces V {V} top {top}")
    rows, at = [], torch.arange(V)
    for off in (-70.0, -1.0, 0.0, 1.0, 60.0):
        for step in (0.5, 40.0, -40.0, 500.0):
            rows.append((top + off + 4.0 * torch.randn(V, generator=gen(len(rows))) - step * (at >= V // 2)).float())
    z = torch.stack(rows)
    B = len(rows)
    u = torch.rand(B, generator=gen(8)).tolist()
    for par in ({}, dict(top_k=[V // 2] * B), dict(top_p=[0.9] * B), dict(min_p=[0.02] * B), dict(top_k=[50] * B, top_p=[0.5] * B)):
        check(z, par, u)
        check(z * 0.001, dict(par, temperature=[0.001] * B), u)
