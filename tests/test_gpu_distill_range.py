"""Lists whose logits are as large as FP32 holds, and the ends of the range of temperatures."""
import pytest
import torch

import paper_2508_21230_amd as pkg
from tests.test_gpu_distill_offsets import check_both, definition, lists

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


@pytest.mark.parametrize("t,v", [(6, 300), (6, 70001)])
@pytest.mark.parametrize("T", [0.25, 0.5, 1.0, 2.0])
def test_lists_of_large_logits(ej, t, v, T):
    """Finite logits, as large as FP32 holds: entries like any others, whatever the temperature."""
    g = torch.Generator(device="cuda").manual_seed(5)
    ids, teacher, weights = lists(t, v, 8, g)
    ids[:, :7] = torch.tensor([0, 1, 2, 3, 4, 5, 6], device="cuda")
    least = torch.finfo(torch.float32).min
    teacher[0] = least          # all alike
    teacher[1] = -least
    teacher[2, 3:] = least      # beside ordinary ones: no share
    teacher[3] = 1e6 + torch.round(16 * teacher[3]) / 16
    teacher[4] = -1e6 + torch.round(16 * teacher[4]) / 16
    z = 2.0 * torch.randn((t, v), generator=g, device="cuda")
    check_both(ej, z, ids, teacher, weights, T)
    _, lse = ej.distill(z, ids, teacher, temperature=T)
    want, off = definition(z, ids, teacher, weights, T)[1::2]
    grad = ej.distill_grad(z, lse, ids, teacher, weights, temperature=T)
    slack = weights[:, None] * T * torch.exp(z.double() / T - lse.double()[:, None]) * 2.0 ** -23 * (2 * lse.double().abs()[:, None] + 2 * z.double().abs() / T + 4)
    assert ((grad.double() - want).abs() <= off + slack).all()


def test_temperatures_at_the_ends_of_the_range(ej):
    """1 / T times log2 e has to be a number that FP32 holds; every T from there on gives one."""
    z = torch.zeros((2, 40), device="cuda")
    ids, teacher, weights = torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.zeros((2, 1), device="cuda"), torch.ones(2, device="cuda")
    for T in (3e-39, 4.2e-39):
        with pytest.raises(pkg.EJoinError):
            ej.distill(z, ids, teacher, temperature=T)
        with pytest.raises(pkg.EJoinError):
            ej.distill_with_grad(z, ids, teacher, weights, temperature=T)
    for T in (4.3e-39, 1e-30, 1e18):
        _, lse = ej.distill(z, ids, teacher, temperature=T)
        assert torch.allclose(lse.cpu(), torch.full((2,), 40.0).log())
