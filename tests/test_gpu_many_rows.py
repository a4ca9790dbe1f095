"""More rows, of scores and of tables, than one launch may have workgroups for."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


@pytest.mark.parametrize("t", [(1 << 22) + 3, (1 << 24) + 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_loss_of_many_rows(ej, t, dtype):
    """Rows of three scores with one entry: log q is elementary.  FP32: a few roundings of numbers below 16 each."""
    gen = torch.Generator(device="cuda").manual_seed(t)
    z = torch.randn((t, 3), generator=gen, device="cuda").to(dtype)
    ids = torch.randint(3, (t, 1), generator=gen, device="cuda", dtype=torch.int32)
    ids[7::11] = -1
    teacher, weights = torch.randn((t, 1), generator=gen, device="cuda"), torch.rand(t, generator=gen, device="cuda")
    there = ids[:, 0] >= 0
    lse = torch.logsumexp(z.double(), dim=1)
    want = torch.where(there, lse - torch.gather(z.double(), 1, ids.clamp(min=0).long())[:, 0], 0.0)
    loss, got_lse = ej.distill(z, ids, teacher)
    assert ((got_lse.double() - lse).abs() <= 64 * 2.0 ** -24).all() and ((loss.double() - want).abs() <= 128 * 2.0 ** -24).all()
    grad = torch.exp(z.double() - lse[:, None])
    grad.scatter_add_(1, ids.clamp(min=0).long(), torch.full((t, 1), -1.0, dtype=torch.float64, device="cuda"))
    grad = torch.where(there[:, None], weights.double()[:, None] * grad, 0.0)
    off = 64 * 2.0 ** -24 + grad.abs() * (2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8) * 1.01
    assert ((ej.distill_grad(z, got_lse, ids, teacher, weights).double() - grad).abs() <= off).all()
    loss2, both = ej.distill_with_grad(z, ids, teacher, weights)
    assert torch.equal(loss2, loss) and ((both.double() - grad).abs() <= off).all()
    assert ej.embed_status() == 0


@pytest.mark.parametrize("t", [5, 3000, 9000])
@pytest.mark.parametrize("v", [(1 << 31) - 1, (1 << 31) - 2, (1 << 28) + 65])
def test_largest_tables(ej, t, v):
    gen = torch.Generator(device="cuda").manual_seed(t)
    tokens = torch.randint(v, (t,), generator=gen, device="cuda")
    tokens[0], tokens[1], tokens[2] = v - 1, 0, v - 1
    g = torch.ones((t, 1), dtype=torch.bfloat16, device="cuda")
    out = torch.full((v, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    ej.lookup_grad(g, tokens, v, out=out)
    rows, counts = torch.unique(tokens, return_counts=True)
    assert torch.equal(out[:, 0][rows], counts.to(torch.bfloat16))
    other = 0
    for at in range(0, v, 1 << 28):
        other += int(torch.count_nonzero(out[at:at + (1 << 28), 0]))
    assert other == rows.numel() and ej.embed_status() == 0
