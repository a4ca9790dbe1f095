"""The loss and its gradient of rows whose scores, or whose lists' logits, share a large offset: the type's lowest value in every place, a million
added to all of them.  Softmaxes depend on differences alone, so the bounds do too.

With D the largest |z - max z| / T among the scores whose share is not zero to 32 bits (it is 110 at most), and E the same of the list's logits: an
exponential is off by the rounding of its argument (3 |argument| 2^-23) and its own (2^-22), a sum over v scores, of which a thread adds v / 64 at
most, by (v / 64 + 32) 2^-23 of itself.  So q is within e = 2^-23 (4 D + v / 64 + 40) of itself, p within f = 2^-23 (4 E + k + 40),
the gradient within weight T (q e + p f) and its own rounding, and the loss within T^2 (e + f) times one plus the largest logarithm in it."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
EPS = 2.0 ** -23
# rows and scores: on both sides of what a workgroup holds, and of the few long rows that are cut into pieces all the same
SIZES = [(4, 900), (4, 32769), (4, 53248), (4, 53249), (64, 60001), (65, 60001), (3, 70001), (300, 66001), (2, 140001)]


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


def definition(z, ids, teacher, weights, T):
    there = (ids >= 0) & (teacher != -torch.inf)
    u = z.double() / T
    tl = (teacher.double() - teacher.double().amax(dim=1, keepdim=True)) / T  # (the difference first: 64 bits do not hold 3e38 + log 7 either)
    some = there.any(dim=1)
    at = ids.clamp(min=0).long()
    log_q = torch.log_softmax(u, dim=1)
    tl = torch.where(there, tl, -torch.inf)
    log_p = torch.where(there, tl - torch.logsumexp(torch.where(some[:, None], tl, 0.0), dim=1)[:, None], -torch.inf)
    p = torch.exp(log_p)
    loss = T * T * torch.where(there & (p > 0), p * (log_p - torch.gather(log_q, 1, at)), 0.0).sum(dim=1)
    at_ids = torch.zeros_like(u).scatter_add_(1, at, torch.where(there, p, 0.0))
    q = torch.exp(log_q)
    scale = weights.double()[:, None] * T
    grad = torch.where(some[:, None], scale * (q - at_ids), 0.0)
    v, k = z.shape[1], ids.shape[1]
    D = torch.where(log_q > -110, (u - u.amax(dim=1, keepdim=True)).abs(), 0.0).amax(dim=1)
    E = torch.where(log_p > -110, (tl - tl.amax(dim=1, keepdim=True)).abs(), 0.0).amax(dim=1)
    e, f = EPS * (4 * D + v / 64 + 40), EPS * (4 * E + k + 40)
    most = 1 + torch.where(there & (p > 0), torch.maximum(log_p.abs(), torch.gather(log_q, 1, at).abs()), 0.0).amax(dim=1)
    off_grad = scale * (q * e[:, None] + at_ids * f[:, None]) + grad.abs() * HALF_ULP[z.dtype] * 1.01 + LEAST[z.dtype]
    return loss, grad, T * T * (e + f) * most, off_grad


def check_both(ej, z, ids, teacher, weights, T):
    want_loss, want, off_loss, off = definition(z, ids, teacher, weights, T)
    loss, grad = ej.distill_with_grad(z, ids, teacher, weights, temperature=T)
    bad = ~((grad.double() - want).abs() <= off)
    assert not bad.any(), (int(bad.sum()), grad[bad][:4], want[bad][:4])
    bad = ~((loss.double() - want_loss).abs() <= off_loss)
    assert not bad.any(), (loss[bad][:4], want_loss[bad][:4])
    held = z.clone()  # in place
    _, out = ej.distill_with_grad(held, ids, teacher, weights, temperature=T, out=held)
    assert torch.equal(out, grad)
    alone, _ = ej.distill(z, ids, teacher, temperature=T)
    bad = ~((alone.double() - want_loss).abs() <= off_loss)
    assert not bad.any(), (alone[bad][:4], want_loss[bad][:4])


def lists(t, v, k, g):
    ids = torch.randint(v, (t, k), generator=g, device="cuda", dtype=torch.int32)
    ids[:, 0] = v - 1
    ids[:, -1] = -1
    return ids, 2.0 * torch.randn((t, k), generator=g, device="cuda"), torch.rand(t, generator=g, device="cuda") + 0.5


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,v", SIZES)
def test_rows_of_the_lowest_value(ej, dtype, t, v):
    g = torch.Generator(device="cuda").manual_seed(t + v)
    ids, teacher, weights = lists(t, v, 12, g)
    z = (2.0 * torch.randn((t, v), generator=g, device="cuda")).to(dtype)
    z[0] = torch.finfo(dtype).min
    z[1] = torch.finfo(dtype).max
    for T in (1.0, 2.0, 0.5):
        check_both(ej, z, ids, teacher, weights, T)


@pytest.mark.parametrize("t,v", SIZES)
@pytest.mark.parametrize("offset", [1e6, -1e6, 3e4])
def test_rows_with_a_common_offset(ej, t, v, offset):
    g = torch.Generator(device="cuda").manual_seed(t + v)
    ids, teacher, weights = lists(t, v, 12, g)
    z = offset + torch.round(32.0 * torch.randn((t, v), generator=g, device="cuda")) / 16  # (multiples of 1 / 16: FP32 holds the sums)
    check_both(ej, z, ids, teacher, weights, 1.5)
