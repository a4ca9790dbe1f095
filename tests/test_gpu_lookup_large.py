"""Lookups whose results are larger than the caches, and of more pieces than 32 bits count; the loss with lists near their longest."""
import pytest
import torch

import paper_2508_21230_amd as pkg
from tests import test_gpu_distill as distill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


@pytest.mark.parametrize("out", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,v,d,dtype,index", [(200003, 5000, 700, torch.float32, torch.int32), (1100000, 300, 130, torch.float16, torch.int64),
                                               (700001, 20000, 200, torch.bfloat16, torch.int32)])
def test_results_larger_than_the_caches(ej, t, v, d, dtype, index, out):
    """To the bit, in memory of their own and within a larger matrix whose rows are not aligned."""
    gen = torch.Generator(device="cuda").manual_seed(t)
    table = torch.randn((v, d), generator=gen, device="cuda").to(dtype)
    tokens = torch.randint(-1, v, (t,), generator=gen, device="cuda").to(index)
    width = (d + 63) // 64 * 64
    assert t * width * 2 > 256 << 20
    whole = torch.full((t + 2, width + 5), 9.0, dtype=out, device="cuda")
    for y in (ej.lookup(table, tokens, scale=0.3, out_dtype=out), ej.lookup(table, tokens, scale=0.3, out=whole[1:-1, 2:-3])):
        for at in range(0, t, 100000):
            tk = tokens[at:at + 100000].long()
            want = torch.where((tk >= 0)[:, None], table[tk.clamp(min=0)].float() * 0.3, 0.0).to(out)
            assert torch.equal(y[at:at + 100000, :d], want) and not y[at:at + 100000, d:].any()
    whole[1:-1, 2:-3] = 9.0
    assert (whole == 9.0).all() and ej.embed_status() == 0


def test_more_pieces_than_32_bits_count(ej):
    t = (1 << 29) + 3001  # rows of eight pieces
    table = torch.arange(5 * 9, device="cuda").view(5, 9).half()
    tokens = (torch.arange(t, device="cuda", dtype=torch.int32) % 6) - 1
    y = ej.lookup(table, tokens)
    for at in (0, (1 << 28) - 5, (1 << 29) - 2000, t - 3000):
        tk = tokens[at:at + 3000].long()
        want = torch.where((tk >= 0)[:, None], table[tk.clamp(min=0)], 0.0)
        assert torch.equal(y[at:at + 3000, :9], want) and not y[at:at + 3000, 9:].any()
    assert ej.embed_status() == 0
    del y, tokens
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,v,k", [(11, 2000, 1024), (7, 50021, 1023), (5, 140001, 1000)])
def test_loss_against_long_lists(ej, dtype, t, v, k):
    distill.check(ej, *distill.made(t, v, k, dtype, twice=True), 2.0)
