"""What the lookups report of tokens stays what it is whatever joins run on the same context."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu


def join_to_host(ej, x, batches, capacity=1 << 20):
    pairs = torch.empty((capacity, 2), dtype=torch.int32, device="cuda")
    host = torch.empty((capacity, 2), dtype=torch.int32, pin_memory=True)
    return ej.selfjoin_pairs_to_host(x, 0.9, batches, pairs, None, host, None)


@pytest.mark.parametrize("n,batches", [(700, 1), (5000, 3)])
def test_a_join_in_batches_leaves_the_report_alone(n, batches):
    ej = pkg.EJoin(0)
    x = torch.rand((n, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).half()
    table, good = torch.randn((10, 64), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    assert ej.embed_status() == 0
    found = join_to_host(ej, x, batches)
    assert found >= n  # (every point is its own neighbour)
    assert ej.embed_status() == 0  # nothing was wrong with any token
    ej.lookup(table, good - 7)
    torch.cuda.synchronize()
    assert join_to_host(ej, x, batches) == found
    assert ej.embed_status() == 3 and ej.embed_status() == 0
    assert join_to_host(ej, x, batches) == found
    ej.lookup(table, good)
    assert ej.embed_status() == 0
    ej.close()


def test_other_joins_leave_it_alone():
    ej = pkg.EJoin(0)
    x = torch.rand((3000, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).half()
    table, bad = torch.randn((10, 64), device="cuda"), torch.full((4,), 10, dtype=torch.int32, device="cuda")
    for join in (lambda: ej.selfjoin_count(x, 0.9), lambda: ej.selfjoin_pairs(x, 0.9, 1 << 20), lambda: ej.selfjoin_count(x[:100], 0.9)):
        ej.lookup(table, bad)
        join()
        assert ej.embed_status() == 3 and ej.embed_status() == 0 and ej.status() == 0
        join()
        assert ej.embed_status() == 0
    ej.close()
