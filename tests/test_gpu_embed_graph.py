"""Graphs of calls that work in the context's memory, replayed after that memory has grown."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu


def test_replays_after_the_memory_has_grown():
    ej = pkg.EJoin(0)
    gen = torch.Generator(device="cuda").manual_seed(4)
    t, v, d = 20000, 3000, 96
    tokens, g = torch.randint(v, (t,), generator=gen, device="cuda", dtype=torch.int32), torch.randn((t, d), generator=gen, device="cuda")
    z = torch.randn((3, 140001), generator=gen, device="cuda")
    ids, teacher, weights = torch.randint(140001, (3, 9), generator=gen, device="cuda"), torch.randn((3, 9), generator=gen, device="cuda"), torch.ones(3, device="cuda")
    x, table = torch.randn((200, 5000), generator=gen, device="cuda"), ej.quantize_f8(torch.randn((300, 5000), generator=gen, device="cuda"))
    grad, dz, scores, loss = torch.empty((v, d), device="cuda"), torch.empty_like(z), torch.empty((200, 300), device="cuda"), torch.empty(3, device="cuda")

    def calls():
        ej.lookup_grad(g, tokens, v, out=grad)
        loss.copy_(ej.distill_with_grad(z, ids, teacher, weights, out=dz)[0])
        ej.scores_f8(x, table, out=scores)

    for _ in range(2):  # (the second finds all the memory it needs)
        calls()
    torch.cuda.synchronize()
    want = [o.clone() for o in (grad, dz, scores, loss)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    free = torch.cuda.mem_get_info()[0]
    sizes = (256 << 20, 300 << 20, 700 << 20)
    for nbytes in sizes:
        ej.embed_reserve(nbytes)
        # memory that the allocation before may have left is in others' hands now
        others = [torch.full((16 << 20,), 7, dtype=torch.int32, device="cuda") for _ in range(8)]
        for _ in range(3):
            for o in (grad, dz, scores, loss):
                o.fill_(3.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip((grad, dz, scores, loss), want))
            assert all((o == 7).all() for o in others)
            calls()  # eager ones work in what there is now
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip((grad, dz, scores, loss), want))
        del others
        torch.cuda.empty_cache()
    assert free - torch.cuda.mem_get_info()[0] < (sizes[-1] + (256 << 20))  # (only what the graph was captured with is kept beside)
    del graph
    ej.close()


def test_memory_is_given_back_without_a_graph():
    ej = pkg.EJoin(0)
    ej.embed_reserve(1 << 20)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for nbytes in (1 << 30, 2 << 30, 3 << 30):
        ej.embed_reserve(nbytes)
    assert free - torch.cuda.mem_get_info()[0] < (3 << 30) + (256 << 20)
    ej.close()
    assert free - torch.cuda.mem_get_info()[0] < 256 << 20
