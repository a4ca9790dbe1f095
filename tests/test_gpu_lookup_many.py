"""The lookup's gradient of many tokens, whose blocks' counts are summed in groups.
Sums of n FP32 values in any order are within n * 2^-23 * sum |g| of the true sum."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


def check(ej, t, v, d, dtype, index, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + t)
    tokens = torch.exp(torch.rand(t, generator=gen, device="cuda", dtype=torch.float64) * torch.log(torch.tensor(float(v), dtype=torch.float64))).long().clamp(1, v) - 1
    tokens = torch.randperm(v, generator=gen, device="cuda")[tokens]  # frequencies as 1 / rank
    tokens[torch.rand(t, generator=gen, device="cuda") < 0.05] = -1
    g = (torch.round(64 * torch.randn((t, d), generator=gen, device="cuda")) / 64).to(dtype)  # (running sums of these are exact in 64 bits)
    got = ej.lookup_grad(g, tokens.to(index), v)
    order = torch.argsort(tokens)[int((tokens < 0).sum()):]
    count = torch.bincount(tokens[order], minlength=v)
    end = torch.cumsum(count, dim=0)

    def sums(x):
        running = torch.nn.functional.pad(torch.cumsum(x[order].double(), dim=0), (0, 0, 1, 0))
        return running[end] - running[end - count]

    assert ((got.double() - sums(g)).abs() <= count[:, None] * 2.0 ** -23 * sums(g.abs())).all()
    assert torch.equal(got, ej.lookup_grad(g, tokens.to(index), v))
    assert ej.embed_status() == 0


# blocks of 2,048 tokens, whose counts are read 32 at a time, or from 256 blocks on summed in groups of 128
@pytest.mark.parametrize("t", [65536, 65537, 70001, 255 * 2048, 255 * 2048 + 1, 256 * 2048, 256 * 2048 + 1, 300 * 2048 + 1, 512 * 2048, 1100 * 2048 + 77])
@pytest.mark.parametrize("v,index", [(300, torch.int64), (40000, torch.int32), (600000, torch.int64)])
def test_many_tokens(ej, t, v, index):
    print(f"lookup_grad {t} of {v}", flush=True)
    check(ej, t, v, 9, torch.float16, index, 1)


def test_many_more_tokens(ej):
    check(ej, 20_000_003, 50000, 4, torch.float32, torch.int32, 2)


def test_time_grows_as_the_number_of_tokens(ej):
    """Four times the tokens take some four times as long (counts of all blocks that every block reads: sixteen times)."""
    def took(t):
        tokens = torch.randint(1000, (t,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
        g, out = torch.ones((t, 1), device="cuda"), torch.empty((1000, 1), device="cuda")
        ej.lookup_grad(g, tokens, 1000, out=out)
        best = 1e9
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ej.lookup_grad(g, tokens, 1000, out=out)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    few, many = took(8 << 20), took(32 << 20)
    print(f"8 M tokens {few:.2f} ms, 32 M {many:.2f} ms", flush=True)
    assert many < 8 * few
