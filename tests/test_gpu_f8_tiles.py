"""Products of so many tiles that every workgroup takes several, whole ones and others: against products of the same rows in 32 bits with exact
values and sums in 64 (in strips).  Bounds as in test_gpu_f8.py: (d + 2) 2^-23 of sum |a b| for FP32 results, 2^-10 of it more for
those of 16 bits, which may come from the 8-bit matrix cores; the result's own rounding on top."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


def rows(ej, n, d, form, seed):
    """Rows whose blocks' scales differ by many powers of two, from row to row and along them."""
    g = torch.Generator(device="cuda").manual_seed(seed + n + d)
    x = torch.randn((n, d), generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (n, 1), generator=g, device="cuda").float())
    for at in range(0, d, 128):
        x[:, at:at + 128] *= torch.exp2(torch.randint(-3, 4, (n, 1), generator=g, device="cuda").float())
    return ej.quantize_f8(x, form)


def check(got, a, b, scale, terms):
    dtype = got.dtype
    a, b = a.float().double(), b.float().double()
    least = (terms + 2) * 2.0 ** -23 + (0.0 if dtype == torch.float32 else 2.0 ** -10)
    bt, bt_abs = b.T.contiguous(), b.abs().T.contiguous()
    for r in range(0, a.shape[0], 1024):
        want = scale * (a[r:r + 1024] @ bt)
        off = least * abs(scale) * (a[r:r + 1024].abs() @ bt_abs) + want.abs() * HALF_ULP[dtype] * 1.01 + LEAST[dtype]
        bad = ~((got[r:r + 1024].double() - want).abs() <= off)
        assert not bad.any(), (r, int(bad.sum()), torch.nonzero(bad)[:3])


# 4,200 x 16,500: 17 x 65 tiles of 256 x 256, 17 x 129 of 256 x 128.  8,300 x 2,100: 33 x 9 and 33 x 17.  5,000 x 3,900: 20 x 16 and 20 x 31.
# 2,048 x 8,192 and 4,096 x 4,096: 256 and 512 whole tiles.  1,025 x 13,000: 5 x 51 (255: the narrow ones, 5 x 102).
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,d,fa,fb", [(4200, 16500, 100, "e4m3", "e4m3"), (4200, 16500, 300, "e5m2", "e4m3"), (8300, 2100, 100, "e4m3", "e5m2"),
                                         (8300, 2100, 600, "e4m3", "e4m3"), (5000, 3900, 200, "e5m2", "e5m2"), (5000, 3900, 960, "e4m3", "e4m3"),
                                         (2048, 8192, 129, "e4m3", "e4m3"), (4096, 4096, 1100, "e5m2", "e4m3"), (1025, 13000, 640, "e4m3", "e5m2")])
def test_products_of_many_tiles(ej, m, n, d, fa, fb, dtype):
    print(f"product {m} x {n}, d = {d}, {fa} {fb}, {dtype}", flush=True)
    a, b = rows(ej, m, d, fa, 1), rows(ej, n, d, fb, 2)
    # results whose rows are aligned, and within a larger matrix with rows that are not
    got = ej.product_f8(a, b, scale=2.0 ** -8, out_dtype=dtype)
    check(got, a, b, 2.0 ** -8, d)
    whole = torch.full((m + 2, n + 5), 7.0, dtype=dtype, device="cuda")
    out = whole[1:-1, 3:-2]
    ej.product_f8(a, b, scale=2.0 ** -8, out_dtype=dtype, out=out)
    assert torch.equal(out, got)
    out.fill_(7.0)
    assert (whole == 7.0).all()
    for _ in range(3):
        assert torch.equal(ej.product_f8(a, b, scale=2.0 ** -8, out_dtype=dtype), got)


@pytest.mark.parametrize("m,d", [(65, 384), (700, 96), (4096, 200)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scores_of_more_rows_than_few(ej, m, d, dtype):
    """Quantised within the call: the product of the same rows, to the bit."""
    g = torch.Generator(device="cuda").manual_seed(m)
    x, table = torch.randn((m, d), generator=g, device="cuda").half(), rows(ej, 20011, d, "e4m3", 3)
    got = ej.scores_f8(x, table, scale=0.125, out_dtype=dtype)
    assert torch.equal(got, ej.product_f8(ej.quantize_f8(x), table, scale=0.125, out_dtype=dtype))
    check(got, ej.quantize_f8(x), table, 0.125, d)
