"""Rows in 8 bits at the ends of what is accepted, and what is refused."""
import pytest
import torch

import paper_2508_21230_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ej():
    e = pkg.EJoin(0)
    yield e
    e.close()


def test_scales_far_apart(ej):
    """Rows of scales 2^24 bytes apart are what 256 rows' 32-bit offsets reach; more is refused."""
    d = 300
    gen = torch.Generator(device="cuda").manual_seed(2)
    a, b = (ej.quantize_f8(torch.exp2(torch.randint(-9, 9, (n, 1), generator=gen, device="cuda").float()) * torch.randn((n, d), generator=gen, device="cuda"))
            for n in (300, 70))
    want = ej.product_f8(a, b, out_dtype=torch.float16), ej.product_f8(a, b), ej.product_f8(b, a)
    room = torch.zeros(300 * ((1 << 24) + (1 << 17)), dtype=torch.uint8, device="cuda")
    far = room.as_strided((300, 4), (1 << 24, 1))
    far.copy_(a.scales)
    wide = pkg.F8Rows(a.values, far, d)
    got = ej.product_f8(wide, b, out_dtype=torch.float16), ej.product_f8(wide, b), ej.product_f8(b, wide)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    too_far = room.as_strided((300, 4), ((1 << 24) + (1 << 17), 1))
    too_far.copy_(a.scales)
    wide = pkg.F8Rows(a.values, too_far, d)
    for call in (lambda: ej.product_f8(wide, b), lambda: ej.product_f8(b, wide), lambda: ej.scores_f8(torch.zeros((3, d), device="cuda"), wide)):
        with pytest.raises(pkg.EJoinError):
            call()
    torch.cuda.synchronize()


def test_rows_of_another_format_are_refused(ej):
    x = torch.randn((70, 200), device="cuda")
    types = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
    for form, other in (("e4m3", "e5m2"), ("e5m2", "e4m3")):
        q = ej.quantize_f8(x, form)
        same = pkg.F8Rows(q.values.view(types[form]), q.scales, 200, form)
        assert torch.equal(same.float(), q.float()) and torch.equal(ej.product_f8(same, q), ej.product_f8(q, q))
        assert torch.equal(pkg.F8Rows(q.values, q.scales.view(torch.float8_e8m0fnu), 200, form).float(), q.float())
        for dtype in (types[other], torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.float8_e8m0fnu, torch.bool):
            with pytest.raises(pkg.EJoinError):
                pkg.F8Rows(q.values.view(dtype), q.scales, 200, form)
        for dtype in (torch.float8_e4m3fn, torch.int8, torch.bool):
            with pytest.raises(pkg.EJoinError):
                pkg.F8Rows(q.values, q.scales.view(dtype), 200, form)


@pytest.mark.parametrize("n,d,dtype", [((1 << 23) + 77, 3, torch.float32), ((1 << 23) - 1, 129, torch.float16), ((1 << 28) + 5, 1, torch.bfloat16)])
def test_rows_in_8_bits_past_2_to_the_23(ej, n, d, dtype):
    """A row's bytes depend on that row alone: those of a large matrix are those of its pieces."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((n, d), generator=gen, device="cuda", dtype=torch.float16 if n > 1 << 27 else torch.float32).to(dtype)
    q = ej.quantize_f8(x)
    for at in (0, 1 << 22, n // 2 + 1, n - 1000):
        piece = ej.quantize_f8(x[at:at + 1000])
        assert torch.equal(q.values[at:at + 1000], piece.values) and torch.equal(q.scales[at:at + 1000], piece.scales)
    if n > 1 << 27:
        at = (1 << 21) * 64 * 2  # (a border between launches)
        piece = ej.quantize_f8(x[at - 70:])
        assert torch.equal(q.values[at - 70:], piece.values) and torch.equal(q.scales[at - 70:], piece.scales)
    del x, q
    torch.cuda.empty_cache()


def test_columns_of_so_many_rows_are_refused(ej):
    """Along the columns a row of the result is as long as X has rows."""
    x = torch.zeros((1 << 23, 2), dtype=torch.float16, device="cuda")
    with pytest.raises(pkg.EJoinError):
        ej.quantize_f8(x, columns=True)
    with pytest.raises(pkg.EJoinError):
        ej.quantize_f8_both(x)
    assert ej.quantize_f8(x[:-1], columns=True).n == 2


@pytest.mark.parametrize("form,most", [("e4m3", 1.875), ("e5m2", 1.75)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_values_stay_finite(ej, form, most, dtype):
    """Held as the largest value of the format below 2^128, by rows, by columns and within the call; products with zeros are zero."""
    m, d = 140, 300
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((m, d), generator=gen, device="cuda").to(dtype)
    top = torch.finfo(dtype).max
    x[3, 7], x[5, 130:140], x[9], x[11, 299] = -top, top, -top, 1.76 * 2.0 ** 127
    want = x[[3, 5, 9, 11]].double()
    rows, columns = ej.quantize_f8_both(x, form)
    for q in (rows, ej.quantize_f8(x, form)):
        got = q.float()
        assert torch.isfinite(got).all()
        assert got[3, 7] == -most * 2.0 ** 127 and (got[5, 130:140] == most * 2.0 ** 127).all() and (got[9] == -most * 2.0 ** 127).all() and got[11, 299] == 1.75 * 2.0 ** 127
        assert (got[3, :7] == 0).all() and (got[3, 128:].double() - want[0, 128:]).abs().max() < 0.3  # (other blocks are as they were)
    for q in (columns, ej.quantize_f8(x, form, columns=True)):
        got = q.float()
        assert torch.isfinite(got).all() and got[7, 3] == -most * 2.0 ** 127 and (got[:, 9] == -most * 2.0 ** 127).all() and got[299, 11] == 1.75 * 2.0 ** 127
    y = torch.randn((200, d), generator=gen, device="cuda") * 2.0 ** -40
    y[:, 7] = 0.0
    y[::2] = 0.0
    b = ej.quantize_f8(y)
    for a in (rows, pkg.F8Rows(rows.values[:20], rows.scales[:20], d, form)):
        exact = a.float().double() @ b.float().double().T.contiguous()
        size = a.float().double().abs() @ b.float().double().abs().T.contiguous()
        for out in (torch.float32, torch.bfloat16):
            got = ej.product_f8(a, b, out_dtype=out).double()
            assert ((got - exact).abs() <= (302 * 2.0 ** -23 + (0.0 if out == torch.float32 else 2.0 ** -8 + 2.0 ** -10)) * size).all()
        assert torch.equal(ej.scores_f8(x[:a.n], b), ej.product_f8(ej.quantize_f8(x[:a.n]), b))
        assert torch.isfinite(ej.scores_f8(x[:a.n], b)).all()
