"""How far sums and roundings of the grouped products and orthogonalised updates are off, by the type of the result.

Products.  One matrix instruction adds 16 products to an accumulator that is cut toward zero, 2^-23 of the sum of magnitudes at most, and its internal
alignment costs as much again.  An accumulator takes 16 instructions (256 products) where the result is fp32, 64 (1024 products) where it has 16 bits, and
is then added in fp32, 2^-24 a time.  What fp32 operands leave out of their nine partial products is below 2^-21 = 4 2^-23.  So

    |error| <= eps(t)/2 |y| + (2 * 16 + 4 + K / 256 / 2 + 1) 2^-23 sum |a||b|      fp32 results
               eps(t)/2 |y| + (2 * 64 + K / 1024 / 2 + 1) 2^-23 sum |a||b|         16-bit results

and operands of one sign, whose errors all point the same way, come nearest to it."""
import pytest

from paper_2112_09335_b200 import binding
from test_gpu_grouped import MUON, code, h, newton_schulz, offsets_of, ortho_tolerance, torch_type  # noqa: F401

pytestmark = pytest.mark.gpu


def limit(got, want, magnitude, K):
    import torch
    units = 2 * 16 + 4 + K / 512 + 1 if got.dtype == torch.float32 else 2 * 64 + K / 2048 + 1
    half = torch.finfo(got.dtype).eps / 2
    return half * want.abs() + units * 2.0**-23 * magnitude * (1 + half)


def positive(*shape, kind, seed):
    import torch
    return (0.5 + 0.5 * torch.rand(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")).to(torch_type(kind))


@pytest.mark.parametrize("kind, out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("k, n", [(1024, 40), (4113, 24), (8000, 264), (8192, 512)])
def test_products_of_one_sign(h, kind, out, k, n):  # noqa: F811
    import torch
    sizes = [300, 0, 41]
    rows = sum(sizes)
    x, w = positive(rows, k, kind=kind, seed=k), positive(3, k, n, kind=kind, seed=n)
    off = offsets_of(sizes)
    y = torch.empty(rows, n, dtype=torch_type(out), device="cuda")
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 3, rows, k, n, type=code(kind), out_type=code(out))
    for g, (lo, hi) in ((0, (0, 300)), (2, (300, rows))):
        want = x[lo:hi].double() @ w[g].double()
        err = (y[lo:hi].double() - want).abs()
        assert not bool((err > limit(y, want, want, k)).any()), float((err / want).max())


@pytest.mark.parametrize("kind, out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("ka, nb", [(40, 24), (57, 131), (256, 256)])
def test_weight_gradients_of_one_sign(h, kind, out, ka, nb):  # noqa: F811
    import torch
    sizes = [9000, 0, 1025, 4097]
    rows = sum(sizes)
    x, d = positive(rows, ka, kind=kind, seed=ka), positive(rows, nb, kind=kind, seed=nb + 1)
    off = offsets_of(sizes)
    dw = torch.empty(4, ka, nb, dtype=torch_type(out), device="cuda")
    h.grouped_product_tn(x.data_ptr(), d.data_ptr(), dw.data_ptr(), off.data_ptr(), 4, rows, ka, nb, type=code(kind), out_type=code(out))
    at = 0
    for g, size in enumerate(sizes):
        want = x[at:at + size].double().T @ d[at:at + size].double()
        err = (dw[g].double() - want).abs()
        assert not bool((err > limit(dw, want, want, size)).any()), float((err / want.clamp(min=1)).max())
        at += size


STEEP = [(8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.5100), (2.3007, -1.6690, 0.4188)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("batch, rows, cols", [(5, 40, 24), (1, 256, 256), (2, 300, 700), (1, 640, 200), (10, 600, 640), (10, 640, 602)])
@pytest.mark.parametrize("strong, floor", [(0, 1.0), (20, 1e-3), (100, 1e-3)])
@pytest.mark.parametrize("coefficients", [[MUON] * 5, [MUON] * 10, STEEP], ids=["5 steps", "10 steps", "steep steps"])
def test_updates_of_16_bits_are_those_of_fp32_rounded(h, kind, batch, rows, cols, strong, floor, coefficients):  # noqa: F811
    """A result of 16 bits is off by its own rounding, which hides what its products have cost; weak directions are lifted, and what they are off with them, by all of the
    steps (products of single halves end 1.5e-3 to 4e-2 off after 5 and 10).  So it has to be the fp32 result, rounded once; that one is held to its own tolerance."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    g = floor * torch.randn(batch, rows, cols, generator=gen, device="cuda")
    if strong:
        g += torch.randn(batch, rows, strong, generator=gen, device="cuda") @ torch.randn(batch, strong, cols, generator=gen, device="cuda")
    g = g.to(torch_type(kind))
    x, y = torch.empty_like(g), torch.empty(g.shape, device="cuda")
    h.orthogonalise(g.data_ptr(), x.data_ptr(), batch, rows, cols, coefficients, scale=0.2, type=code(kind))
    h.orthogonalise(g.data_ptr(), y.data_ptr(), batch, rows, cols, coefficients, scale=0.2, type=code(kind), out_type=binding.F32)
    assert torch.equal(x, y.to(x.dtype))
    want = newton_schulz(g, coefficients, 1e-7, 0.2)
    for i in range(batch):
        rel = float((y[i].double() - want[i]).norm() / want[i].norm())
        assert rel < ortho_tolerance(g[i:i + 1], coefficients, torch.float32), (i, rel)


@pytest.mark.parametrize("k, n", [(7, 5), (64, 40), (100, 256), (129, 70), (331, 264)])
@pytest.mark.parametrize("transposed", [False, True])
def test_fp32_weights_split_once_or_by_tile_give_the_same_bits(h, k, n, transposed):  # noqa: F811
    """Two groups of 500 rows have their weights split once; with three idle groups more they are too few rows for that."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(k)
    x, w = torch.randn(1000, k, generator=gen, device="cuda"), torch.randn(5, *((n, k) if transposed else (k, n)), generator=gen, device="cuda")
    y = [torch.zeros(1000, n, device="cuda") for _ in range(2)]
    for i, sizes in enumerate(([500, 500], [500, 500, 0, 0, 0])):
        off = offsets_of(sizes)
        h.grouped_product(x.data_ptr(), w.data_ptr(), y[i].data_ptr(), off.data_ptr(), len(sizes), 1000, k, n, transpose_w=transposed)
        torch.cuda.synchronize()
    assert torch.equal(y[0], y[1])
