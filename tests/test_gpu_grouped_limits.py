"""Products grouped by expert and orthogonalised updates where sizes and values reach the limits of their formats.  Tolerances of products: those of
test_gpu_grouped.py."""
import pytest

from paper_2112_09335_b200 import binding
from test_gpu_grouped import MUON, bound, code, h, newton_schulz, offsets_of, ortho_tolerance, torch_type, trainer  # noqa: F401

pytestmark = pytest.mark.gpu


def test_weights_whose_split_images_pass_31_bits(h):  # noqa: F811
    """Two fp32 weights of 32768 x 16400: a part of their images is 2^31 bytes and more, so that parts 1 and 2 lie farther than an int reaches."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, n, sizes = 32768, 16400, [300, 290]
    rows = sum(sizes)
    x = torch.randn(rows, k, generator=gen, device="cuda")
    w = torch.empty(2, k, n, device="cuda").normal_(generator=gen)
    y = torch.full((rows, n), 7.0, device="cuda")
    off = offsets_of(sizes)
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 2, rows, k, n)
    torch.cuda.synchronize()
    at = 0
    for g, size in enumerate(sizes):
        a = x[at:at + size].double()
        for lo in (0, n // 2 - 3, n - 130):
            b = w[g, :, lo:lo + 130].double()
            got, want = y[at:at + size, lo:lo + 130], a @ b
            assert not bool(((got.double() - want).abs() > bound(got, want, a.abs() @ b.abs(), k)).any())
        at += size


def test_fp32_products_without_room_for_split_weights():
    """Images of fp32 weights are for speed: where there is no memory for them the call gives the same bits without."""
    import torch
    k, n, groups, rows = 4096, 8192, 8, 2100
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, k, generator=gen, device="cuda")
    w = torch.empty(groups, k, n, device="cuda").normal_(generator=gen)
    y = [torch.zeros(rows, n, device="cuda") for _ in range(2)]
    off = offsets_of([300] * 6 + [0, 300])
    images, hog, s = 3 * groups * k * n * 2, None, torch.cuda.Stream()
    y.append(torch.zeros(rows, n, device="cuda"))
    torch.cuda.synchronize()
    try:
        for i in range(2):
            g = trainer(stream=s.cuda_stream)
            call = lambda to: g.grouped_product(x.data_ptr(), w.data_ptr(), to.data_ptr(), off.data_ptr(), groups, rows, k, n)  # noqa: B023, E731
            try:
                if i == 1:      # memory for half of them is left
                    torch.cuda.empty_cache()
                    hog = torch.empty(torch.cuda.mem_get_info()[0] - images // 2, dtype=torch.uint8, device="cuda")
                    assert torch.cuda.mem_get_info()[0] < images
                call(y[i])
                if i == 1:      # having been made once, the call may be captured
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=s, capture_error_mode="thread_local"):
                        call(y[2])
                    graph.replay()
                    torch.cuda.synchronize()
                    del graph
                torch.cuda.synchronize()
            finally:
                g.destroy()
                binding.release_idle()
    finally:
        del hog
        torch.cuda.empty_cache()
    a, b = x[:300].double(), w[0, :, :200].double()
    assert not bool(((y[0][:300, :200].double() - a @ b).abs() > bound(y[0][:300, :200], a @ b, a.abs() @ b.abs(), k)).any())
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2])


def orthogonalised(h, g, coefficients, eps, scale, out):  # noqa: F811
    import torch
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
    x = torch.full(g.shape, float("nan"), dtype=torch_type(out), device="cuda")
    h.orthogonalise(g.data_ptr(), x.data_ptr(), *g.shape, coefficients, eps=eps, scale=scale, type=code(names[g.dtype]), out_type=code(out))
    return x


SMALL = [(40, 24), (150, 200), (200, 70)]


@pytest.mark.parametrize("kind, out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows, cols", SMALL + [(600, 520)])
def test_norms_far_below_eps(h, kind, out, rows, cols):  # noqa: F811
    """X_0 = G / (||G|| + eps) is then a tiny matrix, as accurate as any other: beside ordinary ones of the same batch, for coefficients with and without a."""
    import torch
    norms = [1.0, 1e-4, 1e-8, 1e-13, 1e-20, 1e-26]
    g = torch.randn(len(norms), rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda", dtype=torch.float64)
    g = (g / torch.linalg.norm(g, dim=(1, 2), keepdim=True) * torch.tensor(norms, device="cuda", dtype=torch.float64)[:, None, None]).to(torch_type(kind))
    for coefficients in ([MUON] * 5, [(1.5, -0.5, 0.0)], [(0.0, 1.25, 0.0)], [(2.0, -1.5, 0.5)] * 12):
        x = orthogonalised(h, g, coefficients, 1.0, 1.0, out)
        want = newton_schulz(g, coefficients, 1.0, 1.0)
        for i in range(len(norms)):
            if float(want[i].norm()) < 1e-32:       # elements among the subnormal results
                continue
            rel = float((x[i].double() - want[i]).norm() / want[i].norm())
            assert rel < ortho_tolerance(g[i:i + 1], coefficients, x.dtype, 1.0), (coefficients, norms[i], rel)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SMALL)
def test_coefficients_that_make_everything_small(h, out, rows, cols):  # noqa: F811
    import torch
    g = torch.randn(2, rows, cols, generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda").to(torch_type(out))
    for coefficients, scale in (([(1e-7, 0.0, 0.0)] * 3, 1e21), ([(1e-9, 0.0, 0.0), MUON], 1e9), ([(0.0, 0.0, 1e-12)], 1e12), ([(0.0, 0.0, 0.0), MUON], 1.0)):
        x = orthogonalised(h, g, coefficients, 1e-7, scale, out)
        want = newton_schulz(g, coefficients, 1e-7, scale)
        if float(want.norm()) == 0:
            assert bool((x == 0).all())
            continue
        rel = float((x.double() - want).norm() / want.norm())
        assert rel < ortho_tolerance(g, coefficients, x.dtype), (coefficients, rel)


@pytest.mark.parametrize("rows", [90, 900])     # weights split tile by tile, and once for all tiles
@pytest.mark.parametrize("ex, ew", [(-108, 0), (-112, 0), (-120, 0), (-130, 0), (-140, 3), (-120, 100), (-130, 120), (0, -125), (-60, -60)])
def test_fp32_elements_near_the_end_of_their_range(h, rows, ex, ew):  # noqa: F811
    """Parts of an fp32 element end at the last bit of a bf16, 2^-133: elements from 2^-110 on are exact sums of theirs, smaller ones are cut there, so that every
    product with one is off by less than 2^-133 of the other factor.  Beyond that the usual tolerance."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    k, n = 96, 40

    def made(e, *shape):
        return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float64) * 2.0**e).float()
    x, w, d = made(ex, rows, k), made(ew, 1, k, n), made(ew, rows, n)
    off = offsets_of([rows])
    cut = lambda a: (a.double().abs() < 2.0**-110).double() * 2.0**-133      # noqa: E731
    for transposed in (False, True):
        v = w.mT.contiguous() if transposed else w
        y = torch.empty(rows, n, device="cuda")
        h.grouped_product(x.data_ptr(), v.data_ptr(), y.data_ptr(), off.data_ptr(), 1, rows, k, n, transpose_w=transposed)
        a, b = x.double(), w[0].double()
        lim = bound(y, a @ b, a.abs() @ b.abs(), k) + cut(x) @ b.abs() + a.abs() @ cut(w[0])
        assert not bool(((y.double() - a @ b).abs() > lim).any())
    dw = torch.empty(k, n, device="cuda")
    h.grouped_product_tn(x.data_ptr(), d.data_ptr(), dw.data_ptr(), off.data_ptr(), 1, rows, k, n)
    a, b = x.double().T, d.double()
    lim = bound(dw, a @ b, a.abs() @ b.abs(), rows) + cut(x).T @ b.abs() + a.abs() @ cut(d)
    assert not bool(((dw.double() - a @ b).abs() > lim).any())


@pytest.mark.parametrize("scale", [1e-33, -3e-30, 1e30])
@pytest.mark.parametrize("rows, cols", SMALL)
def test_scales_near_the_ends_of_fp32(h, scale, rows, cols):  # noqa: F811
    import torch
    g = torch.randn(2, rows, cols, generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda")
    for coefficients in ([MUON] * 5, [(0.5, 0.0, 0.0)], []):
        x = orthogonalised(h, g, coefficients, 1e-7, scale, "f32")
        want = newton_schulz(g, coefficients, 1e-7, scale)
        assert float((x.double() - want).norm() / want.norm()) < ortho_tolerance(g, coefficients, x.dtype), coefficients


@pytest.mark.parametrize("coefficients", [[(3.9, -3.9, 1e-20)], [(2.0, -1.5, 1e-30), MUON], [(-3.9, 3.9, 1e-12)]])
@pytest.mark.parametrize("rows, cols", SMALL)
def test_coefficients_nearly_zero(h, coefficients, rows, cols):  # noqa: F811
    """One strong direction beside weak ones: singular values all over 0 .. 1."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    g = torch.randn(1, rows, cols, generator=gen, device="cuda") * 0.05 + torch.randn(1, rows, 1, generator=gen, device="cuda") @ torch.randn(1, 1, cols, generator=gen, device="cuda")
    x = orthogonalised(h, g, coefficients, 1e-7, 1.0, "f32")
    want = newton_schulz(g, coefficients, 1e-7, 1.0)
    assert float((x.double() - want).norm() / want.norm()) < ortho_tolerance(g, coefficients, x.dtype)
