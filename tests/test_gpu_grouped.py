"""Products grouped by expert, both gradients, and orthogonalised updates against plain fp64 implementations.

Tolerances.  An output of type t is off by half a step, eps(t) / 2 of its value, from rounding, and before that by the sum's error.  Operands
are exact, in one part of 16 bits or three of 8 bits each, whose left-out products are below 2^-21 in all.  Sums are formed in pieces of at
most 256 products in fp32 (16 matrix instructions whose accumulator is cut toward zero, 2^-23 of the sum of magnitudes each, their internal
alignment as much again), which are added in fp32.  So |error| <= eps(t)/2 |y| + (2 * 16 + 8 + K / 256) 2^-23 sum |a||b|.  Where
a whole result is compared in the 2-norm, the same counts against the norm of y for operands of random sign, whose partial sums are no larger.
"""
import numpy as np
import pytest

from paper_2112_09335_b200 import binding

pytestmark = pytest.mark.gpu
NAMES = ("f32", "bf16", "f16")
MUON = (3.4445, -4.7750, 2.0315)


def torch_type(name):
    import torch
    return dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[name]


def code(name):
    return dict(f32=binding.F32, bf16=binding.BF16, f16=binding.F16)[name]


def trainer(stream=0, n=6, community=None):
    """A handle on a small ring of nodes."""
    ptr = np.arange(0, 2 * n + 1, 2)
    col = np.array([sorted(((i - 1) % n, (i + 1) % n)) for i in range(n)]).reshape(-1)
    community = np.zeros(n) if community is None else np.asarray(community)
    return binding.GcnAdmm(n, ptr, col, np.ones((n, 2)), np.zeros(n), np.ones(n), [2, 2], int(community.max()) + 1, community,
                           [np.ones((2, 2), dtype=np.float32)], stream=stream)


@pytest.fixture(scope="module")
def h():
    g = trainer()
    yield g
    g.destroy()


class Matrix:
    """rows x cols inside a larger buffer: `ld` elements a row, `shift` elements behind the buffer's start, NaN around it."""

    def __init__(self, batch, rows, cols, kind, pad=0, shift=0, gap=0, gen=None, scale=1.0, fill=None):
        import torch
        self.ld, self.stride = cols + pad, rows * (cols + pad) + gap
        self.held = torch.full((shift + batch * self.stride + 8,), float("nan"), dtype=torch_type(kind), device="cuda")
        self.view = self.held[shift:].as_strided((batch, rows, cols), (self.stride, self.ld, 1))
        if gen is not None:
            self.view.copy_(torch.randn(batch, rows, cols, generator=gen, device="cuda") * scale)
        if fill is not None:
            self.view.fill_(fill)
        self.at = self.view.data_ptr() if self.view.numel() else 0

    def outside_is_untouched(self):
        import torch
        copy = self.held.clone()
        copy.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(float("nan"))
        return bool(torch.isnan(copy).all())


def bound(got, want, magnitude, K):
    """Elementwise tolerance of the docstring."""
    import torch
    eps = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps   # half a step among subnormal results, at most
    return eps * want.abs() + (40 + K / 256) * 2.0**-23 * magnitude * (1 + eps) + tiny


def close(got, want, magnitude, K):
    import torch
    err = (got.double() - want).abs()
    lim = bound(got, want, magnitude, K)
    worst = (err / lim.clamp(min=1e-300)).max() if err.numel() else torch.zeros(())
    assert not bool((err > lim).any()) and not bool(torch.isnan(err).any()), f"{float(worst):.3g} of the tolerance"
    if got.dtype == torch.float32 and err.numel() > 1000 and K > 1:
        rel = float(err.norm() / want.norm())
        assert rel < (40 + K / 256) * 2.0**-23, rel


def offsets_of(sizes, first=0):
    import torch
    return torch.tensor(np.concatenate([[first], first + np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def run_product(h, sizes, k, n, kind, out, transposed=False, first=0, tail=0, seed=0, x_pad=0, w_pad=0, y_pad=0, shift=0, gap=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = first + int(np.sum(sizes)) + tail
    x = Matrix(1, rows, k, kind, x_pad, shift, gen=gen)
    w = Matrix(len(sizes), *((n, k) if transposed else (k, n)), kind, w_pad, shift, gap, gen=gen, scale=k**-0.5)
    y = Matrix(1, rows, n, out, y_pad, shift, fill=7.0)
    x.view[0, :first], x.view[0, rows - tail:] = float("nan"), float("inf")      # rows of no group reach no result
    off = offsets_of(sizes, first)
    h.grouped_product(x.at, w.at, y.at, off.data_ptr(), len(sizes), rows, k, n, type=code(kind), out_type=code(out), transpose_w=transposed, ldx=x.ld,
                      ldw=w.ld, stride_w=w.stride, ldy=y.ld)
    torch.cuda.synchronize()
    at = first
    for g, size in enumerate(sizes):
        a, b = x.view[0, at:at + size].double(), w.view[g].double()
        b = b.T if transposed else b
        close(y.view[0, at:at + size], a @ b, a.abs() @ b.abs(), k)
        at += size
    assert bool((y.view[0, :first] == 7).all()) and bool((y.view[0, at:] == 7).all())
    assert y.outside_is_untouched()


def run_tn(h, sizes, ka, nb, kind, out, first=0, tail=0, seed=0, x_pad=0, y_pad=0, w_pad=0, shift=0, gap=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = first + int(np.sum(sizes)) + tail
    x, y = Matrix(1, rows, ka, kind, x_pad, shift, gen=gen), Matrix(1, rows, nb, kind, y_pad, shift, gen=gen)
    dw = Matrix(len(sizes), ka, nb, out, w_pad, shift, gap, fill=7.0)
    for m in (x, y):
        m.view[0, :first], m.view[0, rows - tail:] = float("nan"), float("inf")
    off = offsets_of(sizes, first)
    h.grouped_product_tn(x.at, y.at, dw.at, off.data_ptr(), len(sizes), rows, ka, nb, type=code(kind), out_type=code(out), ldx=x.ld, ldy=y.ld, lddw=dw.ld,
                         stride_dw=dw.stride)
    torch.cuda.synchronize()
    at = first
    for g, size in enumerate(sizes):
        a, b = x.view[0, at:at + size].double(), y.view[0, at:at + size].double()
        close(dw.view[g], a.T @ b, a.abs().T @ b.abs(), max(size, 1))
        at += size
    assert dw.outside_is_untouched()


SIZES = [[1], [128], [5, 0, 129, 1], [0, 0, 300], [127, 128, 129, 64, 0], [1] * 40, [700, 3, 0, 260]]
WIDTHS = [(1, 1), (7, 5), (16, 8), (64, 64), (65, 47), (100, 256), (128, 257), (264, 136), (500, 128), (513, 300)]


@pytest.mark.parametrize("kind", NAMES)
@pytest.mark.parametrize("k, n", WIDTHS)
def test_product(h, kind, k, n):
    for i, sizes in enumerate(SIZES):
        for transposed in (False, True):
            run_product(h, sizes, k, n, kind, "f32" if (i + transposed) % 2 else kind, transposed, seed=i)


@pytest.mark.parametrize("kind", NAMES)
@pytest.mark.parametrize("ka, nb", WIDTHS)
def test_product_tn(h, kind, ka, nb):
    for i, sizes in enumerate(SIZES):
        run_tn(h, sizes, ka, nb, kind, "f32" if i % 2 else kind, seed=i)


@pytest.mark.parametrize("k, n", [(1, 1), (7, 5), (64, 40), (100, 256), (129, 70), (200, 130), (331, 264)])
def test_fp32_product_of_many_rows(h, k, n):
    """Enough rows to a group for its weights to be split once for all of them."""
    for transposed in (False, True):
        run_product(h, [1000, 0, 513], k, n, "f32", "f32", transposed, first=3, tail=9)
        run_product(h, [700], k, n, "f32", "f32", transposed, x_pad=1, w_pad=3, y_pad=2, shift=1, gap=5)


LAYOUTS = [dict(x_pad=8, y_pad=16, w_pad=8), dict(x_pad=3, y_pad=1, w_pad=5, gap=7), dict(shift=1), dict(shift=8, gap=8), dict(x_pad=4, y_pad=4, w_pad=4, shift=4)]


@pytest.mark.parametrize("kind", NAMES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_layouts_and_rows_of_no_group(h, kind, layout):
    for k, n in ((72, 136), (61, 130)):
        for transposed in (False, True):
            run_product(h, [30, 0, 200, 65], k, n, kind, kind, transposed, first=17, tail=70, **layout)
        run_tn(h, [30, 0, 200, 65], k, n, kind, "f32", first=17, tail=70, **layout)
        run_tn(h, [30, 0, 200, 65], k, n, kind, kind, first=17, tail=70, **layout)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_larger_ones(h, kind):
    rng = np.random.default_rng(1)
    sizes = rng.multinomial(9000, rng.dirichlet(np.full(13, 0.7)))
    run_product(h, sizes, 1032, 776, kind, kind)
    run_product(h, sizes, 776, 1032, kind, "f32", transposed=True)
    run_product(h, [1] * 8 + [0] * 56, 1024, 1000, kind, kind)
    run_tn(h, sizes, 520, 776, kind, "f32")
    run_tn(h, [20000, 0, 100], 200, 47, kind, "f32")
    run_tn(h, [9000], 16, 7, kind, kind)
    run_tn(h, [40] * 200, 24, 40, kind, "f32")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_tiles_of_256_by_256(h, kind):
    """Widths that fill them and enough rows for all SMs: ends of groups at every place of a tile, idle groups, sums of one chunk and of many."""
    rng = np.random.default_rng(2)
    sizes = np.concatenate([rng.integers(0, 700, 40), [0, 1, 63, 64, 65, 255, 256, 257, 0]])
    for k, n in ((8, 512), (200, 250), (328, 1016)):
        run_product(h, sizes, k, n, kind, kind, first=3, tail=5)
        run_product(h, sizes, k, n, kind, "f32", transposed=True, first=3, tail=5)
    few = rng.integers(0, 64, 200)
    for ka, nb in ((256, 256), (248, 504), (1000, 232)):
        run_tn(h, sizes, ka, nb, kind, "f32", first=3, tail=5)
        run_tn(h, sizes, ka, nb, kind, kind)
    run_tn(h, few, 256, 248, kind, "f32")
    run_tn(h, [30000, 0, 1, 777], 512, 256, kind, "f32")
    run_tn(h, [0, 0], 256, 256, kind, kind)


@pytest.mark.parametrize("kind", NAMES)
def test_sums_shared_by_many_blocks(h, kind):
    """Few tiles and many rows: a tile's sum comes from up to all blocks of the chip; equal and very unequal groups."""
    run_tn(h, [50001], 40, 24, kind, "f32")
    run_tn(h, [30000, 1, 0, 7000], 136, 72, kind, kind)
    run_tn(h, [64 * 37] * 9, 64, 264, kind, "f32")
    run_tn(h, [0, 0, 25000], 130, 7, kind, "f32")


def test_most_groups(h):
    sizes = np.arange(1024) % 3
    run_product(h, sizes, 24, 16, "bf16", "bf16")
    run_tn(h, sizes, 24, 16, "bf16", "f32")
    run_product(h, sizes, 9, 5, "f32", "f32")
    run_tn(h, sizes, 9, 5, "f32", "f32")


@pytest.mark.parametrize("kind", NAMES)
def test_sums_keep_the_range_of_fp32(h, kind):
    """Rows and columns of very different sizes: every product counts with its own exponent."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, n, rows = 96, 40, 150
    span = 30 if kind != "f16" else 4
    ex = torch.randint(-span, span + 1, (k,), generator=gen, device="cuda").double()
    x = (torch.randn(rows, k, generator=gen, device="cuda").double() * 2.0**ex).to(torch_type(kind))
    w = (torch.randn(1, k, n, generator=gen, device="cuda").double() * 2.0**-ex[:, None]).to(torch_type(kind))
    y = torch.empty(rows, n, device="cuda")
    off = offsets_of([rows])
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 1, rows, k, n, type=code(kind), out_type=binding.F32)
    close(y, x.double() @ w[0].double(), x.double().abs() @ w[0].double().abs(), k)


@pytest.mark.parametrize("kind", NAMES)
def test_infinities_and_nan_stay_where_the_formula_has_them(h, kind):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(6)
    for k, n in ((64, 80), (37, 21)):
        x = torch.randn(200, k, generator=gen, device="cuda").to(torch_type(kind))
        w = torch.randn(3, k, n, generator=gen, device="cuda").to(torch_type(kind))
        x[3, 5], x[120, 0], x[199, k - 1] = float("inf"), float("nan"), float("-inf")
        w[1, 2, 7] = float("inf")
        y = torch.empty(200, n, dtype=torch_type(kind), device="cuda")
        off = offsets_of([50, 100, 50])
        h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 3, 200, k, n, type=code(kind))
        bad = torch.zeros(200, n, dtype=torch.bool, device="cuda")
        bad[[3, 120, 199]] = True
        bad[50:150, 7] = True
        assert bool((~torch.isfinite(y) == bad).all())
        dw = torch.empty(3, k, n, dtype=torch_type(kind), device="cuda")
        dy = torch.randn(200, n, generator=gen, device="cuda").to(torch_type(kind))
        h.grouped_product_tn(x.data_ptr(), dy.data_ptr(), dw.data_ptr(), off.data_ptr(), 3, 200, k, n, type=code(kind))
        bad = torch.zeros(3, k, n, dtype=torch.bool, device="cuda")
        bad[0, 5] = bad[1, 0] = bad[2, k - 1] = True
        assert bool((~torch.isfinite(dw) == bad).all())


def test_offsets_outside_of_the_rows_are_cut(h):
    """Negative, descending and too large offsets touch no row outside of the matrices and own no row twice."""
    import torch
    x = torch.randn(100, 16, device="cuda")
    w = torch.randn(4, 16, 8, device="cuda")
    y = torch.full((130, 8), 7.0, device="cuda")
    off = torch.tensor([-50, 20, 10, 60, 1000], dtype=torch.int32, device="cuda")
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 4, 100, 16, 8)
    dw = torch.empty(4, 16, 8, device="cuda")
    dy = torch.randn(100, 8, device="cuda")
    h.grouped_product_tn(x.data_ptr(), dy.data_ptr(), dw.data_ptr(), off.data_ptr(), 4, 100, 16, 8)
    torch.cuda.synchronize()
    d = lambda a, b: a.double() @ b.double()  # noqa: E731
    close(y[:10], d(x[:10], w[0]), d(x[:10].abs(), w[0].abs()), 16)
    close(y[20:60], d(x[20:60], w[2]), d(x[20:60].abs(), w[2].abs()), 16)
    close(y[60:100], d(x[60:], w[3]), d(x[60:].abs(), w[3].abs()), 16)
    assert bool((y[100:] == 7).all())
    for g, (lo, hi) in enumerate(((0, 20), (20, 20), (10, 60), (60, 100))):
        close(dw[g], d(x[lo:hi].T, dy[lo:hi]), d(x[lo:hi].T.abs(), dy[lo:hi].abs()), 50)


def test_no_rows(h):
    import torch
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    h.grouped_product(0, 0, 0, off.data_ptr(), 3, 0, 8, 8)
    dw = torch.full((3, 8, 16), 7.0, device="cuda")
    h.grouped_product_tn(0, 0, dw.data_ptr(), off.data_ptr(), 3, 0, 8, 16)
    torch.cuda.synchronize()
    assert bool((dw == 0).all())
    y = torch.full((5, 8), 7.0, device="cuda")
    x, w = torch.ones(5, 8, device="cuda"), torch.ones(3, 8, 8, device="cuda")
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 3, 5, 8, 8)
    torch.cuda.synchronize()
    assert bool((y == 7).all())


def test_communities_are_the_groups_without_offsets():
    import torch
    community = np.array([2, 0, 1, 1, 0, 2, 2, 0, 1, 2])
    g = trainer(n=10, community=community)
    try:
        perm, ptr = g.index("perm"), g.index("comm_ptr")
        x, w = torch.randn(10, 12, device="cuda"), torch.randn(3, 12, 9, device="cuda")
        rows = x[torch.from_numpy(perm).long().cuda()].contiguous()
        y, dw = torch.empty(10, 9, device="cuda"), torch.empty(3, 12, 9, device="cuda")
        g.grouped_product(rows.data_ptr(), w.data_ptr(), y.data_ptr(), None, 3, 10, 12, 9)
        g.grouped_product_tn(rows.data_ptr(), y.data_ptr(), dw.data_ptr(), None, 3, 10, 12, 9)
        for i, node in enumerate(perm):
            a, b = x[int(node)][None].double(), w[int(community[node])].double()
            close(y[i:i + 1], a @ b, a.abs() @ b.abs(), 12)
        for c in range(3):
            a, b = rows[ptr[c]:ptr[c + 1]].double(), y[ptr[c]:ptr[c + 1]].double()
            close(dw[c], a.T @ b, a.abs().T @ b.abs(), 10)
        for bad in (dict(n_groups=2, rows=10), dict(n_groups=3, rows=9)):
            with pytest.raises(binding.GcnAdmmError) as e:
                g.grouped_product(rows.data_ptr(), w.data_ptr(), y.data_ptr(), None, bad["n_groups"], bad["rows"], 12, 9)
            assert e.value.code == -1
    finally:
        g.destroy()


def test_refusals_leave_the_handle_usable(h):
    import torch
    x, w, y = torch.ones(4, 8, device="cuda"), torch.ones(1, 8, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    off = offsets_of([4])
    host = np.ones((4, 8), dtype=np.float32)
    a = dict(x_dev=x.data_ptr(), w_dev=w.data_ptr(), y_dev=y.data_ptr(), offsets_dev=off.data_ptr(), n_groups=1, rows=4, k=8, n=8)
    for change in (dict(x_dev=host.ctypes.data), dict(y_dev=0), dict(n_groups=0), dict(type=5), dict(ldx=7), dict(offsets_dev=host.ctypes.data),
                   dict(offsets_dev=off.data_ptr() + 2), dict(x_dev=x.data_ptr() + 1), dict(k=0), dict(out_type=binding.F16)):
        with pytest.raises(binding.GcnAdmmError) as e:
            h.grouped_product(**{**a, **change})
        assert e.value.code == -1 and str(e.value)
    with pytest.raises(binding.GcnAdmmError):
        h.orthogonalise(x.data_ptr(), y.data_ptr(), 1, 4, 8, [(5.0, 0.0, 0.0)] * 3)
    with pytest.raises(binding.GcnAdmmError):
        h.orthogonalise(host.ctypes.data, y.data_ptr(), 1, 4, 8, [MUON])
    h.grouped_product(**a)
    torch.cuda.synchronize()
    assert bool((y == 8).all())


def test_offsets_past_32_bits(h):
    """Row numbers times strides pass 2^31 elements in every operand and result."""
    import torch
    ld, rows, k, n = (1 << 21) + 8, 1200, 40, 24
    held = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = held.as_strided((rows, k), (ld, 1))
    y = held[64:].as_strided((rows, n), (ld, 1))
    gen = torch.Generator(device="cuda").manual_seed(3)
    x.copy_(torch.randn(rows, k, generator=gen, device="cuda"))
    y.fill_(7)
    w = torch.randn(2, k, n, generator=gen, device="cuda").bfloat16()
    off = offsets_of([500, 650])
    h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 2, rows, k, n, type=binding.BF16, ldx=ld, ldy=ld)
    torch.cuda.synchronize()
    for g, (lo, hi) in enumerate(((0, 500), (500, 1150))):
        a, b = x[lo:hi].double(), w[g].double()
        close(y[lo:hi].contiguous(), a @ b, a.abs() @ b.abs(), k)
    assert bool((y[1150:] == 7).all())
    far = held.as_strided((2, k, n), (ld * 700, ld, 1))          # weights and gradients that far apart
    dw = torch.empty(2, k, n, device="cuda")
    h.grouped_product_tn(x.data_ptr(), y.data_ptr(), dw.data_ptr(), off.data_ptr(), 2, rows, k, n, type=binding.BF16, out_type=binding.F32, ldx=ld, ldy=ld)
    for g, (lo, hi) in enumerate(((0, 500), (500, 1150))):
        a, b = x[lo:hi].double(), y[lo:hi].double()
        close(dw[g], a.T @ b, a.T.abs() @ b.abs(), hi - lo)
    far.copy_(w)
    z = torch.empty(rows, n, device="cuda")
    xc = torch.randn(rows, k, generator=gen, device="cuda").bfloat16()
    h.grouped_product(xc.data_ptr(), far.data_ptr(), z.data_ptr(), off.data_ptr(), 2, rows, k, n, type=binding.BF16, out_type=binding.F32, ldw=ld, stride_w=ld * 700)
    for g, (lo, hi) in enumerate(((0, 500), (500, 1150))):
        a, b = xc[lo:hi].double(), w[g].double()
        close(z[lo:hi], a @ b, a.abs() @ b.abs(), k)


# ---- orthogonalised updates -------------------------------------------------------------------------

def newton_schulz(g, coefficients, eps, scale):
    """The definition, in fp64."""
    import torch
    x = g.double()
    turn = x.shape[-2] > x.shape[-1]
    x = x.mT if turn else x
    norm = torch.linalg.norm(x, dim=(-2, -1), keepdim=True) + eps
    x = torch.where(norm > 0, x / norm, 0.0)
    for a, b, c in coefficients:
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    x = scale * x
    return x.mT if turn else x


def gradient(batch, rows, cols, kind, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g = torch.randn(batch, rows, cols, generator=gen, device="cuda")
    g += torch.randn(batch, rows, 3, generator=gen, device="cuda") @ torch.randn(batch, 3, cols, generator=gen, device="cuda")
    return (g * 1e-3).to(torch_type(kind))


def ortho_tolerance(g, coefficients, dtype, eps=1e-7):
    """Bound of ||error|| / ||X||.  A step's products are held to u = 2^-19 of their terms (sums of at most 256 products cut toward zero 16 times
    at 2^-23, and added; pairs hold the operands to 2^-22).  These errors have no direction of their own: they spread evenly over the singular
    directions.  An error along direction i is multiplied by |a + 3 b s_i^2 + 5 c s_i^4| in a step, the derivative of s (a + b s^2 + c s^4); parts that
    mix two directions by the divided difference of that map, which lies between derivatives of its interval.  Factor 2 for these.
    bf16 results come from products of halves with the diagonals apart: 2^-12 at most of every element off the diagonals, which is 0.5 to 1.3e-3 of the result
    and has its place between the rounding of a result, 1.7e-3 in the mean (a uniform error of half a step, over sqrt(3)), and eps / 2."""
    import torch
    x = newton_schulz(g, [], eps, 1.0)
    s = torch.linalg.svdvals(x).reshape(-1)
    e = torch.full_like(s, 2.0**-24) * s
    for a, b, c in coefficients:
        gain = (a + 3 * b * s**2 + 5 * c * s**4).abs()
        new = 2.0**-19 * (abs(a) * s + abs(b) * s**3 + abs(c) * s**5).square().mean().sqrt()
        e = gain * e + new
        s = s * (a + b * s**2 + c * s**4)
    return 2 * float(e.norm() / s.norm()) + torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("kind", NAMES)
@pytest.mark.parametrize("batch, rows, cols", [(1, 1, 1), (2, 1, 9), (3, 5, 1), (5, 16, 7), (8, 128, 16), (2, 64, 64), (1, 65, 130), (3, 100, 47),
                                               (1, 128, 256), (2, 129, 128), (1, 257, 300), (1, 500, 128), (1, 300, 767),
                                               (4, 8, 5000), (3, 32, 1100), (3, 1000, 31), (2, 2000, 16), (2, 33, 1000), (2, 24, 1500), (300, 12, 20)])
def test_orthogonalise(h, kind, batch, rows, cols):
    import torch
    for out in {kind, "f32"}:
        for coefficients in ([MUON] * 5, [], [(1.875, -1.25, 0.375)] * 3, [(2.0, -1.5, 0.5), (0.5, 0.0, 0.0)]):
            g = gradient(batch, rows, cols, kind, seed=rows + cols)
            x = torch.full((batch, rows, cols), float("nan"), dtype=torch_type(out), device="cuda")
            h.orthogonalise(g.data_ptr(), x.data_ptr(), batch, rows, cols, coefficients, eps=1e-7, scale=0.2, type=code(kind), out_type=code(out))
            want = newton_schulz(g, coefficients, 1e-7, 0.2)
            rel = float((x.double() - want).norm() / want.norm())
            assert rel < ortho_tolerance(g, coefficients, x.dtype), (out, coefficients, rel)


@pytest.mark.parametrize("kind", NAMES)
@pytest.mark.parametrize("batch, rows, cols", [(16, 600, 700), (16, 712, 600), (10, 600, 640), (10, 640, 602), (1, 1500, 1400)])
def test_orthogonalise_larger_ones(h, kind, batch, rows, cols):
    """Enough tiles for the wider ones, in both orientations."""
    import torch
    g = gradient(batch, rows, cols, kind, seed=rows)
    x = torch.empty_like(g)
    h.orthogonalise(g.data_ptr(), x.data_ptr(), batch, rows, cols, [MUON] * 5, scale=0.2, type=code(kind))
    want = newton_schulz(g, [MUON] * 5, 1e-7, 0.2)
    for i in range(batch):
        rel = float((x[i].double() - want[i]).norm() / want[i].norm())
        assert rel < ortho_tolerance(g[i:i + 1], [MUON] * 5, x.dtype), (i, rel)


def test_orthogonalise_of_spread_singular_values(h):
    """A few strong directions above a weak floor, which the steps lift most: half of a bf16 result's tolerance is left for its rounding, 1.7e-3 in the mean."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    for m, n in ((300, 700), (640, 200)):
        g = torch.randn(1, m, 20, generator=gen, device="cuda") @ torch.randn(1, 20, n, generator=gen, device="cuda")
        g = (g + 1e-3 * torch.randn(1, m, n, generator=gen, device="cuda")).bfloat16()
        x = torch.empty_like(g)
        h.orthogonalise(g.data_ptr(), x.data_ptr(), 1, m, n, [MUON] * 5, type=binding.BF16)
        want = newton_schulz(g, [MUON] * 5, 1e-7, 1.0)
        assert float((x.double() - want).norm() / want.norm()) < torch.finfo(x.dtype).eps / 2


@pytest.mark.parametrize("kind", NAMES)
def test_orthogonalise_layouts(h, kind):
    import torch
    for rows, cols in ((72, 136), (61, 30)):
        for pad, shift, gap in ((8, 0, 8), (3, 1, 5)):
            src = Matrix(3, rows, cols, kind, pad, shift, gap)
            src.view.copy_(gradient(3, rows, cols, kind, 4))
            dst = Matrix(3, rows, cols, kind, pad + 1, shift, gap, fill=7.0)
            args = dict(eps=1e-7, scale=1.0, type=code(kind), ldg=src.ld, stride_g=src.stride)
            h.orthogonalise(src.at, dst.at, 3, rows, cols, [MUON] * 3, ldo=dst.ld, stride_o=dst.stride, **args)
            src_values = src.view.clone()
            want = newton_schulz(src_values, [MUON] * 3, 1e-7, 1.0)
            assert float((dst.view.double() - want).norm() / want.norm()) < ortho_tolerance(src_values, [MUON] * 3, torch_type(kind))
            assert dst.outside_is_untouched()
            h.orthogonalise(src.at, src.at, 3, rows, cols, [MUON] * 3, ldo=src.ld, stride_o=src.stride, **args)       # in place
            torch.cuda.synchronize()
            assert bool((src.view == dst.view).all()) and src.outside_is_untouched()


def test_orthogonalise_edges(h):
    """Zero, non-finite, very large and very small matrices of one batch keep to themselves."""
    import torch
    for rows, cols in ((40, 24), (150, 200)):
        g = gradient(6, rows, cols, "f32", 9)
        g[1] = 0
        g[2, 3, 5] = float("nan")
        g[3, 0, 0] = float("inf")
        g[4] *= 1e33
        g[5] *= 1e-33
        x = torch.empty_like(g)
        h.orthogonalise(g.data_ptr(), x.data_ptr(), 6, rows, cols, [MUON] * 5, eps=0.0)
        want = newton_schulz(g, [MUON] * 5, 0.0, 1.0)
        assert bool((x[1] == 0).all()) and bool(torch.isnan(x[2]).all()) and bool(torch.isnan(x[3]).all())
        for i in (0, 4, 5):
            rel = float((x[i].double() - want[i]).norm() / want[i].norm())
            assert rel < ortho_tolerance(g[i:i + 1], [MUON] * 5, x.dtype, 0.0), (i, rel)


# ---- streams, graphs, repetition --------------------------------------------------------------------

def test_same_bits_every_time(h):
    import torch
    x, w = torch.randn(3000, 136, device="cuda"), torch.randn(5, 136, 72, device="cuda")
    off = offsets_of([2500, 0, 100, 399, 1])
    made = []
    for kind in NAMES:
        a, b = x.to(torch_type(kind)), w.to(torch_type(kind))
        for _ in range(2):
            y, dw, o = torch.empty(3000, 72, dtype=a.dtype, device="cuda"), torch.empty(5, 136, 72, device="cuda"), torch.empty_like(b)
            h.grouped_product(a.data_ptr(), b.data_ptr(), y.data_ptr(), off.data_ptr(), 5, 3000, 136, 72, type=code(kind))
            h.grouped_product_tn(a.data_ptr(), y.data_ptr(), dw.data_ptr(), off.data_ptr(), 5, 3000, 136, 72, type=code(kind), out_type=binding.F32)
            h.orthogonalise(b.data_ptr(), o.data_ptr(), 5, 136, 72, [MUON] * 5, type=code(kind))
            torch.cuda.synchronize()
            made.append((y, dw, o))
        for p, q in zip(made[-1], made[-2]):
            assert torch.equal(p, q)


def test_captured_calls_replay_on_new_data():
    """Two graphs of one handle, its workspace grown between them, on a stream of its own; what the offsets hold may change between replays."""
    import torch
    s = torch.cuda.Stream()
    g = trainer(stream=s.cuda_stream)
    try:
        sizes = {}
        with torch.cuda.stream(s):
            for name, k, n, rows in (("small", 64, 48, 500), ("large", 768, 520, 3001)):
                x, w, y = torch.randn(rows, k, device="cuda"), torch.randn(3, k, n, device="cuda"), torch.zeros(rows, n, device="cuda")
                dw, o, off = torch.empty(3, k, n, device="cuda"), torch.empty(3, k, n, device="cuda"), offsets_of([rows // 2, 0, rows - rows // 2])

                def calls():
                    g.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 3, rows, k, n)
                    g.grouped_product_tn(x.data_ptr(), y.data_ptr(), dw.data_ptr(), off.data_ptr(), 3, rows, k, n)
                    g.orthogonalise(dw.data_ptr(), o.data_ptr(), 3, k, n, [MUON] * 5)
                if name == "large":      # nothing has made room for it
                    graph = torch.cuda.CUDAGraph()
                    with pytest.raises(binding.GcnAdmmError) as e:
                        with torch.cuda.graph(graph, stream=s, capture_error_mode="thread_local"):
                            g.orthogonalise(dw.data_ptr(), o.data_ptr(), 3, k, n, [MUON] * 5)
                    assert e.value.code == -1 and "workspace" in str(e.value)
                calls()
                s.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s, capture_error_mode="thread_local"):
                    calls()
                sizes[name] = (graph, x, w, y, dw, o, off, rows, k)
            for name in ("large", "small", "large", "small"):
                graph, x, w, y, dw, o, off, rows, k = sizes[name]
                x.normal_()
                cut = int(torch.randint(0, rows, (1,)))
                off.copy_(offsets_of([cut, 0, rows - cut]))
                graph.replay()
                s.synchronize()
                for i, (lo, hi) in enumerate(((0, cut), (cut, cut), (cut, rows))):
                    a, b = x[lo:hi].double(), w[i].double()
                    close(y[lo:hi], a @ b, a.abs() @ b.abs(), k)
                    b = y[lo:hi].double()
                    close(dw[i], a.T @ b, a.T.abs() @ b.abs(), max(1, hi - lo))
                want = newton_schulz(dw, [MUON] * 5, 1e-7, 1.0)
                assert float((o.double() - want).norm() / want.norm()) < ortho_tolerance(dw, [MUON] * 5, o.dtype)
        sizes.clear()
    finally:
        s.synchronize()
        g.destroy()


def test_calls_are_counted_and_timed(h):
    import torch
    x, w, y, off = torch.randn(40, 24, device="cuda"), torch.randn(2, 24, 16, device="cuda"), torch.empty(40, 16, device="cuda"), offsets_of([25, 15])
    dw = torch.empty_like(w)

    def calls():
        h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 2, 40, 24, 16)
        h.grouped_product_tn(x.data_ptr(), y.data_ptr(), dw.data_ptr(), off.data_ptr(), 2, 40, 24, 16)
        h.orthogonalise(dw.data_ptr(), dw.data_ptr(), 2, 24, 16, [MUON] * 5)
    calls()
    before = h.launches()
    h.profile(True)
    calls()
    got = h.profile_read()
    h.profile(False)
    for name in ("grouped@24x16", "grouped_tn@24x16", "orthogonalise@24x16"):
        assert got[name]["launches"] >= 1 and got[name]["ms"] > 0 and got[name]["flops"] > 0, got
    assert h.launches() - before == sum(v["launches"] for v in got.values())


def test_a_first_call_may_be_captured():
    """Where no workspace is needed nothing has to have run before."""
    import torch
    s = torch.cuda.Stream()
    g = trainer(stream=s.cuda_stream)
    try:
        with torch.cuda.stream(s):
            x, w = torch.randn(300, 72, device="cuda").half(), torch.randn(2, 72, 40, device="cuda").half()
            y, off = torch.zeros(300, 40, device="cuda"), offsets_of([100, 200])
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s, capture_error_mode="thread_local"):
                g.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 2, 300, 72, 40, type=binding.F16, out_type=binding.F32)
            graph.replay()
            s.synchronize()
        for i, (lo, hi) in enumerate(((0, 100), (100, 300))):
            a, b = x[lo:hi].double(), w[i].double()
            close(y[lo:hi], a @ b, a.abs() @ b.abs(), 72)
        del graph
    finally:
        s.synchronize()
        g.destroy()


def test_a_growing_workspace_holds_a_bounded_amount():
    """Calls that need a little more every time: the outgrown workspaces together are no more than twice the last one, and go with the handle."""
    import torch
    g = trainer()
    try:
        last = torch.randn(1, 2048, 2048, device="cuda")
        out = torch.empty_like(last)
        free = torch.cuda.mem_get_info()[0]
        for side in range(256, 2049, 64):
            g.orthogonalise(last.data_ptr(), out.data_ptr(), 1, side, side, [MUON], ldg=2048, ldo=2048)
        torch.cuda.synchronize()
        # images of X twice, S and P, two halves an element, and grain; half as much again as the step before may have taken
        largest = 4 * 2 * 2 * 2048 * 2048
        assert free - torch.cuda.mem_get_info()[0] <= 3 * 1.5 * largest + (64 << 20)
        want = newton_schulz(last, [MUON], 1e-7, 1.0)
        assert float((out.double() - want).norm() / want.norm()) < ortho_tolerance(last, [MUON], out.dtype)
    finally:
        g.destroy()


def test_two_handles_at_once():
    """Handles on streams of their own share nothing: the same calls side by side give what they give alone."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = [trainer(stream=s.cuda_stream) for s in streams]
    try:
        x, w = torch.randn(5000, 200, device="cuda"), torch.randn(3, 200, 264, device="cuda")
        off = offsets_of([2000, 2900, 100])
        results = []
        torch.cuda.synchronize()
        for _ in range(3):
            outs = []
            for g in made:
                y, dw, o = torch.empty(5000, 264, device="cuda"), torch.empty(3, 200, 264, device="cuda"), torch.empty(3, 200, 264, device="cuda")
                torch.cuda.synchronize()
                outs.append((y, dw, o))
            for g, (y, dw, o) in zip(made, outs):
                g.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), 3, 5000, 200, 264)
                g.grouped_product_tn(x.data_ptr(), y.data_ptr(), dw.data_ptr(), off.data_ptr(), 3, 5000, 200, 264)
                g.orthogonalise(dw.data_ptr(), o.data_ptr(), 3, 200, 264, [MUON] * 5)
            torch.cuda.synchronize()
            results += outs
        for other in results[1:]:
            for p, q in zip(results[0], other):
                assert torch.equal(p, q)
    finally:
        for g in made:
            g.destroy()


# ---- used together ----------------------------------------------------------------------------------

@pytest.mark.parametrize("kind, out", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
def test_gradients_agree_with_differences(h, kind, out):
    """L = sum of r * (x W): along a direction, the difference of L is the product of the gradient with it (L is linear in x and in W)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(11)
    k, n, sizes = 72, 56, [90, 0, 33, 1]
    rows, groups = sum(sizes), len(sizes)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch_type(kind))  # noqa: E731
    x, w, r = make(rows, k), make(groups, k, n), make(rows, n)
    off = offsets_of(sizes)
    t = dict(type=code(kind), out_type=code(out))

    def loss(x, w):
        y = torch.empty(rows, n, device="cuda")
        h.grouped_product(x.data_ptr(), w.data_ptr(), y.data_ptr(), off.data_ptr(), groups, rows, k, n, type=code(kind), out_type=binding.F32)
        return y.double()
    dx, dw = torch.empty(rows, k, dtype=torch_type(out), device="cuda"), torch.empty(groups, k, n, dtype=torch_type(out), device="cuda")
    h.grouped_product(r.data_ptr(), w.data_ptr(), dx.data_ptr(), off.data_ptr(), groups, rows, n, k, transpose_w=True, **t)
    h.grouped_product_tn(x.data_ptr(), r.data_ptr(), dw.data_ptr(), off.data_ptr(), groups, rows, k, n, **t)
    base, R = loss(x, w), r.double()
    for which in ("x", "w"):
        other = make(*(x.shape if which == "x" else w.shape))
        moved = loss(other, w) if which == "x" else loss(x, other)
        terms = R * (moved - base)
        step = (other.double() - x.double(), dx.double()) if which == "x" else (other.double() - w.double(), dw.double())
        got = (step[0] * step[1]).sum()
        # each side's terms are off by the tolerance of its outputs
        K = k if which == "w" else max(k, n)
        slack = (40 + K / 256) * 2.0**-23 * 4
        unit = torch.finfo(torch_type(out)).eps / 2 + slack * 8
        lim = slack * (R.abs() * (moved.abs() + base.abs() + 8 * k**0.5)).sum() + unit * (step[0].abs() * step[1].abs()).sum()
        assert abs(float(terms.sum() - got)) <= float(lim)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_training_steps_of_two_layers_of_experts(h, kind):
    """Forward, both gradients through a ReLU, and the orthogonalised update of both layers' weights, three steps, against fp64 from the
    same state of every step."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(21)
    sizes, widths = [130, 0, 61, 9], (64, 96, 24)
    rows, groups = sum(sizes), len(sizes)
    t = torch_type(kind)
    off = offsets_of(sizes)
    x = torch.randn(rows, widths[0], generator=gen, device="cuda").to(t)
    want_y = torch.randn(rows, widths[2], generator=gen, device="cuda").to(t)
    ws = [torch.randn(groups, a, b, generator=gen, device="cuda") * a**-0.5 for a, b in zip(widths, widths[1:])]
    spans = [(int(a), int(b)) for a, b in zip(off[:-1], off[1:])]
    each = lambda a, f: torch.cat([f(a[lo:hi].double(), g) for g, (lo, hi) in enumerate(spans)])  # noqa: E731
    eps = torch.finfo(t).eps
    for _ in range(3):
        w = [v.to(t) for v in ws]
        a1, a2 = torch.empty(rows, widths[1], dtype=t, device="cuda"), torch.empty(rows, widths[2], dtype=t, device="cuda")
        o = off.data_ptr()
        h.grouped_product(x.data_ptr(), w[0].data_ptr(), a1.data_ptr(), o, groups, rows, widths[0], widths[1], type=code(kind))
        z = torch.relu(a1)
        h.grouped_product(z.data_ptr(), w[1].data_ptr(), a2.data_ptr(), o, groups, rows, widths[1], widths[2], type=code(kind))
        d2 = (a2 - want_y).contiguous()
        dz = torch.empty(rows, widths[1], dtype=t, device="cuda")
        h.grouped_product(d2.data_ptr(), w[1].data_ptr(), dz.data_ptr(), o, groups, rows, widths[2], widths[1], type=code(kind), transpose_w=True)
        d1 = (dz * (a1 > 0)).contiguous()
        dw = [torch.empty_like(v) for v in ws]
        h.grouped_product_tn(x.data_ptr(), d1.data_ptr(), dw[0].data_ptr(), o, groups, rows, widths[0], widths[1], type=code(kind), out_type=binding.F32)
        h.grouped_product_tn(z.data_ptr(), d2.data_ptr(), dw[1].data_ptr(), o, groups, rows, widths[1], widths[2], type=code(kind), out_type=binding.F32)
        steps = [torch.empty_like(v) for v in ws]
        for d, s in zip(dw, steps):
            h.orthogonalise(d.data_ptr(), s.data_ptr(), groups, d.shape[1], d.shape[2], [MUON] * 5, scale=0.05)
        torch.cuda.synchronize()
        # the whole chain in fp64; what a stage is off passes on through at most three products of norms of a few units
        A1 = each(x, lambda r, g: r @ w[0][g].double())
        on = A1 > 0
        A2 = each(torch.relu(A1), lambda r, g: r @ w[1][g].double())
        D2 = A2 - want_y.double()
        D1 = each(D2, lambda r, g: r @ w[1][g].double().T) * on
        full = [torch.stack([u[lo:hi].double().T @ v[lo:hi] for lo, hi in spans]) for u, v in ((x, D1), (torch.relu(A1), D2))]
        lim = 8 * eps + 1e-5
        for d, f in zip(dw, full):
            assert float((d.double() - f).norm() / f.norm()) < lim
            assert bool((d[1] == 0).all())
        for d, s in zip(dw, steps):
            ref = newton_schulz(d, [MUON] * 5, 1e-7, 0.05)
            assert float((s.double() - ref).norm() / ref.norm()) < ortho_tolerance(d, [MUON] * 5, s.dtype)
            assert bool((s[1] == 0).all())
        ws = [v - s for v, s in zip(ws, steps)]
