"""stx_rmsnorm and its backward pass against 64 bits: types, widths around every variant's border, strides, 8-bit output."""
import numpy as np
import pytest
import torch

from paper_2502_16949_amd import binding as B
from tests import gpu_util as G
from tests import ops_ref as R

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# roundings of a row's sum of squares: the square, 64 additions in a thread, 9 over threads, the division and eps; its root halves
# them, then the root and the reciprocal.  y: two products more.
RSTD = (0.5 * (1 + 64 + 9 + 2) + 2) * R.U
Y = RSTD + 2 * R.U


@pytest.fixture(scope="module")
def ctx():
    return B.Context(B.make_config("transe", "l2", 100, 5, 32, 64, 1), G.DEV)


def rows_of(rng, rows, cols, dtype, ld=None, offset=0):
    """A [rows, cols] matrix inside a larger allocation: row stride ld, first element `offset` elements into it."""
    ld = ld or cols
    room = torch.full((offset + rows * ld + 8,), float("nan"), dtype=dtype, device=G.DEV)
    t = room[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    t.copy_(torch.from_numpy(rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal((rows, 1)))))
    return t


SHAPES = [(1, 1), (3, 7), (1, 128), (5, 129), (17, 128), (33, 200), (9, 256), (4, 257), (6, 512), (5, 513), (300, 1001), (7, 1024),
          (3, 1025), (2, 2048), (3, 2049), (2, 4100), (1, 8190), (2, 8193), (1, 16384), (2000, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_backward(ctx, rows, cols, dtype):
    rng = np.random.default_rng(rows * 31 + cols)
    ld, off = (cols + 5, 3) if cols % 2 else (cols, 0)
    x, res, dy, dsum = (rows_of(rng, rows, cols, dtype, ld, off) for _ in range(4))
    w = torch.from_numpy(1 + 0.1 * rng.standard_normal(cols)).float().to(G.DEV)
    total, y, dx = (rows_of(rng, rows, cols, dtype, ld, off).fill_(7.0) for _ in range(3))
    rstd = torch.empty(rows, device=G.DEV)
    q = B.Q8(rows, cols, B.STX_E4M3, G.DEV)
    q.codes.fill_(255)
    eps = 1e-6
    B.stx_rmsnorm(ctx, x, res, w, eps, total, y, q, rstd)
    s, want_y, want_rstd = R.rmsnorm(x, res, w, eps)
    assert torch.equal(total, s)
    assert np.all(np.abs(R.f64(rstd) / want_rstd - 1) <= RSTD)
    half = R.HALF[dtype]
    tiny = 2.0**-25 if dtype == torch.float16 else 0.0       # half a step of fp16's subnormals
    assert np.all(np.abs(R.f64(y) - want_y) <= (Y + half) * np.abs(want_y) + tiny)
    R.check_q8(q, want_y, Y)
    dw = torch.full((cols,), float("nan"), device=G.DEV)
    work = torch.empty(B.stx_rmsnorm_backward_work_bytes(ctx, rows, cols) + 256, dtype=torch.uint8, device=G.DEV)
    B.stx_rmsnorm_backward(ctx, total, w, rstd, dy, dsum, dx, dw, work)
    want, want_dw, size, size_dw = R.rmsnorm_backward(s, w, eps, dy, dsum)
    assert np.all(np.abs(R.f64(dx) - want) <= R.U * size + 3 * RSTD * size + half * np.abs(want) + tiny)
    adds = rows // 1024 + 16 + 64 + 16 + 4                   # rows of a thread, groups, parts of a slice, slices, products
    assert np.all(np.abs(R.f64(dw) - want_dw) <= (adds * R.U + RSTD) * size_dw)
    # what lies between the rows stays as it was
    if ld > cols:
        for t in (total, y, dx):
            assert torch.isnan(t.as_strided((rows, ld - cols), (ld, 1), t.storage_offset() + cols)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_optional_arguments_and_shared_memory(ctx, dtype):
    rng = np.random.default_rng(3)
    rows, cols = 37, 300
    x, res, dy = (rows_of(rng, rows, cols, dtype) for _ in range(3))
    eps = 1e-5
    ones = torch.ones(cols, device=G.DEV)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    rstd = torch.empty(rows, device=G.DEV)
    B.stx_rmsnorm(ctx, x, None, ones, eps, None, y0, None, rstd)
    B.stx_rmsnorm(ctx, x, None, None, eps, None, y1, None, None)
    assert torch.equal(y0, y1)
    # the sum in place of the residual, and of x
    a, b = x.clone(), res.clone()
    B.stx_rmsnorm(ctx, x, b, None, eps, b, y0, None, None)
    B.stx_rmsnorm(ctx, a, res, None, eps, a, y1, None, None)
    assert torch.equal(a, b) and torch.equal(y0, y1) and torch.equal(a, (x.float() + res.float()).to(dtype))
    # only the sum; a gradient in place of dy, without weight, dsum and dweight
    c = torch.empty_like(x)
    B.stx_rmsnorm(ctx, x, res, None, eps, c, None, None, None)
    assert torch.equal(a, c)
    d0, d1 = torch.empty_like(x), dy.clone()
    zero = torch.zeros_like(x)
    B.stx_rmsnorm_backward(ctx, x, ones, rstd, dy, zero, d0, None)
    B.stx_rmsnorm_backward(ctx, x, None, rstd, d1, None, d1, None)
    assert torch.equal(d0, d1)


def test_gradient_against_differences(ctx):
    # dL/dx of L = sum(y * dy) + sum(s * dsum): central differences in 64 bits of the formula
    rng = np.random.default_rng(9)
    rows, cols, eps = 3, 40, 1e-3
    x, dy, dsum = (rows_of(rng, rows, cols, torch.float32) for _ in range(3))
    w = torch.from_numpy(1 + 0.3 * rng.standard_normal(cols)).float().to(G.DEV)
    rstd, y, dx, dw = torch.empty(rows, device=G.DEV), torch.empty_like(x), torch.empty_like(x), torch.empty(cols, device=G.DEV)
    work = torch.empty(B.stx_rmsnorm_backward_work_bytes(ctx, rows, cols) + 256, dtype=torch.uint8, device=G.DEV)
    B.stx_rmsnorm(ctx, x, None, w, eps, None, y, None, rstd)
    B.stx_rmsnorm_backward(ctx, x, w, rstd, dy, dsum, dx, dw, work)

    def loss(xx, ww):
        r = 1 / np.sqrt((xx * xx).mean(1, keepdims=True) + eps)
        return (xx * r * ww * R.f64(dy)).sum() + (xx * R.f64(dsum)).sum()

    x0, w0, h = R.f64(x), R.f64(w), 1e-5
    for i, j in [(0, 0), (1, 17), (2, 39), (0, 20)]:
        e = np.zeros_like(x0)
        e[i, j] = h
        d = (loss(x0 + e, w0) - loss(x0 - e, w0)) / (2 * h)
        assert abs(d - float(dx[i, j])) <= 1e-5 * (1 + abs(d))      # differences: h^2 of the third derivative and 1e-16 / h
        f = np.zeros_like(w0)
        f[j] = h
        d = (loss(x0, w0 + f) - loss(x0, w0 - f)) / (2 * h)
        assert abs(d - float(dw[j])) <= 1e-5 * (1 + abs(d))


def test_rows_that_are_zero_or_not_finite(ctx):
    x = torch.randn(6, 256, device=G.DEV)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 200] = float("inf")
    y, rstd, q = torch.empty_like(x), torch.empty(6, device=G.DEV), B.Q8(6, 256, B.STX_E4M3, G.DEV)
    B.stx_rmsnorm(ctx, x, None, None, 1e-6, None, y, q, rstd)
    assert not y[1].any() and not q.codes[1].any() and (q.scales[1, :2] == 127).all() and float(rstd[1]) == pytest.approx(1e3, rel=1e-6)
    assert y[2].isnan().all() and ((q.codes[2] & 0x7F) == 0x7F).all()
    assert float(rstd[3]) == 0 and y[3, 200].isnan() and not y[3, :200].any()
    _, want, _ = R.rmsnorm(x[[0, 4, 5]], None, None, 1e-6)
    assert np.all(np.abs(R.f64(y[[0, 4, 5]]) - want) <= (Y + R.U) * np.abs(want))


def test_no_rows(ctx):
    x = torch.empty(0, 64, device=G.DEV)
    dw = torch.full((64,), 5.0, device=G.DEV)
    B.stx_rmsnorm(ctx, x, None, None, 1e-6, None, x, None, None)
    B.stx_rmsnorm_backward(ctx, x, None, torch.empty(0, device=G.DEV), x, None, x, dw, torch.empty(256, dtype=torch.uint8, device=G.DEV))
    assert not dw.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 5, 100, 130, 200, 300, 700, 1001, 2000, 4001, 8001, 8300])
def test_codes_behind_the_last_column_are_zeros(ctx, cols, dtype):
    # whatever a row holds: NaN, infinity (rstd 0), nothing but zeros without eps (rstd infinite), a weight that is not finite
    x = torch.randn(7, cols, device=G.DEV).to(dtype)
    x[1, cols // 2], x[2, 0], x[3], x[4, cols - 1] = float("nan"), float("inf"), 0, float("-inf")
    w = torch.ones(cols, device=G.DEV)
    w[cols - 1] = float("inf")
    for weight in (None, w):
        for fmt in (B.STX_E4M3, B.STX_E5M2):
            q = B.Q8(7, cols, fmt, G.DEV)
            q.codes.fill_(0x55)
            B.stx_rmsnorm(ctx, x, None, weight, 0.0, None, None, q, None)
            assert not q.codes[:, cols:].any()
            # all of a row that is NaN or 0 / 0 is NaN codes
            bad = 0x7F if fmt == B.STX_E4M3 else 0x7C
            for row in (1, 3):
                assert ((q.codes[row, :cols] & 0x7F) >= bad).all()


# more rows than the workgroups take at once, so that the next row is under way while this one's gradient is stored
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(40_003, 100), (20_001, 250), (9_001, 500), (5_001, 700), (2_101, 2000), (1_300, 4001), (900, 8000), (700, 9001)])
def test_backward_in_place_of_what_it_reads(ctx, rows, cols, dtype):
    rng = np.random.default_rng(rows)
    s, dy, dsum = (rows_of(rng, rows, cols, dtype) for _ in range(3))
    w = torch.from_numpy(1 + 0.1 * rng.standard_normal(cols)).float().to(G.DEV)
    rstd = torch.empty(rows, device=G.DEV)
    B.stx_rmsnorm(ctx, s, None, w, 1e-6, None, None, None, rstd)
    work = torch.empty(B.stx_rmsnorm_backward_work_bytes(ctx, rows, cols) + 256, dtype=torch.uint8, device=G.DEV)

    def backward(dy, dsum, dx):
        dw = torch.full((cols,), float("nan"), device=G.DEV)
        B.stx_rmsnorm_backward(ctx, s, w, rstd, dy, dsum, dx, dw, work)
        return dx, dw

    want = backward(dy, dsum, torch.empty_like(dy))
    for place in (0, 1):
        d = [dy.clone(), dsum.clone()]
        got = backward(*d, d[place])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    same = backward(dy, dy, torch.empty_like(dy))            # one gradient on both ways, and in its place
    d = dy.clone()
    got = backward(d, d, d)
    assert torch.equal(got[0], same[0]) and torch.equal(got[1], same[1])
