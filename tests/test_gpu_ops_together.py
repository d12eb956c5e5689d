"""RMS norm, rows and products in 8 bits, and AdamW as a program uses them together: a query's row against a whole table, its gradient,
the step; the same captured and replayed, on streams of their own; and sizes whose offsets pass 32 bits."""
import numpy as np
import pytest
import torch

from paper_2502_16949_amd import binding as B
from tests import gpu_util as G
from tests import ops_ref as R
from tests.test_gpu_adamw import H, check
from tests.test_gpu_norm import RSTD, Y, rows_of
from tests.test_gpu_q8 import _q8_of, check_product

pytestmark = pytest.mark.gpu
EPS = 1e-6


def context(stream=None):
    return B.Context(B.make_config("transe", "l2", 100, 5, 32, 64, 1), G.DEV, stream)


class Trainer:
    """Scores m queries of `dim` columns against a table of n rows; g holds the scores' gradient; a step moves table and weight."""

    def __init__(self, ctx, m, n, dim, bits, seed=0, step_dev=None):
        rng = np.random.default_rng(seed)
        t = lambda *s, dtype=torch.bfloat16: torch.from_numpy(rng.standard_normal(s)).to(G.DEV, dtype)  # noqa: E731
        e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device=G.DEV)  # noqa: E731
        f, q8 = torch.float32, lambda r, c: B.Q8(r, c, B.STX_E4M3, G.DEV)  # noqa: E731
        self.ctx, self.bits = ctx, bits
        self.h, self.r, self.g, self.dsum = t(m, dim), t(m, dim), t(m, n) * 1e-2, t(m, dim) * 1e-2
        self.weight, self.table = 1 + 0.1 * t(dim, dtype=f), t(n, dim, dtype=f)
        self.s, self.y, self.rstd, self.scores = e(m, dim), e(m, dim), e(m, dtype=f), e(m, n, dtype=f)
        self.dy, self.dx, self.dweight, self.dtable = e(m, dim), e(m, dim), e(dim, dtype=f), e(n, dim, dtype=f)
        self.q, self.yt, self.wq, self.wt = q8(m, dim), q8(dim, m), q8(n, dim), q8(dim, n)
        self.gq, self.gt = q8(m, n), q8(n, m)
        sizes = [B.stx_q8_matmul_work_bytes(ctx, *s) for s in ((m, n, dim), (m, dim, n), (n, dim, m))]
        sizes.append(B.stx_rmsnorm_backward_work_bytes(ctx, m, dim))
        self.work = torch.empty(max(sizes) + 256, dtype=torch.uint8, device=G.DEV)
        state = lambda k: (torch.zeros(k, device=G.DEV), torch.zeros(k, device=G.DEV)) if bits == 32 else (  # noqa: E731
            torch.zeros(k, dtype=torch.uint8, device=G.DEV), torch.zeros(k, dtype=torch.uint8, device=G.DEV),
            torch.zeros((k + 127) // 128, device=G.DEV), torch.zeros((k + 127) // 128, device=G.DEV))
        self.moments = [state(n * dim), state(dim)]
        self.tensors = B.AdamWTensors([(self.table.view(-1), self.dtable.view(-1), *self.moments[0]), (self.weight, self.dweight, *self.moments[1])],
                                      no_decay=(1,))
        self.hyper = B.make_adamw(**H, bits=bits, seed=5, step_dev=step_dev)

    def score(self):
        c = self.ctx
        B.stx_rmsnorm(c, self.h, self.r, self.weight, EPS, self.s, self.y, self.q, self.rstd)
        B.stx_q8_quantize(c, self.table, self.wq, self.wt)
        B.stx_q8_matmul(c, self.q, self.wq, self.scores, self.work)

    def gradients(self):
        c = self.ctx
        B.stx_q8_quantize(c, self.g, self.gq, self.gt)
        B.stx_q8_quantize(c, self.y, None, self.yt)
        B.stx_q8_matmul(c, self.gq, self.wt, self.dy, self.work)
        B.stx_q8_matmul(c, self.gt, self.yt, self.dtable, self.work)
        B.stx_rmsnorm_backward(c, self.s, self.weight, self.rstd, self.dy, self.dsum, self.dx, self.dweight, self.work)

    def step(self):
        B.stx_adamw_tensors(self.ctx, self.hyper, self.tensors)

    def run(self):
        self.score()
        self.gradients()
        self.step()

    def outputs(self):
        return [self.s, self.y, self.rstd, self.scores, self.dy, self.dx, self.dweight, self.dtable, self.table, self.weight,
                *self.moments[0], *self.moments[1]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("m,n,dim", [(1, 40, 16), (33, 500, 129), (300, 901, 200), (520, 2600, 384)])
def test_a_training_step(m, n, dim, bits):
    t = Trainer(context(), m, n, dim, bits, seed=m)
    table, weight = R.f64(t.table), R.f64(t.weight)
    wb = t.weight.clone()
    t.run()
    s, y, rstd = R.rmsnorm(t.h, t.r, wb, EPS)
    assert torch.equal(t.s, s) and np.all(np.abs(R.f64(t.rstd) / rstd - 1) <= RSTD)
    R.check_q8(t.q, y, Y)
    R.check_q8(t.wq, table)
    R.check_q8(t.wt, np.ascontiguousarray(table.T))
    check_product(t.scores, R.q8_numbers(t.q), R.q8_numbers(t.wq), torch.float32, dim)
    R.check_q8(t.gq, R.f64(t.g))
    R.check_q8(t.gt, np.ascontiguousarray(R.f64(t.g).T))
    R.check_q8(t.yt, np.ascontiguousarray(R.f64(t.y).T))
    check_product(t.dy, R.q8_numbers(t.gq), R.q8_numbers(t.wt), torch.bfloat16, n)
    check_product(t.dtable, R.q8_numbers(t.gt), R.q8_numbers(t.yt), torch.float32, m)
    dx, dw, size, size_dw = R.rmsnorm_backward(s, wb, EPS, t.dy, t.dsum)
    assert np.all(np.abs(R.f64(t.dx) - dx) <= R.U * size + 3 * RSTD * size + R.HALF[torch.bfloat16] * np.abs(dx))
    assert np.all(np.abs(R.f64(t.dweight) - dw) <= ((m // 1024 + 116) * R.U + RSTD) * size_dw)
    for number, (before, after, grad, decay) in enumerate(((table, t.table, t.dtable, True), (weight, t.weight, t.dweight, False))):
        zero = np.zeros((1, before.size))
        check(t.moments[number], after.view(1, -1), before.reshape(1, -1), R.f64(grad).reshape(1, -1), zero, zero, bits, 1, 5, number,
              np.arange(before.size)[None], decay=decay)


def _bits(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_and_replayed(bits):
    m, n, dim = 300, 1500, 200
    stream = torch.cuda.Stream()
    count = torch.ones(1, dtype=torch.int64, device=G.DEV)
    live, ref = Trainer(context(stream), m, n, dim, bits, step_dev=count), Trainer(context(), m, n, dim, bits)
    rng = np.random.default_rng(1)
    inputs = [torch.from_numpy(rng.standard_normal((m, dim))).to(G.DEV, torch.bfloat16) for _ in range(5)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        live.run()
        count.add_(1)
    torch.cuda.synchronize()
    for i, x in enumerate(inputs):
        live.h.copy_(x)
        ref.h.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref.hyper.step = i + 1
        ref.run()
        torch.cuda.synchronize()
        for a, b in zip(live.outputs(), ref.outputs()):
            assert _bits(a, b)
    assert int(count) == 6


def test_two_contexts_on_two_streams():
    sizes = [(300, 1500, 200), (257, 3000, 136)]
    want = []
    for i, s in enumerate(sizes):
        t = Trainer(context(), *s, 8, seed=i)
        for k in range(4):
            t.hyper.step = k + 1
            t.run()
        want.append(t)
    torch.cuda.synchronize()
    got = [Trainer(context(torch.cuda.Stream()), *s, 8, seed=i) for i, s in enumerate(sizes)]
    torch.cuda.synchronize()
    for k in range(4):
        for t in got:
            t.hyper.step = k + 1
            t.run()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(_bits(x, y) for x, y in zip(a.outputs(), b.outputs()))


# ---- sizes ------------------------------------------------------------------------------------------------------------

# more rows than the workgroups of a backward pass take at once, for each number of threads a row
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(40_003, 100), (20_001, 250), (9_001, 500), (5_001, 700), (2_101, 2000), (1_300, 4001), (900, 8000), (700, 9001),
                                       (16_500, 1024), (33_000, 1024)])
def test_norm_of_many_rows(rows, cols, dtype):
    ctx, rng = context(), np.random.default_rng(rows)
    x, dy, dsum = (rows_of(rng, rows, cols, dtype) for _ in range(3))
    w = torch.from_numpy(1 + 0.1 * rng.standard_normal(cols)).float().to(G.DEV)
    y, dx, rstd, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=G.DEV), torch.empty(cols, device=G.DEV)
    q = B.Q8(rows, cols, B.STX_E5M2, G.DEV)
    B.stx_rmsnorm(ctx, x, None, w, EPS, None, y, q, rstd)
    _, want, _ = R.rmsnorm(x, None, w, EPS)
    assert np.all(np.abs(R.f64(y) - want) <= (Y + R.HALF[dtype]) * np.abs(want))
    pick = np.r_[:40, rows - 40:rows]
    part = B.Q8.of(q.codes[pick].contiguous(), q.scales[pick].contiguous(), cols, B.STX_E5M2)
    R.check_q8(part, want[pick], Y)
    work = torch.empty(B.stx_rmsnorm_backward_work_bytes(ctx, rows, cols) + 256, dtype=torch.uint8, device=G.DEV)
    B.stx_rmsnorm_backward(ctx, x, w, rstd, dy, dsum, dx, dw, work)
    want, want_dw, size, size_dw = R.rmsnorm_backward(x, w, EPS, dy, dsum)
    assert np.all(np.abs(R.f64(dx) - want) <= R.U * size + 3 * RSTD * size + R.HALF[dtype] * np.abs(want))
    adds = rows // 256 + 1 + 16 + 16 + 16 + 4                # rows of a thread at most, groups, parts of a slice, slices, products
    assert np.all(np.abs(R.f64(dw) - want_dw) <= (adds * R.U + RSTD) * size_dw)
    kept = dx.clone(), dw.clone()
    B.stx_rmsnorm_backward(ctx, x, w, rstd, dy, dy, dy, dw, work)            # in place of what it reads
    B.stx_rmsnorm_backward(ctx, x, w, rstd, dsum, dsum, dsum, dw, work)
    assert torch.isfinite(dy).all() and torch.isfinite(dsum).all()
    del kept


# tiles of 256 x 256 and 256 x 128 from one block of columns on, outputs beyond the caches with and without whole lines, of a few rows
LARGE = [(4096, 3600, 70), (6200, 1000, 100), (260, 12_400, 640), (6145, 1030, 1300), (7000, 900, 384), (6300, 1024, 200), (4200, 8300, 1100),
         (4200, 8320, 300), (8100, 8448, 128)]


@pytest.mark.parametrize("m,n,k", LARGE)
def test_large_products(m, n, k):
    ctx, rng = context(), np.random.default_rng(m + k)
    (a, x), (b, y) = _q8_of(rng, m, k, 0), _q8_of(rng, n, k, 1)
    pick = np.unique(np.r_[:3, rng.integers(0, m, 150), m - 3:m])
    for dtype, ldo in ((torch.float32, n), (torch.bfloat16, n), (torch.bfloat16, n + 5)):
        room = torch.full((m, ldo), 777.0, dtype=dtype, device=G.DEV)
        work = torch.empty(B.stx_q8_matmul_work_bytes(ctx, m, n, k) + 256, dtype=torch.uint8, device=G.DEV)
        B.stx_q8_matmul(ctx, a, b, room[:, :n], work)
        check_product(room[:, :n][torch.from_numpy(pick).to(G.DEV)], x[pick], y, dtype, k)
        assert (room[:, n:] == 777.0).all()
        whole = room[:, :n].double().sum(1).cpu().numpy()    # every row, by its sum
        want, total = x @ y.sum(0), np.abs(x) @ np.abs(y).sum(0)
        assert np.all(np.abs(whole - want) <= ((16 * -(-k // 128) + 16) * 2.0**-23 + R.HALF[dtype] + (7 * 2.0**-13 if dtype != torch.float32 else 0)) * total)


def test_offsets_beyond_32_bits():
    ctx = context()
    rows, ld, cols = 70_000, 33_000, 130                     # 2.3e9 elements, 130 columns of them in use
    g = torch.Generator(device=G.DEV).manual_seed(1)
    x = torch.empty(rows, ld, dtype=torch.bfloat16, device=G.DEV)[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=g, device=G.DEV))
    small = x.contiguous()
    q, qt, q1, qt1 = B.Q8(rows, cols, 0, G.DEV), B.Q8(cols, rows, 0, G.DEV), B.Q8(rows, cols, 0, G.DEV), B.Q8(cols, rows, 0, G.DEV)
    B.stx_q8_quantize(ctx, x, q, qt)
    B.stx_q8_quantize(ctx, small, q1, qt1)
    assert torch.equal(q.codes, q1.codes) and torch.equal(qt.codes, qt1.codes) and torch.equal(q.scales[:, :2], q1.scales[:, :2])
    y, y1, rstd = torch.empty(rows, ld, dtype=torch.bfloat16, device=G.DEV)[:, :cols], torch.empty_like(small), torch.empty(rows, device=G.DEV)
    B.stx_rmsnorm(ctx, x, None, None, EPS, None, y, None, rstd)
    B.stx_rmsnorm(ctx, small, None, None, EPS, None, y1, None, rstd)
    assert torch.equal(y, y1)
    d1 = torch.empty_like(small)
    B.stx_rmsnorm_backward(ctx, x, None, rstd, y, x, y, None)
    B.stx_rmsnorm_backward(ctx, small, None, rstd, y1, small, d1, None)
    assert torch.equal(y, d1)
    del y, x
    out = torch.empty(rows, ld, device=G.DEV)[:, :300]
    few = B.Q8.of(q.codes[:300].contiguous(), q.scales[:300].contiguous(), cols, 0)
    near = torch.empty(rows, 300, device=G.DEV)
    work = torch.empty(B.stx_q8_matmul_work_bytes(ctx, rows, 300, cols) + 256, dtype=torch.uint8, device=G.DEV)
    B.stx_q8_matmul(ctx, q, few, out, work)
    B.stx_q8_matmul(ctx, q, few, near, work)
    assert torch.equal(out, near)
    check_product(out[-200:], R.q8_numbers(q)[-200:], R.q8_numbers(few), torch.float32, cols)
    # operands whose rows lie as far apart as they may
    far = torch.zeros(300, 1 << 24, dtype=torch.uint8, device=G.DEV)
    far[:, :256] = few.codes[:, :256]
    wide = B.Q8.of(far, few.scales, cols, 0)
    again = torch.empty(rows, 300, device=G.DEV)
    B.stx_q8_matmul(ctx, q, wide, again, work)
    assert torch.equal(again, near)


def test_more_rows_than_one_launch_takes():
    ctx = context()
    rows, cols = (1 << 24) + 3, 1025                         # 256 threads a row
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=G.DEV)
    x[-5:] = torch.randn(5, cols, device=G.DEV)
    rstd = torch.full((rows,), float("nan"), device=G.DEV)
    B.stx_rmsnorm(ctx, x, None, None, EPS, None, None, None, rstd)
    assert not rstd.isnan().any() and rstd[:-5].min() == rstd[:-5].max()
    _, _, want = R.rmsnorm(x[-5:], None, None, EPS)
    assert np.all(np.abs(R.f64(rstd[-5:]) / want - 1) <= RSTD)
    del x, rstd
    rows = (1 << 28) + 5                                     # 16 threads a row
    x = torch.zeros(rows, 1, dtype=torch.bfloat16, device=G.DEV)
    x[-9:] = torch.randn(9, 1, device=G.DEV)
    q = B.Q8(rows, 1, 0, G.DEV)
    q.scales.fill_(200)
    B.stx_q8_quantize(ctx, x, q, None)
    assert (q.scales[:-9, 0] == 127).all()
    part = B.Q8.of(q.codes[-20:].contiguous(), q.scales[-20:].contiguous(), 1, 0)
    R.check_q8(part, R.f64(x[-20:]))
    del x, q
    torch.cuda.empty_cache()


@pytest.mark.parametrize("bits", [32, 8])
def test_tensor_of_more_than_32_bits(bits):
    ctx, n = context(), (1 << 31) + 1027
    p = torch.ones(n, device=G.DEV)
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device=G.DEV)
    g[-2000:] = torch.randn(2000, device=G.DEV).bfloat16()
    like = dict(dtype=torch.float32 if bits == 32 else torch.uint8, device=G.DEV)
    s = [torch.zeros(n, **like), torch.zeros(n, **like)] + ([torch.zeros((n + 127) // 128, device=G.DEV) for _ in range(2)] if bits == 8 else [])
    B.stx_adamw_tensors(ctx, B.make_adamw(**H, bits=bits, seed=3), B.AdamWTensors([(p, g, *s)]))
    first = n // 128 * 128 - 1280
    tail = slice(first, n)
    t = [x[tail] for x in s[:2]] + [x[first // 128:] for x in s[2:]]
    k = n - first
    zero = np.zeros((1, k))
    check(t, p[tail].view(1, -1), np.ones((1, k)), R.f64(g[tail])[None], zero, zero, bits, 1, 3, 0, np.arange(first, n)[None])


def test_small_squares():
    # squares below the normal numbers, and no eps: the quotient follows the formula from the moments that are held
    ctx, n = context(), 4096
    rng = np.random.default_rng(2)
    p = torch.zeros(n, device=G.DEV)
    g = torch.from_numpy(np.exp(rng.uniform(-47, -30, n)) * rng.choice([-1, 1], n)).float().to(G.DEV)
    m, v = torch.zeros(n, device=G.DEV), torch.zeros(n, device=G.DEV)
    h = B.make_adamw(0.01, 0.9, 0.99, 0.0, 0.0, 32, step=3)
    B.stx_adamw_tensors(ctx, h, B.AdamWTensors([(p, g, m, v)]))
    assert (v > 0).all() and (v < 2.0**-126).sum() > 1000 and (v > 2.0**-126).sum() > 100
    want = -0.01 / (1 - 0.9**3) * R.f64(m) / np.sqrt(R.f64(v) / (1 - 0.99**3))
    assert np.all(np.abs(R.f64(p) - want) <= 16 * R.U * np.abs(want))
