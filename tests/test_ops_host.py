"""What the entry points of the operators on rows and tensors refuse, before anything is launched: no GPU needed."""
import ctypes as C
import gc
import types
import weakref

import pytest
import torch

from paper_2502_16949_amd import binding as B

L = B.lib()
P = 4096                                    # an aligned address that is never read


def context(model="transe", dim=32, rel_dim=0, flags=0):
    """A block that begins with the configuration, as a context does: argument checks read no more of it."""
    cfg = B.make_config(model, "l2", 100, 5, dim, 64, 1, rel_dim=rel_dim, flags=flags)
    block = (C.c_char * 65536)()
    C.memmove(block, C.byref(cfg), C.sizeof(cfg))
    return block


def q8(rows=4, cols=200, codes=P, scales=P, ld=256, ld_scale=4, fmt=0, **kw):
    return B.stx_q8(codes, scales, rows, cols, ld, ld_scale, fmt)


def test_struct_sizes():
    assert (C.sizeof(B.stx_q8), C.sizeof(B.stx_adamw), C.sizeof(B.stx_moments), C.sizeof(B.stx_adamw_tensor),
            C.sizeof(B.stx_adamw_state)) == (56, 80, 32, 64, 128)


@pytest.mark.parametrize("kw,status", [
    (dict(), B.STX_OK),                     # no rows: nothing to do
    (dict(ctx=None), B.STX_ERR_NULL),
    (dict(dtype=3), B.STX_ERR_BAD_ARG),
    (dict(rows=-1), B.STX_ERR_BAD_ARG),
    (dict(rows=1 << 31), B.STX_ERR_BAD_ARG),
    (dict(cols=0), B.STX_ERR_BAD_ARG),
    (dict(cols=16385, ld=16385), B.STX_ERR_BAD_ARG),
    (dict(ld=199), B.STX_ERR_BAD_ARG),
    (dict(eps=-1e-6), B.STX_ERR_BAD_ARG),
    (dict(eps=float("nan")), B.STX_ERR_BAD_ARG),
    (dict(rows=4, x=None), B.STX_ERR_NULL),
    (dict(rows=4, y=None), B.STX_ERR_NULL),                 # no output at all
    (dict(rows=4, x=P + 2), B.STX_ERR_BAD_ARG),
    (dict(rows=4, rstd=P + 2), B.STX_ERR_BAD_ARG),
    (dict(rows=4, dtype=B.STX_BF16, x=P + 1), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(rows=5)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(cols=201)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(fmt=2)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(ld=200)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(ld=264)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(ld_scale=2)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(codes=P + 8)), B.STX_ERR_BAD_ARG),
    (dict(rows=4, q=q8(scales=None)), B.STX_ERR_NULL),
])
def test_rmsnorm_refusals(kw, status):
    a = dict(ctx=context(), dtype=B.STX_F32, rows=0, cols=200, ld=200, x=P, res=None, w=None, eps=1e-6, sum=None, y=P, q=None, rstd=None)
    a.update(kw)
    if isinstance(a["q"], B.stx_q8):
        a["q"] = C.byref(a["q"])
    assert L.stx_rmsnorm(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0, dweight=None), B.STX_OK),
    (dict(dtype=-1), B.STX_ERR_BAD_ARG),
    (dict(cols=0), B.STX_ERR_BAD_ARG),
    (dict(ld=100), B.STX_ERR_BAD_ARG),
    (dict(dy=None), B.STX_ERR_NULL),
    (dict(rstd=None), B.STX_ERR_NULL),
    (dict(dx=None), B.STX_ERR_NULL),
    (dict(dsum=P + 1), B.STX_ERR_BAD_ARG),
    (dict(work=None), B.STX_ERR_NULL),
    (dict(work=P + 64), B.STX_ERR_WORKSPACE),
    (dict(work_bytes=100), B.STX_ERR_WORKSPACE),
])
def test_rmsnorm_backward_refusals(kw, status):
    a = dict(ctx=context(), dtype=B.STX_F32, rows=8, cols=200, ld=200, sum=P, w=P, rstd=P, dy=P, dsum=None, dx=P, dweight=P, work=P,
             work_bytes=1 << 20)
    a.update(kw)
    assert L.stx_rmsnorm_backward(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0, q=q8(rows=0)), B.STX_OK),
    (dict(q=None), B.STX_ERR_NULL),
    (dict(dtype=7), B.STX_ERR_BAD_ARG),
    (dict(cols=-1), B.STX_ERR_BAD_ARG),
    (dict(ld=10), B.STX_ERR_BAD_ARG),
    (dict(x=None), B.STX_ERR_NULL),
    (dict(x=P + 2), B.STX_ERR_BAD_ARG),
    (dict(q=q8(rows=3)), B.STX_ERR_BAD_ARG),
    (dict(qt=q8()), B.STX_ERR_BAD_ARG),                     # not the transpose's size
    (dict(qt=q8(rows=200, cols=4, ld=112)), B.STX_ERR_BAD_ARG),
    (dict(rows=1 << 30, cols=1 << 20, ld=1 << 20, q=q8(rows=1 << 30, cols=1 << 20, ld=1 << 20, ld_scale=1 << 13)), B.STX_ERR_UNSUPPORTED),
    (dict(rows=1 << 20, cols=1 << 19, ld=1 << 19, q=None, qt=q8(rows=1 << 19, cols=1 << 20, ld=1 << 20, ld_scale=1 << 13)), B.STX_ERR_UNSUPPORTED),
])
def test_quantize_refusals(kw, status):
    a = dict(ctx=context(), dtype=B.STX_F32, rows=4, cols=200, ld=200, x=P, q=q8(), qt=None)
    a.update(kw)
    for k in ("q", "qt"):
        a[k] = None if a[k] is None else C.byref(a[k])
    assert L.stx_q8_quantize(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(a=q8(rows=0)), B.STX_OK),
    (dict(b=q8(rows=0)), B.STX_OK),
    (dict(a=None), B.STX_ERR_NULL),
    (dict(b=q8(cols=201)), B.STX_ERR_BAD_ARG),
    (dict(a=q8(cols=0), b=q8(cols=0)), B.STX_ERR_BAD_ARG),
    (dict(a=q8(rows=-1)), B.STX_ERR_BAD_ARG),
    (dict(dtype=5), B.STX_ERR_BAD_ARG),
    (dict(ldo=3), B.STX_ERR_BAD_ARG),
    (dict(out=None), B.STX_ERR_NULL),
    (dict(out=P + 2), B.STX_ERR_BAD_ARG),
    (dict(a=q8(ld=(1 << 24) + 16)), B.STX_ERR_UNSUPPORTED),
    (dict(b=q8(ld_scale=(1 << 24) + 4)), B.STX_ERR_UNSUPPORTED),
    (dict(a=q8(rows=1 << 30), b=q8(rows=1 << 30), ldo=1 << 30), B.STX_ERR_UNSUPPORTED),
    (dict(a=q8(rows=(1 << 30) + 1), b=q8(rows=1)), B.STX_ERR_UNSUPPORTED),
    (dict(a=q8(rows=40, cols=100_000, ld=100_096, ld_scale=784), b=q8(rows=40, cols=100_000, ld=100_096, ld_scale=784), ldo=40, work=None), B.STX_ERR_NULL),
    (dict(a=q8(rows=40, cols=100_000, ld=100_096, ld_scale=784), b=q8(rows=40, cols=100_000, ld=100_096, ld_scale=784), ldo=40, work_bytes=4), B.STX_ERR_WORKSPACE),
])
def test_matmul_refusals(kw, status):
    a = dict(ctx=context(), a=q8(), b=q8(), dtype=B.STX_F32, out=P, ldo=4, work=P, work_bytes=1 << 30)
    a.update(kw)
    for k in ("a", "b"):
        a[k] = None if a[k] is None else C.byref(a[k])
    assert L.stx_q8_matmul(*a.values()) == status


def test_work_sizes():
    n = C.c_size_t(7)
    ctx = context()
    assert L.stx_q8_matmul_work_bytes(ctx, 0, 5, 64, C.byref(n)) == B.STX_OK and n.value == 0
    assert L.stx_q8_matmul_work_bytes(ctx, 4, 5, 0, C.byref(n)) == B.STX_ERR_BAD_ARG
    assert L.stx_q8_matmul_work_bytes(ctx, 4, 5, 64, None) == B.STX_ERR_NULL
    assert L.stx_q8_matmul_work_bytes(None, 4, 5, 64, C.byref(n)) == B.STX_ERR_NULL
    assert L.stx_rmsnorm_backward_work_bytes(ctx, 1000, 1001, C.byref(n)) == B.STX_OK and n.value % 256 == 0 and n.value >= 4004
    assert L.stx_rmsnorm_backward_work_bytes(ctx, 1000, 0, C.byref(n)) == B.STX_ERR_BAD_ARG


def hyper(**kw):
    a = dict(lr=0.1, bits=32, step=1)
    a.update(kw)
    return B.make_adamw(**a)


BAD_HYPER = [dict(bits=16), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=1e-40), dict(eps=1e39), dict(step=0),
             dict(weight_decay=float("nan"))]


@pytest.mark.parametrize("kw", BAD_HYPER)
def test_adamw_hyperparameters(kw):
    h = hyper(**kw)
    assert L.stx_adamw_tensors(context(), C.byref(h), None, 0) == B.STX_ERR_BAD_ARG
    assert L.stx_adamw_tensors(context(), C.byref(hyper()), None, 0) == B.STX_OK


@pytest.mark.parametrize("kw,bits,status", [
    (dict(n=0, p=None, g=None), 32, B.STX_OK),
    (dict(n=-1), 32, B.STX_ERR_BAD_ARG),
    (dict(n=(1 << 36) - 4095), 32, B.STX_ERR_BAD_ARG),
    (dict(p=None), 32, B.STX_ERR_NULL),
    (dict(g=None), 32, B.STX_ERR_NULL),
    (dict(p=P + 2), 32, B.STX_ERR_BAD_ARG),
    (dict(g=P + 2), 32, B.STX_ERR_BAD_ARG),
    (dict(m=None), 32, B.STX_ERR_NULL),
    (dict(v=P + 1), 32, B.STX_ERR_BAD_ARG),
    (dict(ms=None), 8, B.STX_ERR_NULL),
    (dict(vs=P + 2), 8, B.STX_ERR_BAD_ARG),
    (dict(dtype=9), 32, B.STX_ERR_BAD_ARG),
    (dict(flags=2), 32, B.STX_ERR_BAD_ARG),
])
def test_adamw_tensor_refusals(kw, bits, status):
    a = dict(p=P, g=P, n=10, m=P, v=P, ms=P, vs=P, dtype=0, flags=0)
    a.update(kw)
    t = B.stx_adamw_tensor(a["p"], a["g"], a["n"], B.stx_moments(a["m"], a["v"], a["ms"], a["vs"]), a["dtype"], a["flags"])
    assert L.stx_adamw_tensors(context(), C.byref(hyper(bits=bits)), C.byref(t), 1) == status


def test_adamw_tensor_counts():
    assert L.stx_adamw_tensors(context(), C.byref(hyper()), None, 1) == B.STX_ERR_NULL
    assert L.stx_adamw_tensors(context(), C.byref(hyper()), None, 65536) == B.STX_ERR_BAD_ARG
    assert L.stx_adamw_tensors(None, C.byref(hyper()), None, 0) == B.STX_ERR_NULL
    assert L.stx_adamw_tensors(context(), None, None, 0) == B.STX_ERR_NULL


def _step(ctx, p=None, g=None, h=None, s=None, b=0):
    inc = B.stx_incidence(b, 1, b * 2, b * 6, *([P] * 10))
    return L.stx_adamw_step(ctx, C.byref(p or B.stx_params(P, P, P, P, None)), C.byref(inc), C.byref(g or B.stx_grads(P, P, P)),
                            C.byref(h or hyper()), C.byref(s or B.stx_adamw_state(*([B.stx_moments(P, P, P, P)] * 4))))


def test_adamw_step_refusals():
    bf16 = B.STX_FLAG_BF16_PROJ
    m = B.stx_moments(P, P, P, P)
    none = B.stx_moments()
    assert _step(context()) == B.STX_OK                     # a batch of nothing
    assert _step(context(), p=B.stx_params()) == B.STX_ERR_NULL
    assert _step(context(), g=B.stx_grads()) == B.STX_ERR_NULL
    assert _step(context(), b=65) == B.STX_ERR_BAD_ARG
    assert _step(context(), h=hyper(bits=4)) == B.STX_ERR_BAD_ARG
    assert _step(context(), s=B.stx_adamw_state(none, m, m, m)) == B.STX_ERR_NULL
    assert _step(context(), s=B.stx_adamw_state(m, none, none, none)) == B.STX_OK
    assert _step(context("transh"), s=B.stx_adamw_state(m, none, m, none)) == B.STX_ERR_NULL
    assert _step(context("transh"), s=B.stx_adamw_state(m, m, none, none)) == B.STX_ERR_NULL
    assert _step(context("transh"), g=B.stx_grads(P, None, None)) == B.STX_ERR_NULL
    assert _step(context("transr", 32, 32, bf16), s=B.stx_adamw_state(m, m, none, none)) == B.STX_ERR_NULL
    assert _step(context("transr", 32, 32, bf16), g=B.stx_grads(P, None, None)) == B.STX_ERR_NULL
    assert _step(context(), s=B.stx_adamw_state(B.stx_moments(P + 4, P), m, m, m)) == B.STX_ERR_BAD_ARG        # rows are read in float4
    assert _step(context(), h=hyper(bits=8), s=B.stx_adamw_state(B.stx_moments(P + 2, P, P, P), m, m, m)) == B.STX_ERR_BAD_ARG
    assert _step(context(), h=hyper(bits=8), s=B.stx_adamw_state(B.stx_moments(P, P), m, m, m)) == B.STX_ERR_NULL
    assert L.stx_adamw_step(None, None, None, None, None, None) == B.STX_ERR_NULL


class _Device:
    """Of a device tensor, what the binding looks at."""

    def __init__(self, dtype, index, n=1):
        self.dtype, self.index, self.n, self.is_cuda = dtype, index, n, True

    def numel(self):
        return self.n

    def get_device(self):
        return self.index

    def data_ptr(self):
        return P if self.n else 0


@pytest.mark.parametrize("name,dtype", [("step_dev", torch.int64), ("grad_scale", torch.float32)])
def test_hyperparameters_in_device_memory(name, dtype):
    ctx = types.SimpleNamespace(index=0, handle=None)       # (no context: the library refuses what the binding lets through)
    none = B.AdamWTensors([])
    for index, error in ((1, AssertionError), (0, B.StxError)):
        h = B.make_adamw(0.1, **{name: _Device(dtype, index)})
        with pytest.raises(error):
            B.stx_adamw_tensors(ctx, h, none)
        inc, grads = types.SimpleNamespace(c=B.stx_incidence()), types.SimpleNamespace(c=B.stx_grads())
        with pytest.raises(error):
            B.stx_adamw_step(ctx, types.SimpleNamespace(c=B.stx_params()), inc, grads, h, types.SimpleNamespace(held={}, c=B.stx_adamw_state()))
    for bad in (_Device(torch.float64, 0), _Device(dtype, 0, 0)):      # (no element: a null pointer, so no factor at all)
        with pytest.raises(AssertionError):
            B.make_adamw(0.1, **{name: bad})
    with pytest.raises(AssertionError):
        B.make_adamw(0.1, step_dev=_Device(torch.int64, 0), grad_scale=_Device(torch.float32, 1))
    t = _Device(dtype, 0)
    kept = weakref.ref(t)
    h = B.make_adamw(0.1, **{name: t})
    del t
    gc.collect()
    assert kept() is not None and h.index == 0
    del h
    gc.collect()
    assert kept() is None


def test_memory_behind_the_last_row():
    room = torch.zeros(64, dtype=torch.uint8)
    for t, width in ((room.view(8, 8)[:, :5], 8), (room.view(8, 8)[:, :1], 4), (room[:20].view(4, 5), 8), (room[3:51].view(6, 8)[:, :5], 8), (room[:0].view(0, 5), 8), (torch.zeros(5, 0, dtype=torch.uint8), 0)):
        assert B._reaches(t, width)
    for t, width in ((torch.zeros(4, 5, dtype=torch.uint8), 8), (room.view(8, 8)[:, 4:5], 8), (room[8:].view(7, 8)[6:, 6:], 4), (room.as_strided((8, 5), (8, 1), 3), 8)):
        assert not B._reaches(t, width)


I31 = (1 << 31) - 1


def test_limits_as_documented():
    """The largest sizes pass their check (and meet a missing pointer), the next ones do not."""
    ctx, x = context(), B.STX_ERR_NULL
    quantize = lambda rows, cols, q, qt, at=None: L.stx_q8_quantize(ctx, 0, rows, cols, max(cols, 1), at, q and C.byref(q), qt and C.byref(qt))  # noqa: E731
    of = lambda rows, cols: q8(rows, cols, ld=(cols + 127) // 128 * 128, ld_scale=((cols + 127) // 128 + 3) // 4 * 4)  # noqa: E731
    wide = I31 - 128
    assert quantize(1, wide, of(1, wide), None) == x and quantize(wide, 1, None, of(1, wide)) == x
    assert quantize(1, wide + 1, of(1, wide + 1), None) == B.STX_ERR_BAD_ARG and quantize(wide + 1, 1, None, of(1, wide + 1)) == B.STX_ERR_BAD_ARG
    assert quantize(I31, 1, of(I31, 1), None) == x and quantize(I31 + 1, 1, of(I31 + 1, 1), None) == B.STX_ERR_BAD_ARG
    # one block of columns more than 2^35; 2^24 blocks of 128 x 128, whole ones and parts
    assert quantize(I31, 17 * 128, of(I31, 17 * 128), None, P) == B.STX_ERR_UNSUPPORTED
    for rows, cols in ((1 << 19, 1 << 19), ((1 << 30) + 1, 129)):
        assert quantize(rows, cols, None, of(cols, rows), P) == B.STX_ERR_UNSUPPORTED
    a30, b14 = of(1 << 30, 128), of(1 << 14, 128)
    product = lambda a, b: L.stx_q8_matmul(ctx, C.byref(a), C.byref(b), 0, None, b.rows, P, 1 << 62)  # noqa: E731
    assert product(a30, b14) == x and product(b14, a30) == x
    assert product(a30, of((1 << 14) + 1, 128)) == B.STX_ERR_UNSUPPORTED and product(of((1 << 30) + 1, 128), b14) == B.STX_ERR_UNSUPPORTED
    assert product(of(3, wide), of(2, wide)) == B.STX_ERR_UNSUPPORTED          # rows of more than 2^24 bytes
    norm = lambda rows: L.stx_rmsnorm(ctx, 0, rows, 64, 64, None, None, None, 1e-6, None, P, None, None)  # noqa: E731
    assert norm(I31) == x and norm(I31 + 1) == B.STX_ERR_BAD_ARG
