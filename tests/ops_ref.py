"""Plain 64-bit forms of the operators on rows and tensors (numpy), written from their formulas, and 8-bit formats as numbers."""
from __future__ import annotations

import numpy as np
import torch

U = 2.0**-24                               # half a step of fp32, relative
HALF = {torch.float32: U, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}   # at most half a step, relative to the value
BLOCK = 128
FORMATS = {0: (torch.float8_e4m3fn, 3, -6, 448.0), 1: (torch.float8_e5m2, 2, -14, 57344.0)}


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def blocked(x, fill=0.0):
    """[rows, cols] -> [rows, blocks, 128]."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    out = np.full((rows, nb * BLOCK), fill, x.dtype)
    out[:, :cols] = x
    return out.reshape(rows, nb, BLOCK)


def decode(codes, fmt):
    """uint8 codes as numbers."""
    return torch.from_numpy(np.ascontiguousarray(codes)).view(FORMATS[fmt][0]).to(torch.float64).numpy()


def held(codes, scales, cols, fmt=0):
    """The numbers that a matrix in 8 bits stands for (uint8 arrays)."""
    nb = -(-cols // BLOCK)
    x = decode(codes[:, :nb * BLOCK], fmt).reshape(len(codes), nb, BLOCK)
    return (x * 2.0 ** (scales[:, :nb].astype(np.float64) - 127.0)[..., None]).reshape(len(codes), -1)[:, :cols]


def q8_numbers(q):
    return held(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.cols, q.format)


def scale_byte(most, fmt):
    """Exponent byte of the smallest power of two, 2^-126 at least, that brings `most` to the format's largest number."""
    top = FORMATS[fmt][3]
    e = np.ceil(np.log2(np.maximum(most, 1e-300) / top))
    e = np.where(most > top * 2.0**e, e + 1, np.where(most <= top * 2.0 ** (e - 1), e - 1, e))
    return np.where(most > 0, np.maximum(e, -126) + 127, 127).astype(np.int64)


def step_at(x, fmt):
    """The step between neighbouring codes at |x| (the one above it)."""
    _, bits, low, _ = FORMATS[fmt]
    e = np.floor(np.log2(np.maximum(np.abs(x), 1e-300)))
    e = np.where(2.0**e > np.abs(x), e - 1, np.where(2.0 ** (e + 1) <= np.abs(x), e + 1, e))
    return 2.0 ** (np.maximum(e, low) - bits)


def check_q8(q, y, slack=0.0):
    """q holds y: right scales, every code the nearest, where y is known up to a relative `slack`; zeros behind the columns."""
    fmt, top = q.format, FORMATS[q.format][3]
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    rows, cols = y.shape
    nb = -(-cols // BLOCK)
    assert codes.shape[0] == rows and not codes[:, cols:nb * BLOCK].any()
    b = blocked(y)
    most = np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1)
    got = scales[:, :nb].astype(np.int64)
    assert np.all((got == scale_byte(most * (1 - slack), fmt)) | (got == scale_byte(most * (1 + slack), fmt)))
    down = 2.0 ** (127.0 - got)[..., None]
    v, x = decode(codes[:, :nb * BLOCK], fmt).reshape(b.shape), b * down
    fine = np.isfinite(x)
    if fmt == 0:
        assert np.isnan(v[~fine]).all()
    else:
        assert np.array_equal(v[~fine], x[~fine], equal_nan=True)
    x, v = x[fine], v[fine]
    assert np.all(np.abs(v) <= top)
    assert np.all(np.abs(v - x) <= 0.5 * step_at(np.abs(x) * (1 + slack), fmt) + slack * np.abs(x))


# ---- RMS norm ---------------------------------------------------------------------------------------------------

def rmsnorm(x, residual, weight, eps):
    """(s as a tensor of x's type, y, rstd) with s rounded to x's type as the interface says."""
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = f64(s)
    rstd = 1.0 / np.sqrt((f * f).mean(1) + eps)
    w = 1.0 if weight is None else f64(weight)
    return s, f * rstd[:, None] * w, rstd


def rmsnorm_backward(s, weight, eps, dy, dsum):
    """(dx, dweight, and what their rounding errors are relative to)."""
    f, d = f64(s), f64(dy)
    n = f.shape[1]
    rstd = 1.0 / np.sqrt((f * f).mean(1, keepdims=True) + eps)
    a = d * (1.0 if weight is None else f64(weight))
    dx = rstd * (a - f * rstd**2 * (a * f).sum(1, keepdims=True) / n)
    size = rstd * (np.abs(a) * 8 + np.abs(f) * rstd**2 * (80 + 8) * (np.abs(a * f)).sum(1, keepdims=True) / n)
    if dsum is not None:
        dx, size = dx + f64(dsum), size + 2 * np.abs(f64(dsum))
    return dx, (d * f * rstd).sum(0), size, np.abs(d * f * rstd).sum(0)


# ---- AdamW ------------------------------------------------------------------------------------------------------

def splitmix(seed, ctr):
    """Output number ctr (array of uint64) of the SplitMix64 sequence seeded with `seed`."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + (np.asarray(ctr, np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def noise(seed, step, tensor, index):
    """(for m, for v) in [0, 1) of the elements `index`."""
    key = splitmix(seed, (step << 16) + tensor)
    u = splitmix(key, np.asarray(index, np.uint64) >> np.uint64(1))
    u = np.where(np.asarray(index) % 2 == 1, u >> np.uint64(32), u)
    return (u & np.uint64(0xFFFF)).astype(np.float64) / 65536, ((u >> np.uint64(16)) & np.uint64(0xFFFF)).astype(np.float64) / 65536


def adamw(p, g, m, v, h, step, decay=True, scale=1.0):
    """(p, m, v) in 64 bits from arrays of numbers."""
    g = g * scale
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    if decay:
        p = p - h["lr"] * h["weight_decay"] * p
    return p - h["lr"] * (m / (1 - h["beta1"]**step)) / (np.sqrt(v / (1 - h["beta2"]**step)) + h["eps"]), m, v


def check_moment(codes, scales, x, err, u, fmt):
    """8-bit codes [rows, width] and scales [rows, blocks] hold x, known up to err, rounded by the random numbers u."""
    top = FORMATS[fmt][3]
    b, eb, ub = blocked(x), blocked(err), blocked(u)
    most, off = np.abs(b).max(-1), eb.max(-1)
    live = most >= 2.0**-100
    assert np.all(np.abs(scales - np.where(live, most / top, 0.0)) <= (off + 2 * U * most) / top)
    v = blocked(decode(codes, fmt))
    assert not v[~live].any()
    safe = np.where(live, most, 1.0)[..., None]
    y = np.where(live[..., None], b * top / safe, 0.0)
    a, got = np.abs(y), np.abs(v)
    # its own error, the block's largest, and two roundings
    near = np.where(live[..., None], eb * top / safe, 0) + a * (off[..., None] / safe + 4 * U) + 2.0**-40
    assert np.all((np.sign(v) == np.sign(y)) | (v == 0) | (a <= near))
    floor = lambda t: np.minimum(np.floor(t / step_at(t, fmt) + ub) * step_at(t, fmt), top)  # noqa: E731
    # 16 random bits against the bits that are dropped: a value below the smallest normal number has its own last bits rounded first
    edge = step_at(a, fmt) * 2.0**-16
    low, high = floor(np.maximum(a - near - edge, 0)), floor(a + near + edge)
    if fmt == 1:
        low, high = (np.where(a > 0, np.maximum(t, 2.0**-16), t) for t in (low, high))
    assert np.all((got >= low) & (got <= high))
    assert np.mean(low != high) < 0.01 or a.size < 4096
