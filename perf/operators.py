"""The cases by which the speed of the 8-bit training operators is measured, each in its plain form and through the library.

Four operators, used one after the other by a program that scores queries against every entity of a table and trains through it:

  norm     a query row is a sum (head row + relation row): RMS norm of x + residual, with the result also as 8-bit codes and a
           scale for each block of 128 columns; in training its backward pass.
  product  scores of queries against a table held in 8 bits, and in training the two products of their gradient, whose operands
           are quantised along the other axis.
  adamw    one step over many dense tensors, moments in 32 or in 8 bits.
  rows     one step over the touched rows of a batch's tables, moments in 32 or in 8 bits.

8-bit codes are the OCP formats.  A block's scale in `norm` and `product` is the smallest power of two, at least 2**-126, that
brings its largest finite magnitude to at most the largest finite code, held as a byte (exponent + 127); a block of zeros has
scale 1.  Moments have a 32-bit scale for each block of 128 elements and are rounded by given random numbers: see _moments.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                                   # True: the library's calls; False: elementary torch operations

DEV = "cuda:0"
BLOCK = 128
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15 - 2**64, 0xBF58476D1CE4E5B9 - 2**64, 0x94D049BB133111EB - 2**64
HYPER = {"lr": 4e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}


def listed():
    return [
        # one query of a link-prediction service: its row summed, normalised and quantised; latency is all there is
        {"name": "norm_one_query", "op": "norm", "rows": 1, "cols": 1_024, "dtype": "bf16", "train": False},
        # the queries of one batch of the ordinary benchmark (32,768 positives) at the paper's width
        {"name": "norm_queries", "op": "norm", "rows": 32_768, "cols": 1_024, "dtype": "bf16", "train": False},
        # a training step's norm, both directions, fp32 rows of an odd number of columns
        {"name": "norm_train_ragged", "op": "norm", "rows": 20_011, "cols": 1_001, "dtype": "f32", "train": True},
        # one query scored against all entities of an FB15k-sized table
        {"name": "score_one_query", "op": "product", "m": 1, "n": 14_951, "k": 1_024, "dtype": "bf16", "out": "f32", "train": False},
        # an evaluation's batch of queries against the same table
        {"name": "score_batch", "op": "product", "m": 4_096, "n": 14_951, "k": 1_024, "dtype": "bf16", "out": "bf16", "train": False},
        # a training step's gradient of those scores: towards the queries and towards the table
        {"name": "score_gradients", "op": "product", "m": 8_192, "n": 14_951, "k": 1_024, "dtype": "bf16", "out": "f32", "train": True},
        # the largest product: a square one, where only the matrix cores count
        {"name": "product_square", "op": "product", "m": 8_192, "n": 8_192, "k": 8_192, "dtype": "bf16", "out": "bf16", "train": False},
        # the smallest model's tensors (tables of 1,000 and 20 rows of 32, a weight, a few vectors): launches and the host
        {"name": "adamw_tiny_8", "op": "adamw", "sizes": "32000,640,1024,32,32,7", "bits": 8, "grad": "f32"},
        # FB15k-sized tables of the paper's width, a projection and its vectors, moments in 32 bits
        {"name": "adamw_wide_32", "op": "adamw", "sizes": "15309824,1377280,1048576,1024,1024,14951", "bits": 32, "grad": "f32"},
        # the largest table, 4 M entities of 128, gradients in bf16, moments in 8 bits
        {"name": "adamw_4m_8", "op": "adamw", "sizes": "512000000,128000,16384,128", "bits": 8, "grad": "bf16"},
        # the headline benchmark's batch: some 14,000 touched rows of 128, moments in 8 bits
        {"name": "rows_mid_8", "op": "rows", "model": "transe", "n_ent": 15_000, "n_rel": 1_350, "dim": 128, "batch": 32_768,
         "n_neg": 1, "bits": 8},
        # the largest table's batch: about a million touched rows, spread over 2 GB, moments in 32 bits
        {"name": "rows_4m_32", "op": "rows", "model": "toruse", "n_ent": 4_000_000, "n_rel": 1_000, "dim": 128, "batch": 262_144,
         "n_neg": 4, "bits": 32},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "product", "product", "adamw", "rows"])
    if op == "norm":
        cols = rng.choice([_log_int(rng, 1, 8_192), 8 * _log_int(rng, 4, 1_024)])
        return {"op": op, "rows": _log_int(rng, 1, max(2, min(131_072, 67_000_000 // cols))), "cols": cols,
                "dtype": rng.choice(sorted(DTYPES)), "train": rng.random() < 0.5}
    if op == "product":
        train = rng.random() < 0.4
        m, n = _log_int(rng, 1, 16_384), _log_int(rng, 1, 40_559)
        k = rng.choice([_log_int(rng, 1, 8_192), 4 * _log_int(rng, 8, 256)])
        k = max(1, min(k, int(5.0e11 / (m * n * (2 if train else 1)))))
        return {"op": op, "m": m, "n": n, "k": k, "dtype": rng.choice(sorted(DTYPES)), "out": rng.choice(["f32", "bf16"]), "train": train}
    if op == "adamw":
        sizes = [_log_int(rng, 1, 20_000_000) for _ in range(_log_int(rng, 1, 200))]
        while sum(sizes) > 100_000_000:
            sizes.pop()
        return {"op": op, "sizes": ",".join(map(str, sizes)), "bits": rng.choice([8, 32]), "grad": rng.choice(sorted(DTYPES))}
    dim, n_neg = 4 * _log_int(rng, 4, 256), rng.choice([0, 1, 1, 2, 4])
    n_ent = _log_int(rng, 1_000, min(4_000_000, 400_000_000 // dim))
    return {"op": op, "model": rng.choice(["transe", "transe", "toruse", "transh"]), "n_ent": n_ent, "n_rel": _log_int(rng, 11, 1_350),
            "dim": dim, "batch": max(1, min(_log_int(rng, 1, 262_144), 60_000_000 // dim // (1 + n_neg))), "n_neg": n_neg,
            "bits": rng.choice([8, 32])}


# ---- inputs ---------------------------------------------------------------------------------------------------

class _State:
    pass


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _spread(g, rows, cols):
    """Rows of different sizes, as trained rows are: normal values times a size per row and per column."""
    x = _randn(g, rows, cols)
    x *= torch.exp(0.5 * _randn(g, rows, 1))
    x *= torch.exp(0.5 * _randn(g, 1, cols))
    return x


def _first_moments(g, n, bits, width):
    """Moments after some steps: what a program holds before the call."""
    m = _randn(g, n) * 1e-3
    v = _randn(g, n).square_() * 1e-6 + m * m
    if bits == 32:
        return {"m": m, "v": v}
    blocks = _blocks(m.view(-1, width) if width else m.view(1, -1))
    m_scale = blocks.abs().amax(-1) / 448.0
    codes = (blocks / m_scale.unsqueeze(-1)).to(E4M3)
    vb = _blocks(v.view(-1, width) if width else v.view(1, -1))
    v_scale = vb.amax(-1) / 57344.0
    vcodes = (vb / v_scale.unsqueeze(-1)).to(E5M2)
    shape = (n // width, width) if width else (1, n)
    flat = lambda c: c.view(torch.uint8).view(shape[0], -1)[:, :shape[1]].reshape(-1).contiguous()  # noqa: E731
    return {"m": flat(codes), "v": flat(vcodes), "m_scale": m_scale.contiguous(), "v_scale": v_scale.contiguous()}


def _tables(c):
    """(name, rows, first column) of the tables of a `rows` case: which columns of the incidence matrix their rows are."""
    n, r = c["n_ent"], c["n_rel"]
    if c["model"] in ("transe", "toruse"):
        return [("ent", n + r, 0)]
    return [("ent", n, 0), ("rel", r, n), ("w", r, n)]


def prepare(case, seed):
    """Rows, tables, gradients and moments, as a program holds them before the call; the library's handles around them."""
    c, s, g = case, _State(), _gen(seed)
    s.case = c
    if own:
        from paper_2502_16949_amd import binding as B
        s.B = B
    if c["op"] == "norm":
        dt, rows, cols = DTYPES[c["dtype"]], c["rows"], c["cols"]
        s.x, s.res = _spread(g, rows, cols).to(dt), _randn(g, rows, cols).to(dt)
        s.weight, s.eps = 1.0 + 0.1 * _randn(g, cols), 1e-6
        if c["train"]:
            s.dy, s.dsum = _randn(g, rows, cols).to(dt), _randn(g, rows, cols).to(dt)
        if own:
            s.ctx = _context(B)
            s.sum, s.rstd = torch.empty_like(s.x), torch.empty(rows, device=DEV)
            if c["train"]:
                s.y, s.dx, s.dweight = torch.empty_like(s.x), torch.empty_like(s.x), torch.empty(cols, device=DEV)
                s.work = torch.empty(B.stx_rmsnorm_backward_work_bytes(s.ctx, rows, cols) + 256, dtype=torch.uint8, device=DEV)
            else:
                s.q = B.Q8(rows, cols, B.STX_E4M3, DEV)
        return s
    if c["op"] == "product":
        dt, m, n, k = DTYPES[c["dtype"]], c["m"], c["n"], c["k"]
        s.x = _spread(g, m, k).to(dt)
        table = _spread(g, n, k)
        if c["train"]:
            s.table = table
            s.ds = (_randn(g, m, n) / math.sqrt(n)).to(dt)
        else:                                 # held in 8 bits, quantised once
            s.codes, s.scales = _quantized(table)
        if own:
            s.ctx = _context(B)
            dev = dict(device=DEV)
            if c["train"]:
                s.ds_q, s.ds_qt = B.Q8(m, n, B.STX_E4M3, DEV), B.Q8(n, m, B.STX_E4M3, DEV)
                s.x_qt, s.table_qt = B.Q8(k, m, B.STX_E4M3, DEV), B.Q8(k, n, B.STX_E4M3, DEV)
                s.dx, s.dtable = torch.empty(m, k, dtype=DTYPES[c["out"]], **dev), torch.empty(n, k, dtype=DTYPES[c["out"]], **dev)
                need = max(B.stx_q8_matmul_work_bytes(s.ctx, m, k, n), B.stx_q8_matmul_work_bytes(s.ctx, n, k, m))
            else:
                s.x_q = B.Q8(m, k, B.STX_E4M3, DEV)
                s.table_q = B.Q8.of(s.codes, s.scales, k, B.STX_E4M3)
                s.scores = torch.empty(m, n, dtype=DTYPES[c["out"]], **dev)
                need = B.stx_q8_matmul_work_bytes(s.ctx, m, n, k)
            s.work = torch.empty(need + 256, dtype=torch.uint8, **dev)
        return s
    s.step, s.seed = 7, 1234567 + int(seed)
    if c["op"] == "adamw":
        s.tensors = []
        for n in map(int, c["sizes"].split(",")):
            t = _first_moments(g, n, c["bits"], 0)
            t["p"], t["g"] = _randn(g, n) * 0.1, (_randn(g, n) * 1e-3).to(DTYPES[c["grad"]])
            s.tensors.append(t)
        if own:
            s.ctx = _context(B)
            s.hyper = B.make_adamw(bits=c["bits"], step=s.step, seed=s.seed, **HYPER)
            s.handle = B.AdamWTensors([(t["p"], t["g"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale")) for t in s.tensors])
        return s
    b, k, dim, n, r = c["batch"], c["n_neg"], c["dim"], c["n_ent"], c["n_rel"]
    i32 = dict(generator=g, device=DEV, dtype=torch.int32)
    skew = lambda hi, size: (torch.rand(size, generator=g, device=DEV).pow_(4.0) * hi).to(torch.int32).clamp_(max=hi - 1)  # noqa: E731
    h, rel, t = skew(n, b), skew(r, b), skew(n, b)
    neg_h, neg_t = h.repeat_interleave(k), torch.randint(0, n, (b * k,), **i32)
    s.touched = torch.unique(torch.cat([h, t, neg_t, rel + n])).long()
    s.grad = _randn(g, len(s.touched), dim) * 1e-3
    s.grad_w = _randn(g, len(s.touched), dim) * 1e-3 if c["model"] == "transh" else None
    s.tables = {}
    for name, rows, _ in _tables(c):
        s.tables[name] = _first_moments(g, rows * dim, c["bits"], dim)
        p = _randn(g, rows, dim) * 0.1
        s.tables[name]["p"] = (p - torch.floor(p)).remainder_(1.0) if c["model"] == "toruse" else p
    if own:
        s.ctx = B.Context(B.make_config(c["model"], "l2" if c["model"] != "toruse" else "torus_l2", n, r, dim, b, k), DEV)
        s.inc, s.grads = B.Incidence(s.ctx), B.Grads(s.ctx)
        B.stx_build_incidence(s.ctx, h, rel, t, neg_h if k else None, neg_t if k else None, k, s.inc)
        s.grads.rows[:len(s.touched)].copy_(s.grad)
        if s.grad_w is not None:
            s.grads.w_rows[:len(s.touched)].copy_(s.grad_w)
        s.params = B.Params(s.tables["ent"]["p"], *((s.tables["rel"]["p"], s.tables["w"]["p"]) if c["model"] == "transh" else ()))
        s.hyper = B.make_adamw(bits=c["bits"], step=s.step, seed=s.seed, **HYPER)
        s.moments = B.AdamWState(**{name: (t["m"], t["v"], t.get("m_scale"), t.get("v_scale")) for name, t in s.tables.items()})
    return s


def _context(B):
    """The context of a small model: what a program has whose tables the dense operators work on."""
    return B.Context(B.make_config("transe", "l2", 1_000, 20, 32, 64, 1), DEV)


# ---- one pass -------------------------------------------------------------------------------------------------

def run(s):
    return {"norm": _run_norm, "product": _run_product, "adamw": _run_adamw, "rows": _run_rows}[s.case["op"]](s)


def _values(q, cols):
    """Codes and scales of a library operand as the values they stand for."""
    return q.codes[:, :cols].view(E4M3), q.scales[:, :-(-cols // BLOCK)].view(E8M0)


def _run_norm(s):
    c = s.case
    if own:
        B = s.B
        if not c["train"]:
            B.stx_rmsnorm(s.ctx, s.x, s.res, s.weight, s.eps, s.sum, None, s.q, None)
            return s.sum, _values(s.q, c["cols"])
        B.stx_rmsnorm(s.ctx, s.x, s.res, s.weight, s.eps, s.sum, s.y, None, s.rstd)
        B.stx_rmsnorm_backward(s.ctx, s.sum, s.weight, s.rstd, s.dy, s.dsum, s.dx, s.dweight, s.work)
        return s.sum, s.y, s.rstd, s.dx, s.dweight
    dt = s.x.dtype
    total = (s.x.float() + s.res.float()).to(dt)
    f = total.float()
    rstd = 1.0 / torch.sqrt((f * f).mean(1) + s.eps)
    y = f * rstd.unsqueeze(1) * s.weight
    if not c["train"]:
        codes, scales = _quantize(y)
        return total, (codes[:, :c["cols"]], scales)
    a = s.dy.float() * s.weight
    inner = (a * f).mean(1) * rstd * rstd
    dx = (a - f * inner.unsqueeze(1)) * rstd.unsqueeze(1) + s.dsum.float()
    # (a long sum over rows of either sign: what 32 bits round in it shows where it comes near zero)
    dweight = (s.dy.float() * f * rstd.unsqueeze(1)).sum(0, dtype=torch.float64).float()
    return total, y.to(dt), rstd, dx.to(dt), dweight


def _blocks(x):
    """[rows, cols] -> [rows, blocks, 128], zeros behind the last column."""
    pad = -x.shape[1] % BLOCK
    return torch.nn.functional.pad(x, (0, pad)).view(x.shape[0], -1, BLOCK)


def _quantize(x):
    """Rows as e4m3 codes [rows, cols rounded up to whole blocks] and powers of two [rows, blocks]."""
    blocks = _blocks(x.float())
    size = blocks.abs()
    most = torch.where(torch.isfinite(size), size, 0.0).amax(-1)
    frac, exp = torch.frexp(most)             # most = frac 2**exp, 1/2 <= frac < 1, and 448 = 0.875 * 2**9
    exp = (exp - 9 + (frac > 0.875).to(exp.dtype)).clamp_(min=-126)
    exp = torch.where(most > 0, exp, 0)
    down = ((127 - exp) << 23).to(torch.int32).view(torch.float32)
    codes = (blocks * down.unsqueeze(-1)).to(E4M3)
    return codes.view(x.shape[0], -1), (exp + 127).to(torch.uint8).view(E8M0)


def _quantized(x):
    """_quantize in the layout in which the library holds it: rows of whole blocks, scales padded to four bytes."""
    codes, scales = _quantize(x)
    room = torch.full((x.shape[0], -(-scales.shape[1] // 4) * 4), 127, dtype=torch.uint8, device=DEV)
    room[:, :scales.shape[1]] = scales.view(torch.uint8)
    return codes.view(torch.uint8), room


def _dequantize(codes, scales, cols):
    blocks = -(-cols // BLOCK)
    up = (scales[:, :blocks].view(torch.uint8).to(torch.int32) << 23).view(torch.float32)
    return (codes.view(E4M3).float().view(codes.shape[0], blocks, BLOCK) * up.unsqueeze(-1)).view(codes.shape[0], -1)


def _rounded(x):
    """What is left of x after its rows are held in 8 bits."""
    return _dequantize(*_quantize(x), x.shape[1])[:, :x.shape[1]]


def _run_product(s):
    c = s.case
    if own:
        B = s.B
        if not c["train"]:
            B.stx_q8_quantize(s.ctx, s.x, s.x_q, None)
            B.stx_q8_matmul(s.ctx, s.x_q, s.table_q, s.scores, s.work)
            return s.scores, _values(s.x_q, c["k"])
        B.stx_q8_quantize(s.ctx, s.ds, s.ds_q, s.ds_qt)
        B.stx_q8_quantize(s.ctx, s.x, None, s.x_qt)
        B.stx_q8_quantize(s.ctx, s.table, None, s.table_qt)
        B.stx_q8_matmul(s.ctx, s.ds_q, s.table_qt, s.dx, s.work)
        B.stx_q8_matmul(s.ctx, s.ds_qt, s.x_qt, s.dtable, s.work)
        return s.dx, s.dtable
    out = DTYPES[c["out"]]
    if not c["train"]:
        codes, scales = _quantize(s.x)
        scores = _dequantize(codes, scales, c["k"]) @ _dequantize(s.codes, s.scales, c["k"]).T
        return scores.to(out), (codes[:, :c["k"]], scales)
    dx = _rounded(s.ds) @ _rounded(s.table.T).T
    dtable = _rounded(s.ds.T) @ _rounded(s.x.T).T
    return dx.to(out), dtable.to(out)


def _mix(z):
    """The output function of SplitMix64 on 64-bit integers that wrap."""
    z = (z ^ ((z >> 30) & (2**34 - 1))) * MIX1
    z = (z ^ ((z >> 27) & (2**37 - 1))) * MIX2
    return z ^ ((z >> 31) & (2**33 - 1))


def _noise(seed, step, tensor, index):
    """16 random bits for each moment of the elements `index` of a tensor: SplitMix64 output number index / 2 of the sequence
    whose seed is output step 2**16 + tensor of the one seeded with `seed`; an even element takes the low 32 bits, an odd one
    the high ones, the first moment the lower half of them."""
    first = torch.tensor((seed + GOLDEN * ((step << 16) + tensor + 1) + 2**63) % 2**64 - 2**63, dtype=torch.int64, device=DEV)
    z = _mix(_mix(first) + GOLDEN * ((index >> 1) + 1)) >> (32 * (index & 1))
    return (z & 0xFFFF).to(torch.int32), ((z >> 16) & 0xFFFF).to(torch.int32)


def _round(x, noise, drop, tiny, top):
    """x >= 0 to an 8-bit format that keeps 23 - drop bits of the mantissa, up or down by the noise; below `tiny` the format's
    steps are all alike, and above `top` there is nothing."""
    low = x < tiny
    z = torch.where(low, x + tiny, x)
    z = ((z.view(torch.int32) + (noise << (drop - 16))) & -(1 << drop)).view(torch.float32)
    return torch.where(low, z - tiny, z).clamp_(max=top)


def _moments(new, noise, drop, tiny, top, least):
    """Values [rows, width] as codes and a scale for each block of 128: the block's largest magnitude over the format's largest
    number (0, with codes of 0, where the largest is below 2**-100).  `least`: the smallest code of a value that is not 0."""
    rows, width = new.shape
    blocks = _blocks(new)
    most = blocks.abs().amax(-1, keepdim=True)
    live = most >= 2.0**-100
    scale = torch.where(live, most * (1.0 / top), 0.0)
    x = torch.where(live, blocks.abs() * (top / most), 0.0)
    x = _round(x, _blocks(noise), drop, tiny, top)
    x = torch.where((x == 0) & live & (blocks != 0), least, x)
    return torch.copysign(x, blocks).view(rows, -1)[:, :width], scale.squeeze(-1)


def _adamw(p, g, m, v, step):
    """One step on fp32 values: the new p, m and v.  Every operation is rounded once."""
    h = HYPER
    one = lambda b: torch.tensor(1.0 - b, dtype=torch.float64).float().item()  # noqa: E731
    m = m * h["beta1"] + g * one(h["beta1"])
    v = v * h["beta2"] + (g * g) * one(h["beta2"])
    size = h["lr"] / (1.0 - h["beta1"] ** step)
    root = 1.0 / math.sqrt(1.0 - h["beta2"] ** step)
    p = p - p * (h["lr"] * h["weight_decay"])
    return p - (m * size) / (torch.sqrt(v) * root + h["eps"]), m, v


def _adamw_values(t, p, g, pick, tensor, index, s):
    """A step on the rows `pick` of a tensor with its moments; returns the new p rows and stores the moments."""
    rows, width = p.shape
    if s.case["bits"] == 32:
        m, v = t["m"].view(-1, width), t["v"].view(-1, width)
        p, m[pick], v[pick] = _adamw(p, g, m[pick], v[pick], s.step)
        return p
    mc, vc = t["m"].view(-1, width), t["v"].view(-1, width)
    blocks = -(-width // BLOCK)
    m_scale, v_scale = t["m_scale"].view(-1, blocks), t["v_scale"].view(-1, blocks)
    spread = lambda scale: scale[pick].repeat_interleave(BLOCK, 1)[:, :width]  # noqa: E731
    p, m, v = _adamw(p, g, mc[pick].view(E4M3).float() * spread(m_scale), vc[pick].view(E5M2).float() * spread(v_scale), s.step)
    m_noise, v_noise = _noise(s.seed, s.step, tensor, index)
    m, m_scale[pick] = _moments(m, m_noise, 20, 2.0**-6, 448.0, 0.0)
    mc[pick] = m.to(E4M3).view(torch.uint8)
    v, v_scale[pick] = _moments(v, v_noise, 21, 2.0**-14, 57344.0, 2.0**-16)
    vc[pick] = v.to(E5M2).view(torch.uint8)
    return p


def _updated(tensors, bits):
    if bits == 32:
        return [(t["p"], t["m"], t["v"]) for t in tensors]
    return [(t["p"], t["m"].view(E4M3), t["v"].view(E5M2), t["m_scale"], t["v_scale"]) for t in tensors]


def _few(outs):
    """The outputs of many tensors end to end, so that they are a few outputs."""
    return [torch.cat([o.view(torch.uint8).reshape(-1) if o.element_size() == 1 else o.reshape(-1) for o in kind]).view(kind[0].dtype)
            for kind in zip(*outs)] if len(outs) > 10 else outs


def _run_adamw(s):
    if own:
        s.hyper.step = s.step
        s.B.stx_adamw_tensors(s.ctx, s.hyper, s.handle)
    else:
        for i, t in enumerate(s.tensors):
            n = t["p"].numel()
            t["p"].copy_(_adamw_values(t, t["p"].view(1, n), t["g"].view(1, n).float(), slice(None), i,
                                       torch.arange(n, device=DEV).view(1, n), s).view(-1))
    s.step += 1
    return _few(_updated(s.tensors, s.case["bits"]))


def _run_rows(s):
    c = s.case
    if own:
        s.hyper.step = s.step
        s.B.stx_adamw_step(s.ctx, s.params, s.inc, s.grads, s.hyper, s.moments)
        s.step += 1
        return _updated(s.tables.values(), c["bits"])
    for i, (name, rows, first) in enumerate(_tables(c)):
        t = s.tables[name]
        mine = (s.touched >= first) & (s.touched < first + rows)
        pick = s.touched[mine] - first
        grad = (s.grad_w if name == "w" else s.grad)[mine]
        index = pick.unsqueeze(1) * c["dim"] + torch.arange(c["dim"], device=DEV)
        p = _adamw_values(t, t["p"][pick], grad, pick, i, index, s)
        if c["model"] == "toruse":            # only the fractional part is kept
            p = p - torch.floor(p)
            p = torch.where(p >= 1.0, 0.0, p)
        t["p"][pick] = p
    s.step += 1
    return _updated(s.tables.values(), c["bits"])


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    """Every input read once and every output written once; the arithmetic of the formulas."""
    c = case
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}
    if c["op"] == "norm":
        n, e = float(c["rows"]) * c["cols"], size[c["dtype"]]
        if c["train"]:                        # x, residual, dy, dsum in; sum, y, dx out
            return {"bytes": n * e * 7 + 4.0 * (2 * c["cols"] + c["rows"]), "flops": 16.0 * n}
        return {"bytes": n * (3 * e + 1.0 + 1.0 / BLOCK) + 4.0 * c["cols"], "flops": 7.0 * n}
    if c["op"] == "product":
        m, n, k = float(c["m"]), float(c["n"]), float(c["k"])
        e, o = size[c["dtype"]], size[c["out"]]
        if c["train"]:
            return {"bytes": m * n * e + m * k * e + n * k * 4.0 + (m + n) * k * o, "flops": 4.0 * m * n * k}
        return {"bytes": m * k * (e + 1.0) + n * k * (1.0 + 1.0 / BLOCK) + m * n * o, "flops": 2.0 * m * n * k}
    if c["op"] == "adamw":
        n, g = float(sum(map(int, c["sizes"].split(",")))), size[c["grad"]]
    else:
        b, k, ents = c["batch"], c["n_neg"], c["n_ent"]
        # the entities that 2 b heads and tails (the first ids most often) and b k uniform negative tails touch
        share = np.diff((np.arange(ents + 1) / ents) ** 0.25)
        ent = float(-np.expm1(-2.0 * b * share).sum())
        ent += (ents - ent) * -math.expm1(-float(b * k) / ents)
        rel = min(c["n_rel"], b)
        n = (ent + rel * (2 if c["model"] == "transh" else 1)) * c["dim"]
        g = 4.0
    per = 8.0 + g + (16.0 if c["bits"] == 32 else 4.0 + 16.0 / BLOCK)
    return {"bytes": n * per, "flops": n * (14.0 if c["bits"] == 32 else 40.0)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, from the formulas in 64 bits; 8-bit codes as the numbers nearest to them."""
    held = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "adamw": _exact_adamw, "rows": _exact_rows}[case["op"]](held, case)


def _exact_norm(s, c):
    low = lambda t: t.to(DTYPES[c["dtype"]]).double()  # noqa: E731
    total = low(s.x.double() + s.res.double())   # the sum is rounded to its type before the norm is taken
    rms = torch.sqrt(total.pow(2).sum(1) / c["cols"] + s.eps)
    unit = total / rms[:, None]
    y = unit * s.weight.double()
    if not c["train"]:
        return total, _exact_codes(y)
    a = s.dy.double() * s.weight.double()
    dx = (a - unit * (a * unit).sum(1, keepdim=True) / c["cols"]) / rms[:, None] + s.dsum.double()
    return total, y, 1.0 / rms, dx, (s.dy.double() * unit).sum(0)


def _exact_steps(x, bits, low, top):
    """x to the nearest number with `bits` bits behind its leading one, exponents from `low` on; ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0**-1000)))
    e = torch.where(torch.exp2(e) > x.abs(), e - 1, torch.where(torch.exp2(e + 1) <= x.abs(), e + 1, e)).clamp(min=low)
    step = torch.exp2(e - bits)
    return (torch.round(x / step) * step).clamp(-top, top)


def _exact_codes(x):
    rows, cols = x.shape
    whole = torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.float64, device=x.device)
    whole[:, :cols] = x
    whole = whole.reshape(rows, -1, 128)
    most = whole.abs().amax(2)
    e = torch.ceil(torch.log2(most.clamp(min=2.0**-1000) / 448.0))
    e = torch.where(most > 448.0 * torch.exp2(e), e + 1, torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e))
    scale = torch.where(most > 0, torch.exp2(e.clamp(min=-126)), 1.0)
    return _exact_steps(whole / scale[..., None], 3, -6, 448.0).reshape(rows, -1)[:, :cols], scale


def _exact_held(x):
    codes, scale = _exact_codes(x.double())
    return codes * scale.repeat_interleave(128, 1)[:, :codes.shape[1]]


def _exact_product(s, c):
    if c["train"]:
        return _exact_held(s.ds) @ _exact_held(s.table.T).T.contiguous(), _exact_held(s.ds.T) @ _exact_held(s.x.T).T.contiguous()
    codes, scale = _exact_codes(s.x.double())
    table = s.codes[:, :c["k"]].view(E4M3).double() * torch.exp2(s.scales.double() - 127.0).repeat_interleave(128, 1)[:, :c["k"]]
    x = codes * scale.repeat_interleave(128, 1)[:, :c["k"]]
    return x @ table.T.contiguous(), (codes, scale)


def _exact_bits(seed, step, tensor, index):
    """The random bits of the elements, as numbers in [0, 1)."""
    word = lambda v: ((v + 2**63) % 2**64) - 2**63  # noqa: E731
    shift = lambda z, n: torch.bitwise_and(torch.bitwise_right_shift(z, n), (1 << (64 - n)) - 1)  # noqa: E731

    def out(z):
        z = torch.bitwise_xor(z, shift(z, 30)) * word(0xBF58476D1CE4E5B9)
        z = torch.bitwise_xor(z, shift(z, 27)) * word(0x94D049BB133111EB)
        return torch.bitwise_xor(z, shift(z, 31))

    key = out(torch.full((1,), word(seed + 0x9E3779B97F4A7C15 * (step * 65536 + tensor + 1)), dtype=torch.int64, device=DEV))
    z = out(key + (torch.div(index, 2, rounding_mode="floor") + 1) * word(0x9E3779B97F4A7C15))
    z = torch.where(index % 2 == 1, shift(z, 32), z)
    return torch.bitwise_and(z, 65535).double() / 65536, torch.bitwise_and(shift(z, 16), 65535).double() / 65536


def _exact_store(x, u, bits, low, top, least):
    rows, width = x.shape
    blocks = -(-width // 128)
    room = lambda t: torch.nn.functional.pad(t, (0, blocks * 128 - width)).reshape(rows, blocks, 128)  # noqa: E731
    b = room(x)
    most = b.abs().amax(2, keepdim=True)
    live = most >= 2.0**-100
    y = torch.where(live, b.abs() * top / most.clamp(min=2.0**-1000), 0.0)
    e = torch.floor(torch.log2(y.clamp(min=2.0**-1000)))
    e = torch.where(torch.exp2(e) > y, e - 1, torch.where(torch.exp2(e + 1) <= y, e + 1, e)).clamp(min=low)
    step = torch.exp2(e - bits)
    q = (torch.floor(y / step + room(u)) * step).clamp(max=top)
    q = torch.where((q == 0) & (y > 0), least, q) * torch.sign(b)
    return q.reshape(rows, -1)[:, :width], torch.where(live, most / top, 0.0)[..., 0]


def _exact_step(c, s, t, p, g, pick, tensor, index):
    """(p, m, v[, m_scale, v_scale]) of the rows `pick`."""
    width = p.shape[1]
    h, step = HYPER, s.step
    m, v = t["m"].view(-1, width)[pick], t["v"].view(-1, width)[pick]
    if c["bits"] == 8:
        blocks = -(-width // 128)
        wide = lambda x: x.view(-1, blocks)[pick].double().repeat_interleave(128, 1)[:, :width]  # noqa: E731
        m, v = m.view(E4M3).double() * wide(t["m_scale"]), v.view(E5M2).double() * wide(t["v_scale"])
    m = h["beta1"] * m.double() + (1 - h["beta1"]) * g
    v = h["beta2"] * v.double() + (1 - h["beta2"]) * g * g
    p = p * (1 - h["lr"] * h["weight_decay"]) - h["lr"] * (m / (1 - h["beta1"] ** step)) / (torch.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"])
    if c["bits"] == 32:
        return p, m, v
    um, uv = _exact_bits(s.seed, step, tensor, index)
    m, m_scale = _exact_store(m, um, 3, -6, 448.0, 0.0)
    v, v_scale = _exact_store(v, uv, 2, -14, 57344.0, 2.0**-16)
    return p, m, v, m_scale, v_scale


def _exact_adamw(s, c):
    outs = []
    for i, t in enumerate(s.tensors):
        n = t["p"].numel()
        got = _exact_step(c, s, t, t["p"].double().view(1, n), t["g"].double().view(1, n), slice(None), i, torch.arange(n, device=DEV).view(1, n))
        outs.append([x.reshape(-1) for x in got])
        t.clear()
    return [torch.cat(kind) for kind in zip(*outs)] if len(outs) > 10 else outs


def _exact_rows(s, c):
    outs = []
    for i, (name, rows, first) in enumerate(_tables(c)):
        t = s.tables[name]
        mine = (s.touched >= first) & (s.touched < first + rows)
        pick = s.touched[mine] - first
        index = pick[:, None] * c["dim"] + torch.arange(c["dim"], device=DEV)[None]
        grad = (s.grad_w if name == "w" else s.grad)[mine].double()
        new = list(_exact_step(c, s, t, t["p"][pick].double(), grad, pick, i, index))
        if c["model"] == "toruse":
            part = new[0] - torch.floor(new[0])
            new[0] = torch.where(part.float() >= 1.0, 0.0, part)   # (part of the definition: 0 where it rounds to 1)
        whole = [t["p"].double(), t["m"].double(), t["v"].double()]
        if c["bits"] == 8:
            whole = [whole[0], t["m"].view(E4M3).double(), t["v"].view(E5M2).double(), t["m_scale"].double(), t["v_scale"].double()]
        for all_rows, mine_rows in zip(whole, new):
            all_rows.view(rows, -1)[pick] = mine_rows
        outs.append(whole)
    return outs
