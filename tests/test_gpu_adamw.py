"""stx_adamw_tensors and stx_adamw_step against 64 bits, moments in 32 and in 8 bits."""
import numpy as np
import pytest
import torch

from paper_2502_16949_amd import binding as B
from tests import gpu_util as G
from tests import ops_ref as R

pytestmark = pytest.mark.gpu

H = {"lr": 3e-3, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "weight_decay": 0.1}
# m and v: products, sums and the constants' own roundings
MV = 5 * R.U


@pytest.fixture(scope="module")
def ctx():
    return B.Context(B.make_config("transe", "l2", 100, 5, 32, 64, 1), G.DEV)


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(G.DEV, dtype)


def moments(rng, rows, width, bits):
    """(tensors, m, v as numbers): random ones, in 8 bits as codes and scales."""
    nb = -(-width // 128)
    if bits == 32:
        m, v = rng.standard_normal((rows, width)) * 1e-2, rng.standard_normal((rows, width)) ** 2 * 1e-4
        t = dev(m), dev(v)
        return t, R.f64(t[0]), R.f64(t[1])
    mc, vc = rng.integers(0, 256, (rows, width), dtype=np.uint8), rng.integers(0, 0x7C, (rows, width), dtype=np.uint8)
    mc[(mc & 0x7F) == 0x7F] = 0
    ms, vs = (rng.uniform(0.5, 1, (rows, nb)).astype(np.float32) * f for f in (1e-5, 1e-9))
    t = dev(mc, torch.uint8), dev(vc, torch.uint8), dev(ms), dev(vs)
    wide = lambda s: np.repeat(s.astype(np.float64), 128, 1)[:, :width]  # noqa: E731
    return t, R.decode(mc, 0) * wide(ms), R.decode(vc, 1) * wide(vs)


def check(t, p_got, p, g, m, v, bits, step, seed, number, index, decay=True, scale=1.0, wrap=None):
    """One tensor's rows after a step against the numbers before it."""
    want, wm, wv = R.adamw(p, g, m, v, H, step, decay, scale)
    size_m = np.abs(H["beta1"] * m) + np.abs((1 - H["beta1"]) * g * scale)
    move = np.abs(want - p)
    root = np.sqrt(wv / (1 - H["beta2"] ** step)) + H["eps"]
    part = H["lr"] / (1 - H["beta1"] ** step) * size_m / root           # m's own error, through the quotient
    tol = 4 * R.U * (np.abs(p) + move) + 16 * R.U * (move + part) + 1e-30
    if wrap:
        tol += R.U                                                       # p - floor(p) is rounded once, below 1
    got = R.f64(p_got)
    assert np.all(np.abs((wrap or (lambda d: d))(got - want)) <= tol)
    if bits == 32:
        assert np.all(np.abs(R.f64(t[0]) - wm) <= MV * size_m + 1e-40) and np.all(np.abs(R.f64(t[1]) - wv) <= MV * wv + 1e-40)
        return
    um, uv = R.noise(seed, step, number, index)
    R.check_moment(t[0].cpu().numpy().reshape(wm.shape), R.f64(t[2]).reshape(len(wm), -1), wm, MV * size_m, um, 0)
    R.check_moment(t[1].cpu().numpy().reshape(wv.shape), R.f64(t[3]).reshape(len(wv), -1), wv, MV * wv, uv, 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [4, 0, 127, 128, 129, 4096, 4097], [20_001, 3], [513] * 101 + [0]])
def test_tensors(ctx, sizes, gtype, bits):
    rng = np.random.default_rng(len(sizes) + bits)
    held, before = [], []
    for i, n in enumerate(sizes):
        room = torch.full((n + 5,), 55.0, device=G.DEV)
        p = room[i % 2:i % 2 + n]                            # the second tensor begins 4 bytes into its allocation
        p.copy_(dev(rng.standard_normal(n)))
        g = dev(rng.standard_normal(n) * 1e-2, gtype)
        t, m, v = moments(rng, 1, n, bits) if n else ((torch.empty(0, device=G.DEV),) * 2 if bits == 32 else
                                                      (torch.empty(0, dtype=torch.uint8, device=G.DEV),) * 2 + (torch.empty(0, device=G.DEV),) * 2, None, None)
        held.append((p, g, *(x.view(-1) for x in t)))
        before.append((room, R.f64(p)[None], R.f64(g)[None], m, v))
    step, seed = 5, 991
    scale = torch.tensor([0.5], device=G.DEV)
    h = B.make_adamw(**H, bits=bits, step=step, seed=seed, grad_scale=scale)
    B.stx_adamw_tensors(ctx, h, B.AdamWTensors(held, no_decay=(2,)))
    for i, ((room, p, g, m, v), (pt, _, *t)) in enumerate(zip(before, held)):
        if p.size:
            check(t, pt[None], p, g, m, v, bits, step, seed, i, np.arange(p.size)[None], decay=i != 2, scale=0.5)
        assert (room[:i % 2] == 55.0).all() and (room[i % 2 + p.size:] == 55.0).all()


def test_first_step_from_zero(ctx):
    # m and v of zero, t = 1: every element moves by lr against its gradient's sign
    for bits in (32, 8):
        n = 1000
        p, g = torch.zeros(n, device=G.DEV), torch.randn(n, device=G.DEV)
        g[17] = 0
        t = [torch.zeros(n, device=G.DEV) for _ in range(2)] if bits == 32 else \
            [torch.zeros(n, dtype=torch.uint8, device=G.DEV) for _ in range(2)] + [torch.zeros(8, device=G.DEV) for _ in range(2)]
        h = B.make_adamw(lr=0.1, eps=0.0 if bits == 32 else 1e-12, bits=bits, step=1)
        B.stx_adamw_tensors(ctx, h, B.AdamWTensors([(p, g, *t)]))
        want = -0.1 * torch.sign(g)
        keep = torch.arange(n, device=G.DEV) != 17
        assert torch.allclose(p[keep], want[keep], rtol=1e-6)
        assert (p[17].isnan() if bits == 32 else p[17] == 0)     # 0 / (0 + 0) is what the formula says without eps


def test_eight_bit_average_keeps_small_changes(ctx):
    # v falls by 1 % a step where the gradient is 0 while its block's largest stays: a rounding to nearest would hold it
    n = 128 * 400
    g = torch.zeros(n, device=G.DEV)
    g[::128] = 1.0
    p, codes = torch.zeros(n, device=G.DEV), [torch.zeros(n, dtype=torch.uint8, device=G.DEV) for _ in range(2)]
    scales = [torch.zeros(n // 128, device=G.DEV) for _ in range(2)]
    codes[1].fill_(0x3C)                                     # v = 1.0 everywhere, the largest 57344
    codes[1][::128] = 0x7B
    scales[1].fill_(1e-4)
    held = B.AdamWTensors([(p, g, *codes, *scales)])
    h = B.make_adamw(lr=0.0, beta2=0.99, bits=8, seed=5)
    for step in range(1, 41):
        h.step = step
        B.stx_adamw_tensors(ctx, h, held)
    v = R.decode(codes[1].cpu().numpy(), 1).reshape(-1, 128)[:, 1:] * R.f64(scales[1])[:, None]
    # each step's rounding has at most a quarter of a step squared as variance, a step is at most 1/4 of the value, and over 40 steps
    # and 50,800 elements the average is off by less than five of its deviations
    assert abs(v.mean() / (1e-4 * 0.99**40) - 1) <= 5 * np.sqrt(40 / 16 / 16 / v.size)


def test_non_finite_gradient_spoils_its_block_only(ctx):
    for bad in (float("nan"), float("inf")):
        n = 512
        p, g = torch.zeros(n, device=G.DEV), torch.ones(n, device=G.DEV)
        g[200] = bad
        t = [torch.zeros(n, dtype=torch.uint8, device=G.DEV) for _ in range(2)] + [torch.zeros(4, device=G.DEV) for _ in range(2)]
        B.stx_adamw_tensors(ctx, B.make_adamw(lr=0.1, bits=8, step=1), B.AdamWTensors([(p, g, *t)]))
        assert p.isnan().sum() == 1 and p[200].isnan()
        for s in t[2:]:
            assert s.isnan().tolist() == [False, True, False, False]


def test_step_from_device_memory(ctx):
    rng = np.random.default_rng(8)
    for bits in (32, 8):
        n = 700
        outs = []
        for device_step in (False, True):
            r = np.random.default_rng(8)
            p, g = dev(r.standard_normal(n)), dev(r.standard_normal(n))
            t, _, _ = moments(r, 1, n, bits)
            where = torch.tensor([123], dtype=torch.int64, device=G.DEV) if device_step else None
            h = B.make_adamw(**H, bits=bits, step=0 if device_step else 123, seed=77, step_dev=where)
            B.stx_adamw_tensors(ctx, h, B.AdamWTensors([(p, g, *(x.view(-1) for x in t))]))
            outs.append([p, *t])
        for a, b in zip(*outs):
            assert torch.equal(a, b)
    del rng


# ---- touched rows ---------------------------------------------------------------------------------------------------

def _model(model, n_ent, n_rel, dim, rel_dim, b, k, seed, flags=0):
    dist = "torus_l1" if model == "toruse" else "l2"
    ctx = B.Context(B.make_config(model, dist, n_ent, n_rel, dim, b, k, rel_dim=rel_dim, flags=flags), G.DEV)
    rng = np.random.default_rng(seed)
    h, t = (G.dev_i32(rng.integers(0, n_ent, b)) for _ in range(2))
    r = G.dev_i32(rng.integers(0, n_rel, b))
    nh, nt = (G.dev_i32(rng.integers(0, n_ent, b * k)) for _ in range(2))
    inc, grads = B.Incidence(ctx), B.Grads(ctx)
    B.stx_build_incidence(ctx, h, r, t, nh if k else None, nt if k else None, k, inc)
    stacked = model in ("transe", "toruse")
    ent = dev(rng.uniform(0, 1, (n_ent + (n_rel if stacked else 0), dim)))
    rel = None if stacked else dev(rng.standard_normal((n_rel, rel_dim or dim)))
    w = dev(rng.standard_normal((n_rel, dim))) if model == "transh" else None
    proj = dev(rng.standard_normal((n_rel, rel_dim, dim))) if model == "transr" else None
    for gt in (grads.rows, grads.w_rows, grads.proj):
        if gt is not None:
            gt.copy_(dev(rng.standard_normal(tuple(gt.shape)) * 1e-2))
    return ctx, inc, grads, B.Params(ent, rel, w=w, proj=proj), rng


MODELS = [("transe", 300, 7, 4, 0), ("transe", 200, 9, 32, 0), ("toruse", 500, 3, 64, 0), ("transe", 60, 4, 128, 0), ("toruse", 90, 5, 200, 0),
          ("transe", 400, 11, 516, 0), ("transe", 100, 8, 1024, 0), ("transh", 150, 12, 100, 0), ("transh", 80, 6, 256, 0),
          ("transr", 120, 9, 32, 96), ("transr", 70, 5, 128, 64)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("model,n_ent,n_rel,dim,rel_dim", MODELS)
def test_touched_rows(model, n_ent, n_rel, dim, rel_dim, bits):
    flags = {"transr": B.STX_FLAG_BF16_PROJ, "transh": 0}.get(model, 0)
    ctx, inc, grads, params, rng = _model(model, n_ent, n_rel, dim, rel_dim, 23, 2, dim + bits, flags)
    names = [n for n in ("ent", "rel", "w", "proj") if getattr(params, n) is not None]
    held, before = {}, {}
    for n in names:
        t = getattr(params, n)
        rows, width = t.shape[0], t.numel() // t.shape[0]
        held[n], m, v = moments(rng, rows, width, bits)
        before[n] = (R.f64(t).reshape(rows, width), m, v, [x.clone() for x in held[n]], t.clone())
    step, seed = 9, 31337
    B.stx_adamw_step(ctx, params, inc, grads, B.make_adamw(**H, bits=bits, step=step, seed=seed), B.AdamWState(**held))
    torch.cuda.synchronize()
    u = int(inc.n_touched.item())
    cols = inc.at_touched_cols[:u].cpu().numpy().astype(np.int64)
    for number, n in enumerate(("ent", "rel", "w", "proj")):
        if n not in names:
            continue
        p, m, v, t0, p0 = before[n]
        rows, width = p.shape
        first = 0 if n == "ent" else n_ent
        seg = np.nonzero((cols >= first) & (cols < first + rows))[0]
        pick = cols[seg] - first
        if n == "proj":
            g = R.f64(grads.proj).reshape(rows, width)[pick]
        else:
            g = R.f64(grads.w_rows if n == "w" else grads.rows)[seg][:, :width]
        now = getattr(params, n).reshape(rows, width)
        index = pick[:, None] * width + np.arange(width)
        wrap = (lambda d: d - np.round(d)) if model == "toruse" else None
        if model == "toruse":
            assert float(now.min()) >= 0 and float(now.max()) < 1
        check([x.reshape(rows, -1)[torch.from_numpy(pick).to(G.DEV)] for x in held[n]], now[torch.from_numpy(pick).to(G.DEV)], p[pick], g, m[pick],
              v[pick], bits, step, seed, number, index, wrap=wrap)
        rest = torch.ones(rows, dtype=torch.bool, device=G.DEV)
        rest[torch.from_numpy(pick).to(G.DEV)] = False
        assert torch.equal(now[rest], p0.reshape(rows, width)[rest])
        for a, b in zip(held[n], t0):
            assert torch.equal(a.reshape(rows, -1)[rest], b.reshape(rows, -1)[rest])


@pytest.mark.parametrize("bits", [32, 8])
def test_transh_normals_stay_unit(bits):
    ctx, inc, grads, params, _ = _model("transh", 100, 20, 128, 0, 16, 1, 3, B.STX_FLAG_RENORM_W)
    state = B.AdamWState.zeros(params, bits)
    before = params.w.clone()
    B.stx_adamw_step(ctx, params, inc, grads, B.make_adamw(**H, bits=bits, step=1), state)
    moved = (params.w != before).any(1)
    assert 0 < int(moved.sum()) < 20
    assert torch.allclose(params.w[moved].norm(dim=1), torch.ones(int(moved.sum()), device=G.DEV), rtol=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_rows_and_tensors_agree(ctx, bits):
    # a batch that touches every row of a table whose width is whole blocks: both calls do the same
    n_ent, n_rel, dim = 40, 5, 128
    c = B.Context(B.make_config("transe", "l2", n_ent, n_rel, dim, 200, 0), G.DEV)
    ids = np.arange(200)
    inc, grads = B.Incidence(c), B.Grads(c)
    B.stx_build_incidence(c, G.dev_i32(ids % n_ent), G.dev_i32(ids % n_rel), G.dev_i32((ids + 1) % n_ent), None, None, 0, inc)
    grads.rows.normal_()
    a, g = torch.randn(n_ent + n_rel, dim, device=G.DEV), grads.rows.clone()
    b = a.clone()
    sa, sb = B.AdamWState.zeros(B.Params(a), bits), B.AdamWState.zeros(B.Params(b), bits)
    held = B.AdamWTensors([(b.view(-1), g.view(-1), *(None if t is None else t.view(-1) for t in sb.held["ent"].keep))])
    for step in (1, 2, 3):
        h = B.make_adamw(**H, bits=bits, step=step, seed=4)
        B.stx_adamw_step(c, B.Params(a), inc, grads, h, sa)
        B.stx_adamw_tensors(ctx, h, held)
    assert torch.equal(a, b)
    for x, y in zip(sa.held["ent"].keep, sb.held["ent"].keep):
        assert x is None or torch.equal(x, y)


def test_step_invalidates_a_stored_forward():
    ctx, inc, grads, params, _ = _model("transe", 100, 5, 32, 0, 16, 1, 3)
    scores, loss = torch.empty(32, device=G.DEV), torch.empty(1, device=G.DEV)
    B.stx_forward(ctx, inc, params, scores, loss)
    B.stx_adamw_step(ctx, params, inc, grads, B.make_adamw(**H, step=1), B.AdamWState.zeros(params))
    with pytest.raises(B.StxError) as e:
        B.stx_backward(ctx, inc, params, grads)
    assert e.value.status == B.STX_ERR_STATE


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("model,dim,rel_dim", [("toruse", 64, 0), ("transh", 100, 0), ("transr", 32, 96)])
def test_touched_rows_step_and_scale_from_device_memory(model, dim, rel_dim, bits):
    outs = []
    for device in (False, True):
        ctx, inc, grads, params, rng = _model(model, 120, 9, dim, rel_dim, 23, 2, 7, B.STX_FLAG_BF16_PROJ if model == "transr" else 0)
        names = [n for n in ("ent", "rel", "w", "proj") if getattr(params, n) is not None]
        held = {n: moments(rng, getattr(params, n).shape[0], getattr(params, n)[0].numel(), bits)[0] for n in names}
        if device:                                           # made here and dropped: the hyperparameters keep them
            h = B.make_adamw(**H, bits=bits, step=0, seed=8, step_dev=torch.tensor([41], dtype=torch.int64, device=G.DEV),
                             grad_scale=torch.tensor([0.25], device=G.DEV))
        else:
            h = B.make_adamw(**H, bits=bits, step=41, seed=8)
            for g in (grads.rows, grads.w_rows, grads.proj):
                if g is not None:
                    g.mul_(0.25)                             # a power of two: the products are the same
        B.stx_adamw_step(ctx, params, inc, grads, h, B.AdamWState(**held))
        outs.append([getattr(params, n) for n in names] + [t for n in names for t in held[n]])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
