"""Thin ctypes binding of libstx (include/stx.h): same names, argument marshalling only.

PyTorch is used for device memory and the stream; every step of the method runs in the library's
HIP kernels.  There is no CPU fallback: if libstx.so is missing or a call fails, this raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstx.so")

STX_OK = 0
STX_ERR_NULL, STX_ERR_BAD_ARG, STX_ERR_INDEX_RANGE, STX_ERR_WORKSPACE = 1, 2, 3, 4
STX_ERR_STATE, STX_ERR_UNSUPPORTED, STX_ERR_HIP, STX_ERR_STATIC_LIMIT = 5, 6, 7, 8
STX_STATIC_WORK_BYTES = 96 << 20
STX_TRANSE, STX_TRANSH, STX_TRANSR, STX_TORUSE = 0, 1, 2, 3
STX_L1, STX_L2, STX_TORUS_L1, STX_TORUS_L2, STX_L2_SQ = 0, 1, 2, 3, 4
STX_SUM, STX_MEAN = 0, 1
STX_FLAG_RENORM_W, STX_FLAG_BF16_PROJ = 1, 2
STX_DISTMULT, STX_COMPLEX, STX_ROTATE = 0, 1, 2
STX_TAIL, STX_HEAD = 0, 1
STX_F32, STX_BF16, STX_F16 = 0, 1, 2
STX_E4M3, STX_E5M2 = 0, 1
STX_ADAMW_NO_DECAY = 1

MODELS = {"transe": STX_TRANSE, "transh": STX_TRANSH, "transr": STX_TRANSR, "toruse": STX_TORUSE}
DTYPES = {torch.float32: STX_F32, torch.bfloat16: STX_BF16, torch.float16: STX_F16}
DISTS = {"l1": STX_L1, "l2": STX_L2, "torus_l1": STX_TORUS_L1, "torus_l2": STX_TORUS_L2, "l2_sq": STX_L2_SQ}

EXPORTS = ["stx_workspace_bytes", "stx_create", "stx_destroy", "stx_sample_negatives", "stx_build_incidence",
           "stx_check_indices", "stx_spmm", "stx_spmm_semiring", "stx_spmm_semiring_t", "stx_spmm_semiring_t_static", "stx_rank", "stx_rank_work_bytes", "stx_rmsnorm", "stx_rmsnorm_backward", "stx_rmsnorm_backward_work_bytes",
           "stx_q8_quantize", "stx_q8_matmul", "stx_q8_matmul_work_bytes", "stx_adamw_tensors", "stx_adamw_step", "stx_forward", "stx_backward", "stx_sgd_step", "stx_backward_sgd", "stx_train_step", "stx_profile_kernel",
           "stx_profile_every", "stx_profile_read", "stx_profile_dump", "stx_copy_f32", "stx_read_sectors", "stx_status_string"]


class StxError(RuntimeError):
    def __init__(self, call: str, status: int):
        self.status = status
        super().__init__(f"{call}: {status_string(status)} (status {status})")


class stx_config(C.Structure):
    _fields_ = [("model", C.c_int32), ("dist", C.c_int32), ("reduce", C.c_int32), ("dim", C.c_int32),
                ("rel_dim", C.c_int32), ("n_ent", C.c_int64), ("n_rel", C.c_int64), ("margin", C.c_float),
                ("max_batch", C.c_int32), ("max_neg", C.c_int32), ("flags", C.c_uint32)]


class stx_params(C.Structure):
    _fields_ = [("ent", C.c_void_p), ("rel", C.c_void_p), ("w", C.c_void_p), ("proj", C.c_void_p),
                ("rel_weight", C.c_void_p)]


class stx_incidence(C.Structure):
    _fields_ = [("b", C.c_int32), ("k", C.c_int32), ("n_rows", C.c_int64), ("nnz", C.c_int64),
                ("a_rowptr", C.c_void_p), ("a_colidx", C.c_void_p), ("a_vals", C.c_void_p),
                ("at_touched_cols", C.c_void_p), ("at_seg_ptr", C.c_void_p), ("at_row_idx", C.c_void_p),
                ("at_sign", C.c_void_p), ("at_seg_id", C.c_void_p), ("at_packed", C.c_void_p),
                ("n_touched", C.c_void_p)]


class stx_grads(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("w_rows", C.c_void_p), ("proj", C.c_void_p)]


class stx_batch(C.Structure):
    _fields_ = [("h", C.c_void_p), ("r", C.c_void_p), ("t", C.c_void_p), ("b", C.c_int32), ("k", C.c_int32),
                ("seed", C.c_uint64), ("epoch", C.c_uint64), ("m_total", C.c_int64), ("global_offset", C.c_int64),
                ("neg_h", C.c_void_p), ("neg_t", C.c_void_p), ("next", C.c_void_p)]


class stx_q8(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64),
                ("ld_scale", C.c_int64), ("format", C.c_int32)]


class stx_adamw(C.Structure):
    held, index = (), None                     # device tensors that it points to (make_adamw), and their device
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("step", C.c_int64), ("step_dev", C.c_void_p), ("grad_scale", C.c_void_p),
                ("seed", C.c_uint64), ("bits", C.c_int32)]


class stx_moments(C.Structure):
    _fields_ = [("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class stx_adamw_tensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("n", C.c_int64), ("s", stx_moments), ("g_dtype", C.c_int32),
                ("flags", C.c_uint32)]


class stx_adamw_state(C.Structure):
    _fields_ = [("ent", stx_moments), ("rel", stx_moments), ("w", stx_moments), ("proj", stx_moments)]


_lib = None


def lib():
    """Load libstx.so from the package directory.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2502_16949_amd.build); "
                               "there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        L.stx_workspace_bytes.argtypes = [C.POINTER(stx_config), C.POINTER(C.c_size_t)]
        L.stx_create.argtypes = [C.POINTER(stx_config), vp, C.c_size_t, vp, C.POINTER(vp)]
        L.stx_destroy.argtypes = [vp]
        L.stx_sample_negatives.argtypes = [vp, vp, vp, vp, i64, i32, u64, u64, i64, i64, vp, vp]
        L.stx_build_incidence.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, C.POINTER(stx_incidence)]
        L.stx_check_indices.argtypes = [vp, C.POINTER(i64)]
        L.stx_spmm.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), vp]
        L.stx_spmm_semiring.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), i32, vp]
        L.stx_spmm_semiring_t.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), i32, vp, vp,
                                          C.POINTER(stx_grads)]
        L.stx_spmm_semiring_t_static.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), i32, vp,
                                                 C.POINTER(stx_grads)]
        L.stx_rank.argtypes = [vp, C.POINTER(stx_params), vp, vp, vp, i64, i32, vp, vp, vp, vp, C.c_size_t]
        L.stx_rank_work_bytes.argtypes = [vp, i64, C.POINTER(C.c_size_t)]
        L.stx_forward.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), vp, vp]
        L.stx_backward.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), C.POINTER(stx_grads)]
        L.stx_sgd_step.argtypes = [vp, C.POINTER(stx_params), C.POINTER(stx_incidence), C.POINTER(stx_grads),
                                   C.c_float]
        L.stx_backward_sgd.argtypes = [vp, C.POINTER(stx_incidence), C.POINTER(stx_params), C.POINTER(stx_grads),
                                       C.c_float]
        L.stx_train_step.argtypes = [vp, C.POINTER(stx_batch), C.POINTER(stx_incidence), C.POINTER(stx_params),
                                     C.POINTER(stx_grads), C.c_float, vp, vp]
        L.stx_rmsnorm.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, C.c_float, vp, vp, C.POINTER(stx_q8), vp]
        L.stx_rmsnorm_backward_work_bytes.argtypes = [vp, i64, i64, C.POINTER(C.c_size_t)]
        L.stx_rmsnorm_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t]
        L.stx_q8_quantize.argtypes = [vp, i32, i64, i64, i64, vp, C.POINTER(stx_q8), C.POINTER(stx_q8)]
        L.stx_q8_matmul_work_bytes.argtypes = [vp, i64, i64, i64, C.POINTER(C.c_size_t)]
        L.stx_q8_matmul.argtypes = [vp, C.POINTER(stx_q8), C.POINTER(stx_q8), i32, vp, i64, vp, C.c_size_t]
        L.stx_adamw_tensors.argtypes = [vp, C.POINTER(stx_adamw), C.POINTER(stx_adamw_tensor), i32]
        L.stx_adamw_step.argtypes = [vp, C.POINTER(stx_params), C.POINTER(stx_incidence), C.POINTER(stx_grads),
                                     C.POINTER(stx_adamw), C.POINTER(stx_adamw_state)]
        L.stx_profile_kernel.argtypes = [vp, C.c_char_p, i32]
        L.stx_profile_every.argtypes = [vp, i32]
        L.stx_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i32)]
        L.stx_profile_dump.argtypes = [vp, C.c_char_p, C.c_size_t]
        L.stx_copy_f32.argtypes = [vp, vp, vp, i64]
        L.stx_read_sectors.argtypes = [vp, vp, i64, i32, i64, vp]
        L.stx_status_string.argtypes = [C.c_int]
        L.stx_status_string.restype = C.c_char_p
        for name in EXPORTS[:-1]:
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().stx_status_string(status).decode()


def _check(call: str, status: int):
    if status != STX_OK:
        raise StxError(call, status)


def _ptr(t):
    return None if t is None else t.data_ptr()


def make_config(model, dist, n_ent, n_rel, dim, max_batch, max_neg, rel_dim=0, margin=1.0, reduce=STX_SUM,
                flags=0) -> stx_config:
    model = MODELS[model] if isinstance(model, str) else model
    dist = DISTS[dist] if isinstance(dist, str) else dist
    return stx_config(model, dist, reduce, dim, rel_dim or dim, n_ent, n_rel, margin, max_batch, max_neg, flags)


def stx_workspace_bytes(cfg: stx_config) -> int:
    n = C.c_size_t(0)
    _check("stx_workspace_bytes", lib().stx_workspace_bytes(C.byref(cfg), C.byref(n)))
    return n.value


class Context:
    """Owns the workspace tensor and the stx_ctx handle."""

    def __init__(self, cfg: stx_config, device="cuda:0", stream: torch.cuda.Stream | None = None):
        self.cfg = cfg
        self.device = torch.device(device)
        self.index = torch.cuda.current_device() if self.device.index is None else self.device.index
        nbytes = stx_workspace_bytes(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        _check("stx_create", lib().stx_create(C.byref(cfg), self._ws_ptr, nbytes, self.stream.cuda_stream,
                                              C.byref(h)))
        self.handle = h

    @property
    def rows_max(self):
        return self.cfg.max_batch * (1 + self.cfg.max_neg)

    @property
    def cols_max(self):
        return min(3 * self.rows_max, self.cfg.n_ent + self.cfg.n_rel)

    @property
    def ld(self):
        return max(self.cfg.dim, self.cfg.rel_dim)

    def close(self):
        if self.handle:
            lib().stx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Incidence:
    """Device arrays of one stx_incidence, sized for the context's maxima."""

    def __init__(self, ctx: Context):
        dev, rows, nnz, cols = ctx.device, ctx.rows_max, 3 * ctx.rows_max, ctx.cols_max
        i32 = dict(dtype=torch.int32, device=dev)
        self.a_rowptr = torch.empty(rows + 1, **i32)
        self.a_colidx = torch.empty(nnz, **i32)
        self.a_vals = torch.empty(nnz, dtype=torch.float32, device=dev)
        self.at_touched_cols = torch.empty(cols, **i32)
        self.at_seg_ptr = torch.empty(cols + 1, **i32)
        self.at_row_idx = torch.empty(nnz, **i32)
        self.at_sign = torch.empty(nnz, dtype=torch.int8, device=dev)
        self.at_seg_id = torch.empty(nnz, **i32)
        self.at_packed = torch.empty(nnz, **i32)
        self.n_touched = torch.zeros(1, **i32)
        self.c = stx_incidence(0, 0, 0, 0, *(t.data_ptr() for t in (
            self.a_rowptr, self.a_colidx, self.a_vals, self.at_touched_cols, self.at_seg_ptr, self.at_row_idx,
            self.at_sign, self.at_seg_id, self.at_packed, self.n_touched)))

    @property
    def n_rows(self):
        return self.c.n_rows

    @property
    def nnz(self):
        return self.c.nnz


class Grads:
    def __init__(self, ctx: Context):
        f32 = dict(dtype=torch.float32, device=ctx.device)
        self.rows = torch.empty(ctx.cols_max, ctx.ld, **f32)
        self.w_rows = torch.empty(ctx.cols_max, ctx.ld, **f32) if ctx.cfg.model == STX_TRANSH else None
        self.proj = (torch.empty(ctx.cfg.n_rel, ctx.cfg.rel_dim, ctx.cfg.dim, **f32)
                     if ctx.cfg.model == STX_TRANSR else None)
        self.c = stx_grads(_ptr(self.rows), _ptr(self.w_rows), _ptr(self.proj))


class Params:
    def __init__(self, ent, rel=None, w=None, proj=None, rel_weight=None):
        self.ent, self.rel, self.w, self.proj, self.rel_weight = ent, rel, w, proj, rel_weight
        for t in (ent, rel, w, proj, rel_weight):
            assert t is None or (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous())
        self.c = stx_params(_ptr(ent), _ptr(rel), _ptr(w), _ptr(proj), _ptr(rel_weight))


def _i32dev(t):
    assert t is None or (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous())
    return _ptr(t)


def stx_sample_negatives(ctx: Context, h, r, t, k, seed, epoch, m_total, global_offset, neg_h, neg_t):
    m = h.numel()
    assert neg_h.numel() >= m * k and neg_t.numel() >= m * k
    _check("stx_sample_negatives",
           lib().stx_sample_negatives(ctx.handle, _i32dev(h), _i32dev(r), _i32dev(t), m, k, seed, epoch, m_total,
                                      global_offset, _i32dev(neg_h), _i32dev(neg_t)))


def stx_build_incidence(ctx: Context, h, r, t, neg_h, neg_t, k, inc: Incidence):
    b = h.numel()
    assert r.numel() == b and t.numel() == b
    assert k == 0 or (neg_h.numel() >= b * k and neg_t.numel() >= b * k)
    _check("stx_build_incidence",
           lib().stx_build_incidence(ctx.handle, _i32dev(h), _i32dev(r), _i32dev(t), _i32dev(neg_h),
                                     _i32dev(neg_t), b, k, C.byref(inc.c)))


def stx_check_indices(ctx: Context) -> int:
    n = C.c_int64(0)
    st = lib().stx_check_indices(ctx.handle, C.byref(n))
    if st not in (STX_OK, STX_ERR_INDEX_RANGE):
        raise StxError("stx_check_indices", st)
    return n.value


def stx_spmm(ctx: Context, inc: Incidence, p: Params, c_out):
    assert c_out.is_cuda and c_out.dtype == torch.float32 and c_out.is_contiguous()
    assert c_out.numel() >= inc.n_rows * ctx.cfg.dim
    _check("stx_spmm", lib().stx_spmm(ctx.handle, C.byref(inc.c), C.byref(p.c), c_out.data_ptr()))


def stx_spmm_semiring(ctx: Context, inc: Incidence, p: Params, kind: int, z_out):
    assert z_out.is_cuda and z_out.dtype == torch.float32 and z_out.is_contiguous()
    assert z_out.numel() >= inc.n_rows * ctx.cfg.dim
    _check("stx_spmm_semiring", lib().stx_spmm_semiring(ctx.handle, C.byref(inc.c), C.byref(p.c), kind,
                                                        z_out.data_ptr()))


def stx_spmm_semiring_t(ctx: Context, inc: Incidence, p: Params, kind: int, gz, work, g: Grads):
    for t in (gz, work):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    assert gz.numel() >= inc.n_rows * ctx.cfg.dim and work.numel() >= 3 * inc.n_rows * ctx.cfg.dim
    _check("stx_spmm_semiring_t", lib().stx_spmm_semiring_t(ctx.handle, C.byref(inc.c), C.byref(p.c), kind,
                                                            gz.data_ptr(), work.data_ptr(), C.byref(g.c)))


def stx_spmm_semiring_t_static(ctx: Context, inc: Incidence, p: Params, kind: int, gz, g: Grads):
    assert gz.is_cuda and gz.dtype == torch.float32 and gz.is_contiguous()
    assert gz.numel() >= inc.n_rows * ctx.cfg.dim
    _check("stx_spmm_semiring_t_static", lib().stx_spmm_semiring_t_static(ctx.handle, C.byref(inc.c), C.byref(p.c),
                                                                          kind, gz.data_ptr(), C.byref(g.c)))


def stx_rank_work_bytes(ctx: Context, nq: int) -> int:
    n = C.c_size_t(0)
    _check("stx_rank_work_bytes", lib().stx_rank_work_bytes(ctx.handle, nq, C.byref(n)))
    return n.value


def stx_rank(ctx: Context, p: Params, h, r, t, side: int, true_score, n_less, n_equal, work=None):
    """work: a uint8 device tensor of at least stx_rank_work_bytes(nq) + 256 bytes (TransR), else None."""
    nq = h.numel()
    assert r.numel() == nq and t.numel() == nq
    assert true_score.is_cuda and true_score.dtype == torch.float32 and true_score.numel() >= nq
    for c in (n_less, n_equal):
        assert c.is_cuda and c.dtype == torch.int32 and c.is_contiguous() and c.numel() >= nq
    wp, wb = None, 0
    if work is not None:
        assert work.is_cuda and work.dtype == torch.uint8 and work.is_contiguous()
        wp = (work.data_ptr() + 255) // 256 * 256
        wb = work.numel() - (wp - work.data_ptr())
    _check("stx_rank", lib().stx_rank(ctx.handle, C.byref(p.c), _i32dev(h), _i32dev(r), _i32dev(t), nq, side,
                                      true_score.data_ptr(), n_less.data_ptr(), n_equal.data_ptr(), wp, wb))


def stx_forward(ctx: Context, inc: Incidence, p: Params, scores, loss):
    assert scores.is_cuda and scores.dtype == torch.float32 and scores.numel() >= inc.n_rows
    assert loss.is_cuda and loss.dtype == torch.float32 and loss.numel() >= 1
    _check("stx_forward", lib().stx_forward(ctx.handle, C.byref(inc.c), C.byref(p.c), scores.data_ptr(),
                                            loss.data_ptr()))


def stx_backward(ctx: Context, inc: Incidence, p: Params, g: Grads):
    _check("stx_backward", lib().stx_backward(ctx.handle, C.byref(inc.c), C.byref(p.c), C.byref(g.c)))


def stx_sgd_step(ctx: Context, p: Params, inc: Incidence, g: Grads, lr: float):
    _check("stx_sgd_step", lib().stx_sgd_step(ctx.handle, C.byref(p.c), C.byref(inc.c), C.byref(g.c), lr))


def stx_backward_sgd(ctx: Context, inc: Incidence, p: Params, g, lr: float):
    """g may be None for TransE / TorusE (no gradient rows are written)."""
    gp = C.byref(g.c) if g is not None else None
    _check("stx_backward_sgd", lib().stx_backward_sgd(ctx.handle, C.byref(inc.c), C.byref(p.c), gp, lr))


def make_batch(h, r, t, k, seed, epoch, m_total, global_offset, neg_h, neg_t, next_batch=None) -> "stx_batch":
    """Argument block of stx_train_step; the tensors (and next_batch, the block of the call that follows, if
    given) must stay alive while it is in use.  link_batches() chains a list of them."""
    b = h.numel()
    assert r.numel() == b and t.numel() == b
    assert k == 0 or (neg_h.numel() >= b * k and neg_t.numel() >= b * k)
    return stx_batch(_i32dev(h), _i32dev(r), _i32dev(t), b, k, seed, epoch, m_total, global_offset,
                     _i32dev(neg_h) if k else None, _i32dev(neg_t) if k else None,
                     C.addressof(next_batch) if next_batch is not None else None)


def link_batches(batches, cyclic=False):
    """Sets every block's `next` to the block after it (the last one's to the first when cyclic)."""
    for i, bt in enumerate(batches):
        nxt = batches[(i + 1) % len(batches)] if (cyclic or i + 1 < len(batches)) else None
        bt.next = C.addressof(nxt) if nxt is not None else None
    return batches


def stx_train_step(ctx: Context, batch, inc: Incidence, p: Params, g, lr: float, scores, loss):
    assert scores.is_cuda and scores.dtype == torch.float32 and scores.numel() >= batch.b * (1 + batch.k)
    assert loss.is_cuda and loss.dtype == torch.float32 and loss.numel() >= 1
    gp = C.byref(g.c) if g is not None else None
    _check("stx_train_step", lib().stx_train_step(ctx.handle, C.byref(batch), C.byref(inc.c), C.byref(p.c), gp, lr,
                                                  scores.data_ptr(), loss.data_ptr()))


def _reaches(t, width):
    """Whether a matrix of bytes lies in memory that goes on to `width` bytes of its last row."""
    return t.shape[0] == 0 or width == 0 or t.untyped_storage().nbytes() - t.storage_offset() >= (t.shape[0] - 1) * t.stride(0) + width


class Q8:
    """A matrix in 8 bits: `codes` (rows x cols rounded up to 128) and `scales` (rows x blocks rounded up to 4), uint8."""

    def __init__(self, rows, cols, format=STX_E4M3, device="cuda:0"):
        blocks = (cols + 127) // 128
        self._set(torch.zeros(rows, blocks * 128, dtype=torch.uint8, device=device),
                  torch.full((rows, (blocks + 3) // 4 * 4), 127, dtype=torch.uint8, device=device), cols, format)

    @classmethod
    def of(cls, codes, scales, cols, format=STX_E4M3):
        """Around tensors that a program holds already; the codes behind the last column are 0, and rows of scales are read in
        words, the last one too."""
        q = cls.__new__(cls)
        q._set(codes, scales, cols, format)
        return q

    def _set(self, codes, scales, cols, format):
        for t in (codes, scales):
            assert t.is_cuda and t.dtype == torch.uint8 and t.dim() == 2 and t.stride(1) == 1 and t.shape[0] == codes.shape[0]
        blocks = (cols + 127) // 128
        assert codes.shape[1] >= blocks * 128 and scales.shape[1] >= blocks and _reaches(scales, (blocks + 3) // 4 * 4)
        self.codes, self.scales, self.rows, self.cols, self.format = codes, scales, codes.shape[0], cols, format
        self.index = codes.get_device()
        assert scales.get_device() == self.index
        self.c = stx_q8(_ptr(codes), _ptr(scales), codes.shape[0], cols, codes.stride(0), scales.stride(0), format)
        self.ref = C.byref(self.c)


def _rows2d(ctx, first, *others):
    """(dtype, rows, cols, ld) of matrices of one type, shape and row stride on the context's device; others may be None."""
    dtype, shape, stride, index = first.dtype, first.shape, first.stride(), ctx.index
    rows, cols = shape
    assert first.get_device() == index and (stride[1] == 1 or cols == 1)
    ld = stride[0] if rows > 1 else cols
    for t in others:
        if t is not None:
            assert t.dtype is dtype and t.get_device() == index and t.shape == shape
            s = t.stride()
            assert s == stride or ((s[1] == 1 or cols == 1) and (s[0] == ld or rows <= 1))
    return DTYPES[dtype], rows, cols, ld


def _f32dev(ctx, t, n):
    if t is None:
        return None
    assert t.get_device() == ctx.index and t.dtype is torch.float32 and t.is_contiguous() and t.numel() >= n
    return t.data_ptr()


def _work(ctx, work):
    """(pointer, bytes) of the aligned part of a uint8 scratch tensor."""
    if work is None:
        return None, 0
    assert work.get_device() == ctx.index and work.dtype is torch.uint8 and work.is_contiguous()
    at = work.data_ptr()
    wp = (at + 255) // 256 * 256
    return wp, max(0, work.numel() - (wp - at))


def _q8(ctx, q):
    if q is None:
        return None
    assert q.index == ctx.index
    return q.ref


def stx_rmsnorm(ctx: Context, x, residual, weight, eps: float, sum, y, q, rstd):
    """Rows are matrices of one type, shape and row stride; sum, y, q (Q8) and rstd may be None, as may residual and weight."""
    dtype, rows, cols, ld = _rows2d(ctx, x, residual, sum, y)
    _check("stx_rmsnorm", lib().stx_rmsnorm(ctx.handle, dtype, rows, cols, ld, _ptr(x), _ptr(residual), _f32dev(ctx, weight, cols),
                                            eps, _ptr(sum), _ptr(y), _q8(ctx, q), _f32dev(ctx, rstd, rows)))


def stx_rmsnorm_backward_work_bytes(ctx: Context, rows: int, cols: int) -> int:
    n = C.c_size_t(0)
    _check("stx_rmsnorm_backward_work_bytes", lib().stx_rmsnorm_backward_work_bytes(ctx.handle, rows, cols, C.byref(n)))
    return n.value


def stx_rmsnorm_backward(ctx: Context, sum, weight, rstd, dy, dsum, dx, dweight, work=None):
    """work: a uint8 device tensor of at least stx_rmsnorm_backward_work_bytes(rows, cols) + 256 bytes, or None without dweight."""
    dtype, rows, cols, ld = _rows2d(ctx, sum, dy, dsum, dx)
    wp, wb = _work(ctx, work)
    _check("stx_rmsnorm_backward",
           lib().stx_rmsnorm_backward(ctx.handle, dtype, rows, cols, ld, _ptr(sum), _f32dev(ctx, weight, cols), _f32dev(ctx, rstd, rows),
                                      _ptr(dy), _ptr(dsum), _ptr(dx), _f32dev(ctx, dweight, cols), wp, wb))


def stx_q8_quantize(ctx: Context, x, q, qt):
    """q (rows x cols) and / or qt (cols x rows) from a matrix; one of them may be None."""
    dtype, rows, cols, ld = _rows2d(ctx, x)
    _check("stx_q8_quantize", lib().stx_q8_quantize(ctx.handle, dtype, rows, cols, ld, _ptr(x), _q8(ctx, q), _q8(ctx, qt)))


def stx_q8_matmul_work_bytes(ctx: Context, rows_a: int, rows_b: int, cols: int) -> int:
    n = C.c_size_t(0)
    _check("stx_q8_matmul_work_bytes", lib().stx_q8_matmul_work_bytes(ctx.handle, rows_a, rows_b, cols, C.byref(n)))
    return n.value


def stx_q8_matmul(ctx: Context, a: Q8, b: Q8, out, work=None):
    """out = A B^T.  work: a uint8 device tensor of at least stx_q8_matmul_work_bytes(...) + 256 bytes, or None where that is 0."""
    dtype, rows, cols, ldo = _rows2d(ctx, out)
    assert (rows, cols) == (a.rows, b.rows)
    wp, wb = _work(ctx, work)
    _check("stx_q8_matmul", lib().stx_q8_matmul(ctx.handle, _q8(ctx, a), _q8(ctx, b), dtype, _ptr(out), ldo, wp, wb))


def make_adamw(lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, bits=32, step=1, seed=0, step_dev=None,
               grad_scale=None) -> stx_adamw:
    """Hyperparameters; a program sets .step before every call.  step_dev (int64) and grad_scale (float32) are device tensors, of
    which the first element counts, on the device of the calls' context; the result keeps them alive."""
    h = stx_adamw(lr, beta1, beta2, eps, weight_decay, step, _ptr(step_dev), _ptr(grad_scale), seed, bits)
    for t, dtype in ((step_dev, torch.int64), (grad_scale, torch.float32)):
        if t is not None:
            assert t.is_cuda and t.dtype == dtype and t.numel() > 0 and h.index in (None, t.get_device())
            h.index = t.get_device()
    h.held = step_dev, grad_scale
    return h


class _Moments:
    """m and v of one tensor (float32, or uint8 codes with float32 scales)."""

    def __init__(self, m, v, m_scale=None, v_scale=None):
        self.bits, self.n, self.blocks = 32 if m_scale is None else 8, m.numel(), 0 if m_scale is None else m_scale.numel()
        self.index, self.keep = m.get_device(), (m, v, m_scale, v_scale)
        for t in (m, v):
            assert t.is_cuda and t.dtype == (torch.float32 if self.bits == 32 else torch.uint8) and t.numel() == self.n
        for t in (m_scale, v_scale):
            assert (t is None) == (self.bits == 32)
            assert t is None or (t.dtype == torch.float32 and t.numel() == self.blocks)
        assert all(t is None or (t.is_contiguous() and t.get_device() == self.index) for t in self.keep)
        self.c = stx_moments(*(_ptr(t) for t in self.keep))


class AdamWTensors:
    """The tensors of stx_adamw_tensors: (p, g, m, v[, m_scale, v_scale]) each; m and v are float32, or uint8 codes with a float32
    scale for each 128 elements.  no_decay: positions of tensors without weight decay.  Addresses are taken here, once: a program
    whose gradients are new tensors every step makes a new one every step, or keeps its gradients where they are."""

    def __init__(self, tensors, no_decay=()):
        self.keep, self.n = [], len(tensors)
        self.c = (stx_adamw_tensor * max(1, self.n))()
        for i, (p, g, *s) in enumerate(tensors):
            s = _Moments(*s)
            assert p.is_cuda and p.dtype == torch.float32 and p.is_contiguous() and p.numel() == g.numel() == s.n
            assert g.is_contiguous() and p.get_device() == g.get_device() == s.index
            assert s.bits == 32 or s.blocks == (s.n + 127) // 128
            self.c[i] = stx_adamw_tensor(_ptr(p), _ptr(g), s.n, s.c, DTYPES[g.dtype], STX_ADAMW_NO_DECAY if i in no_decay else 0)
            self.keep.append((p, g, s))
        self.places = {(s.index, s.bits) for _, _, s in self.keep}


class AdamWState:
    """Moments of the tables that a model has, (m, v[, m_scale, v_scale]) each, laid out as the tables."""

    def __init__(self, ent, rel=None, w=None, proj=None):
        self.held = {name: _Moments(*t) for name, t in (("ent", ent), ("rel", rel), ("w", w), ("proj", proj)) if t is not None}
        self.c = stx_adamw_state(**{name: s.c for name, s in self.held.items()})

    @classmethod
    def zeros(cls, p: Params, bits=32):
        def one(t):
            if t is None:
                return None
            like = lambda: torch.zeros(t.shape, dtype=torch.float32 if bits == 32 else torch.uint8, device=t.device)  # noqa: E731
            scale = lambda: torch.zeros(t.shape[0], (t[0].numel() + 127) // 128, device=t.device)  # noqa: E731
            return (like(), like()) if bits == 32 else (like(), like(), scale(), scale())
        return cls(one(p.ent), one(p.rel), one(p.w), one(p.proj))


def stx_adamw_tensors(ctx: Context, h: stx_adamw, tensors: AdamWTensors):
    assert (tensors.n == 0 or tensors.places == {(ctx.index, h.bits)}) and h.index in (None, ctx.index)
    _check("stx_adamw_tensors", lib().stx_adamw_tensors(ctx.handle, C.byref(h), tensors.c, tensors.n))


def stx_adamw_step(ctx: Context, p: Params, inc: Incidence, g: Grads, h: stx_adamw, s: AdamWState):
    assert h.index in (None, ctx.index)
    for name, m in s.held.items():
        t = getattr(p, name)
        assert t is None or (m.n == t.numel() and (m.index, m.bits) == (ctx.index, h.bits) and
                             (m.bits == 32 or m.blocks == t.shape[0] * ((m.n // t.shape[0] + 127) // 128)))
    _check("stx_adamw_step", lib().stx_adamw_step(ctx.handle, C.byref(p.c), C.byref(inc.c), C.byref(g.c), C.byref(h), C.byref(s.c)))


def stx_profile_kernel(ctx: Context, kernel_name, max_records: int):
    name = None if kernel_name is None else kernel_name.encode()
    _check("stx_profile_kernel", lib().stx_profile_kernel(ctx.handle, name, max_records))


def stx_profile_every(ctx: Context, every: int):
    _check("stx_profile_every", lib().stx_profile_every(ctx.handle, every))


def stx_profile_read(ctx: Context):
    """(mean microseconds per bracketed launch, number of launches recorded)."""
    avg, n = C.c_double(0), C.c_int32(0)
    _check("stx_profile_read", lib().stx_profile_read(ctx.handle, C.byref(avg), C.byref(n)))
    return avg.value, n.value


def stx_copy_f32(ctx: Context, dst, src):
    assert dst.numel() == src.numel() and dst.dtype == src.dtype == torch.float32
    _check("stx_copy_f32", lib().stx_copy_f32(ctx.handle, dst.data_ptr(), src.data_ptr(), src.numel()))


def stx_read_sectors(ctx: Context, src, n_slots: int, slot_bytes: int, n_reads: int, sink):
    assert src.is_cuda and src.numel() * src.element_size() >= n_slots * slot_bytes
    assert sink.is_cuda and sink.dtype == torch.float32 and sink.numel() >= 16384
    _check("stx_read_sectors", lib().stx_read_sectors(ctx.handle, src.data_ptr(), n_slots, slot_bytes, n_reads,
                                                      sink.data_ptr()))


def stx_profile_dump(ctx: Context) -> dict:
    """{kernel name: (mean microseconds, launches)} of everything recorded since the last read."""
    buf = C.create_string_buffer(8192)
    _check("stx_profile_dump", lib().stx_profile_dump(ctx.handle, buf, len(buf)))
    out = {}
    for ln in buf.value.decode().splitlines():
        name, us, n = ln.split()
        out[name] = (float(us), int(n))
    return out
