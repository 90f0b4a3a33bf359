"""ctypes binding of libkurtail (argument marshalling only).

Every function here forwards to the C entry point of the same name declared in
include/kurtail.h; all arithmetic runs in the CUDA library.  torch is used for
device memory and streams only.  There is no fallback: if the shared library is
missing the import of this module's `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# KURTAIL_LIB names another build of the same library (e.g. one compiled with other nvcc flags) to load instead
LIB_PATH = os.environ.get("KURTAIL_LIB") or os.path.join(_HERE, "libkurtail.so")

KT_BF16, KT_F32, KT_F64 = 0, 1, 2
STATUS = {0: "KT_OK", 1: "KT_ERR_INVALID_ARG", 2: "KT_ERR_SHAPE", 3: "KT_ERR_ALIGN", 4: "KT_ERR_WORKSPACE",
          5: "KT_ERR_ARCH", 6: "KT_ERR_CUDA", 7: "KT_ERR_NONFINITE", 8: "KT_ERR_TIMEOUT", 9: "KT_ERR_TOO_LARGE",
          10: "KT_ERR_COOPERATIVE", 11: "KT_ERR_REDUCE",
          12: "KT_ERR_CACHE"}


class KtError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}")


class kt_mat(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64)]


class kt_config(C.Structure):
    _fields_ = [("kappa_target", C.c_float), ("cayley_iters", C.c_int32), ("q", C.c_float), ("eps", C.c_float),
                ("polish_thresh", C.c_float), ("retract_terms", C.c_int32), ("guard_every", C.c_int32),
                ("forward_terms", C.c_int32), ("small_d_fused", C.c_int32), ("small_d_orth", C.c_int32),
                ("optimizer", C.c_int32), ("beta1", C.c_float), ("beta2", C.c_float), ("adam_eps", C.c_float),
                ("norm_iters", C.c_int32), ("backward_mode", C.c_int32), ("cta_pairs", C.c_int32), ("loss_mode", C.c_int32), ("rmsnorm", C.c_int32), ("rms_eps", C.c_float),
                ("wait_limit_ms", C.c_int32), ("forward_bf16", C.c_int32)]


class kt_quant_spec(C.Structure):
    _fields_ = [("bits", C.c_int32), ("asymmetric", C.c_int32), ("clip", C.c_float), ("clip_mode", C.c_int32)]


class kt_adam_state(C.Structure):
    _fields_ = [("v", C.c_double), ("step", C.c_int32), ("reserved", C.c_int32)]


class kt_fit_report(C.Structure):
    _fields_ = [("steps_done", C.c_int32), ("degenerate_rows", C.c_int32), ("loss_first", C.c_double),
                ("loss_last", C.c_double), ("orth_err", C.c_double), ("alpha_last", C.c_float),
                ("w_norm_last", C.c_float), ("loss_history", C.POINTER(C.c_double)), ("w_op_last", C.c_float),
                ("series_terms_last", C.c_int32), ("p0_terms_last", C.c_int32), ("guards_run", C.c_int32)]


class kt_kv_cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_steps", C.c_void_p), ("v_steps", C.c_void_p),
                ("pages", C.c_int32), ("heads", C.c_int32), ("page_size", C.c_int32), ("head_dim", C.c_int32),
                ("bits", C.c_int32)]


class kt_kv_batch(C.Structure):
    _fields_ = [("row_starts", C.c_void_p), ("lengths", C.c_void_p), ("page_table", C.c_void_p),
                ("n_seqs", C.c_int32), ("table_ld", C.c_int32), ("max_rows", C.c_int32), ("max_length", C.c_int32)]


class kt_profile(C.Structure):
    _fields_ = [("launches_total", C.c_int64), ("gemm_launches", C.c_int32 * 8), ("gemm_ms", C.c_float * 8)]


EXPORTS = ["kt_default_config", "kt_create", "kt_destroy", "kt_status_string", "kt_workspace_bytes",
           "kt_set_workspace", "kt_init_rotation", "kt_kurtosis_loss", "kt_loss_grad", "kt_row_moments",
           "kt_rotate", "kt_orth_step", "kt_adam_step", "kt_orth_error", "kt_fit", "kt_fit_layers",
           "kt_fit_shared_workspace_bytes", "kt_fit_shared", "kt_fit_host", "kt_fit_sharded", "kt_fit_shared_sharded",
           "kt_test_wait_timeout",
           "kt_quant4_error", "kt_quant4_codes", "kt_quant_error", "kt_quant_codes", "kt_quant_error_given",
           "kt_rowmax_success", "kt_profile_begin", "kt_profile_end",
           "kt_kurtosis_loss_noalloc", "kt_rmsnorm_quant", "kt_kv_append", "kt_kv_scratch_bytes", "kt_kv_attend",
           "kt_check"]

# int32 reduce(void* user, void* dev_ptr, int64 count, int32 dtype, void* cuda_stream)
REDUCE_FN = C.CFUNCTYPE(C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p)

_lib = _serving = None


class _Missing:
    """Stands for _serving.so where it cannot be used: the serving calls raise the reason, all others need only the library."""

    def __init__(self, why):
        self._why = why

    def __getattr__(self, name):
        raise ImportError(self._why)


def _load_serving():
    """The module that reads the serving calls' tensors, built beside the library."""
    from . import build
    try:
        from . import _serving as module
    except ImportError as e:
        return _Missing(f"the serving calls need _serving.so; build with: python -m paper_2503_01483_b200.build ({e})")
    named = getattr(module, "built_for", "another version of this library")
    if named != build.built_for():
        return _Missing(f"_serving.so was built for {named}, this is {build.built_for()}; build with: "
                        "python -m paper_2503_01483_b200.build")
    return module


def lib():
    """Loads libkurtail.so (built by paper_2503_01483_b200.build).  Raises if absent."""
    global _lib, _serving
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2503_01483_b200.build` "
                                "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    dp = C.POINTER(C.c_double)
    L.kt_default_config.argtypes = [C.POINTER(kt_config)]
    L.kt_default_config.restype = None
    L.kt_create.argtypes = [C.POINTER(vp), C.POINTER(kt_config), vp]
    L.kt_destroy.argtypes = [vp]
    L.kt_destroy.restype = None
    L.kt_status_string.argtypes = [i32]
    L.kt_status_string.restype = C.c_char_p
    L.kt_workspace_bytes.argtypes = [vp, i64, i64, i32, C.POINTER(C.c_size_t)]
    L.kt_set_workspace.argtypes = [vp, vp, C.c_size_t]
    L.kt_init_rotation.argtypes = [vp, vp, i64, i32]
    L.kt_kurtosis_loss.argtypes = [vp, kt_mat, vp, dp]
    L.kt_loss_grad.argtypes = [vp, kt_mat, vp, vp, dp]
    L.kt_row_moments.argtypes = [vp, kt_mat, vp, vp]
    L.kt_rotate.argtypes = [vp, kt_mat, vp, vp]
    L.kt_orth_step.argtypes = [vp, vp, vp, i64, f32]
    L.kt_adam_step.argtypes = [vp, vp, vp, vp, C.POINTER(kt_adam_state), i64, f32]
    L.kt_orth_error.argtypes = [vp, vp, i64, dp]
    L.kt_fit.argtypes = [vp, kt_mat, vp, i32, f32, C.POINTER(kt_fit_report)]
    L.kt_fit_layers.argtypes = [vp, C.POINTER(kt_mat), C.POINTER(vp), i32, i32, i32, f32, C.POINTER(kt_fit_report)]
    L.kt_fit_shared_workspace_bytes.argtypes = [vp, i64, i32, i64, C.POINTER(C.c_size_t)]
    L.kt_fit_shared.argtypes = [vp, C.POINTER(kt_mat), i32, i64, C.POINTER(i32), i32, vp, i32, f32,
                                C.POINTER(kt_fit_report)]
    L.kt_fit_host.argtypes = [vp, kt_mat, vp, vp, vp, i32, f32, C.POINTER(kt_fit_report)]
    L.kt_fit_sharded.argtypes = [vp, kt_mat, vp, i64, REDUCE_FN, vp, i32, f32, C.POINTER(kt_fit_report)]
    L.kt_fit_shared_sharded.argtypes = [vp, C.POINTER(kt_mat), i32, i64, C.POINTER(i32), i32, vp, i64, REDUCE_FN, vp,
                                        i32, f32, C.POINTER(kt_fit_report)]
    L.kt_test_wait_timeout.argtypes = [vp, i32]
    L.kt_quant4_error.argtypes = [vp, kt_mat, vp, dp]
    L.kt_quant4_codes.argtypes = [vp, vp, i64, i64, vp, vp]
    L.kt_quant_error.argtypes = [vp, kt_mat, vp, C.POINTER(kt_quant_spec), dp]
    L.kt_quant_codes.argtypes = [vp, vp, i64, i64, C.POINTER(kt_quant_spec), vp, vp, vp]
    L.kt_quant_error_given.argtypes = [vp, vp, i64, i64, C.POINTER(kt_quant_spec), dp]
    L.kt_rowmax_success.argtypes = [vp, kt_mat, vp, vp, dp]
    L.kt_kurtosis_loss_noalloc.argtypes = [kt_mat, vp, vp, vp]
    mp, cp, bp = C.POINTER(kt_mat), C.POINTER(kt_kv_cache), C.POINTER(kt_kv_batch)
    L.kt_rmsnorm_quant.argtypes = [vp, kt_mat, mp, mp, vp, C.c_double, C.POINTER(kt_quant_spec), vp, vp, mp]
    L.kt_kv_append.argtypes = [vp, cp, bp, mp, kt_mat, kt_mat, vp, i64, i32, C.POINTER(kt_quant_spec), mp, mp, mp]
    L.kt_kv_scratch_bytes.argtypes = [vp, cp, bp, i32, C.POINTER(C.c_size_t)]
    L.kt_kv_attend.argtypes = [vp, cp, bp, kt_mat, kt_mat, vp, f32, i32, i32, vp, C.c_size_t]
    L.kt_check.argtypes = [vp]
    L.kt_profile_begin.argtypes = [vp]
    L.kt_profile_end.argtypes = [vp, C.POINTER(kt_profile)]
    for name in EXPORTS:
        fn = getattr(L, name)
        if name not in ("kt_default_config", "kt_destroy", "kt_status_string"):
            fn.restype = i32
    _serving = _load_serving()
    if not isinstance(_serving, _Missing):
        _serving.bind(*(C.cast(getattr(L, n), vp).value for n in ("kt_rmsnorm_quant", "kt_kv_append", "kt_kv_attend")))
    _lib = L
    return L


def default_config(**overrides):
    cfg = kt_config()
    lib().kt_default_config(C.byref(cfg))
    for k, v in overrides.items():
        setattr(cfg, k, v)
    return cfg


def _check(st, where):
    if st != 0:
        raise KtError(st, where)


def as_mat(X: torch.Tensor) -> kt_mat:
    """Describes a 2-D row-major torch tensor (bf16 or f32, device or host)."""
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be 2-D with unit column stride")
    if X.dtype == torch.bfloat16:
        dt = KT_BF16
    elif X.dtype == torch.float32:
        dt = KT_F32
    else:
        raise ValueError("X must be bfloat16 or float32")
    return kt_mat(X.data_ptr(), dt, 0, X.shape[0], X.shape[1], X.stride(0))


def _rep_dict(rep, hist):
    return dict(steps_done=rep.steps_done, degenerate_rows=rep.degenerate_rows, loss_first=rep.loss_first,
                loss_last=rep.loss_last, orth_err=rep.orth_err, alpha_last=rep.alpha_last,
                w_norm_last=rep.w_norm_last, loss_history=list(hist) if hist is not None else None,
                w_op_last=rep.w_op_last, series_terms_last=rep.series_terms_last, p0_terms_last=rep.p0_terms_last,
                guards_run=rep.guards_run)


def kurtosis_loss_noalloc(X, R, loss_dev, stream=None):
    """kt_kurtosis_loss_noalloc: the loss without a context, a workspace or any allocation.
    `loss_dev` is a caller-owned float64 device tensor of one element; the call is stream
    ordered (synchronise before reading it).  Raises KtError(9) above N 16384 / d 1024."""
    sp = C.c_void_p(stream.cuda_stream if stream is not None else 0)
    with torch.cuda.device(X.device):     # the call works on the current device's copy of the built-in array
        _check(lib().kt_kurtosis_loss_noalloc(as_mat(X), R.data_ptr(), loss_dev.data_ptr(), sp),
               "kt_kurtosis_loss_noalloc")


def _need(cond, what):
    if not cond:
        raise ValueError(what)


class KvCache:
    """A paged, quantised KV cache: the tensors of a kt_kv_cache.

    k_codes, v_codes: uint8 [pages, heads, page_size, head_dim * bits / 8]; k_steps, v_steps: float32
    [pages, heads, page_size, 2] (scale, shift); all dense, on one device.  KvCache.empty() allocates them.
    """

    def __init__(self, k_codes, v_codes, k_steps, v_steps, bits):
        _need(bits in (4, 8), "bits must be 4 or 8")
        for c in (k_codes, v_codes):
            _need(c.dtype == torch.uint8 and c.dim() == 4 and c.is_contiguous() and c.shape == k_codes.shape
                  and c.device == k_codes.device, "codes must be dense uint8 [pages, heads, page_size, bytes]")
        for t in (k_steps, v_steps):
            _need(t.dtype == torch.float32 and t.is_contiguous() and t.shape == (*k_codes.shape[:3], 2)
                  and t.device == k_codes.device, "steps must be dense float32 [pages, heads, page_size, 2]")
        self.k_codes, self.v_codes, self.k_steps, self.v_steps, self.bits = k_codes, v_codes, k_steps, v_steps, bits
        self.index = k_codes.get_device()
        self.pages, self.heads, self.page_size, held = k_codes.shape
        self.head_dim = held * 8 // bits
        self.scale = self.head_dim ** -0.5   # of the attention's scores, unless another is given
        self._c = kt_kv_cache(k_codes.data_ptr(), v_codes.data_ptr(), k_steps.data_ptr(), v_steps.data_ptr(),
                              self.pages, self.heads, self.page_size, self.head_dim, bits)
        self._ref, self._at = C.byref(self._c), C.addressof(self._c)

    @classmethod
    def empty(cls, pages, heads, page_size, head_dim, bits, device="cuda:0"):
        """A cache of zeros."""
        codes = [torch.zeros((pages, heads, page_size, head_dim * bits // 8), dtype=torch.uint8, device=device)
                 for _ in range(2)]
        steps = [torch.zeros((pages, heads, page_size, 2), device=device) for _ in range(2)]
        return cls(*codes, *steps, bits)


class KvBatch:
    """The sequences of a call (kt_kv_batch) and the scratch of their attention; made by Context.kv_batch().

    The three index tensors may be rewritten in place between calls and between replays of a captured graph, within
    max_rows and max_length (lowered to what page_table's own columns hold, where it is columns of a wider table).  max_rows
    chooses the attention's kernel for all sequences of a call: single tokens beside a prompt are served faster by a call of
    their own.  Two calls that may overlap need two KvBatch objects (each owns one scratch buffer).
    """

    def __init__(self, row_starts, lengths, page_table, max_rows, max_length):
        for t in (row_starts, lengths, page_table):
            _need(t.dtype == torch.int32 and t.device == row_starts.device, "indices must be int32, on one device")
        _need(lengths.dim() == 1 and lengths.is_contiguous() and lengths.numel() >= 1, "lengths must be dense, 1-D")
        _need(row_starts.shape == (lengths.numel() + 1,) and row_starts.is_contiguous(),
              "row_starts must be dense, one more than lengths")
        _need(page_table.dim() == 2 and page_table.shape[0] == lengths.numel() and page_table.shape[1] >= 1
              and page_table.stride(1) == 1, "page_table must be [sequences, pages]")
        self.row_starts, self.lengths, self.page_table = row_starts, lengths, page_table
        self.max_rows, self.max_length = int(max_rows), int(max_length)
        _need(abs(self.max_rows) < 2**31 and abs(self.max_length) < 2**31, "max_rows and max_length must fit 32 bits")
        self.index = row_starts.get_device()
        ld = page_table.stride(0) if page_table.shape[0] > 1 else page_table.shape[1]
        _need(page_table.shape[1] <= ld < 2**31, "page_table rows overlap, or lie 2^31 entries apart")
        self._c = kt_kv_batch(row_starts.data_ptr(), lengths.data_ptr(), page_table.data_ptr(), lengths.numel(), ld,
                              self.max_rows, self.max_length)
        self._ref, self._at = C.byref(self._c), C.addressof(self._c)
        self.q_heads, self.scratch, self._scratch_ptr, self._scratch_bytes = 0, None, 0, 0
        self._page_size = 0 if ld > page_table.shape[1] else None   # of a table that is columns of a wider one

    def _own_columns(self, cache):
        """The kernels know a table's pitch and take it for its width: of a table that is columns of a wider one, its own
        columns bound the lengths, for caches of this page size."""
        if self._page_size is not None:
            self._page_size = cache.page_size
            self._c.max_length = self.max_length = min(self.max_length, self.page_table.shape[1] * cache.page_size)

    def _fits(self, cache, index):
        if self.index != index or cache.index != index:
            raise ValueError("cache and batch must be on the context's device")
        if self._page_size is not None and self._page_size != cache.page_size:
            raise ValueError("a page table that is columns of a wider one needs the batch of Context.kv_batch, and caches of "
                             "that call's page size")


class Context:
    """Owns a kt_ctx and (optionally) a torch-allocated workspace."""

    def __init__(self, device="cuda:0", stream=None, **cfg_overrides):
        self.device = torch.device(device)
        self.stream = stream
        self._ws = None
        self._ws_bytes = 0
        self._h = C.c_void_p()
        cfg = default_config(**cfg_overrides)
        with torch.cuda.device(self.device):
            self._index = torch.cuda.current_device()
            sp = C.c_void_p(stream.cuda_stream if stream is not None else 0)
            _check(lib().kt_create(C.byref(self._h), C.byref(cfg), sp), "kt_create")
        self._at = self._h.value

    def close(self):
        if self._h:
            lib().kt_destroy(self._h)
            self._h = C.c_void_p()
            self._at = 0
        self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- workspace --------------------------------------------------------
    def workspace_bytes(self, N, d, x_dtype=KT_BF16):
        n = C.c_size_t()
        _check(lib().kt_workspace_bytes(self._h, N, d, x_dtype, C.byref(n)), "kt_workspace_bytes")
        return n.value

    def ensure_workspace(self, N, d, x_dtype=KT_BF16):
        need = self.workspace_bytes(N, d, x_dtype)
        if need > self._ws_bytes:
            self._ws = None
            self._ws = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
            base = (self._ws.data_ptr() + 255) // 256 * 256
            _check(lib().kt_set_workspace(self._h, C.c_void_p(base), need), "kt_set_workspace")
            self._ws_bytes = need

    def _prep(self, X):
        m = as_mat(X)
        self.ensure_workspace(m.rows, m.cols, m.dtype)
        return m

    # -- entry points (same names as the C ABI, without the kt_ prefix) -----
    def init_rotation(self, d, kind):
        R = torch.empty((d, d), dtype=torch.float32, device=self.device)
        k = {"identity": 0, "hadamard": 1}[kind] if isinstance(kind, str) else kind
        _check(lib().kt_init_rotation(self._h, R.data_ptr(), d, k), "kt_init_rotation")
        return R

    def kurtosis_loss(self, X, R):
        m = self._prep(X)
        out = C.c_double()
        _check(lib().kt_kurtosis_loss(self._h, m, R.data_ptr(), C.byref(out)), "kt_kurtosis_loss")
        return out.value

    def loss_grad(self, X, R, dR=None, want_loss=True):
        m = self._prep(X)
        if dR is None:
            dR = torch.empty_like(R)
        out = C.c_double()
        _check(lib().kt_loss_grad(self._h, m, R.data_ptr(), dR.data_ptr(), C.byref(out) if want_loss else None),
               "kt_loss_grad")
        return (out.value if want_loss else None), dR

    def row_moments(self, X, R):
        m = self._prep(X)
        mom = torch.empty((m.rows, 4), dtype=torch.float32, device=self.device)
        _check(lib().kt_row_moments(self._h, m, R.data_ptr(), mom.data_ptr()), "kt_row_moments")
        return mom

    def rotate(self, X, R):
        m = self._prep(X)
        Y = torch.empty((m.rows, m.cols), dtype=torch.float32, device=self.device)
        _check(lib().kt_rotate(self._h, m, R.data_ptr(), Y.data_ptr()), "kt_rotate")
        return Y

    def orth_step(self, R, dR, lr):
        d = R.shape[0]
        self.ensure_workspace(1, d, KT_BF16)
        _check(lib().kt_orth_step(self._h, R.data_ptr(), dR.data_ptr(), d, lr), "kt_orth_step")
        return R

    def adam_step(self, R, dR, M, state, lr):
        """kt_adam_step.  `state` is a dict(v=float, step=int), zero before the first step; updated in place."""
        d = R.shape[0]
        self.ensure_workspace(1, d, KT_BF16)
        st = kt_adam_state(float(state["v"]), int(state["step"]), 0)
        _check(lib().kt_adam_step(self._h, R.data_ptr(), dR.data_ptr(), M.data_ptr(), C.byref(st), d, lr),
               "kt_adam_step")
        state["v"], state["step"] = st.v, st.step
        return R

    def orth_error(self, R):
        d = R.shape[0]
        self.ensure_workspace(1, d, KT_BF16)
        out = C.c_double()
        _check(lib().kt_orth_error(self._h, R.data_ptr(), d, C.byref(out)), "kt_orth_error")
        return out.value

    def fit(self, X, R, steps, lr, history=False):
        m = self._prep(X)
        rep = kt_fit_report()
        hist = (C.c_double * max(steps, 1))() if history else None
        if history:
            rep.loss_history = C.cast(hist, C.POINTER(C.c_double))
        _check(lib().kt_fit(self._h, m, R.data_ptr(), steps, lr, C.byref(rep)), "kt_fit")
        return _rep_dict(rep, hist[:steps] if history else None)

    def fit_layers(self, Xs, Rs, steps, lr, first_layer=0):
        L = len(Xs)
        mats = (kt_mat * L)(*[as_mat(X) for X in Xs])
        self.ensure_workspace(mats[0].rows, mats[0].cols, mats[0].dtype)
        ptrs = (C.c_void_p * L)(*[R.data_ptr() for R in Rs])
        reps = (kt_fit_report * L)()
        _check(lib().kt_fit_layers(self._h, mats, ptrs, L, first_layer, steps, lr, reps), "kt_fit_layers")
        return [_rep_dict(r, None) for r in reps]

    def fit_shared(self, Xs, rows_per_sample, order, batch, R, steps, lr, history=False):
        """kt_fit_shared: one R for the equally shaped buffers Xs; `order` is a sequence of steps*batch sample ids."""
        nb = len(Xs)
        mats = (kt_mat * nb)(*[as_mat(X) for X in Xs])
        self._shared_workspace(rows_per_sample, batch, mats[0].cols)
        ids = (C.c_int32 * (steps * batch))(*[int(v) for v in order[:steps * batch]])
        rep = kt_fit_report()
        hist = (C.c_double * steps)() if history and steps > 0 else None
        if hist is not None:
            rep.loss_history = C.cast(hist, C.POINTER(C.c_double))
        _check(lib().kt_fit_shared(self._h, mats, nb, rows_per_sample, ids, batch, R.data_ptr(), steps, lr,
                                   C.byref(rep)), "kt_fit_shared")
        return _rep_dict(rep, hist)

    def _shared_workspace(self, rows_per_sample, batch, d):
        need = C.c_size_t()
        _check(lib().kt_fit_shared_workspace_bytes(self._h, rows_per_sample, batch, d, C.byref(need)),
               "kt_fit_shared_workspace_bytes")
        if need.value > self._ws_bytes:
            self._ws = None
            self._ws = torch.empty(need.value + 256, dtype=torch.uint8, device=self.device)
            base = (self._ws.data_ptr() + 255) // 256 * 256
            _check(lib().kt_set_workspace(self._h, C.c_void_p(base), need.value), "kt_set_workspace")
            self._ws_bytes = need.value

    def fit_sharded(self, X_local, R, rows_total, reduce, steps, lr, history=False):
        """kt_fit_sharded.  `reduce` is None (a single shard) or a Python callable
        reduce(dev_ptr, count, dtype, cuda_stream) -> 0 that enqueues an in-place sum all-reduce."""
        m = self._prep(X_local)
        rep = kt_fit_report()
        hist = (C.c_double * max(steps, 1))() if history else None
        if history:
            rep.loss_history = C.cast(hist, C.POINTER(C.c_double))
        cb = REDUCE_FN(lambda user, ptr, count, dtype, stream: int(reduce(ptr, count, dtype, stream))) \
            if reduce is not None else C.cast(None, REDUCE_FN)
        _check(lib().kt_fit_sharded(self._h, m, R.data_ptr(), rows_total, cb, None, steps, lr, C.byref(rep)),
               "kt_fit_sharded")
        return _rep_dict(rep, hist[:steps] if history else None)

    def fit_shared_sharded(self, Xs, rows_per_sample, order, batch, R, rows_total, reduce, steps, lr, history=False):
        """kt_fit_shared_sharded: this process's share (`batch` samples per step, its own `order`) of every minibatch."""
        nb = len(Xs)
        mats = (kt_mat * nb)(*[as_mat(X) for X in Xs])
        self._shared_workspace(rows_per_sample, batch, mats[0].cols)
        ids = (C.c_int32 * (steps * batch))(*[int(v) for v in order[:steps * batch]])
        rep = kt_fit_report()
        hist = (C.c_double * steps)() if history and steps > 0 else None
        if hist is not None:
            rep.loss_history = C.cast(hist, C.POINTER(C.c_double))
        cb = REDUCE_FN(lambda user, ptr, count, dtype, stream: int(reduce(ptr, count, dtype, stream))) \
            if reduce is not None else C.cast(None, REDUCE_FN)
        _check(lib().kt_fit_shared_sharded(self._h, mats, nb, rows_per_sample, ids, batch, R.data_ptr(), rows_total,
                                           cb, None, steps, lr, C.byref(rep)), "kt_fit_shared_sharded")
        return _rep_dict(rep, hist)

    def test_wait_timeout(self, limit_ms):
        _check(lib().kt_test_wait_timeout(self._h, limit_ms), "kt_test_wait_timeout")

    def fit_host(self, X_host, X_staging, R_host, R_dev, steps, lr):
        m = as_mat(X_host)
        self.ensure_workspace(m.rows, m.cols, m.dtype)
        rep = kt_fit_report()
        _check(lib().kt_fit_host(self._h, m, X_staging.data_ptr(), R_host.data_ptr(), R_dev.data_ptr(), steps, lr,
                                 C.byref(rep)), "kt_fit_host")
        return _rep_dict(rep, None)

    def quant4_error(self, X, R):
        m = self._prep(X)
        out = C.c_double()
        _check(lib().kt_quant4_error(self._h, m, R.data_ptr(), C.byref(out)), "kt_quant4_error")
        return out.value

    def quant_error(self, X, R, bits=4, asymmetric=False, clip=1.0, clip_mode=0):
        m = self._prep(X)
        spec = kt_quant_spec(bits, int(asymmetric), clip, clip_mode)
        out = C.c_double()
        _check(lib().kt_quant_error(self._h, m, R.data_ptr(), C.byref(spec), C.byref(out)), "kt_quant_error")
        return out.value

    def quant_codes(self, Y, bits=4, asymmetric=False, clip=1.0, clip_mode=0):
        N, d = Y.shape
        spec = kt_quant_spec(bits, int(asymmetric), clip, clip_mode)
        codes = torch.empty((N, d), dtype=torch.int16, device=Y.device)
        scales = torch.empty((N,), dtype=torch.float32, device=Y.device)
        shifts = torch.empty((N,), dtype=torch.float32, device=Y.device)
        _check(lib().kt_quant_codes(self._h, Y.data_ptr(), N, d, C.byref(spec), codes.data_ptr(), scales.data_ptr(),
                                    shifts.data_ptr()), "kt_quant_codes")
        return codes, scales, shifts

    def quant_error_given(self, Y, bits=4, asymmetric=False, clip=1.0, clip_mode=0):
        N, d = Y.shape
        self.ensure_workspace(N, max(128, (d + 127) // 128 * 128), KT_BF16)
        spec = kt_quant_spec(bits, int(asymmetric), clip, clip_mode)
        out = C.c_double()
        _check(lib().kt_quant_error_given(self._h, Y.data_ptr(), N, d, C.byref(spec), C.byref(out)),
               "kt_quant_error_given")
        return out.value

    # -- the rotated, quantised model ------------------------------------------
    def _new(self, shape, dtype):
        """An output, allocated on the context's stream, whose kernels write it."""
        with torch.cuda.stream(self.stream or torch.cuda.default_stream(self._index)):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def rmsnorm_quant(self, x, residual=None, residual_out=None, gain=None, eps=1e-6, bits=8, clip=1.0, codes=None,
                      scales=None, values=None):
        """kt_rmsnorm_quant on x (N x d, bf16 or f32).  Returns (codes, scales, values).

        bits in 2..8; bits=None: no quantisation, `values` (allocated in x's type if not given) receives the normalised
        rows.  codes (int8) are allocated if neither codes nor values is given; an output that is neither given nor
        allocated comes back as None."""
        if bits is None:
            _need(codes is None and scales is None, "bits=None has no codes and no scales")
            if values is None:
                values = self._new(x.shape, x.dtype)
        else:
            if codes is None and values is None:
                codes = self._new(x.shape, torch.int8)
            if scales is None:
                scales = self._new(x.shape[:1], torch.float32)
        st = _serving.rmsnorm_quant(self._at, self._index, x, residual, residual_out, gain, eps, bits, clip, codes, scales,
                                    values)
        if st:
            raise KtError(st, "kt_rmsnorm_quant")
        return codes, scales, values

    def kv_batch(self, cache, q_heads, row_starts, lengths, page_table, max_rows, max_length):
        """A KvBatch with the scratch that kv_attend needs for this cache and head count (make it before capturing a graph
        that uses it)."""
        batch = KvBatch(row_starts, lengths, page_table, max_rows, max_length)
        batch._own_columns(cache)
        batch._fits(cache, self._index)
        n = C.c_size_t()
        _check(lib().kt_kv_scratch_bytes(self._h, cache._ref, batch._ref, q_heads, C.byref(n)), "kt_kv_scratch_bytes")
        batch.q_heads = q_heads
        if n.value:
            batch.scratch = self._new((n.value + 256,), torch.uint8)
            batch._scratch_ptr = (batch.scratch.data_ptr() + 255) // 256 * 256
            batch._scratch_bytes = n.value
        return batch

    def kv_append(self, cache, batch, q, k, v, rope=None, hadamard=False, asymmetric=True, clip=1.0, q_out=None,
                  k_values=None, v_values=None):
        """kt_kv_append.  q (None: keys and values only), k, v: rows x heads*head_dim, bf16 or f32.  Returns q_out, the
        turned queries in bf16 (allocated if not given; may be q itself)."""
        batch._fits(cache, self._index)
        if q is not None and q_out is None:
            q_out = self._new(q.shape, torch.bfloat16)
        st = _serving.kv_append(self._at, self._index, cache._at, batch._at, q, k, v, rope, hadamard, asymmetric, clip,
                                q_out, k_values, v_values)
        if st:
            raise KtError(st, "kt_kv_append")
        return q_out

    def kv_attend(self, cache, batch, q, out=None, lse=None, scale=None, causal=True, window=0):
        """kt_kv_attend.  q: rows x q_heads*head_dim bf16; scale: 1/sqrt(head_dim) if not given; lse: float32
        rows x q_heads to be filled, or None.  Returns out (allocated if not given: rows that no sequence owns, or of a
        sequence out of bounds, are then whatever the memory held)."""
        batch._fits(cache, self._index)
        if out is None:
            out = self._new(q.shape, torch.bfloat16)
        st = _serving.kv_attend(self._at, self._index, cache._at, batch._at, q, out, lse,
                                cache.scale if scale is None else scale, causal, window, batch._scratch_ptr,
                                batch._scratch_bytes)
        if st:
            raise KtError(st, "kt_kv_attend")
        return out

    def check(self):
        """kt_check: synchronises, and raises what the stream-ordered calls left (KT_ERR_TIMEOUT, KT_ERR_CACHE)."""
        _check(lib().kt_check(self._h), "kt_check")

    def rowmax_success(self, X, R_a, R_b=None):
        m = self._prep(X)
        out = C.c_double()
        _check(lib().kt_rowmax_success(self._h, m, R_a.data_ptr(), R_b.data_ptr() if R_b is not None else None,
                                       C.byref(out)), "kt_rowmax_success")
        return out.value

    def profile_begin(self):
        _check(lib().kt_profile_begin(self._h), "kt_profile_begin")

    def profile_end(self):
        pr = kt_profile()
        _check(lib().kt_profile_end(self._h, C.byref(pr)), "kt_profile_end")
        names = ["forward", "backward_a", "backward_b", "square", "quant", "fused"]
        return dict(launches_total=pr.launches_total,
                    gemm={n: dict(launches=pr.gemm_launches[i], ms=pr.gemm_ms[i]) for i, n in enumerate(names)})

    def quant4_codes(self, Y):
        N, d = Y.shape
        codes = torch.empty((N, d), dtype=torch.int8, device=self.device)
        scales = torch.empty((N,), dtype=torch.float32, device=self.device)
        _check(lib().kt_quant4_codes(self._h, Y.data_ptr(), N, d, codes.data_ptr(), scales.data_ptr()),
               "kt_quant4_codes")
        return codes, scales
