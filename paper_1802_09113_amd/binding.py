"""Thin ctypes binding of libssn_hip.so (C ABI in include/ssn.h).

Argument marshalling only: torch tensors supply device pointers and the current HIP stream, every
step of the method runs inside the library's kernels.  There is no fallback: if the library has not
been built (python -m paper_1802_09113_amd.build) importing this module's `lib()` raises.
"""
import ctypes
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libssn_hip.so")

SSN_F32, SSN_F64, SSN_F16, SSN_BF16 = 0, 1, 2, 3
SSN_DENSE_ROWMAJOR, SSN_CSR = 0, 1
SSN_SCALE_MEAN, SSN_SCALE_SUM = 0, 1
SSN_OK = 0
SSN_SOLVE_NO_LOOKAHEAD = 1
SSN_SOLVE_NO_PHASE_TIMES = 2
SSN_SOLVE_NO_MARGIN_CACHE = 4
SSN_E_INVALID_ARG, SSN_E_BAD_LABEL, SSN_E_BAD_INDEX, SSN_E_NOT_PREPARED = -1, -2, -3, -4
SSN_E_ALLOC, SSN_E_HIP, SSN_E_NONFINITE, SSN_E_UNSUPPORTED, SSN_E_TOO_LARGE = -5, -6, -7, -8, -9
SSN_STATIC_WORKSPACE_BYTES = 48 << 20

EXPORTS = [
    "ssn_strerror", "ssn_last_error", "ssn_create", "ssn_destroy", "ssn_set_stream", "ssn_objective",
    "ssn_gradient", "ssn_gradient_sampled", "ssn_hess_prepare", "ssn_hess_apply", "ssn_hessvec", "ssn_cg", "ssn_linesearch",
    "ssn_predict", "ssn_solve", "ssn_axpy", "ssn_normalize_columns", "ssn_objective_dev", "ssn_gradient_dev",
    "ssn_accuracy", "ssn_vec_to_rowmajor", "ssn_rowmajor_to_vec", "ssn_hessvec_static",
    "ssn_logprobs", "ssn_logprobs_workspace", "ssn_logprobs_grad", "ssn_q4_quantize", "ssn_q4_margins",
    "ssn_q4_margins_workspace",
]
BENCH_EXPORTS = ["ssn_time_kernel", "ssn_dense_path", "ssn_sampled_slices", "ssn_direction_form"]          # include/ssn_bench.h


class ssn_desc(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int64), ("p", ctypes.c_int64),
        ("C", ctypes.c_int32), ("dtype", ctypes.c_int32), ("layout", ctypes.c_int32), ("scale", ctypes.c_int32),
        ("lam", ctypes.c_double),
        ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
        ("rowptr", ctypes.c_void_p), ("colidx", ctypes.c_void_p), ("vals", ctypes.c_void_p), ("nnz", ctypes.c_int64),
        ("labels", ctypes.c_void_p),
        ("ldw", ctypes.c_int64),
        ("stream", ctypes.c_void_p),
    ]


class ssn_cg_info(ctypes.Structure):
    _fields_ = [("iters", ctypes.c_int32), ("flags", ctypes.c_int32), ("rel_res", ctypes.c_double),
                ("gnorm", ctypes.c_double)]


class ssn_params(ctypes.Structure):
    _fields_ = [
        ("iters", ctypes.c_int32), ("T", ctypes.c_int32), ("imax", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("nS", ctypes.c_int64),
        ("eps", ctypes.c_double), ("theta", ctypes.c_double), ("beta", ctypes.c_double), ("rho", ctypes.c_double),
        ("S_all", ctypes.c_void_p), ("test", ctypes.c_void_p),
        ("Sg_all", ctypes.c_void_p), ("nSg", ctypes.c_int64),
    ]


class ssn_iter_record(ctypes.Structure):
    _fields_ = [
        ("f", ctypes.c_double), ("gnorm", ctypes.c_double), ("cg_rel_res", ctypes.c_double), ("alpha", ctypes.c_double),
        ("test_acc", ctypes.c_double),
        ("ms_grad", ctypes.c_double), ("ms_prepare", ctypes.c_double), ("ms_cg", ctypes.c_double),
        ("ms_linesearch", ctypes.c_double), ("ms_update", ctypes.c_double),
        ("cg_iters", ctypes.c_int32), ("ls_evals", ctypes.c_int32), ("ls_ok", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class ssn_rows(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int64), ("C", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reference", ctypes.c_int32),
        ("Z", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("allowed", ctypes.c_void_p), ("ld_allowed", ctypes.c_int64),
        ("labels", ctypes.c_void_p), ("m", ctypes.c_int32), ("k", ctypes.c_int32), ("stream", ctypes.c_void_p),
    ]


class ssn_q4(ctypes.Structure):
    _fields_ = [("p", ctypes.c_int64), ("K", ctypes.c_int64), ("group", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("packed", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


_lib = None


def lib():
    """Load the HIP library; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1802_09113_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.ssn_strerror.restype = ctypes.c_char_p
        L.ssn_strerror.argtypes = [ctypes.c_int]
        L.ssn_last_error.restype = ctypes.c_char_p
        L.ssn_last_error.argtypes = [ctypes.c_void_p]
        vp, dp, ip = ctypes.c_void_p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)
        L.ssn_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(ssn_desc)]
        L.ssn_destroy.argtypes = [vp]
        L.ssn_set_stream.argtypes = [vp, vp]
        L.ssn_objective.argtypes = [vp, vp, dp]
        L.ssn_gradient.argtypes = [vp, vp, vp, dp]
        L.ssn_gradient_sampled.argtypes = [vp, vp, vp, ctypes.c_int64, vp, dp]
        L.ssn_hess_prepare.argtypes = [vp, vp, vp, ctypes.c_int64]
        L.ssn_hess_apply.argtypes = [vp, vp, vp]
        L.ssn_hessvec.argtypes = [vp, vp, vp, ctypes.c_int64, vp, vp]
        L.ssn_cg.argtypes = [vp, vp, ctypes.c_double, ctypes.c_int32, vp, ctypes.POINTER(ssn_cg_info), dp]
        L.ssn_linesearch.argtypes = [vp, vp, vp, vp, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_int32,
                                     dp, dp, ip, ip]
        L.ssn_predict.argtypes = [vp, vp, vp, dp]
        L.ssn_solve.argtypes = [vp, vp, ctypes.POINTER(ssn_params), ctypes.POINTER(ssn_iter_record), ctypes.c_int32, ip]
        L.ssn_axpy.argtypes = [vp, ctypes.c_double, vp, vp]
        L.ssn_time_kernel.argtypes = [vp, ctypes.c_int32, vp, ctypes.c_int32, dp]
        L.ssn_dense_path.argtypes = [vp]
        L.ssn_sampled_slices.argtypes = [vp]
        L.ssn_direction_form.argtypes = [vp]
        L.ssn_normalize_columns.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, vp, ctypes.c_int64,
                                            vp, vp, vp, ctypes.c_int64, vp, vp]
        L.ssn_objective_dev.argtypes = [vp, vp, vp]
        L.ssn_gradient_dev.argtypes = [vp, vp, vp, vp]
        L.ssn_accuracy.argtypes = [vp, ctypes.POINTER(ssn_desc), vp, dp]
        L.ssn_vec_to_rowmajor.argtypes = [vp, vp, vp]
        L.ssn_rowmajor_to_vec.argtypes = [vp, vp, vp]
        L.ssn_hessvec_static.argtypes = [ctypes.POINTER(ssn_desc), vp, vp, ctypes.c_int64, vp, vp]
        i32, i64, lp, rows, q4 = (ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ssn_rows),
                                  ctypes.POINTER(ssn_q4))
        L.ssn_logprobs.argtypes = [rows, vp, vp, vp, vp, vp, vp, vp, i64]
        L.ssn_logprobs_workspace.argtypes = [rows, lp]
        L.ssn_logprobs_grad.argtypes = [rows, vp, vp, vp, vp, vp, vp, vp, vp, i64]
        L.ssn_q4_quantize.argtypes = [q4, i32, vp, i64, i64, vp]
        L.ssn_q4_margins.argtypes = [q4, i32, i64, vp, i64, i32, vp, i64, vp, i64, vp]
        L.ssn_q4_margins_workspace.argtypes = [q4, i32, i64, lp]
        for name in EXPORTS + BENCH_EXPORTS:
            fn = getattr(L, name)
            if fn.restype is not ctypes.c_char_p:
                fn.restype = ctypes.c_int
        _lib = L
    return _lib


def ssn_normalize_columns(X=None, csr=None, p=None):
    """Unit-column-norm preprocessing of Sec. 4, in place on device tensors: X (n x p, row-major, float32 / float64)
    or csr = (rowptr int32, colidx int32, vals).  Returns the column norms before scaling (float64, device)."""
    if X is not None:
        assert X.is_cuda and X.dim() == 2 and X.stride(1) == 1
        n, p = X.shape
        norms = torch.empty(p, dtype=torch.float64, device=X.device)
        dt = 0 if X.dtype == torch.float32 else 1
        st = lib().ssn_normalize_columns(0, dt, n, p, _ptr(X), X.stride(0), None, None, None, 0, _ptr(norms), None)
    else:
        rowptr, colidx, vals = csr
        assert rowptr.is_cuda and rowptr.dtype == torch.int32 and colidx.dtype == torch.int32
        n = rowptr.shape[0] - 1
        norms = torch.empty(int(p), dtype=torch.float64, device=vals.device)
        dt = 0 if vals.dtype == torch.float32 else 1
        st = lib().ssn_normalize_columns(1, dt, n, int(p), None, 0, _ptr(rowptr), _ptr(colidx), _ptr(vals), vals.shape[0],
                                         _ptr(norms), None)
    if st != 0:
        raise SsnError(st, "ssn_normalize_columns")
    return norms


class SsnError(RuntimeError):
    def __init__(self, status, detail=""):
        self.status = status
        name = lib().ssn_strerror(status).decode()
        super().__init__(f"ssn status {status} ({name}) {detail}")


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def make_desc(labels, C, lam, X=None, csr=None, p=None, scale="mean", ldw=None, stream=None):
    """An ssn_desc for device tensors (and the list of tensors it borrows, to be kept alive by the caller)."""
    assert labels.is_cuda and labels.dtype == torch.int32
    keep = [labels]
    d = ssn_desc()
    d.n, d.C, d.lam = labels.shape[0], C, lam
    d.scale = {"mean": SSN_SCALE_MEAN, "sum": SSN_SCALE_SUM}[scale]
    d.labels = labels.data_ptr()
    if X is not None:
        assert X.is_cuda and X.dim() == 2 and X.stride(1) == 1
        d.layout, d.X, d.ldx, d.p = SSN_DENSE_ROWMAJOR, X.data_ptr(), X.stride(0), X.shape[1]
        tdtype = X.dtype
        keep.append(X)
    else:
        rowptr, colidx, vals = csr
        assert rowptr.dtype == torch.int32 and colidx.dtype == torch.int32
        d.layout, d.p, d.nnz = SSN_CSR, p, vals.shape[0]
        d.rowptr, d.colidx, d.vals = rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr()
        tdtype = vals.dtype
        keep += [rowptr, colidx, vals]
    d.dtype = {torch.float32: SSN_F32, torch.float64: SSN_F64}[tdtype]
    d.ldw = int(ldw) if ldw is not None else int(C) - 1
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    d.stream = stream
    return d, keep


def ssn_hessvec_static(desc, W, S, V, HV):
    """The product of Context.ssn_hessvec without a context and without any allocation: desc from make_desc,
    W, V, HV p x ldw device blocks, S int32 device indices.  Returns the status (0 = ok)."""
    assert S.is_cuda and S.dtype == torch.int32 and S.is_contiguous()
    return lib().ssn_hessvec_static(ctypes.byref(desc), _ptr(W), _ptr(S), S.shape[0], _ptr(V), _ptr(HV))


class Context:
    """One data set resident on the GPU.  Methods carry the names of the C entry points."""

    def __init__(self, labels, C, lam, X=None, csr=None, p=None, scale="mean", ldw=None, stream=None):
        d, self._keep = make_desc(labels, C, lam, X=X, csr=csr, p=p, scale=scale, ldw=ldw, stream=stream)
        self.tdtype = X.dtype if X is not None else csr[2].dtype
        self.n, self.p, self.C, self.K = int(d.n), int(d.p), int(C), int(C) - 1
        self.ldw = int(d.ldw)
        self.device = labels.device
        self._h = ctypes.c_void_p()
        st = lib().ssn_create(ctypes.byref(self._h), ctypes.byref(d))
        if st != SSN_OK:
            self._h = None
            raise SsnError(st, "in ssn_create")

    def close(self):
        if getattr(self, "_h", None):
            lib().ssn_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st):
        if st != SSN_OK:
            raise SsnError(st, lib().ssn_last_error(self._h).decode())

    def ssn_set_stream(self, stream):
        """stream: a hipStream_t handle as an integer (e.g. torch.cuda.Stream().cuda_stream), or None for the default."""
        self._check(lib().ssn_set_stream(self._h, ctypes.c_void_p(stream) if stream else None))

    def new_block(self):
        """An uninitialised p x ldw block of the context's dtype."""
        return torch.empty((self.p, self.ldw), dtype=self.tdtype, device=self.device)

    def _blk(self, t):
        assert t.is_cuda and t.dtype == self.tdtype and t.shape[0] == self.p and t.stride(0) == self.ldw and t.stride(1) == 1
        return _ptr(t)

    def ssn_objective(self, W):
        f = ctypes.c_double()
        self._check(lib().ssn_objective(self._h, self._blk(W), ctypes.byref(f)))
        return f.value

    def ssn_gradient(self, W, G=None, want_f=True):
        G = self.new_block() if G is None else G
        f = ctypes.c_double()
        self._check(lib().ssn_gradient(self._h, self._blk(W), self._blk(G), ctypes.byref(f) if want_f else None))
        return G, (f.value if want_f else None)

    def ssn_objective_dev(self, W, f_dev):
        """f_dev: a one-element float64 device tensor that receives f(W); nothing is read back."""
        assert f_dev.is_cuda and f_dev.dtype == torch.float64
        self._check(lib().ssn_objective_dev(self._h, self._blk(W), _ptr(f_dev)))

    def ssn_gradient_dev(self, W, G, f_dev):
        assert f_dev.is_cuda and f_dev.dtype == torch.float64
        self._check(lib().ssn_gradient_dev(self._h, self._blk(W), self._blk(G), _ptr(f_dev)))

    def ssn_accuracy(self, test_desc, W):
        acc = ctypes.c_double()
        self._check(lib().ssn_accuracy(self._h, ctypes.byref(test_desc), self._blk(W), ctypes.byref(acc)))
        return acc.value

    def ssn_vec_to_rowmajor(self, vec, block=None):
        assert vec.is_cuda and vec.dtype == self.tdtype and vec.is_contiguous() and vec.numel() == self.p * self.K
        block = self.new_block() if block is None else block
        self._check(lib().ssn_vec_to_rowmajor(self._h, _ptr(vec), self._blk(block)))
        return block

    def ssn_rowmajor_to_vec(self, block, vec=None):
        vec = torch.empty(self.p * self.K, dtype=self.tdtype, device=self.device) if vec is None else vec
        assert vec.is_cuda and vec.dtype == self.tdtype and vec.is_contiguous() and vec.numel() == self.p * self.K
        self._check(lib().ssn_rowmajor_to_vec(self._h, self._blk(block), _ptr(vec)))
        return vec

    def ssn_gradient_sampled(self, W, S, G=None, want_f=True):
        assert S.is_cuda and S.dtype == torch.int32 and S.is_contiguous()
        G = self.new_block() if G is None else G
        f = ctypes.c_double()
        self._check(lib().ssn_gradient_sampled(self._h, self._blk(W), _ptr(S), S.shape[0], self._blk(G),
                                               ctypes.byref(f) if want_f else None))
        return G, (f.value if want_f else None)

    def ssn_hess_prepare(self, W, S):
        assert S.is_cuda and S.dtype == torch.int32 and S.is_contiguous()
        self._S = S
        self._check(lib().ssn_hess_prepare(self._h, self._blk(W), _ptr(S), S.shape[0]))

    def ssn_hess_apply(self, V, HV=None):
        HV = self.new_block() if HV is None else HV
        self._check(lib().ssn_hess_apply(self._h, self._blk(V), self._blk(HV)))
        return HV

    def ssn_hessvec(self, W, S, V, HV=None):
        assert S.is_cuda and S.dtype == torch.int32 and S.is_contiguous()
        self._S = S
        HV = self.new_block() if HV is None else HV
        self._check(lib().ssn_hessvec(self._h, self._blk(W), _ptr(S), S.shape[0], self._blk(V), self._blk(HV)))
        return HV

    def ssn_cg(self, G, theta, T, P=None, want_trace=True):
        P = self.new_block() if P is None else P
        info = ssn_cg_info()
        tr = (ctypes.c_double * (3 * max(T, 1)))()
        self._check(lib().ssn_cg(self._h, self._blk(G), theta, T, self._blk(P), ctypes.byref(info),
                                 tr if want_trace else None))
        it = info.iters
        out = dict(p=P, iters=it, flags=info.flags, rel_res=info.rel_res, gnorm=info.gnorm)
        if want_trace:
            out.update(alpha=[tr[3 * k] for k in range(it)], rnorm=[tr[3 * k + 1] for k in range(it)],
                       sHs=[tr[3 * k + 2] for k in range(it)])
        return out

    def ssn_linesearch(self, W, P, G, fW, beta=1e-4, rho=0.5, imax=10):
        a, fn = ctypes.c_double(), ctypes.c_double()
        ne, ok = ctypes.c_int32(), ctypes.c_int32()
        self._check(lib().ssn_linesearch(self._h, self._blk(W), self._blk(P), self._blk(G), fW, beta, rho, imax,
                                         ctypes.byref(a), ctypes.byref(fn), ctypes.byref(ne), ctypes.byref(ok)))
        return dict(alpha=a.value, f_new=fn.value, n_eval=ne.value, ok=ok.value)

    def ssn_predict(self, W, want_pred=True):
        pred = torch.empty(self.n, dtype=torch.int32, device=self.device) if want_pred else None
        acc = ctypes.c_double()
        self._check(lib().ssn_predict(self._h, self._blk(W), _ptr(pred), ctypes.byref(acc)))
        return pred, acc.value

    def ssn_axpy(self, alpha, P, W):
        self._check(lib().ssn_axpy(self._h, alpha, self._blk(P), self._blk(W)))

    def ssn_dense_path(self):
        return lib().ssn_dense_path(self._h)

    def ssn_sampled_slices(self):
        return lib().ssn_sampled_slices(self._h)

    def ssn_direction_form(self):
        return lib().ssn_direction_form(self._h)

    def ssn_time_kernel(self, which, M, reps):
        ms = ctypes.c_double()
        self._check(lib().ssn_time_kernel(self._h, which, self._blk(M), reps, ctypes.byref(ms)))
        return ms.value

    def ssn_solve(self, W, S_all, eps=0.0, theta=1e-4, T=10, beta=1e-4, rho=0.5, imax=10, test=None, Sg_all=None,
                  lookahead=True, phase_times=True, margin_cache=True):
        """S_all: (iters, nS) int32 device tensor; Sg_all (optional): (iters, nSg) gradient samples.  W is updated
        in place; returns (records, iterations done).  lookahead=False sets SSN_SOLVE_NO_LOOKAHEAD,
        phase_times=False SSN_SOLVE_NO_PHASE_TIMES."""
        assert S_all.is_cuda and S_all.dtype == torch.int32 and S_all.is_contiguous() and S_all.dim() == 2
        pr = ssn_params()
        if Sg_all is not None:
            assert Sg_all.is_cuda and Sg_all.dtype == torch.int32 and Sg_all.is_contiguous() and Sg_all.dim() == 2
            assert Sg_all.shape[0] == S_all.shape[0]
            pr.Sg_all, pr.nSg = Sg_all.data_ptr(), Sg_all.shape[1]
        pr.iters, pr.nS = S_all.shape
        pr.T, pr.imax, pr.eps, pr.theta, pr.beta, pr.rho = T, imax, eps, theta, beta, rho
        pr.S_all = S_all.data_ptr()
        pr.flags = ((0 if lookahead else SSN_SOLVE_NO_LOOKAHEAD) | (0 if phase_times else SSN_SOLVE_NO_PHASE_TIMES)
                    | (0 if margin_cache else SSN_SOLVE_NO_MARGIN_CACHE))
        pr.test = test._h if test is not None else None
        log = (ssn_iter_record * max(int(pr.iters), 1))()
        done = ctypes.c_int32()
        self._check(lib().ssn_solve(self._h, self._blk(W), ctypes.byref(pr), log, int(pr.iters), ctypes.byref(done)))
        fields = [f[0] for f in ssn_iter_record._fields_ if f[0] != "reserved"]
        nrec = min(done.value + 1, int(pr.iters))
        return [{k: getattr(log[i], k) for k in fields} for i in range(nrec)], done.value


# ---- a softmax layer over many classes -----------------------------------------------------------------------------
# The smallest of these calls are a kernel of a few microseconds: what the binding does around them is kept to plain
# attribute reads and one library call where no workspace is needed.  They take and return plain data: torch records no graph
# of them, and a gradient is asked for with ssn_logprobs_grad.

_DTYPE = {torch.float32: SSN_F32, torch.float64: SSN_F64, torch.float16: SSN_F16, torch.bfloat16: SSN_BF16}
_STAT = {torch.float32: torch.float32, torch.float16: torch.float32, torch.bfloat16: torch.float32, torch.float64: torch.float64}


def _raw_stream(dev):
    """The current stream of a device as a hipStream_t: from torch's table of handles where this torch has that accessor
    (0.1 us), else from a stream object (1.1 us)."""
    handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return handle(dev) if handle else torch.cuda.current_stream(dev).cuda_stream


def _ld(t, n, width):
    """Leading dimension of an n x width matrix whose rows are contiguous (the stride of a single row means nothing)."""
    ld, step = t.stride()
    assert step == 1 or width == 1, "rows must be contiguous"
    return ld if n > 1 else width


def _elsewhere(t):
    """Whether t lives on another device than the current one (kernels go to its device's current stream)."""
    assert t.is_cuda
    return t.get_device() != torch.cuda.current_device()


def _rows(Z, labels, k, reference, allowed, dev):
    n, width = Z.shape
    reference = 1 if reference else 0
    C = width + reference
    at_allowed, ld_allowed, at_labels, m = None, 0, None, 0
    if allowed is not None:
        words = (C + 31) // 32
        assert allowed.get_device() == dev and allowed.dtype is torch.int32 and allowed.shape[-1] == words
        assert allowed.stride(-1) == 1 or words == 1
        assert allowed.dim() == 1 or (allowed.dim() == 2 and allowed.shape[0] == n)
        at_allowed, ld_allowed = allowed.data_ptr(), 0 if allowed.dim() == 1 else allowed.stride(0) if n > 1 else words
    if labels is not None:
        assert labels.get_device() == dev and labels.dtype is torch.int32 and labels.is_contiguous()
        shape = labels.shape
        assert shape[0] == n and len(shape) <= 2
        at_labels, m = labels.data_ptr(), shape[1] if len(shape) == 2 else 1
    return ssn_rows(n, C, _DTYPE[Z.dtype], reference, Z.data_ptr(), _ld(Z, n, width), at_allowed, ld_allowed, at_labels, m, k,
                    _raw_stream(dev)), n, m


def _data(t, dtype, count, dev):
    """The address of a contiguous tensor of `count` elements, or None."""
    if t is None:
        return None
    assert t.dtype is dtype and t.numel() == count and t.get_device() == dev and t.is_contiguous()
    return t.data_ptr()


def ssn_logprobs(Z, labels=None, k=0, reference=False, allowed=None, out=None):
    """Log probabilities of given classes, entropy and the k most probable classes of rows of margins.

    Z: n x C device tensor (float32, float64, float16, bfloat16), rows contiguous; with reference=True n x (C - 1), and
    class C - 1 has margin zero.  labels: int32, (n,) or (n, m), negative = padding.  allowed: int32 words of bits, (n,
    ceil(C / 32)) or one row of words for all.  Returns a dict of logp (shaped like labels), maxpart, logpart, entropy
    and, with k > 0, top_ids and top_logp; `out` may bring any of them (missing or None: entropy, maxpart and logpart are
    then not computed, the others allocated).  Nothing of it requires a gradient, whatever Z does: ssn_logprobs_grad is the
    backward pass, to be called by itself or by a torch.autograd.Function of the caller's."""
    if _elsewhere(Z):
        with torch.cuda.device(Z.device):
            return ssn_logprobs(Z, labels, k, reference, allowed, out)
    dev, stat = Z.get_device(), _STAT[Z.dtype]
    d, n, m = _rows(Z, labels, k, reference, allowed, dev)
    if out is None:
        out = {name: torch.empty(n, dtype=stat, device=Z.device) for name in ("maxpart", "logpart", "entropy")}
    get = out.get
    if labels is not None and get("logp") is None:
        out["logp"] = torch.empty(labels.shape, dtype=stat, device=Z.device)
    if k and get("top_ids") is None:
        out["top_ids"] = torch.empty((n, k), dtype=torch.int32, device=Z.device)
    if k and get("top_logp") is None:
        out["top_logp"] = torch.empty((n, k), dtype=stat, device=Z.device)
    args = (ctypes.byref(d), _data(out["logp"], stat, n * m, dev) if m else None, _data(get("maxpart"), stat, n, dev),
            _data(get("logpart"), stat, n, dev), _data(get("entropy"), stat, n, dev),
            _data(out["top_ids"], torch.int32, n * k, dev) if k else None,
            _data(out["top_logp"], stat, n * k, dev) if k else None)
    L = lib()
    st = L.ssn_logprobs(*args, None, 0)
    if st == SSN_E_TOO_LARGE:                       # rows split over workgroups
        size = ctypes.c_int64()
        st = L.ssn_logprobs_workspace(args[0], ctypes.byref(size))
        if st == SSN_OK:
            work = torch.empty(size.value, dtype=torch.uint8, device=Z.device)
            st = L.ssn_logprobs(*args, work.data_ptr(), size.value)
    if st != SSN_OK:
        raise SsnError(st, "in ssn_logprobs")
    return out


def ssn_logprobs_grad(Z, labels, forward, dlogp=None, dlse=None, dentropy=None, reference=False, allowed=None, dZ=None):
    """The gradient with respect to Z of sum dlogp * logp + sum dlse * (maxpart + logpart) + sum dentropy * entropy; forward
    is what ssn_logprobs returned for Z, labels, reference and allowed.  dZ: like Z, or Z itself."""
    if _elsewhere(Z):
        with torch.cuda.device(Z.device):
            return ssn_logprobs_grad(Z, labels, forward, dlogp, dlse, dentropy, reference, allowed, dZ)
    dev, stat = Z.get_device(), _STAT[Z.dtype]
    d, n, m = _rows(Z, labels, 0, reference, allowed, dev)
    if dZ is None:
        dZ = torch.empty(Z.shape, dtype=Z.dtype, device=Z.device)
    assert dZ.get_device() == dev and dZ.dtype is Z.dtype and dZ.shape == Z.shape
    st = lib().ssn_logprobs_grad(
        ctypes.byref(d), _data(forward["logp"], stat, n * m, dev) if m else None, _data(forward["maxpart"], stat, n, dev),
        _data(forward["logpart"], stat, n, dev), _data(forward["entropy"], stat, n, dev) if dentropy is not None else None,
        _data(dlogp, stat, n * m, dev), _data(dlse, stat, n, dev), _data(dentropy, stat, n, dev), dZ.data_ptr(), _ld(dZ, *dZ.shape))
    if st != SSN_OK:
        raise SsnError(st, "in ssn_logprobs_grad")
    return dZ


class Q4Block(NamedTuple):
    """A p x K weight block in 4 bits (ssn_q4 of ssn.h): packed uint8, scales bfloat16, both contiguous device tensors."""
    packed: torch.Tensor
    scales: torch.Tensor
    p: int
    K: int
    group: int


def _q4(block, dev):
    packed, scales, p, K, group = block
    tiles = -(-K // 16) * -(-p // 128)
    assert group in (32, 64, 128)
    return ssn_q4(p, K, group, 0, _data(packed, torch.uint8, tiles * 1024, dev), _data(scales, torch.bfloat16, tiles * 2048 // group, dev))


def ssn_q4_quantize(W, group=32):
    """A p x K weight block (any strides, float32 / float64 / float16 / bfloat16; a K x p layer as its transpose) in 4 bits,
    one scale for each class and `group` features."""
    if _elsewhere(W):
        with torch.cuda.device(W.device):
            return ssn_q4_quantize(W, group)
    assert group in (32, 64, 128)
    (p, K), (sj, sc) = W.shape, W.stride()
    tiles, blocks = -(-K // 16), -(-p // 128)
    block = Q4Block(torch.empty((tiles, blocks, 64, 16), dtype=torch.uint8, device=W.device),
                    torch.empty((tiles, blocks, 16, 128 // group), dtype=torch.bfloat16, device=W.device), p, K, group)
    dev = W.get_device()
    d = _q4(block, dev)
    st = lib().ssn_q4_quantize(ctypes.byref(d), _DTYPE[W.dtype], W.data_ptr(), sj if p > 1 else 1, sc if K > 1 else 1,
                               _raw_stream(dev))
    if st != SSN_OK:
        raise SsnError(st, "in ssn_q4_quantize")
    return block


def ssn_q4_margins(block, X, Z=None):
    """Margins X W of n x p rows (float32, float16, bfloat16; rows contiguous) with a block in 4 bits: n x K, of X's type
    unless a float32 Z is given."""
    if _elsewhere(X):
        with torch.cuda.device(X.device):
            return ssn_q4_margins(block, X, Z)
    dev = X.get_device()
    d = _q4(block, dev)
    n, p = X.shape
    assert p == d.p
    if Z is None:
        Z = torch.empty((n, d.K), dtype=X.dtype, device=X.device)
    assert Z.get_device() == dev and Z.shape == (n, d.K)
    dt, st, L = _DTYPE[X.dtype], _raw_stream(dev), lib()
    args = (ctypes.byref(d), dt, n, X.data_ptr(), _ld(X, n, p), _DTYPE[Z.dtype], Z.data_ptr(), _ld(Z, n, d.K))
    status = L.ssn_q4_margins(*args, None, 0, st)
    if status == SSN_E_TOO_LARGE:                   # parts of the features, each with sums of its own
        size = ctypes.c_int64()
        status = L.ssn_q4_margins_workspace(args[0], dt, n, ctypes.byref(size))
        if status == SSN_OK:
            work = torch.empty(size.value, dtype=torch.uint8, device=X.device)
            status = L.ssn_q4_margins(*args, work.data_ptr(), size.value, st)
    if status != SSN_OK:
        raise SsnError(status, "in ssn_q4_margins")
    return Z
