"""Python binding of libpdb (serially-equivalent sparse SGD on one GPU).

Argument marshalling only: every step of the method runs in the CUDA kernels
of ``csrc/`` behind the C ABI declared in ``include/pdb.h``.  The functions
below carry the C names and forward torch tensors' device pointers and the
current CUDA stream.  There is no CPU fallback: if the compiled library is
missing or cannot load, every call raises.
"""
from __future__ import annotations

import ctypes
import glob
import os
import subprocess
import threading
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
_CSRC = os.path.join(_HERE, "csrc")
_INCLUDE = os.path.join(_ROOT, "include")
_LIBDIR = os.path.join(_HERE, "_lib")
LIB_PATH = os.path.join(_LIBDIR, "libpdb.so")
ARCH = "-gencode=arch=compute_103a,code=sm_103a"
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-fmad=false", "-Xcompiler", "-fPIC", ARCH, f"-I{_INCLUDE}"]

PDB_OK, PDB_EINVAL, PDB_ERANGE, PDB_EDUP, PDB_ENOMEM, PDB_ECUDA, PDB_ETIMEOUT, PDB_EFAULT, PDB_ESTATE = \
    0, -1, -2, -3, -4, -5, -6, -7, -8
PDB_ETOOBIG = -9
NOALLOC_MAX_COLS = 1 << 20
PDB_LOSS_LOGISTIC, PDB_LOSS_SQUARED, PDB_LOSS_HINGE = 0, 1, 2
PDB_SCHED_LEVELS, PDB_SCHED_READY, PDB_SCHED_CHAIN, PDB_SCHED_AUTO, PDB_SCHED_WINDOW = 0, 1, 2, 3, 4
PDB_SSP_COUNT, PDB_SSP_PREFIX = 1, 2
PDB_TYPE_FLOAT, PDB_TYPE_BFLOAT, PDB_TYPE_HALF = 0, 1, 2

_lock = threading.Lock()
_lib = None


class PdbError(RuntimeError):
    def __init__(self, code: int, what: str = ""):
        self.code = code
        msg = _strerror(code)
        super().__init__(f"{what}: {msg} ({code})" if what else f"{msg} ({code})")


def _sources():
    return sorted(glob.glob(os.path.join(_CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(_CSRC, "*.cuh")) + [os.path.join(_INCLUDE, "pdb.h")]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile libpdb.so in-tree for sm_103a (nvcc, one object per .cu, in parallel)."""
    with _lock:
        os.makedirs(_LIBDIR, exist_ok=True)
        if (not force and os.path.exists(LIB_PATH)
                and os.path.getmtime(LIB_PATH) >= max(os.path.getmtime(p) for p in _deps())):
            return LIB_PATH
        objs = []

        def compile_one(src):
            obj = os.path.join(_LIBDIR, os.path.basename(src)[:-3] + f".{os.getpid()}.o")
            cmd = ["nvcc", *NVCC_FLAGS, "-c", src, "-o", obj]
            if verbose:
                cmd += ["-Xptxas", "-v"]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed for {src}:\n{r.stderr}")
            if verbose:
                print(r.stderr)
            return obj

        with ThreadPoolExecutor(max_workers=len(_sources())) as ex:
            objs = list(ex.map(compile_one, _sources()))
        tmp = f"{LIB_PATH}.{os.getpid()}.tmp"
        r = subprocess.run(["nvcc", "-shared", ARCH, "-o", tmp, *objs], capture_output=True, text=True)
        for o in objs:
            os.remove(o)
        if r.returncode != 0:
            raise RuntimeError(f"link of libpdb.so failed:\n{r.stderr}")
        os.replace(tmp, LIB_PATH)
        return LIB_PATH


class pdb_csr(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_cols", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("row_ptr", ctypes.c_void_p), ("col", ctypes.c_void_p), ("val", ctypes.c_void_p)]


class pdb_opts(ctypes.Structure):
    """Launch and wait options (zeroed = defaults).  The calls also take a dict of
    the same fields; a torch tensor given as `trace` passes its device pointer."""
    _fields_ = [("blocks_per_sm", ctypes.c_int32), ("ticket_chunk", ctypes.c_int32),
                ("wait_timeout_s", ctypes.c_double), ("trace", ctypes.c_void_p), ("ssp_gates", ctypes.c_int32)]


class pdb_stats(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_cols", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("n_levels", ctypes.c_int64), ("max_level_width", ctypes.c_int64), ("max_chain", ctypes.c_int64),
                ("ms_build", ctypes.c_double), ("ms_schedule", ctypes.c_double), ("ms_sgd", ctypes.c_double),
                ("ms_bsp", ctypes.c_double), ("ms_sgd_kernels", ctypes.c_double), ("sched_mode", ctypes.c_int64)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class pdb_mat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("stride", ctypes.c_int64), ("type", ctypes.c_int32)]


class pdb_ids(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("wide", ctypes.c_int32)]


EXPORTS = ["pdb_build_conflicts", "pdb_conflicts_arrays", "pdb_schedule_build", "pdb_schedule_levels",
           "pdb_schedule_ready",
           "pdb_sgd_epoch", "pdb_bsp_epoch", "pdb_status", "pdb_get_stats", "pdb_conflicts_free",
           "pdb_schedule_free", "pdb_strerror", "pdb_memcpy", "pdb_eval_expf", "pdb_eval_grad", "pdb_launch_count",
           "pdb_sgd_epoch_ready_noalloc", "pdb_ssp_epoch", "pdb_bsp_plan_build", "pdb_bsp_plan_batches",
           "pdb_bsp_coef", "pdb_bsp_apply", "pdb_bsp_plan_free",
           "pdb_tokens_create", "pdb_tokens_free", "pdb_tokens_status",
           "pdb_tokens_set_wait_limit", "pdb_embed", "pdb_embed_grad", "pdb_logprobs",
           "pdb_logprobs_grad", "pdb_distill"]


def load(path: str | None = None):
    """Load libpdb.so (building it first if it is absent or stale); raises if that fails."""
    global _lib
    if _lib is None:
        lib = ctypes.CDLL(path or build())
        P, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        PP = ctypes.POINTER(ctypes.c_void_p)
        lib.pdb_build_conflicts.argtypes = [ctypes.POINTER(pdb_csr), PP, P]
        lib.pdb_conflicts_arrays.argtypes = [P, PP, PP, PP, PP, PP, P]
        lib.pdb_schedule_build.argtypes = [P, I32, PP, P]
        lib.pdb_schedule_levels.argtypes = [P, PP, PP, PP, ctypes.POINTER(I64), P]
        lib.pdb_schedule_ready.argtypes = [P, PP, PP]
        lib.pdb_sgd_epoch.argtypes = [ctypes.POINTER(pdb_csr), P, P, P, P, I32, ctypes.c_float, I32,
                                      ctypes.POINTER(pdb_opts), P]
        lib.pdb_bsp_epoch.argtypes = [ctypes.POINTER(pdb_csr), P, P, P, I32, ctypes.c_float, I64, I32,
                                      ctypes.POINTER(pdb_opts), P]
        lib.pdb_status.argtypes = [P, P]
        lib.pdb_get_stats.argtypes = [P, P, ctypes.POINTER(pdb_stats)]
        lib.pdb_conflicts_free.argtypes = [P]
        lib.pdb_conflicts_free.restype = None
        lib.pdb_schedule_free.argtypes = [P]
        lib.pdb_schedule_free.restype = None
        lib.pdb_strerror.argtypes = [I32]
        lib.pdb_strerror.restype = ctypes.c_char_p
        lib.pdb_memcpy.argtypes = [P, P, ctypes.c_size_t, P]
        lib.pdb_eval_expf.argtypes = [P, P, I64, P]
        lib.pdb_eval_grad.argtypes = [P, P, P, I64, I32, P]
        lib.pdb_sgd_epoch_ready_noalloc.argtypes = [ctypes.POINTER(pdb_csr), P, P, P, I32, ctypes.c_float, I32, P]
        lib.pdb_ssp_epoch.argtypes = [ctypes.POINTER(pdb_csr), P, P, P, P, I32, ctypes.c_float, I32, I64, P,
                                      ctypes.POINTER(pdb_opts), P]
        lib.pdb_bsp_plan_build.argtypes = [P, I64, PP, P]
        lib.pdb_bsp_plan_batches.argtypes = [P]
        lib.pdb_bsp_plan_batches.restype = I64
        lib.pdb_bsp_coef.argtypes = [P, ctypes.POINTER(pdb_csr), P, P, I32, ctypes.c_float, I64, I64, P, P]
        lib.pdb_bsp_apply.argtypes = [P, P, I64, P, P]
        lib.pdb_bsp_plan_free.argtypes = [P]
        lib.pdb_bsp_plan_free.restype = None
        M, J, F32 = ctypes.POINTER(pdb_mat), ctypes.POINTER(pdb_ids), ctypes.c_float
        lib.pdb_tokens_create.argtypes = [I64, I64, PP, P]
        lib.pdb_tokens_free.argtypes = [P]
        lib.pdb_tokens_free.restype = None
        lib.pdb_tokens_status.argtypes = [P, P]
        lib.pdb_tokens_set_wait_limit.argtypes = [P, I64]
        lib.pdb_embed.argtypes = [P, M, J, F32, I64, M, P]
        lib.pdb_embed_grad.argtypes = [P, J, M, F32, I64, I32, M, P]
        lib.pdb_logprobs.argtypes = [P, M, J, F32, I64, P, P, P, I64, P, P, P]
        lib.pdb_logprobs_grad.argtypes = [P, M, J, F32, I64, P, P, P, P, M, P]
        lib.pdb_distill.argtypes = [P, M, J, M, P, F32, P, P, M, P]
        lib.pdb_launch_count.argtypes = []
        lib.pdb_launch_count.restype = I64
        _lib = lib
    return _lib


def _strerror(code: int) -> str:
    try:
        return load().pdb_strerror(int(code)).decode()
    except Exception:  # the library itself failed to load
        return f"error {code}"


def _check(rc: int, what: str):
    if rc != PDB_OK:
        raise PdbError(rc, what)


_raw_stream = None


def _find_raw_stream():
    import torch
    # the current stream's address without the Python object around it (3 us less per call), where torch has it
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    torch.cuda.init()
    device = torch._C._cuda_getDevice
    return lambda: raw(device())


def _stream(stream):
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            _raw_stream = _find_raw_stream()
        return ctypes.c_void_p(_raw_stream())
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


class Csr:
    """CSR examples on the device: int64 row_ptr, int32 col, float32 val (or None)."""

    def __init__(self, row_ptr, col, val, n_cols: int):
        self.row_ptr, self.col, self.val, self.n_cols = row_ptr, col, val, int(n_cols)
        self.struct = pdb_csr(row_ptr.numel() - 1, self.n_cols, col.numel(), _ptr(row_ptr), _ptr(col), _ptr(val))

    @classmethod
    def from_problem(cls, problem, device="cuda"):
        import torch
        row_ptr = torch.from_numpy(problem.row_ptr).to(device)
        col = torch.from_numpy(problem.col).to(device)
        val = None if problem.val is None else torch.from_numpy(problem.val).to(device)
        return cls(row_ptr, col, val, problem.n_cols)


class Conflicts:
    """Owns a pdb_conflicts handle."""

    def __init__(self, handle, n_rows, n_cols, nnz):
        self.handle = handle
        self.n_rows, self.n_cols, self.nnz = n_rows, n_cols, nnz

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pdb_conflicts_free(self.handle)
            self.handle = None


class Schedule:
    """Owns a pdb_schedule handle (keeps its conflicts alive)."""

    def __init__(self, handle, conflicts, mode):
        self.handle, self.conflicts, self.mode = handle, conflicts, mode

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pdb_schedule_free(self.handle)
            self.handle = None


def pdb_build_conflicts(X: Csr, stream=None) -> Conflicts:
    """Validate X and build its per-feature occurrence chains (Definitions 1-3,
    Section 5); errors the device finds surface through pdb_status."""
    h = ctypes.c_void_p()
    _check(load().pdb_build_conflicts(ctypes.byref(X.struct), ctypes.byref(h), _stream(stream)),
           "pdb_build_conflicts")
    return Conflicts(h, X.struct.n_rows, X.struct.n_cols, X.struct.nnz)


def pdb_conflicts_arrays(c: Conflicts, stream=None) -> dict:
    """Borrowed device pointers (ints) of csc_pos, feat_ptr, prev, next, rank."""
    ptrs = [ctypes.c_void_p() for _ in range(5)]
    _check(load().pdb_conflicts_arrays(c.handle, *[ctypes.byref(p) for p in ptrs], _stream(stream)),
           "pdb_conflicts_arrays")
    return dict(zip(["csc_pos", "feat_ptr", "prev", "next", "rank"], [p.value for p in ptrs]))


def pdb_schedule_build(c: Conflicts, mode: int, stream=None) -> Schedule:
    """Schedule for pdb_sgd_epoch: PDB_SCHED_LEVELS (Theorem 3), READY, WINDOW,
    CHAIN or AUTO (include/pdb.h describes each)."""
    h = ctypes.c_void_p()
    _check(load().pdb_schedule_build(c.handle, int(mode), ctypes.byref(h), _stream(stream)), "pdb_schedule_build")
    return Schedule(h, c, mode)


def pdb_schedule_levels(s: Schedule, stream=None) -> dict:
    """Borrowed device pointers (ints) of a LEVELS schedule's level, order and
    level_ptr arrays, and its number of levels (waits for the schedule)."""
    ptrs = [ctypes.c_void_p() for _ in range(3)]
    L = ctypes.c_int64()
    _check(load().pdb_schedule_levels(s.handle, *[ctypes.byref(p) for p in ptrs], ctypes.byref(L), _stream(stream)),
           "pdb_schedule_levels")
    return dict(level=ptrs[0].value, order=ptrs[1].value, level_ptr=ptrs[2].value, n_levels=L.value)


def pdb_schedule_ready(s: Schedule) -> dict:
    """Borrowed device pointers (ints) of the READY schedule's gate and records arrays."""
    ptrs = [ctypes.c_void_p() for _ in range(2)]
    _check(load().pdb_schedule_ready(s.handle, *[ctypes.byref(p) for p in ptrs]), "pdb_schedule_ready")
    return dict(gate=ptrs[0].value, records=ptrs[1].value)


def _opts(opts):
    if opts is None:
        return None
    if isinstance(opts, pdb_opts):
        return ctypes.byref(opts)
    kw = dict(opts)
    if kw.get("trace") is not None and not isinstance(kw["trace"], int):
        kw["trace"] = kw["trace"].data_ptr()     # a torch uint64/int64 tensor on the device
    return ctypes.byref(pdb_opts(**kw))


def pdb_sgd_epoch(X: Csr, y, c: Conflicts, s: Schedule, w, loss: int, eta: float, n_epochs: int, opts=None,
                  stream=None):
    """n_epochs of SGD over X in data order, serially equivalent (Algorithm 1,
    Theorem 2): w (float32, n_cols, on the device) is updated in place."""
    _check(load().pdb_sgd_epoch(ctypes.byref(X.struct), _ptr(y), c.handle, s.handle, _ptr(w), int(loss), float(eta),
                                int(n_epochs), _opts(opts), _stream(stream)), "pdb_sgd_epoch")


def pdb_ssp_epoch(X: Csr, y, c: Conflicts, s: Schedule, w, loss: int, eta: float, n_epochs: int, delay: int,
                  coef=None, opts=None, stream=None):
    """SGD with admissible delay (Section 7) under a READY schedule; opts may set
    ssp_gates to PDB_SSP_COUNT (default) or PDB_SSP_PREFIX.  delay = 0 is
    pdb_sgd_epoch's result bit for bit."""
    _check(load().pdb_ssp_epoch(ctypes.byref(X.struct), _ptr(y), c.handle, s.handle, _ptr(w), int(loss), float(eta),
                                int(n_epochs), int(delay), _ptr(coef), _opts(opts), _stream(stream)),
           "pdb_ssp_epoch")


def pdb_bsp_epoch(X: Csr, y, c: Conflicts, w, loss: int, eta: float, batch: int, n_epochs: int, opts=None,
                  stream=None):
    """The BSP comparison (Algorithm 2a): `batch` examples between barriers,
    margins at the batch-start weights, ordered per-feature sums."""
    _check(load().pdb_bsp_epoch(ctypes.byref(X.struct), _ptr(y), c.handle, _ptr(w), int(loss), float(eta),
                                int(batch), int(n_epochs), _opts(opts), _stream(stream)), "pdb_bsp_epoch")


class BspPlan:
    """Owns a pdb_bsp_plan handle (keeps its conflicts alive)."""

    def __init__(self, handle, conflicts, batch):
        self.handle, self.conflicts, self.batch = handle, conflicts, int(batch)
        self.n_batches = int(load().pdb_bsp_plan_batches(handle))

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pdb_bsp_plan_free(self.handle)
            self.handle = None


def pdb_bsp_plan_build(c: Conflicts, batch: int, stream=None) -> BspPlan:
    """The (batch, feature, example) order of c's pairs for the data-parallel
    BSP split of Algorithm 2a (synchronizes)."""
    h = ctypes.c_void_p()
    _check(load().pdb_bsp_plan_build(c.handle, int(batch), ctypes.byref(h), _stream(stream)), "pdb_bsp_plan_build")
    return BspPlan(h, c, min(int(batch), max(1, c.n_rows)) if c.n_rows > 0 else int(batch))


def pdb_bsp_coef(plan: BspPlan, X: Csr, y, w, loss: int, eta: float, row_begin: int, row_end: int, coef,
                 stream=None):
    """coef[i - row_begin] = eta * dloss/dm of rows [row_begin, row_end) at w
    (the rows lie inside one batch)."""
    _check(load().pdb_bsp_coef(plan.handle, ctypes.byref(X.struct), _ptr(y), _ptr(w), int(loss), float(eta),
                               int(row_begin), int(row_end), _ptr(coef), _stream(stream)), "pdb_bsp_coef")


def pdb_bsp_apply(plan: BspPlan, w, batch_index: int, coef, stream=None):
    """The write half of batch `batch_index` from all of its coefficients."""
    _check(load().pdb_bsp_apply(plan.handle, _ptr(w), int(batch_index), _ptr(coef), _stream(stream)),
           "pdb_bsp_apply")


def rank_rows(r0: int, r1: int, rank: int, world: int) -> tuple[int, int]:
    """The contiguous share of rows [r0, r1) that rank `rank` of `world` computes
    (the first (r1 - r0) % world ranks take one row more)."""
    n = r1 - r0
    q, extra = divmod(n, world)
    lo = r0 + rank * q + min(rank, extra)
    return lo, lo + q + (1 if rank < extra else 0)


def bsp_epoch_data_parallel(X: Csr, y, c: Conflicts, w, loss: int, eta: float, batch: int, n_epochs: int,
                            group=None, plan: BspPlan | None = None, ops=None, stream=None):
    """Algorithm 2a over the ranks of a torch.distributed group, each holding
    the whole data and a replica of w: per batch every rank computes the
    coefficients of its share of the rows (pdb_bsp_coef), the shares are
    all-gathered in rank order (= row order), and every rank applies the
    batch (pdb_bsp_apply).  Without an initialized process group it runs on
    one rank.  The result equals pdb_bsp_epoch's bit for bit.

    `ops` replaces the three library calls (coef, apply, all_gather) with
    callables of the same meaning; the CPU tests use it to check the
    partitioning without a GPU."""
    import torch
    import torch.distributed as dist
    world = dist.get_world_size(group) if dist.is_available() and dist.is_initialized() else 1
    rank = dist.get_rank(group) if world > 1 else 0
    if ops is None:
        plan = plan or pdb_bsp_plan_build(c, batch, stream)
        n_batches, B = plan.n_batches, plan.batch

        def coef_fn(r0, r1, out):
            pdb_bsp_coef(plan, X, y, w, loss, eta, r0, r1, out, stream)

        def apply_fn(b, coef):
            pdb_bsp_apply(plan, w, b, coef, stream)

        def gather_fn(parts, mine):
            if world == 1:
                return
            if dist.get_backend(group) == "nccl":
                dist.all_gather(parts, mine, group=group)
            else:                              # gloo: host tensors
                host = [torch.empty(p.numel(), dtype=p.dtype) for p in parts]
                dist.all_gather(host, mine.cpu(), group=group)
                for p, h in zip(parts, host):
                    p.copy_(h)
        device = w.device
    else:
        coef_fn, apply_fn, gather_fn = ops["coef"], ops["apply"], ops["gather"]
        n_batches, B = ops["n_batches"], ops["batch"]
        device = ops.get("device", "cpu")
    n_rows = X.struct.n_rows if hasattr(X, "struct") else ops["n_rows"]
    coef = torch.empty(max(B, 1), dtype=torch.float32, device=device)
    for _ in range(n_epochs):
        for b in range(n_batches):
            r0, r1 = b * B, min(n_rows, (b + 1) * B)
            bounds = [rank_rows(r0, r1, r, world) for r in range(world)]
            # one slice per rank, padded to the longest so that every all_gather part has one size
            width = max(hi - lo for lo, hi in bounds)
            if world == 1:
                coef_fn(r0, r1, coef[: r1 - r0])
                apply_fn(b, coef[: r1 - r0])
                continue
            parts = [torch.zeros(width, dtype=torch.float32, device=device) for _ in range(world)]
            lo, hi = bounds[rank]
            coef_fn(lo, hi, parts[rank][: hi - lo])
            gather_fn(parts, parts[rank])
            for r, (l2, h2) in enumerate(bounds):
                coef[l2 - r0: h2 - r0].copy_(parts[r][: h2 - l2])
            apply_fn(b, coef[: r1 - r0])


def pdb_sgd_epoch_ready_noalloc(X: Csr, y, gate_ptr: int, w, loss: int, eta: float, n_epochs: int,
                                stream=None) -> int:
    """READY-schedule SGD epochs that allocate no device memory (scratch is a
    fixed array inside the library, up to NOALLOC_MAX_COLS features).  For
    callers that cannot let a library allocate while they train, e.g. a
    server whose own memory pool owns the whole device.  Synchronizes the
    stream and returns the status code (PDB_OK on success)."""
    return int(load().pdb_sgd_epoch_ready_noalloc(ctypes.byref(X.struct), _ptr(y), ctypes.c_void_p(gate_ptr), _ptr(w),
                                                  int(loss), float(eta), int(n_epochs), _stream(stream)))


def pdb_status(c: Conflicts, stream=None) -> int:
    """Synchronize the stream and return the first error a kernel recorded in c
    (PDB_OK when none)."""
    return int(load().pdb_status(c.handle, _stream(stream)))


def pdb_get_stats(c: Conflicts, s: Schedule | None = None) -> dict:
    """Sizes, level counts and CUDA-event timings of the last calls on c (and s)
    as a dict; synchronizes the device."""
    st = pdb_stats()
    _check(load().pdb_get_stats(c.handle, None if s is None else s.handle, ctypes.byref(st)), "pdb_get_stats")
    return st.as_dict()


def pdb_memcpy(dst_ptr: int, src_ptr: int, nbytes: int, stream=None):
    """Stream-ordered copy between device or host pointers (ints)."""
    _check(load().pdb_memcpy(ctypes.c_void_p(dst_ptr), ctypes.c_void_p(src_ptr), int(nbytes), _stream(stream)),
           "pdb_memcpy")


def pdb_eval_grad(m, y, out, loss: int, stream=None):
    """out = the library's device loss derivative at margins m and labels y
    (float32 device tensors of one length)."""
    _check(load().pdb_eval_grad(_ptr(m), _ptr(y), _ptr(out), m.numel(), int(loss), _stream(stream)), "pdb_eval_grad")


def pdb_eval_expf(x, out, stream=None):
    """out = the library's device exponential of x (float32 tensors), for tests."""
    _check(load().pdb_eval_expf(_ptr(x), _ptr(out), x.numel(), _stream(stream)), "pdb_eval_expf")


class Tokens:
    """Owns a pdb_tokens handle: workspace and status word of the token operators."""

    def __init__(self, handle, device):
        self.handle, self.device = handle, device

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pdb_tokens_free(self.handle)
            self.handle = None


class _Types(dict):
    """Matrix types and id widths by torch dtype, filled when torch is first needed (this module does not import it)."""

    def __missing__(self, dtype):
        if not self:
            import torch
            self.update({torch.float32: PDB_TYPE_FLOAT, torch.bfloat16: PDB_TYPE_BFLOAT, torch.float16: PDB_TYPE_HALF,
                         torch.int32: "int32", torch.int64: "int64"})
        return self.get(dtype)


_types = _Types()


def _refuse(what, why):
    raise PdbError(PDB_EINVAL, f"{what}: {why}")


def _mat(t, tok, what):
    """A pdb_mat of a 2-D device tensor whose rows are contiguous."""
    kind = _types[t.dtype]
    if kind.__class__ is not int:
        _refuse(what, f"float32, bfloat16 or float16 wanted, got {t.dtype}")
    stride = t.stride()
    if len(stride) != 2 or t.get_device() != tok.device:
        _refuse(what, f"a matrix on cuda:{tok.device} wanted, got {tuple(t.shape)} on {t.device}")
    rows, cols = t.shape
    if (stride[1] != 1 and cols > 1) or (stride[0] < cols and rows > 1):
        _refuse(what, f"rows of neighbouring elements that do not overlap wanted, got strides {stride}")
    return pdb_mat(t.data_ptr(), rows, cols, stride[0], kind)


def _ids(t, tok, what):
    """A pdb_ids of a vector of ids."""
    kind = _types[t.dtype]
    if kind.__class__ is not str:
        _refuse(what, f"int32 or int64 wanted, got {t.dtype}")
    stride = t.stride()
    if len(stride) != 1 or t.get_device() != tok.device:
        _refuse(what, f"a vector on cuda:{tok.device} wanted, got {tuple(t.shape)} on {t.device}")
    return pdb_ids(t.data_ptr(), t.numel(), stride[0], kind == "int64")


def _rows_of_ids(t, tok, what):
    """A pdb_ids of a matrix of ids whose rows are contiguous."""
    kind = _types[t.dtype]
    if kind.__class__ is not str:
        _refuse(what, f"int32 or int64 wanted, got {t.dtype}")
    stride = t.stride()
    if len(stride) != 2 or t.get_device() != tok.device:
        _refuse(what, f"a matrix on cuda:{tok.device} wanted, got {tuple(t.shape)} on {t.device}")
    if stride[1] != 1 and t.shape[1] > 1:
        _refuse(what, f"rows of neighbouring elements wanted, got strides {stride}")
    return pdb_ids(t.data_ptr(), t.numel(), stride[0], kind == "int64")


def _vec(t, n, tok, what, kind=PDB_TYPE_FLOAT):
    """The pointer of n contiguous device words (None stays None)."""
    if t is None:
        return None
    if _types[t.dtype] != kind or t.get_device() != tok.device or t.numel() != n or not t.is_contiguous():
        _refuse(what, f"{n} contiguous {'int32' if kind == 'int32' else 'float32'} on cuda:{tok.device} wanted, "
                      f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def pdb_tokens_create(max_tokens: int = 0, max_dim: int = 0, stream=None) -> Tokens:
    """Workspace and status word of the token operators, for pdb_embed_grad
    calls of at most max_tokens ids and max_dim columns (the other calls need neither)."""
    import torch
    h = ctypes.c_void_p()
    _check(load().pdb_tokens_create(int(max_tokens), int(max_dim), ctypes.byref(h), _stream(stream)),
           "pdb_tokens_create")
    return Tokens(h, torch.cuda.current_device())


def pdb_tokens_status(tok: Tokens, stream=None) -> int:
    """Synchronize the stream and return the first error a kernel recorded in tok
    (PDB_ERANGE: an id out of range; PDB_OK when none)."""
    return int(load().pdb_tokens_status(tok.handle, _stream(stream)))


def pdb_tokens_set_wait_limit(tok: Tokens, tries: int):
    """Tries of a device-side wait in later calls on tok (0: none, every such call ends with PDB_ETIMEOUT)."""
    _check(load().pdb_tokens_set_wait_limit(tok.handle, tries), "pdb_tokens_set_wait_limit")


def pdb_embed(tok: Tokens, table, ids, out, scale: float = 1.0, pad: int = -1, stream=None):
    """out[i] = scale * table[ids[i]] (Definition 3's reads); rows of zeros for ids equal to pad.
    table (vocab, dim) and out (n, dim) in float32, bfloat16 or float16, each its own; ids n int32 or int64."""
    _check(load().pdb_embed(tok.handle, _mat(table, tok, "pdb_embed table"), _ids(ids, tok, "pdb_embed ids"), scale,
                            pad, _mat(out, tok, "pdb_embed out"), _stream(stream)), "pdb_embed")


def pdb_embed_grad(tok: Tokens, ids, dout, dtable, scale: float = 1.0, pad: int = -1, accumulate: bool = False,
                   stream=None):
    """dtable[v] = scale * sum of dout[i] over ids[i] = v, in an order fixed by their number (pieces of 32 in data
    order, the pieces as the header says); every row is written.  accumulate=True adds to the rows that occur and leaves the others: with the table for
    dtable and scale = -eta * scale, the SGD step in place."""
    _check(load().pdb_embed_grad(tok.handle, _ids(ids, tok, "pdb_embed_grad ids"),
                                 _mat(dout, tok, "pdb_embed_grad dout"), scale, pad, accumulate,
                                 _mat(dtable, tok, "pdb_embed_grad dtable"), _stream(stream)), "pdb_embed_grad")


def pdb_logprobs(tok: Tokens, logits, ids=None, logp=None, lse=None, entropy=None, top_logp=None, top_ids=None,
                 scale: float = 1.0, ignore: int = -100, stream=None):
    """Per row of logits (times scale, the inverse temperature): logp of the token ids[r], log-sum-exp, entropy,
    and the top_logp.shape[1] most probable tokens, each where its output tensor (float32; top_ids int32) is given."""
    z = _mat(logits, tok, "pdb_logprobs logits")
    n, k = z.rows, 0
    top = top_ids if top_logp is None else top_logp
    if top is not None:
        if top.dim() != 2:
            _refuse("pdb_logprobs top", f"(rows, k) wanted, got {tuple(top.shape)}")
        k = top.shape[1]
    if (ids is None) != (logp is None):
        _refuse("pdb_logprobs", "ids and logp go together")
    _check(load().pdb_logprobs(
        tok.handle, z, None if ids is None else _ids(ids, tok, "pdb_logprobs ids"), scale, ignore,
        _vec(logp, n, tok, "pdb_logprobs logp"), _vec(lse, n, tok, "pdb_logprobs lse"),
        _vec(entropy, n, tok, "pdb_logprobs entropy"), k, _vec(top_logp, n * k, tok, "pdb_logprobs top_logp"),
        _vec(top_ids, n * k, tok, "pdb_logprobs top_ids", "int32"), _stream(stream)), "pdb_logprobs")


def pdb_logprobs_grad(tok: Tokens, logits, ids, lse, entropy, dlogp, dentropy, dlogits, scale: float = 1.0,
                      ignore: int = -100, stream=None):
    """dlogits = the gradient of sum(dlogp * logp + dentropy * entropy), with lse and entropy as pdb_logprobs gave
    them.  dlogp (with ids) or dentropy (with entropy) may be None; dlogits may be logits itself."""
    z = _mat(logits, tok, "pdb_logprobs_grad logits")
    n = z.rows
    _check(load().pdb_logprobs_grad(
        tok.handle, z, None if ids is None else _ids(ids, tok, "pdb_logprobs_grad ids"), scale, ignore,
        _vec(lse, n, tok, "pdb_logprobs_grad lse"), _vec(entropy, n, tok, "pdb_logprobs_grad entropy"),
        _vec(dlogp, n, tok, "pdb_logprobs_grad dlogp"), _vec(dentropy, n, tok, "pdb_logprobs_grad dentropy"),
        _mat(dlogits, tok, "pdb_logprobs_grad dlogits"), _stream(stream)), "pdb_logprobs_grad")


def pdb_distill(tok: Tokens, logits, top_ids, top_logits, loss=None, teacher_lse=None, weight=None, dlogits=None,
                temperature: float = 1.0, stream=None):
    """Loss per row of the student's logits against a teacher's top_logits (rows, K) at the tokens top_ids (a
    negative id: an empty slot), and, where dlogits is given, the gradient of sum(weight * loss).  With
    teacher_lse (log-sum-exp of all the teacher's logits / temperature) the rest of the teacher's
    probability stands in one bucket; else its slots are renormalised.  dlogits may be logits itself."""
    z = _mat(logits, tok, "pdb_distill logits")
    n = z.rows
    t = _mat(top_logits, tok, "pdb_distill top_logits")
    if top_ids.shape != top_logits.shape:
        _refuse("pdb_distill", f"top_ids {tuple(top_ids.shape)} and top_logits {tuple(top_logits.shape)} differ in shape")
    _check(load().pdb_distill(
        tok.handle, z, _rows_of_ids(top_ids, tok, "pdb_distill top_ids"), t,
        _vec(teacher_lse, n, tok, "pdb_distill teacher_lse"), temperature, _vec(loss, n, tok, "pdb_distill loss"),
        _vec(weight, n, tok, "pdb_distill weight"),
        None if dlogits is None else _mat(dlogits, tok, "pdb_distill dlogits"), _stream(stream)), "pdb_distill")


def check_tokens(tok: Tokens, stream=None):
    """Synchronize and raise PdbError if a kernel recorded an error in tok."""
    rc = pdb_tokens_status(tok, stream)
    if rc != PDB_OK:
        raise PdbError(rc, "device status")


def pdb_launch_count() -> int:
    """Kernels this process has launched through the library so far."""
    return int(load().pdb_launch_count())


def pdb_strerror(code: int) -> str:
    return _strerror(code)


def device_array(ptr: int, n: int, dtype, stream=None):
    """Copy n elements of a borrowed device array into a new torch tensor."""
    import torch
    out = torch.empty(n, dtype=dtype, device="cuda")
    if n:
        pdb_memcpy(out.data_ptr(), ptr, n * out.element_size(), stream)
    return out


def check_status(c: Conflicts, stream=None):
    """Synchronize and raise PdbError if a kernel recorded an error in c."""
    rc = pdb_status(c, stream)
    if rc != PDB_OK:
        raise PdbError(rc, "device status")
