"""Python binding of the esspt C-ABI (argument marshalling only).

Every method maps to one `esspt_*` entry point of include/esspt.h.  PyTorch
provides device memory (the workspaces are torch tensors) and the CUDA
stream; every computation runs in the library's CUDA kernels.  There is no
CPU fallback: if the library or a GPU is missing, construction fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libesspt.so")

OK, EINVAL, ESTATE, ENOSPC, ESTALE, ECUDA = range(6)
STATUS_NAMES = {OK: "OK", EINVAL: "EINVAL", ESTATE: "ESTATE", ENOSPC: "ENOSPC", ESTALE: "ESTALE", ECUDA: "ECUDA"}
MODELS = {"ssp": 0, "essp": 1, "external": 2, "vap": 3, "ssp_row": 4}

# Every entry point declared in include/esspt.h.
EXPORTS = (
    "esspt_workspace_bytes", "esspt_create", "esspt_destroy", "esspt_table_init", "esspt_get", "esspt_inc",
    "esspt_clock", "esspt_set_schedule", "esspt_poll", "esspt_read_schedule", "esspt_read_table",
    "esspt_last_error", "esspt_mf_workspace_bytes", "esspt_mf_scratch_bytes", "esspt_mf_load",
    "esspt_mf_sgd_clock", "esspt_mf_objective", "esspt_mf_minibatch_size", "esspt_mf_export_minibatch",
    "esspt_mf_stage_minibatch", "esspt_mf_stage_bytes", "esspt_set_profile_events",
    "esspt_mf_worker_objective_noalloc",
    "esspt_mf_sequential_work_bytes", "esspt_mf_sgd_clock_sequential",
    "esspt_softmax_workspace_bytes", "esspt_softmax_create", "esspt_softmax_destroy", "esspt_softmax_loss",
    "esspt_softmax_distill", "esspt_softmax_poll", "esspt_softmax_last_error",
    "esspt_embed_workspace_bytes", "esspt_embed_create", "esspt_embed_destroy", "esspt_embed_lookup",
    "esspt_embed_gradient", "esspt_embed_poll", "esspt_embed_last_error",
    "esspt_norm_workspace_bytes", "esspt_norm_create", "esspt_norm_destroy", "esspt_norm_forward",
    "esspt_norm_backward", "esspt_norm_last_error",
    "esspt_adamw_moment_values", "esspt_adamw_workspace_bytes", "esspt_adamw_create", "esspt_adamw_destroy",
    "esspt_adamw_step", "esspt_adamw_moments", "esspt_adamw_load", "esspt_adamw_steps", "esspt_adamw_last_error",
)


class EssptError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class Config(ctypes.Structure):
    _fields_ = [
        ("n_rows", ctypes.c_int64),
        ("row_width", ctypes.c_int32),
        ("num_workers", ctypes.c_int32),
        ("staleness", ctypes.c_int32),
        ("model", ctypes.c_int32),
        ("phased", ctypes.c_int32),
        ("essp_max_delay", ctypes.c_int32),
        ("essp_p", ctypes.c_double),
        ("seed", ctypes.c_uint64),
        ("stream", ctypes.c_void_p),
        ("vap_v0", ctypes.c_double),
    ]


class SoftmaxConfig(ctypes.Structure):
    _fields_ = [
        ("max_rows", ctypes.c_int64),
        ("n_items", ctypes.c_int64),
        ("width", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("max_top", ctypes.c_int32),
        ("backward", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
    ]


class EmbedConfig(ctypes.Structure):
    _fields_ = [
        ("max_tokens", ctypes.c_int64),
        ("n_rows", ctypes.c_int64),
        ("width", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("backward", ctypes.c_int32),
        ("stream", ctypes.c_void_p),
    ]


class NormConfig(ctypes.Structure):
    _fields_ = [
        ("max_rows", ctypes.c_int64),
        ("width", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32),
        ("backward", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("stream", ctypes.c_void_p),
    ]


class AdamWTensor(ctypes.Structure):
    _fields_ = [
        ("d_param", ctypes.c_void_p),
        ("d_copy", ctypes.c_void_p),
        ("count", ctypes.c_int64),
        ("weight_decay", ctypes.c_float),
    ]


class AdamWConfig(ctypes.Structure):
    _fields_ = [
        ("n_tensors", ctypes.c_int32),
        ("state_bits", ctypes.c_int32),
        ("copy_dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("seed", ctypes.c_uint64),
        ("stream", ctypes.c_void_p),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libesspt.so (built by `build()`); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"esspt CUDA library not built: {LIB_PATH} is missing (run __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    sig = {
        "esspt_workspace_bytes": (SZ, [P]),
        "esspt_create": (ctypes.c_int, [P, P, SZ, P]),
        "esspt_destroy": (ctypes.c_int, [P]),
        "esspt_table_init": (ctypes.c_int, [P, P]),
        "esspt_get": (ctypes.c_int, [P, I32, P, I64, P, P]),
        "esspt_inc": (ctypes.c_int, [P, I32, P, P, I64]),
        "esspt_clock": (ctypes.c_int, [P]),
        "esspt_set_schedule": (ctypes.c_int, [P, P]),
        "esspt_poll": (ctypes.c_int, [P]),
        "esspt_read_schedule": (ctypes.c_int, [P, P, P]),
        "esspt_read_table": (ctypes.c_int, [P, I32, P]),
        "esspt_last_error": (ctypes.c_char_p, [P]),
        "esspt_mf_workspace_bytes": (SZ, [P, I64, I64, I32]),
        "esspt_mf_scratch_bytes": (SZ, [P, I64, I64, I32]),
        "esspt_mf_load": (ctypes.c_int, [P, P, P, P, P, I64, P, I64, I32, P, SZ, P, SZ]),
        "esspt_mf_sgd_clock": (ctypes.c_int, [P, ctypes.c_float, ctypes.c_float, I32, P]),
        "esspt_mf_sequential_work_bytes": (SZ, [P]),
        "esspt_mf_sgd_clock_sequential": (ctypes.c_int, [P, ctypes.c_float, ctypes.c_float, I32, P, P, SZ]),
        "esspt_mf_objective": (ctypes.c_int, [P, I32, ctypes.c_float, P, P, P]),
        "esspt_mf_minibatch_size": (ctypes.c_int, [P, I32, P]),
        "esspt_mf_export_minibatch": (ctypes.c_int, [P, I32, P, P, P, P]),
        "esspt_mf_stage_bytes": (SZ, [P]),
        "esspt_mf_stage_minibatch": (ctypes.c_int, [P, I32, P, P, P, P, P, SZ, P]),
        "esspt_set_profile_events": (ctypes.c_int, [P, P, P]),
        "esspt_mf_worker_objective_noalloc": (ctypes.c_int, [P, I32, ctypes.c_float, P, P]),
        "esspt_softmax_workspace_bytes": (SZ, [P]),
        "esspt_softmax_create": (ctypes.c_int, [P, P, SZ, P]),
        "esspt_softmax_destroy": (ctypes.c_int, [P]),
        "esspt_softmax_loss": (ctypes.c_int, [P, P, I64, P, I64, P, I64, P, ctypes.c_float, P, P, P, P]),
        "esspt_softmax_distill": (ctypes.c_int, [P, P, I64, P, I64, P, P, I32, I64, P, ctypes.c_float, P, P, P, P]),
        "esspt_softmax_poll": (ctypes.c_int, [P]),
        "esspt_softmax_last_error": (ctypes.c_char_p, [P]),
        "esspt_embed_workspace_bytes": (SZ, [P]),
        "esspt_embed_create": (ctypes.c_int, [P, P, SZ, P]),
        "esspt_embed_destroy": (ctypes.c_int, [P]),
        "esspt_embed_lookup": (ctypes.c_int, [P, P, I64, P, I64, ctypes.c_float, P]),
        "esspt_embed_gradient": (ctypes.c_int, [P, P, P, I64, I64, ctypes.c_float, I32, P]),
        "esspt_embed_poll": (ctypes.c_int, [P]),
        "esspt_embed_last_error": (ctypes.c_char_p, [P]),
        "esspt_norm_workspace_bytes": (SZ, [P]),
        "esspt_norm_create": (ctypes.c_int, [P, P, SZ, P]),
        "esspt_norm_destroy": (ctypes.c_int, [P]),
        "esspt_norm_forward": (ctypes.c_int, [P, P, I64, I64, P, P, P, P, P]),
        "esspt_norm_backward": (ctypes.c_int, [P, P, I64, P, I64, I64, P, P, P, P, P, P]),
        "esspt_norm_last_error": (ctypes.c_char_p, [P]),
        "esspt_adamw_moment_values": (I64, [P, P]),
        "esspt_adamw_workspace_bytes": (SZ, [P, P]),
        "esspt_adamw_create": (ctypes.c_int, [P, P, P, SZ, P]),
        "esspt_adamw_destroy": (ctypes.c_int, [P]),
        "esspt_adamw_step": (ctypes.c_int, [P, P, ctypes.c_float, P, P]),
        "esspt_adamw_moments": (ctypes.c_int, [P, P, P]),
        "esspt_adamw_load": (ctypes.c_int, [P, P, P, I64]),
        "esspt_adamw_steps": (ctypes.c_int, [P, P]),
        "esspt_adamw_last_error": (ctypes.c_char_p, [P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return int(t)


def _dev_tensor(x, dtype, device) -> torch.Tensor:
    if isinstance(x, torch.Tensor):
        return x.to(device=device, dtype=dtype).contiguous()
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype, device=device)


class Table:
    """A stale-synchronous parameter table on one GPU (one `esspt_ctx`)."""

    def __init__(self, n_rows: int, K: int, P: int, s: int, model: str = "ssp", phased: bool = True,
                 seed: int = 8043, essp_p: float = 0.7, essp_max_delay: int = 3, vap_v0: float = 0.0,
                 device=None, stream=None):
        if not torch.cuda.is_available():
            raise RuntimeError("esspt needs a CUDA device")
        L = self._lib = lib()
        self.device = torch.device(device if device is not None else "cuda")
        # as the tensors on it name it
        self._on = self.device if self.device.index is not None else torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.cfg = Config(n_rows, K, P, s, MODELS[model], int(phased), essp_max_delay, essp_p,
                          seed & 0xFFFFFFFFFFFFFFFF, ctypes.c_void_p(self.stream.cuda_stream), vap_v0)
        self.n_rows, self.K, self.P, self.s, self.model = n_rows, K, P, s, model
        nbytes = L.esspt_workspace_bytes(ctypes.byref(self.cfg))
        if nbytes == 0:
            raise EssptError(EINVAL, "invalid table configuration")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        st = L.esspt_create(ctypes.byref(self.cfg), self.workspace.data_ptr(), nbytes, ctypes.byref(h))
        if st != OK:
            raise EssptError(st, L.esspt_last_error(None).decode())
        self._h = h
        self.mf_workspace = None
        self.n_users = None

    # -- plumbing -----------------------------------------------------------
    def _dev(self, x, dtype) -> torch.Tensor:
        if isinstance(x, torch.Tensor) and x.dtype is dtype and x.device == self._on and x.is_contiguous():
            return x  # the usual call: nothing to convert
        return _dev_tensor(x, dtype, self.device)

    def _check(self, st: int) -> None:
        if st != OK:
            raise EssptError(st, lib().esspt_last_error(self._h).decode())

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().esspt_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- table API ----------------------------------------------------------
    def table_init(self, rows) -> None:
        """esspt_table_init: version 0 from (n_rows, K) fp32 values."""
        t = _dev_tensor(rows, torch.float32, self.device)
        assert t.numel() == self.n_rows * self.K
        self._check(lib().esspt_table_init(self._h, t.data_ptr()))
        self._keep = t

    def get(self, worker: int, row_ids, out=None, want_version: bool = False):
        """esspt_get: rows of `worker`'s read version; returns (rows, version or None)."""
        ids = self._dev(row_ids, torch.int32)
        if out is None:
            out = torch.empty((ids.numel(), self.K), dtype=torch.float32, device=self.device)
        self._keep_ids = ids
        if not want_version:
            st = self._lib.esspt_get(self._h, worker, ids.data_ptr(), ids.numel(), out.data_ptr(), None)
            if st != OK:
                self._check(st)
            return out, None
        ver = ctypes.c_int32(-1)
        self._check(self._lib.esspt_get(self._h, worker, ids.data_ptr(), ids.numel(), out.data_ptr(),
                                        ctypes.byref(ver)))
        return out, ver.value

    def inc(self, worker: int, row_ids, deltas) -> None:
        """esspt_inc: additive updates into the version being written."""
        ids = self._dev(row_ids, torch.int32)
        d = self._dev(deltas, torch.float32)
        n = ids.numel()
        assert d.numel() == n * self.K
        self._keep_inc = (ids, d)
        st = self._lib.esspt_inc(self._h, worker, ids.data_ptr(), d.data_ptr(), n)
        if st != OK:
            self._check(st)

    def clock(self) -> None:
        """esspt_clock: all workers tick."""
        self._check(lib().esspt_clock(self._h))

    def set_schedule(self, v) -> None:
        """esspt_set_schedule (external model)."""
        a = np.ascontiguousarray(v, dtype=np.int32)
        assert a.shape == (self.P,)
        self._check(lib().esspt_set_schedule(self._h, a.ctypes.data))

    def poll(self) -> None:
        """esspt_poll: synchronise and raise on a latched device error."""
        self._check(lib().esspt_poll(self._h))

    def read_schedule(self):
        """esspt_read_schedule: (v_p(c) as int32[P], c)."""
        v = np.empty(self.P, dtype=np.int32)
        c = ctypes.c_int32()
        self._check(lib().esspt_read_schedule(self._h, v.ctypes.data, ctypes.byref(c)))
        return v, c.value

    @property
    def clock_index(self) -> int:
        c = ctypes.c_int32()
        self._check(lib().esspt_read_schedule(self._h, None, ctypes.byref(c)))
        return c.value

    def read_table(self, version: int, out=None) -> torch.Tensor:
        """esspt_read_table: a final version still in the ring."""
        if out is None:
            out = torch.empty((self.n_rows, self.K), dtype=torch.float32, device=self.device)
        self._check(lib().esspt_read_table(self._h, version, out.data_ptr()))
        return out

    # -- matrix factorisation -----------------------------------------------
    def mf_load(self, i, j, D, minibatch, worker, n_users: int, F: int) -> None:
        """esspt_mf_load: observed entries and their worker / minibatch partition."""
        L = lib()
        di = _dev_tensor(i, torch.int32, self.device)
        dj = _dev_tensor(j, torch.int32, self.device)
        dD = _dev_tensor(D, torch.float32, self.device)
        dm = _dev_tensor(minibatch, torch.uint8, self.device)
        dw = _dev_tensor(worker, torch.int32, self.device)
        n_obs = di.numel()
        ws = L.esspt_mf_workspace_bytes(self._h, n_obs, n_users, F)
        sc = L.esspt_mf_scratch_bytes(self._h, n_obs, n_users, F)
        if ws == 0 or sc == 0:
            raise EssptError(EINVAL, "invalid MF sizes")
        self.mf_workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
        scratch = torch.empty(sc, dtype=torch.uint8, device=self.device)
        self._check(L.esspt_mf_load(self._h, di.data_ptr(), dj.data_ptr(), dD.data_ptr(), dm.data_ptr(), n_obs,
                                    dw.data_ptr(), n_users, F, self.mf_workspace.data_ptr(), ws,
                                    scratch.data_ptr(), sc))
        del scratch, di, dj, dD, dm, dw
        # the sort scratch and the input copies can be tens of GB: hand them back
        torch.cuda.empty_cache()
        self.n_users, self.F, self.n_obs = n_users, F, n_obs
        self._obj_scratch = torch.zeros(2, dtype=torch.float64, device=self.device)

    def mf_sgd_clock(self, eta: float, lam: float, cap: int = 0, sq_loss: torch.Tensor | None = None) -> None:
        """esspt_mf_sgd_clock: one fused clock of MF-SGD (+ CLOCK)."""
        self._check(lib().esspt_mf_sgd_clock(self._h, eta, lam, cap, _ptr(sq_loss)))

    def mf_sgd_clock_sequential(self, eta: float, lam: float, cap: int = 0,
                                sq_loss: torch.Tensor | None = None) -> None:
        """esspt_mf_sgd_clock_sequential: one clock with read-my-writes SGD inside each worker.
        The work buffer is allocated here (torch) on first use and kept."""
        need = lib().esspt_mf_sequential_work_bytes(self._h)
        if getattr(self, "_seq_work", None) is None or self._seq_work.numel() < need:
            self._seq_work = torch.empty(max(need, 16), dtype=torch.uint8, device=self.device)
        self._check(lib().esspt_mf_sgd_clock_sequential(self._h, eta, lam, cap, _ptr(sq_loss),
                                                        self._seq_work.data_ptr(), self._seq_work.numel()))

    def mf_objective(self, version: int, lam: float):
        """esspt_mf_objective: (sum e^2, sum [e^2 + lam(|L_i|^2+|R_j|^2)]) at `version`."""
        sq = ctypes.c_double()
        pen = ctypes.c_double()
        self._check(lib().esspt_mf_objective(self._h, version, lam, self._obj_scratch.data_ptr(), ctypes.byref(sq),
                                             ctypes.byref(pen)))
        return sq.value, pen.value

    def mf_minibatch_size(self, b: int) -> int:
        """esspt_mf_minibatch_size."""
        n = ctypes.c_int64()
        self._check(lib().esspt_mf_minibatch_size(self._h, b, ctypes.byref(n)))
        return n.value

    def mf_export_minibatch(self, b: int, pin: bool = True, out=None):
        """esspt_mf_export_minibatch: (u, j, D, uoff) host tensors of minibatch b,
        written into `out` (four contiguous host tensors of the right sizes) if given."""
        n = self.mf_minibatch_size(b)
        if out is not None:
            u, j, D, uoff = out
            assert u.numel() == n and j.numel() == n and D.numel() == n and uoff.numel() == self.n_users + 1
            assert u.dtype == j.dtype == uoff.dtype == torch.int32 and D.dtype == torch.float32
            assert all(x.is_contiguous() and x.device.type == "cpu" for x in out)
        else:
            mk = lambda k, dt: torch.empty(k, dtype=dt, pin_memory=pin)  # noqa: E731
            u, j, D, uoff = mk(n, torch.int32), mk(n, torch.int32), mk(n, torch.float32), mk(self.n_users + 1, torch.int32)
        self._check(lib().esspt_mf_export_minibatch(self._h, b, u.data_ptr(), j.data_ptr(), D.data_ptr(),
                                                    uoff.data_ptr()))
        return u, j, D, uoff

    def mf_stage_minibatch(self, b: int, u, j, D, uoff, stream=None) -> None:
        """esspt_mf_stage_minibatch: asynchronous host-to-device copy of minibatch b
        on `stream` (a torch.cuda.Stream; None = the table's stream).  The device
        staging buffer is allocated here (torch) on first use and kept."""
        need = lib().esspt_mf_stage_bytes(self._h)
        if getattr(self, "_stage", None) is None or self._stage.numel() < need:
            self._stage = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        st = None if stream is None else ctypes.c_void_p(stream.cuda_stream)
        self._check(lib().esspt_mf_stage_minibatch(self._h, b, u.data_ptr(), j.data_ptr(), D.data_ptr(),
                                                   uoff.data_ptr(), self._stage.data_ptr(), self._stage.numel(), st))

    def set_profile_events(self, before, after) -> None:
        """esspt_set_profile_events: torch.cuda.Event pair (created) or None."""
        if before is None:
            self._check(lib().esspt_set_profile_events(self._h, None, None))
        else:
            self._check(lib().esspt_set_profile_events(self._h, before.cuda_event, after.cuda_event))

    def mf_worker_objective_noalloc(self, version: int, lam: float):
        """esspt_mf_worker_objective_noalloc: per-worker (sum e^2, penalised sum)
        as two float64[P] arrays, computed without any device allocation."""
        sq = np.empty(self.P, dtype=np.float64)
        pen = np.empty(self.P, dtype=np.float64)
        self._check(lib().esspt_mf_worker_objective_noalloc(self._h, version, lam, sq.ctypes.data, pen.ctypes.data))
        return sq, pen

    @classmethod
    def for_workload(cls, w, data, partition, **kw) -> "Table":
        """A table for an MF workload (gen.workloads.Workload) with data loaded."""
        t = cls(w.n_users + w.n_items, w.K, w.P, w.s, model=w.model, seed=w.sched_seed, essp_p=w.essp_p,
                essp_max_delay=w.essp_max_delay, vap_v0=w.vap_v0, **kw)
        wp, mb = partition
        t.mf_load(data.i, data.j, data.D, mb, wp, w.n_users, w.F)
        t.table_init(np.concatenate([data.L0, data.R0]))
        return t


class SoftmaxResult(NamedTuple):
    """loss and lse, fp32[n]; the gradients are None after a forward pass."""

    loss: torch.Tensor
    lse: torch.Tensor
    grad_h: torch.Tensor | None
    grad_w: torch.Tensor | None


class SoftmaxHead:
    """Softmax over a catalogue of `n_items` rows (one `esspt_softmax` handle).

    `loss` is cross entropy against one item per row, `distill` the divergence
    from a teacher's top logits; both give the gradients of the weighted sum of
    the rows' losses as tensors: there is no autograd graph, a program hands them on
    itself (`h.backward(r.grad_h)`).  The n x n_items scores are not kept (but for calls
    of up to 8 rows, and of up to 128 where that is faster: at most 8 n_items or 2^24 of
    them, in the workspace).  The workspace is allocated here once.  Work runs on `stream` (default: the current one at
    construction); a call from another current stream is ordered after the work
    queued there, and that stream's later work after the call.  Calls may be captured
    in a CUDA graph, where `stream` is the captured one.
    """

    def __init__(self, max_rows: int, n_items: int, width: int, dtype=torch.float32, max_top: int = 1,
                 backward: bool = True, device=None, stream=None):
        self._h = None
        if not torch.cuda.is_available():
            raise RuntimeError("esspt needs a CUDA device")
        L = self._lib = lib()
        if dtype not in DTYPES:
            raise EssptError(EINVAL, f"dtype must be one of {', '.join(str(d) for d in DTYPES)}")
        device = torch.device(device if device is not None else "cuda")
        self.device = device if device.index is not None else torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.max_rows, self.n_items, self.width, self.dtype = max_rows, n_items, width, dtype
        self.max_top, self.backward = max_top, backward
        cfg = SoftmaxConfig(max_rows, n_items, width, DTYPES[dtype], max_top, int(backward),
                            ctypes.c_void_p(self.stream.cuda_stream))
        nbytes = L.esspt_softmax_workspace_bytes(ctypes.byref(cfg))
        if nbytes == 0:
            raise EssptError(EINVAL, "invalid softmax configuration")
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            st = L.esspt_softmax_create(ctypes.byref(cfg), self.workspace.data_ptr(), nbytes, ctypes.byref(h))
        if st != OK:
            raise EssptError(st, L.esspt_softmax_last_error(None).decode())
        self._h = h

    def _check(self, st: int) -> None:
        if st != OK:
            raise EssptError(st, self._lib.esspt_softmax_last_error(self._h).decode())

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.esspt_softmax_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _rows(self, x, n, name) -> torch.Tensor:
        """`x` as rows that the library reads in place; another layout is copied."""
        if not isinstance(x, torch.Tensor) or x.dtype is not self.dtype or x.device != self.device:
            raise EssptError(EINVAL, f"{name} must be a {self.dtype} tensor on {self.device}")
        if x.dim() != 2 or x.shape[1] != self.width or (n is not None and x.shape[0] != n):
            raise EssptError(EINVAL, f"{name} has shape {tuple(x.shape)}, not ({n if n is not None else 'n'}, {self.width})")
        if (x.stride(1) != 1 and self.width > 1) or (x.shape[0] > 1 and x.stride(0) < self.width):
            x = x.contiguous()
        return x

    def _list(self, x, shape, dtype, name) -> torch.Tensor:
        if not isinstance(x, torch.Tensor) or x.device != self.device or tuple(x.shape) != tuple(shape):
            raise EssptError(EINVAL, f"{name} must be a tensor of shape {tuple(shape)} on {self.device}")
        if x.dtype is not dtype or not x.is_contiguous():
            if x.dtype.is_floating_point != dtype.is_floating_point:
                raise EssptError(EINVAL, f"{name} must hold {dtype} values")
            if x.dtype is torch.int64:  # ids past 32 bits stay outside the catalogue
                x = x.clamp(-1, 2**31 - 1)
            x = x.to(dtype).contiguous()
        return x

    def _out(self, x, shape, name) -> torch.Tensor:
        if x is None:
            return torch.empty(shape, dtype=self.dtype, device=self.device)
        if x.dtype is not self.dtype or x.device != self.device or tuple(x.shape) != shape or not x.is_contiguous():
            raise EssptError(EINVAL, f"{name} must be a contiguous {self.dtype} tensor of shape {shape} on {self.device}")
        return x

    def _call(self, head, ids, logits, tail) -> int:
        if logits is None:
            return self._lib.esspt_softmax_loss(*head, ids.data_ptr(), *tail)
        return self._lib.esspt_softmax_distill(*head, ids.data_ptr(), logits.data_ptr(), ids.shape[1], *tail)

    def _run(self, h, w, ids, logits, weight, inv_temperature, backward, grad_h, grad_w) -> SoftmaxResult:
        if backward is None:
            backward = self.backward
        h = self._rows(h, None, "h")
        w = self._rows(w, self.n_items, "w")
        n = h.shape[0]
        if n > self.max_rows:
            raise EssptError(EINVAL, f"{n} rows, more than max_rows = {self.max_rows}")
        if weight is not None:
            weight = self._list(weight, (n,), torch.float32, "weight")
        loss = torch.empty(n, dtype=torch.float32, device=self.device)
        lse = torch.empty(n, dtype=torch.float32, device=self.device)
        if backward:
            grad_h = self._out(grad_h, (n, self.width), "grad_h")
            grad_w = self._out(grad_w, (self.n_items, self.width), "grad_w")
        else:
            grad_h = grad_w = None
        cur = torch.cuda.current_stream(self.device)
        elsewhere = cur.cuda_stream != self.stream.cuda_stream
        if elsewhere:
            self.stream.wait_stream(cur)
        tail = (n, _ptr(weight), inv_temperature, loss.data_ptr(), lse.data_ptr(), _ptr(grad_h), _ptr(grad_w))
        head = (self._h, h.data_ptr(), h.stride(0) if n > 1 else self.width, w.data_ptr(),
                w.stride(0) if self.n_items > 1 else self.width)
        if torch.cuda.current_device() == self.device.index:
            st = self._call(head, ids, logits, tail)
        else:
            with torch.cuda.device(self.device):
                st = self._call(head, ids, logits, tail)
        if elsewhere:
            cur.wait_stream(self.stream)
        if st != OK:
            self._check(st)
        return SoftmaxResult(loss, lse, grad_h, grad_w)

    def loss(self, h, w, targets, weight=None, inv_temperature: float = 1.0, backward: bool | None = None, grad_h=None,
             grad_w=None) -> SoftmaxResult:
        """esspt_softmax_loss: rows h (n, width) against w (n_items, width), targets
        int32 (n,), a negative one marking an ignored row; weight fp32 (n,).  Rows of h
        and w may be strided.  backward defaults to the handle's."""
        targets = self._list(targets, (h.shape[0],), torch.int32, "targets")
        return self._run(h, w, targets, None, weight, inv_temperature, backward, grad_h, grad_w)

    def distill(self, h, w, ids, logits, weight=None, inv_temperature: float = 1.0, backward: bool | None = None,
                grad_h=None, grad_w=None) -> SoftmaxResult:
        """esspt_softmax_distill: ids int32 and teacher logits fp32, both (n, top); an
        id < 0 is an absent entry."""
        if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
            raise EssptError(EINVAL, "ids must be a tensor of shape (n, top)")
        ids = self._list(ids, (h.shape[0], ids.shape[1]), torch.int32, "ids")
        logits = self._list(logits, tuple(ids.shape), torch.float32, "logits")
        return self._run(h, w, ids, logits, weight, inv_temperature, backward, grad_h, grad_w)

    def poll(self) -> None:
        """esspt_softmax_poll: synchronise and raise on a target or id outside the catalogue."""
        self._check(self._lib.esspt_softmax_poll(self._h))


_current_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


class _Operator:
    """What the handles of the operators on rows share: where they run, errors, the end.

    Work runs on `stream` (default: the current one at construction).  A call from
    another current stream is ordered after the work queued there, and that stream's later
    work after the call.  Calls may be captured in a CUDA graph, where `stream` is the
    captured one.
    """

    _name = ""

    def _open(self, dtype, device, stream):
        self._h = None
        if not torch.cuda.is_available():
            raise RuntimeError("esspt needs a CUDA device")
        self._lib = lib()
        if dtype not in DTYPES:
            raise EssptError(EINVAL, f"dtype must be one of {', '.join(str(d) for d in DTYPES)}")
        device = torch.device(device if device is not None else "cuda")
        self.device = device if device.index is not None else torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.dtype = dtype
        self._stream_ptr, self._index = self.stream.cuda_stream, self.device.index

    def _create(self, *config) -> None:
        """The workspace and the handle of a configuration (and what else its calls take)."""
        nbytes = getattr(self._lib, f"esspt_{self._name}_workspace_bytes")(*config)
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            st = getattr(self._lib, f"esspt_{self._name}_create")(*config, self.workspace.data_ptr(), nbytes, ctypes.byref(h))
        if st != OK:
            raise EssptError(st, getattr(self._lib, f"esspt_{self._name}_last_error")(None).decode())
        self._h = h

    def _check(self, st: int) -> None:
        if st != OK:
            raise EssptError(st, getattr(self._lib, f"esspt_{self._name}_last_error")(self._h).decode())

    def _call(self, call, *args) -> None:
        """One of the library's calls, in order with the current stream."""
        if _current_stream(self._index) == self._stream_ptr and _current_device() == self._index:
            st = call(self._h, *args)  # the usual call
        else:
            current = torch.cuda.current_stream(self.device)
            elsewhere = current.cuda_stream != self._stream_ptr
            if elsewhere:
                self.stream.wait_stream(current)
            with torch.cuda.device(self.device):
                st = call(self._h, *args)
            if elsewhere:
                current.wait_stream(self.stream)
        if st != OK:
            self._check(st)

    def _wait(self, call, *args) -> None:
        """One of the library's calls that wait for the stream: of the default stream, the handle's device's."""
        with torch.cuda.device(self.device):
            self._check(call(self._h, *args))

    def close(self) -> None:
        if getattr(self, "_h", None):
            with torch.cuda.device(self.device):
                getattr(self._lib, f"esspt_{self._name}_destroy")(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _rows(self, x, n, width, dtype, name) -> torch.Tensor:
        """`x` as rows that the library reads in place; another layout is copied."""
        if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.device != self.device:
            raise EssptError(EINVAL, f"{name} must be a {dtype} tensor on {self.device}")
        shape = x.shape
        if len(shape) != 2 or shape[1] != width or (n is not None and shape[0] != n):
            raise EssptError(EINVAL, f"{name} has shape {tuple(shape)}, not ({n if n is not None else 'n'}, {width})")
        if not x.is_contiguous() and ((x.stride(1) != 1 and width > 1) or (shape[0] > 1 and x.stride(0) < width)):
            x = x.contiguous()
        return x

    def _values(self, x, shape, dtype, name) -> torch.Tensor:
        """`x`, read as contiguous values."""
        if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.device != self.device or x.shape != shape:
            raise EssptError(EINVAL, f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return x if x.is_contiguous() else x.contiguous()

    def _out(self, x, shape, dtype, name) -> torch.Tensor:
        if x is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.device != self.device or x.shape != shape or not x.is_contiguous():
            raise EssptError(EINVAL, f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return x


def _stride(x) -> int:
    """Values from one row to the next."""
    return x.stride(0) if x.shape[0] != 1 else x.shape[1]


class Embedding(_Operator):
    """Rows of a table of `n_rows` by id, and the gradient back to it (one `esspt_embed` handle).

    `lookup` gives scale * w[ids], zeros where an id is negative (padding); `gradient`
    sums scale * grad over the tokens of each row, in a fixed order: the same inputs
    give the same bits.  There is no autograd graph.  The workspace is allocated here once.
    """

    __doc__ += _Operator.__doc__.split("\n", 1)[1]
    _name = "embed"

    def __init__(self, max_tokens: int, n_rows: int, width: int, dtype=torch.float32, backward: bool = True, device=None,
                 stream=None):
        self._open(dtype, device, stream)
        self.max_tokens, self.n_rows, self.width, self.backward = max_tokens, n_rows, width, backward
        self._create(ctypes.byref(EmbedConfig(max_tokens, n_rows, width, DTYPES[dtype], int(backward),
                                              ctypes.c_void_p(self._stream_ptr))))

    def _ids(self, ids) -> torch.Tensor:
        if not isinstance(ids, torch.Tensor) or ids.device != self.device or ids.dim() != 1:
            raise EssptError(EINVAL, f"ids must be a tensor of shape (n,) on {self.device}")
        if ids.shape[0] > self.max_tokens:
            raise EssptError(EINVAL, f"{ids.shape[0]} ids, more than max_tokens = {self.max_tokens}")
        if ids.dtype is not torch.int32:
            if ids.dtype is not torch.int64:
                raise EssptError(EINVAL, "ids must hold torch.int32 values")
            ids = ids.clamp(-1, 2**31 - 1).to(torch.int32)  # (past 32 bits is outside the table all the same)
        return ids if ids.is_contiguous() else ids.contiguous()

    def lookup(self, w, ids, scale: float = 1.0, out=None) -> torch.Tensor:
        """esspt_embed_lookup: rows of w (n_rows, width), which may be strided, by ids
        int32 (n,)."""
        ids = self._ids(ids)
        w = self._rows(w, self.n_rows, self.width, self.dtype, "w")
        n = ids.shape[0]
        if out is None:
            out = torch.empty((n, self.width), dtype=self.dtype, device=self.device)
        else:
            out = self._out(out, (n, self.width), self.dtype, "out")
        self._call(self._lib.esspt_embed_lookup, w.data_ptr(), _stride(w), ids.data_ptr(), n, scale, out.data_ptr())
        return out

    def gradient(self, ids, grad, scale: float = 1.0, grad_w=None, accumulate: bool = False) -> torch.Tensor:
        """esspt_embed_gradient: from grad (n, width), which may be strided, that of a
        whole table; with `accumulate` added to grad_w, whose other rows stay as they are."""
        ids = self._ids(ids)
        n = ids.shape[0]
        grad = self._rows(grad, n, self.width, self.dtype, "grad")
        if accumulate and grad_w is None:
            raise EssptError(EINVAL, "accumulate needs a grad_w")
        grad_w = self._out(grad_w, (self.n_rows, self.width), self.dtype, "grad_w")
        self._call(self._lib.esspt_embed_gradient, ids.data_ptr(), grad.data_ptr(), _stride(grad), n, scale,
                   int(bool(accumulate)), grad_w.data_ptr())
        return grad_w

    def poll(self) -> None:
        """esspt_embed_poll: synchronise and raise on an id outside the table."""
        self._wait(self._lib.esspt_embed_poll)


class NormResult(NamedTuple):
    """y, and fp32[n] of a row's mean and 1 / standard deviation for the backward pass."""

    y: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor


class NormGradients(NamedTuple):
    grad_x: torch.Tensor | None
    grad_weight: torch.Tensor | None
    grad_bias: torch.Tensor | None


class LayerNorm(_Operator):
    """Layer norm of rows, forward and backward (one `esspt_norm` handle).

    Weights and their gradients are `weight_dtype` (default: the rows').  There is no
    autograd graph: a program keeps mean and rstd of `forward` for `backward`.
    """

    __doc__ += _Operator.__doc__.split("\n", 1)[1]
    _name = "norm"

    def __init__(self, max_rows: int, width: int, dtype=torch.float32, weight_dtype=None, eps: float = 1e-5,
                 backward: bool = True, device=None, stream=None):
        self._open(dtype, device, stream)
        weight_dtype = weight_dtype if weight_dtype is not None else dtype
        if weight_dtype not in DTYPES:
            raise EssptError(EINVAL, f"weight_dtype must be {dtype} or torch.float32")
        self.max_rows, self.width, self.weight_dtype, self.eps, self.backwards = max_rows, width, weight_dtype, eps, backward
        self._shape = (width,)
        self._create(ctypes.byref(NormConfig(max_rows, width, DTYPES[dtype], DTYPES[weight_dtype], int(backward), eps,
                                             ctypes.c_void_p(self._stream_ptr))))

    def _n(self, x) -> int:
        if x.shape[0] > self.max_rows:
            raise EssptError(EINVAL, f"{x.shape[0]} rows, more than max_rows = {self.max_rows}")
        return x.shape[0]

    def forward(self, x, weight=None, bias=None, y=None) -> NormResult:
        """esspt_norm_forward: rows x (n, width), which may be strided; weight and bias
        (width,), or None for 1 and 0."""
        x = self._rows(x, None, self.width, self.dtype, "x")
        n = self._n(x)
        if weight is not None:
            weight = self._values(weight, self._shape, self.weight_dtype, "weight")
        if bias is not None:
            bias = self._values(bias, self._shape, self.weight_dtype, "bias")
        if y is None:
            y = torch.empty((n, self.width), dtype=self.dtype, device=self.device)
        else:
            y = self._out(y, (n, self.width), self.dtype, "y")
        mean = torch.empty(n, dtype=torch.float32, device=self.device)
        rstd = torch.empty_like(mean)
        self._call(self._lib.esspt_norm_forward, x.data_ptr(), _stride(x), n, _ptr(weight), _ptr(bias), y.data_ptr(),
                   mean.data_ptr(), rstd.data_ptr())
        return NormResult(y, mean, rstd)

    def backward(self, dy, x, mean, rstd, weight=None, grad_x=None, need_x: bool = True, need_weights: bool = True) -> NormGradients:
        """esspt_norm_backward: from dy and the x, mean, rstd and weight of a forward pass;
        need_x and need_weights say which gradients are wanted."""
        x = self._rows(x, None, self.width, self.dtype, "x")
        n = self._n(x)
        dy = self._rows(dy, n, self.width, self.dtype, "dy")
        mean, rstd = self._values(mean, (n,), torch.float32, "mean"), self._values(rstd, (n,), torch.float32, "rstd")
        if weight is not None:
            weight = self._values(weight, self._shape, self.weight_dtype, "weight")
        grad_x = self._out(grad_x, (n, self.width), self.dtype, "grad_x") if need_x else None
        dw = db = None
        if need_weights:
            dw = torch.empty(self.width, dtype=self.weight_dtype, device=self.device)
            db = torch.empty_like(dw)
        self._call(self._lib.esspt_norm_backward, dy.data_ptr(), _stride(dy), x.data_ptr(), _stride(x), n, _ptr(weight),
                   mean.data_ptr(), rstd.data_ptr(), _ptr(grad_x), _ptr(dw), _ptr(db))
        return NormGradients(grad_x, dw, db)


class Moments(NamedTuple):
    """Of all tensors in flat order (`AdamW.places`): m, and v (32 bits) or sqrt(v) (8 bits, bf16)."""

    m: torch.Tensor
    second: torch.Tensor


class AdamW(_Operator):
    """AdamW steps over many fp32 tensors at once (one `esspt_adamw` handle).

    `params` are updated in place and may not share memory; where `copies` has a 16-bit tensor, it is rewritten
    from its parameter and the parameter's gradients are of its type.  `weight_decay`:
    one for all, or one each.  With `state_bits` 8 moments are held in 8 bits, rounded up or down by a hash of
    `seed`, the step and the value's place.  The handle keeps references to the tensors.
    """

    __doc__ += _Operator.__doc__.split("\n", 1)[1]
    _name = "adamw"

    def __init__(self, params, copies=None, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, state_bits: int = 32,
                 seed: int = 0, device=None, stream=None):
        params = list(params)
        copies = [None] * len(params) if copies is None else list(copies)
        if device is None and params and isinstance(params[0], torch.Tensor) and params[0].is_cuda:
            device = params[0].device
        self._open(torch.float32, device, stream)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(params)
        if len(copies) != len(params) or len(decay) != len(params):
            raise EssptError(EINVAL, f"{len(params)} params, {len(copies)} copies, {len(decay)} weight decays")
        kinds = {c.dtype for c in copies if isinstance(c, torch.Tensor)}
        if len(kinds) > 1 or not kinds <= {torch.bfloat16, torch.float16}:
            raise EssptError(EINVAL, "copies must all be bf16, or all fp16")
        copy_dtype = kinds.pop() if kinds else torch.bfloat16
        self.places, self._like, end = [], [], 0
        recs = (AdamWTensor * max(1, len(params)))()
        for k, (p, c) in enumerate(zip(params, copies)):
            self._in_place(p, None, torch.float32, f"params[{k}]")
            if c is not None:
                self._in_place(c, p.shape, copy_dtype, f"copies[{k}]")
            recs[k] = AdamWTensor(_ptr(p), _ptr(c), p.numel(), decay[k])
            self.places.append(end)
            self._like.append((p.shape, torch.float32 if c is None else copy_dtype))
            end += -(-p.numel() // 128) * 128
        self.params, self.copies, self.state_bits, self.values = params, copies, state_bits, end
        self._grads = (ctypes.c_void_p * max(1, len(params)))()
        self._create(ctypes.byref(AdamWConfig(len(params), state_bits, DTYPES[copy_dtype], 0, betas[0], betas[1], eps,
                                              seed & 0xFFFFFFFFFFFFFFFF, ctypes.c_void_p(self._stream_ptr))), recs)
        if state_bits == 32:
            both = self.workspace[:8 * end].view(torch.float32)
            self._moments = Moments(both[:end], both[end:])

    def _in_place(self, x, shape, dtype, name) -> None:
        if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.device != self.device or not x.is_contiguous() or (
                shape is not None and x.shape != shape):
            raise EssptError(EINVAL, f"{name} must be a contiguous {dtype} tensor on {self.device}"
                             + (f" of shape {tuple(shape)}" if shape is not None else ""))

    def _scalar(self, x, name):
        if x is None:
            return None
        if not isinstance(x, torch.Tensor) or x.dtype is not torch.float32 or x.device != self.device or x.numel() != 1:
            raise EssptError(EINVAL, f"{name} must be one fp32 value on {self.device}")
        return x

    def step(self, grads, lr, grad_scale=None) -> None:
        """esspt_adamw_step: one step along `grads`, one for each parameter, None to leave it as it is.
        `lr` is a number or one fp32 value on the device, `grad_scale` such a value or None."""
        if len(grads) != len(self._like):
            raise EssptError(EINVAL, f"{len(grads)} gradients for {len(self._like)} params")
        kept, at, on = [], [], self.device
        for g, (shape, dtype) in zip(grads, self._like):
            if g is None:
                at.append(None)
                continue
            if not isinstance(g, torch.Tensor) or g.dtype is not dtype or g.shape != shape or g.device != on:
                raise EssptError(EINVAL, f"grads[{len(at)}] must be a {dtype} tensor of shape {tuple(shape)} on {on}")
            if not g.is_contiguous():
                g = g.contiguous()
                kept.append(g)
            at.append(g.data_ptr())
        self._grads[:] = at
        scale = self._scalar(grad_scale, "grad_scale")
        d_lr = self._scalar(lr, "lr") if isinstance(lr, torch.Tensor) else None
        self._call(self._lib.esspt_adamw_step, self._grads, 0.0 if d_lr is not None else lr, _ptr(d_lr), _ptr(scale))

    def moments(self) -> Moments:
        """The moments in flat order: with 32 bits the state itself, with 8 what its codes stand for
        (esspt_adamw_moments)."""
        n = self.values
        if self.state_bits == 32:
            if _current_stream(self._index) != self._stream_ptr:
                torch.cuda.current_stream(self.device).wait_stream(self.stream)
            return self._moments
        m, second = torch.empty((2, n), dtype=torch.bfloat16, device=self.device).unbind()
        self._call(self._lib.esspt_adamw_moments, m.data_ptr(), second.data_ptr())
        return Moments(m, second)

    def load(self, m, second, step: int) -> None:
        """esspt_adamw_load: moments as `moments` gives them (any floating type), and the number of steps taken."""
        dtype = torch.float32 if self.state_bits == 32 else torch.bfloat16
        for x in (m, second):
            if not isinstance(x, torch.Tensor) or x.device != self.device or x.shape != (self.values,) or not x.is_floating_point():
                raise EssptError(EINVAL, f"moments must be floating-point tensors of shape ({self.values},) on {self.device}")
        m, second = m.to(dtype).contiguous(), second.to(dtype).contiguous()
        self._call(self._lib.esspt_adamw_load, m.data_ptr(), second.data_ptr(), step)

    @property
    def steps(self) -> int:
        """esspt_adamw_steps: steps taken so far (synchronises)."""
        n = ctypes.c_int64()
        self._wait(self._lib.esspt_adamw_steps, ctypes.byref(n))
        return n.value
