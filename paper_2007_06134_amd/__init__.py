"""ADPSGD hot path on MI355X: Python side of the C ABI in ``include/adpsgd.h``.

``_native`` holds the ctypes binding (functions named as in C).  ``Adpsgd``
below owns one context together with its torch-allocated device buffers;
torch supplies only device memory and the HIP stream.
"""
from __future__ import annotations

import contextlib
from typing import Optional

import numpy as np

from ._native import (  # noqa: F401
    AdpsgdError, EDEVICE, EINVAL, ENONFINITE, ESTATE, EXPORTED, LAUNCH_DEVICE, LAUNCH_HOST, LAUNCH_HYBRID,
    LIB_PATH, LR_CONST, LR_COSINE, MX_E2M1, MX_E4M3, adpsgd_average_noalloc, adpsgd_mx_rows,
    LR_STEP, LR_WARMUP_STEP, OK, PERIOD_ADAPTIVE, PERIOD_ALG1, PERIOD_CONST, adpsgd_average, adpsgd_buffers, adpsgd_destroy,
    adpsgd_get_state, adpsgd_get_timing, adpsgd_hparams, adpsgd_init, adpsgd_last_error,
    adpsgd_local_steps, adpsgd_lr, adpsgd_normal_dump, adpsgd_philox_dump, adpsgd_reset, adpsgd_run,
    adpsgd_run_traced, adpsgd_step_rec,
    adpsgd_sched_init, adpsgd_sched_on_sync, adpsgd_sched_step, adpsgd_schedule, adpsgd_set_launch_policy, adpsgd_set_state, adpsgd_set_timing,
    adpsgd_get_step_launch, adpsgd_set_step_launch,
    adpsgd_padded_row_stride, adpsgd_state, adpsgd_step_average, adpsgd_sync_rec, adpsgd_timing,
    adpsgd_workspace_bytes, make_hparams,
)
from . import mx as _mx
from .mx import MxRows, mx_average, mx_dequantize, mx_product, mx_quantize  # noqa: F401


def hparams_of(w) -> adpsgd_hparams:
    """hparams from any object with the fields of the C struct (e.g. a workload)."""
    return make_hparams(seed=w.seed, sigma=w.sigma, momentum=w.momentum, weight_decay=w.weight_decay,
                        h_lo=w.h_lo, h_hi=w.h_hi, lr_kind=w.lr_kind, lr0=w.lr0,
                        total_steps=w.total_steps, period_mode=w.period_mode, p_init=w.p_init,
                        k_s=w.k_s, thr_lo=w.thr_lo, thr_hi=w.thr_hi,
                        sync_warmup_steps=getattr(w, "sync_warmup_steps", 0),
                        p_switch_step=getattr(w, "p_switch_step", 0), p_after=getattr(w, "p_after", 0),
                        avg_momentum=getattr(w, "avg_momentum", False), p_max=getattr(w, "p_max", 0))


class Adpsgd:
    """One ADPSGD context with its device buffers on a torch device.

    x, m: float32 [K, P]; h, xstar: float32 [P]; workspace: uint8 sized by
    adpsgd_workspace_bytes.  The stream is the torch stream current at
    construction (or the one passed in).  With pad_rows (default), x, m, h and
    xstar are views of the rows of ONE [2K + 2, row_stride] buffer (x rows,
    then m rows, then h, then xstar), row_stride = adpsgd_padded_row_stride(P):
    256 n floats with n odd.  Every row then starts on a 1 KB boundary (the
    kernels move whole float4 groups, and each 64-lane wave's 1 KB of a row is
    one aligned kilobyte), and the rows that a kernel streams together start an
    odd number of kilobytes apart, which measures fastest on MI355X.
    pad_rows=False allocates x and m as packed [K, P] buffers and h and xstar
    on their own.
    """

    def __init__(self, K: int, offsets, hp: adpsgd_hparams, device="cuda", stream=None, pad_rows: bool = True):
        import torch
        self.torch = torch
        off = np.ascontiguousarray(np.asarray(offsets, dtype=np.int64))
        self.K, self.P, self.T = int(K), int(off[-1]), len(off) - 1
        self.offsets = off
        self.hp = hp
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("the ADPSGD library runs on a GPU device only")
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        nbytes = adpsgd_workspace_bytes(self.K, self.P, off)
        if nbytes == 0:
            raise ValueError("invalid K, P or tensor offsets")
        alloc = dict(device=self.device, dtype=torch.float32)
        K = self.K
        if pad_rows:
            self.row_stride = adpsgd_padded_row_stride(self.P)
            self._rows = torch.empty((2 * K + 2, self.row_stride), **alloc)
            self._x_rows, self._m_rows = self._rows[:K], self._rows[K:2 * K]
            self.h, self.xstar = self._rows[2 * K, :self.P], self._rows[2 * K + 1, :self.P]
        else:
            self.row_stride = self.P
            self._x_rows = torch.empty((K, self.P), **alloc)
            self._m_rows = torch.empty((K, self.P), **alloc)
            self.h = torch.empty((self.P,), **alloc)
            self.xstar = torch.empty((self.P,), **alloc)
        self.x = self._x_rows[:, :self.P]
        self.m = self._m_rows[:, :self.P]
        self.workspace = torch.empty((nbytes,), device=self.device, dtype=torch.uint8)
        self.buf = adpsgd_buffers(x=self._x_rows.data_ptr(), m=self._m_rows.data_ptr(), h=self.h.data_ptr(),
                                  xstar=self.xstar.data_ptr(), workspace=self.workspace.data_ptr(),
                                  workspace_bytes=nbytes, stream=self.stream.cuda_stream,
                                  row_stride=self.row_stride)
        # the state of average_mx (made by its first call or by mx_begin).  _mx_lost: syncs of fp32
        # replicas have moved the model that the workers share, and mx_base is not that model.
        self.mx_base = self.mx_residual = None
        self._mx_lost = False
        self._mx_rows = self._mx_offsets = None
        with torch.cuda.device(self.device):
            self.ctx = adpsgd_init(self.K, self.P, off, hp, self.buf)

    @classmethod
    def from_workload(cls, w, device="cuda", stream=None, pad_rows: bool = True) -> "Adpsgd":
        return cls(w.K, w.offsets(), hparams_of(w), device=device, stream=stream, pad_rows=pad_rows)

    # -- the hot path
    def local_steps(self, n: int) -> None:
        adpsgd_local_steps(self.ctx, n)

    def average(self) -> np.ndarray:
        return self._following(adpsgd_average, lambda var: 1, self.T)

    def step_average(self) -> np.ndarray:
        return self._following(adpsgd_step_average, lambda var: 1, self.T)

    def _following(self, call, syncs, *args, **kw):
        """call(self.ctx, ...), which synchronizes fp32 replicas syncs(result) times.  Where it ends with
        such a sync mx_base follows (if average_mx is in use), else it is lost."""
        try:
            out = call(self.ctx, *args, **kw)
        except (TypeError, ValueError):
            raise                              # (of arguments: nothing ran)
        except BaseException as e:
            if getattr(e, "code", None) != EINVAL:
                self._mx_lost = True
            raise
        if syncs(out):
            self._mx_lost = True
            if self.mx_base is not None and self.get_state().cnt == 0:
                self.mx_begin()
        return out

    @contextlib.contextmanager
    def _mx_scope(self):
        """The engine's device and stream, without gradients; not in inference mode, as the tensors of
        average_mx are written outside it, too."""
        torch = self.torch
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream), torch.inference_mode(False), torch.no_grad():
            yield

    def average_mx(self, format: int = MX_E2M1, error_feedback: bool = True, products: bool = False):
        """The synchronization with microscaled messages in place of fp32 replicas: every worker sends
        its difference from mx_base, the model after the last sync (0 at first, as the replicas),
        in `format`; all replicas become mx_base + the mean of what was sent, which is the new mx_base.
        With error_feedback what a worker's message left out (mx_residual) is added to its next one;
        a message without it, and a sync of fp32 replicas, end what is owed.

        Returns the per-tensor variances of what was sent, for ``schedule`` (and, with products, the
        workers' inner products [T, K, K] as ``mx_product`` gives them).  Like ``average`` it restarts
        the counter and waits for the stream; momentum stays local (with avg_momentum it is refused).

        Syncs of fp32 replicas may come between: mx_base follows ``average``, ``step_average`` and a run that
        ends with a sync.  Where it could not follow (those calls, or the state of another run, before the first
        of this one; a run that stepped on past its last sync) the call is refused until ``mx_begin`` names a
        base: a message would be most of a model in a few bits.  mx_base and mx_residual belong to a
        checkpoint, next to x and m (``mx_begin`` takes them back); reset() zeroes them."""
        torch = self.torch
        if self.hp.avg_momentum:
            raise ValueError("average_mx keeps the momentum local; the hyper-parameters ask for avg_momentum")
        if products and self.K > 256:      # (before anything is sent)
            raise ValueError("products are for at most 256 workers")
        if self._mx_lost:
            raise AdpsgdError(ESTATE, "the workers' shared model has moved past mx_base: call mx_begin right behind a "
                                      "sync, or with the model after the last one")
        with self._mx_scope():
            if self.mx_base is None:
                self.mx_base = torch.zeros((self.P,), device=self.device, dtype=torch.float32)
            if error_feedback and self.mx_residual is None:
                self.mx_residual = torch.zeros_like(self._x_rows)[:, :self.P]
            if self._mx_rows is None or self._mx_rows.format != format:
                self._mx_rows = MxRows.empty(self.K, self.P, format, self.device)
            if self._mx_offsets is None:
                self._mx_offsets = torch.from_numpy(self.offsets).to(self.device)
            # (all memory before anything is sent, so that a call that fails has moved nothing)
            rows, off = self._mx_rows, self._mx_offsets
            made = _mx.average_buffers(rows, self.T, off)
            made_c = _mx.product_buffers(rows, self.T, off) if products else None
            mx_quantize(self.x, self.mx_base, self.mx_residual if error_feedback else None, out=rows)
            if not error_feedback and self.mx_residual is not None:
                self.mx_residual.zero_()
            c = mx_product(rows, off, _buffers=made_c) if products else None
            _, var = mx_average(rows, off, self.mx_base, x=self.x, base_out=self.mx_base, _buffers=made)
            st = self.get_state()
            st.cnt = 0
            self.set_state(st)
            out = var.cpu().numpy()
            if c is not None:
                out = (out, c.cpu().numpy())
        return out

    def mx_begin(self, base=None, residual=None) -> None:
        """Sets what the next ``average_mx`` starts from: mx_base to base [P], the model that all workers know,
        and mx_residual to residual [K, P], what each one's messages still owe (zero by default).  float32
        tensors on any device, copied.  Without a base it is what the replicas hold now: right behind a sync
        of fp32 replicas, or where every row of x was just given the model to start from."""
        torch = self.torch
        for name, t, shape in (("base", base, (self.P,)), ("residual", residual, (self.K, self.P))):
            if t is not None and (t.dtype is not torch.float32 or t.shape != shape):
                raise ValueError(f"{name} must be float32 {list(shape)}")
        if base is None and self.get_state().cnt != 0:
            raise ValueError("the workers have stepped on since the last sync: base must be given")
        self.stream.wait_stream(torch.cuda.current_stream(self.device))
        with self._mx_scope():
            to_base, to_residual = self.mx_base, self.mx_residual
            if to_base is None:
                to_base = torch.empty((self.P,), device=self.device, dtype=torch.float32)
            if to_residual is None and residual is not None:
                to_residual = torch.empty_like(self._x_rows)[:, :self.P]
            to_base.copy_(self.x[0] if base is None else base)
            if residual is not None:
                to_residual.copy_(residual)
            elif to_residual is not None:
                to_residual.zero_()
            for t in (base, residual):         # (the caller may drop them before the copies have run)
                if t is not None and t.device == to_base.device:
                    t.record_stream(self.stream)
        self.mx_base, self.mx_residual, self._mx_lost = to_base, to_residual, False

    def schedule(self, var: np.ndarray) -> int:
        return adpsgd_schedule(self.ctx, var)

    def run(self, n_steps: int, log_cap: Optional[int] = None, with_var: bool = True):
        return self._following(adpsgd_run, lambda out: out[2], n_steps, self.T, log_cap=log_cap, with_var=with_var)

    def run_traced(self, n_steps: int, log_cap: Optional[int] = None, with_var: bool = True):
        return self._following(adpsgd_run_traced, lambda out: out[2], n_steps, self.T, log_cap=log_cap, with_var=with_var)

    def reset(self) -> None:
        adpsgd_reset(self.ctx)
        self._mx_lost = False
        with self.torch.cuda.stream(self.stream):
            for t in (self.mx_base, self.mx_residual):
                if t is not None:
                    t.zero_()

    # -- state, timing
    def get_state(self) -> adpsgd_state:
        return adpsgd_get_state(self.ctx)

    def set_state(self, st: adpsgd_state) -> None:
        t = self.get_state().t
        adpsgd_set_state(self.ctx, st)
        if st.t != t and self.mx_base is None:     # (another run's replicas, whose last sync is not known here)
            self._mx_lost = True

    @property
    def step_launch(self) -> tuple:
        """(threads per block, LDS bytes reserved per block, chunks of a row an
        XCD takes in a run) of the plain local step."""
        return adpsgd_get_step_launch(self.ctx)

    def set_step_launch(self, block: int, lds_bytes: int = 0, row_chunks: int = 1) -> None:
        adpsgd_set_step_launch(self.ctx, block, lds_bytes, row_chunks)

    def set_launch_policy(self, policy: int) -> None:
        adpsgd_set_launch_policy(self.ctx, policy)

    def set_timing(self, every=True) -> None:
        adpsgd_set_timing(self.ctx, every)

    def get_timing(self) -> adpsgd_timing:
        return adpsgd_get_timing(self.ctx)

    def close(self) -> None:
        if getattr(self, "ctx", None):
            adpsgd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def write_sync_log(path: str, recs: np.ndarray, var: Optional[np.ndarray] = None) -> int:
    """Append one JSON line per sync record (t, p, S, C2, gamma, margin and, when
    given, the per-tensor variances) to `path`; returns the number written."""
    import json
    with open(path, "a") as f:
        for j, r in enumerate(recs):
            row = {"t": int(r["t"]), "p": int(r["p"]), "S": float(r["S"]), "C2": float(r["C2"]),
                   "gamma": float(r["gamma"]),
                   "margin": None if np.isnan(r["margin"]) else float(r["margin"])}
            if var is not None:
                row["var"] = [float(v) for v in var[j]]
            f.write(json.dumps(row) + "\n")
    return len(recs)
