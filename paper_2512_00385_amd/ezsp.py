"""Thin Python binding of the C ABI in ``include/ezsp.h`` (libezsp.so).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Tensors must already live on the current HIP device; outputs and
the workspace are allocated with torch on that device, and the call is
enqueued on torch's current stream.  There is no fallback: when the
library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libezsp.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_NONFINITE = -2
ERR_RANGE = -3
ERR_WORKSPACE = -4
ERR_DEVICE = -5
ERR_NOT_CONVERGED = -6
F_ENERGY = 1
F_LINK_ISOLATED = 2

ENTRY_POINTS = (
    "ezsp_knn_workspace_size", "ezsp_knn",
    "ezsp_partition_workspace_size", "ezsp_partition",
    "ezsp_partition_from_knn",
    "ezsp_component_stats_workspace_size", "ezsp_component_stats",
    "ezsp_status_string", "ezsp_last_error",
    "ezsp_profile_enable", "ezsp_profile_read", "ezsp_profile_only",
    "ezsp_grid_subsample_workspace_size", "ezsp_grid_subsample",
    "ezsp_edge_loss_workspace_size", "ezsp_edge_loss",
    "ezsp_purity_workspace_size", "ezsp_purity",
    "ezsp_embed_mlp", "ezsp_sync_status", "ezsp_knn_noalloc",
    "ezsp_knn_walk_stats",
    "ezsp_layer_norm", "ezsp_layer_norm_backward_workspace_size",
    "ezsp_layer_norm_backward",
    "ezsp_linear_workspace_size", "ezsp_linear",
    "ezsp_linear_backward_workspace_size", "ezsp_linear_backward",
    "ezsp_gated_ff_workspace_size", "ezsp_gated_ff",
    "ezsp_gated_ff_backward_workspace_size", "ezsp_gated_ff_backward",
    "ezsp_rms_norm", "ezsp_rms_norm_backward_workspace_size",
    "ezsp_rms_norm_backward", "ezsp_dropout",
    "ezsp_log_probs_workspace_size", "ezsp_log_probs",
    "ezsp_log_probs_backward",
    "ezsp_cross_attention_workspace_size", "ezsp_cross_attention",
    "ezsp_cross_attention_backward_workspace_size",
    "ezsp_cross_attention_backward",
)


class Params(ctypes.Structure):
    """Mirror of ezsp_params."""
    _fields_ = [("k", ctypes.c_int32), ("n_levels", ctypes.c_int32),
                ("lambdas", ctypes.c_void_p), ("min_size", ctypes.c_void_p),
                ("max_rounds", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class LossStats(ctypes.Structure):
    """Mirror of ezsp_loss_stats."""
    _fields_ = [("loss", ctypes.c_double), ("n_edges", ctypes.c_int64),
                ("n_intra", ctypes.c_int64), ("n_inter", ctypes.c_int64),
                ("n_intra_kept", ctypes.c_int64)]


class PurityStats(ctypes.Structure):
    """Mirror of ezsp_purity_stats."""
    _fields_ = [("miou", ctypes.c_double), ("purity", ctypes.c_double),
                ("n_present", ctypes.c_int64)]


class EzspError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str):
        super().__init__(f"{where}: {status_string(code)} ({code}): {detail}")
        self.code = code


_lib = None


def load() -> ctypes.CDLL:
    """Load libezsp.so (built by ``paper_2512_00385_amd/build.py``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with "
            "`python paper_2512_00385_amd/build.py` (or __graft_entry__.build())")
    lib = ctypes.CDLL(LIB_PATH)
    P, i32, i64, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                       ctypes.c_size_t)
    sig = {
        "ezsp_knn_workspace_size": (sz, [i64, i32]),
        "ezsp_knn": (ctypes.c_int, [P, i64, i32, P, P, P, sz, P]),
        "ezsp_partition_workspace_size": (sz, [i64, i32, P]),
        "ezsp_partition": (ctypes.c_int, [P, P, i64, i32, P, P, P, P, P, sz,
                                          P]),
        "ezsp_partition_from_knn": (ctypes.c_int, [P, P, i64, i32, P, P, P, P,
                                                   P, sz, P]),
        "ezsp_component_stats_workspace_size": (sz, [i64, i64, i32]),
        "ezsp_component_stats": (ctypes.c_int, [P, i64, i64, P, i32, P, P, P,
                                                P, P, sz, P]),
        "ezsp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "ezsp_last_error": (ctypes.c_char_p, []),
        "ezsp_profile_enable": (ctypes.c_int, [ctypes.c_int]),
        "ezsp_profile_read": (ctypes.c_int, [ctypes.c_char_p, P, P, P]),
        "ezsp_profile_only": (ctypes.c_int, [ctypes.c_char_p]),
        "ezsp_grid_subsample_workspace_size": (sz, [i64]),
        "ezsp_grid_subsample": (ctypes.c_int, [P, i64, ctypes.c_float, P, P,
                                               P, sz, P]),
        "ezsp_edge_loss_workspace_size": (sz, [i64, i32]),
        "ezsp_edge_loss": (ctypes.c_int, [P, i64, i32, P, i32, P, P,
                                          ctypes.c_double, ctypes.c_double,
                                          P, P, P, P, P, sz, P]),
        "ezsp_purity_workspace_size": (sz, [i64, i64, i32]),
        "ezsp_purity": (ctypes.c_int, [P, i64, i64, P, i32, P, P, P, P, sz,
                                       P]),
        "ezsp_embed_mlp": (ctypes.c_int, [P, i64, i32, i32, i32, P, P, P, P,
                                          P, P, P, P]),
        "ezsp_sync_status": (ctypes.c_int, [P, sz, P]),
        "ezsp_knn_noalloc": (ctypes.c_int, [P, i64, i32, P, P, P]),
        "ezsp_knn_walk_stats": (ctypes.c_int, [P, i64, i32, P, P, P, P, sz,
                                               P]),
        "ezsp_layer_norm": (ctypes.c_int, [P, i64, i32, i64, i32, P, P,
                                           ctypes.c_double, P, i64, i32, P,
                                           P, P]),
        "ezsp_layer_norm_backward_workspace_size": (sz, [i64, i32]),
        "ezsp_layer_norm_backward": (ctypes.c_int, [
            P, i64, i32, P, i64, i32, i64, i32, P, P, P, P, i64, P, i64, P, P,
            P, sz, P]),
        "ezsp_linear_workspace_size": (sz, [i64, i32, i32]),
        "ezsp_linear": (ctypes.c_int, [P, i64, i64, i32, i32, i32, P, P, i32,
                                       P, i64, P, i64, i32, P, i64, P, sz,
                                       P]),
        "ezsp_linear_backward_workspace_size": (sz, [i64, i32, i32, i32]),
        "ezsp_linear_backward": (ctypes.c_int, [
            P, i64, i32, P, i64, i64, i32, i32, i32, P, P, i64, i32, P, i64,
            P, P, P, sz, P]),
        "ezsp_gated_ff_workspace_size": (sz, [i64, i32, i32]),
        "ezsp_gated_ff": (ctypes.c_int, [P, i64, i64, i32, i32, i32, P, P, P,
                                         P, i32, P, i64, P, P, i64, P, sz,
                                         P]),
        "ezsp_gated_ff_backward_workspace_size": (sz, [i64, i32, i32, i32]),
        "ezsp_gated_ff_backward": (ctypes.c_int, [
            P, i64, P, i64, i64, i32, i32, i32, P, P, P, P, i64, i32, P, i64,
            P, P, P, P, P, sz, P]),
        "ezsp_rms_norm": (ctypes.c_int, [
            P, i64, i32, i64, i32, P, i64, P, i64, i32, P, ctypes.c_double, P,
            i64, i32, P, P, P]),
        "ezsp_rms_norm_backward_workspace_size": (sz, [i64, i32]),
        "ezsp_rms_norm_backward": (ctypes.c_int, [
            P, i64, i32, P, i64, i32, i64, i32, P, P, P, i64, P, i64, P, P,
            sz, P]),
        "ezsp_dropout": (ctypes.c_int, [
            P, i64, i32, i64, i32, ctypes.c_double, ctypes.c_uint64,
            ctypes.c_uint64, P, P, i64, P, i64, i32, P]),
        "ezsp_log_probs_workspace_size": (sz, [i64, i32, i32]),
        "ezsp_log_probs": (ctypes.c_int, [
            P, i64, i32, i64, i32, P, P, P, P, i32, P, P, P, sz, P]),
        "ezsp_log_probs_backward": (ctypes.c_int, [
            P, P, P, i64, i32, i64, i32, P, P, P, P, i64, P]),
        "ezsp_cross_attention_workspace_size": (sz, [i64, i64, i32, i32,
                                                     i32]),
        "ezsp_cross_attention": (ctypes.c_int, [
            P, i64, i64, P, i64, P, i64, i64, i32, i32, i32, i32, P, P, i64,
            P, ctypes.c_double, P, i64, P, P, sz, P]),
        "ezsp_cross_attention_backward_workspace_size": (sz, [
            i64, i64, i32, i32, i32]),
        "ezsp_cross_attention_backward": (ctypes.c_int, [
            P, i64, P, i64, i64, P, i64, P, i64, i64, P, i64, P, i32, i32,
            i32, i32, P, P, i64, P, ctypes.c_double, P, i64, P, i64, P, i64,
            P, sz, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().ezsp_status_string(int(code)).decode()


def last_error() -> str:
    return load().ezsp_last_error().decode()


def profile_enable(on: bool = True):
    """Start (clearing the totals) or stop per-stage event timing."""
    load().ezsp_profile_enable(1 if on else 0)


def profile_only(stage=None):
    """Time only `stage` (None: every stage) while profiling is on."""
    load().ezsp_profile_only(stage.encode() if stage else None)


STAGES = ("morton_sort", "knn_query", "graph_build", "select", "union",
          "stats", "contract", "compose", "tail", "link")
EXTRA_STAGES = ("grid_subsample", "edge_loss", "purity", "embed_mlp",
                "layer_norm", "linear", "gated_ff", "rms_norm",
                "dropout", "log_probs", "cross_attention")


def profile_read(stage: str):
    """(launches, total milliseconds, algorithmic bytes) of a stage."""
    n = ctypes.c_int64(0)
    ms = ctypes.c_double(0.0)
    nb = ctypes.c_double(0.0)
    load().ezsp_profile_read(stage.encode(), ctypes.byref(n), ctypes.byref(ms),
                             ctypes.byref(nb))
    return int(n.value), float(ms.value), float(nb.value)


def _check(code: int, where: str):
    if code != OK:
        raise EzspError(code, where, last_error())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dev_tensor(t, dtype, name, cols=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if cols is not None and (t.dim() != 2 or t.shape[1] != cols):
        raise ValueError(f"{name} must have shape [n, {cols}]")
    return t.contiguous()


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _workspace(nbytes: int, device):
    if nbytes == 0:
        raise EzspError(ERR_INVALID_ARG, "workspace size", "invalid sizes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _params(k, lambdas, min_size, max_rounds, energy, link=False):
    lam = np.ascontiguousarray(np.atleast_1d(np.asarray(lambdas, np.float64)))
    ms = None
    if min_size is not None:
        ms = np.ascontiguousarray(np.atleast_1d(np.asarray(min_size,
                                                           np.int64)))
        if ms.shape != lam.shape:
            raise ValueError("min_size needs one value per level")
    p = Params(int(k), int(lam.shape[0]), lam.ctypes.data,
               None if ms is None else ms.ctypes.data, int(max_rounds),
               (F_ENERGY if energy else 0) | (F_LINK_ISOLATED if link else 0))
    return p, lam, ms  # keep the arrays alive with the struct


class Pending:
    """The workspace of a stream-asynchronous call, kept alive until its
    device-detected errors have been checked (ezsp_sync_status)."""

    def __init__(self, ws, nbytes, device, where):
        self.ws, self.nbytes, self.device, self.where = ws, nbytes, device, where

    def check(self):
        """Synchronise the stream; raise EzspError for a device error."""
        _check(load().ezsp_sync_status(_ptr(self.ws), self.nbytes,
                                       _stream(self.device)), self.where)


def knn(xyz: torch.Tensor, k: int, want_d2: bool = False, sync: bool = True):
    """Exact kNN (ezsp_knn): nbr [n, k] int32 (and d2 [n, k] fp32).  With
    sync=False the call returns right after enqueuing, with a Pending whose
    check() reports device errors: (nbr, [d2,] pending)."""
    lib = load()
    xyz = _dev_tensor(xyz, torch.float32, "xyz", 3)
    n = xyz.shape[0]
    dev = xyz.device
    nbr = torch.empty((n, k), dtype=torch.int32, device=dev)
    d2 = torch.empty((n, k), dtype=torch.float32, device=dev) \
        if want_d2 else None
    nbytes = lib.ezsp_knn_workspace_size(n, k)
    ws = _workspace(nbytes, dev)
    _check(lib.ezsp_knn(_ptr(xyz), n, int(k), _ptr(nbr), _ptr(d2), _ptr(ws),
                        nbytes, _stream(dev)), "ezsp_knn")
    pending = Pending(ws, nbytes, dev, "ezsp_knn")
    if sync:
        pending.check()
        return (nbr, d2) if want_d2 else nbr
    return ((nbr, d2) if want_d2 else (nbr,)) + (pending,)


def knn_walk_stats(xyz: torch.Tensor, k: int):
    """ezsp_knn_walk_stats: (nbr [n, k] int32, 16-point buckets scanned and
    inner nodes entered per 64-point query group, each [ceil(n / 64)]
    int32)."""
    lib = load()
    xyz = _dev_tensor(xyz, torch.float32, "xyz", 3)
    n = xyz.shape[0]
    dev = xyz.device
    g = (n + 63) // 64
    nbr = torch.empty((n, k), dtype=torch.int32, device=dev)
    scans = torch.empty(g, dtype=torch.int32, device=dev)
    nodes = torch.empty(g, dtype=torch.int32, device=dev)
    nbytes = lib.ezsp_knn_workspace_size(n, k)
    ws = _workspace(nbytes, dev)
    _check(lib.ezsp_knn_walk_stats(_ptr(xyz), n, int(k), _ptr(nbr),
                                   _ptr(scans), _ptr(nodes), _ptr(ws), nbytes,
                                   _stream(dev)), "ezsp_knn_walk_stats")
    Pending(ws, nbytes, dev, "ezsp_knn_walk_stats").check()
    return nbr, scans, nodes


def partition_workspace_size(n: int, d: int, k: int, n_levels: int = 1):
    p, _, _ = _params(k, [0.0] * n_levels, None, 0, False)
    return load().ezsp_partition_workspace_size(n, d, ctypes.byref(p))


class Partitioner:
    """Reusable call state for ezsp_partition: the workspace is allocated
    once, so repeated calls on the same sizes allocate nothing new."""

    def __init__(self, n: int, d: int, k: int, lambdas, min_size=None,
                 max_rounds: int = 0, energy: bool = False, device=None,
                 link: bool = False):
        self.lib = load()
        self.n, self.d, self.k = int(n), int(d), int(k)
        self.device = torch.device(device or "cuda")
        self.params, self._lam, self._ms = _params(k, lambdas, min_size,
                                                   max_rounds, energy, link)
        self.L = int(self._lam.shape[0])
        self.nbytes = self.lib.ezsp_partition_workspace_size(
            self.n, self.d, ctypes.byref(self.params))
        self.ws = _workspace(self.nbytes, self.device)
        self.labels = torch.empty((self.L, self.n), dtype=torch.int32,
                                  device=self.device)
        self.n_comp = np.zeros(self.L, np.int64)
        self.energy = np.zeros(self.L, np.float64) if energy else None

    def __call__(self, xyz: torch.Tensor, emb: torch.Tensor):
        xyz = _dev_tensor(xyz, torch.float32, "xyz", 3)
        emb = _dev_tensor(emb, torch.float32, "emb", self.d)
        if xyz.shape[0] != self.n or emb.shape[0] != self.n:
            raise ValueError("xyz/emb do not have n rows")
        rc = self.lib.ezsp_partition(
            _ptr(xyz), _ptr(emb), self.n, self.d, ctypes.byref(self.params),
            _ptr(self.labels), self.n_comp.ctypes.data,
            None if self.energy is None else self.energy.ctypes.data,
            _ptr(self.ws), self.nbytes, _stream(self.device))
        _check(rc, "ezsp_partition")
        return self.labels, self.n_comp.copy(), \
            None if self.energy is None else self.energy.copy()


def partition(xyz: torch.Tensor, emb: torch.Tensor, k: int, lambdas,
              min_size=None, max_rounds: int = 0, energy: bool = False,
              link: bool = False):
    """kNN graph + merge ladder (ezsp_partition); link: prepare_graph's
    linking of isolated nodes (EZSP_F_LINK_ISOLATED).

    Returns (labels [L, n] int32 on the device, n_comp int64 numpy [L],
    energy float64 numpy [L] or None)."""
    emb = _dev_tensor(emb, torch.float32, "emb")
    if emb.dim() != 2:
        raise ValueError("emb must have shape [n, d]")
    part = Partitioner(xyz.shape[0], emb.shape[1], k, lambdas, min_size,
                       max_rounds, energy, xyz.device, link)
    labels, nc, en = part(xyz, emb)
    return labels, nc, en


def partition_from_knn(nbr: torch.Tensor, emb: torch.Tensor, lambdas,
                       min_size=None, max_rounds: int = 0,
                       energy: bool = False):
    """Merge ladder on a given neighbour table (ezsp_partition_from_knn)."""
    lib = load()
    nbr = _dev_tensor(nbr, torch.int32, "nbr")
    emb = _dev_tensor(emb, torch.float32, "emb")
    if nbr.dim() != 2 or emb.dim() != 2 or nbr.shape[0] != emb.shape[0]:
        raise ValueError("nbr [n, k] and emb [n, d] needed")
    n, k = nbr.shape
    d = emb.shape[1]
    dev = emb.device
    p, lam, ms = _params(k, lambdas, min_size, max_rounds, energy)
    L = lam.shape[0]
    # from_knn needs no kNN scratch; the xyz query is an upper bound
    nbytes = lib.ezsp_partition_workspace_size(n, d, ctypes.byref(p))
    ws = _workspace(nbytes, dev)
    labels = torch.empty((L, n), dtype=torch.int32, device=dev)
    n_comp = np.zeros(L, np.int64)
    en = np.zeros(L, np.float64) if energy else None
    rc = lib.ezsp_partition_from_knn(
        _ptr(nbr), _ptr(emb), n, d, ctypes.byref(p), _ptr(labels),
        n_comp.ctypes.data, None if en is None else en.ctypes.data, _ptr(ws),
        nbytes, _stream(dev))
    _check(rc, "ezsp_partition_from_knn")
    return labels, n_comp, en


def component_stats(labels: torch.Tensor, n_comp: int, emb: torch.Tensor,
                    xyz: torch.Tensor | None = None, sync: bool = True):
    """Size, mean embedding and centroid per superpoint.  With sync=False
    the call returns right after enqueuing: (size, mean, centroid,
    pending), pending.check() reporting device errors."""
    lib = load()
    labels = _dev_tensor(labels, torch.int32, "labels")
    emb = _dev_tensor(emb, torch.float32, "emb")
    n, d = emb.shape
    dev = emb.device
    if xyz is not None:
        xyz = _dev_tensor(xyz, torch.float32, "xyz", 3)
    size = torch.empty(n_comp, dtype=torch.int64, device=dev)
    mean = torch.empty((n_comp, d), dtype=torch.float32, device=dev)
    cen = torch.empty((n_comp, 3), dtype=torch.float32, device=dev) \
        if xyz is not None else None
    nbytes = lib.ezsp_component_stats_workspace_size(n, int(n_comp), d)
    ws = _workspace(nbytes, dev)
    _check(lib.ezsp_component_stats(_ptr(labels), n, int(n_comp), _ptr(emb),
                                    d, _ptr(xyz), _ptr(size), _ptr(mean),
                                    _ptr(cen), _ptr(ws), nbytes,
                                    _stream(dev)), "ezsp_component_stats")
    pending = Pending(ws, nbytes, dev, "ezsp_component_stats")
    if sync:
        pending.check()
        return size, mean, cen
    return size, mean, cen, pending


def grid_subsample(xyz: torch.Tensor, h: float) -> torch.Tensor:
    """Indices (increasing, int32) of the point kept in every occupied cell
    of a regular grid of spacing h: the cell's smallest point index."""
    lib = load()
    xyz = _dev_tensor(xyz, torch.float32, "xyz", 3)
    n = xyz.shape[0]
    keep = torch.empty(n, dtype=torch.int32, device=xyz.device)
    n_keep = ctypes.c_int64(0)
    nbytes = lib.ezsp_grid_subsample_workspace_size(n)
    ws = _workspace(nbytes, xyz.device)
    _check(lib.ezsp_grid_subsample(_ptr(xyz), n, float(h), _ptr(keep),
                                   ctypes.byref(n_keep), _ptr(ws), nbytes,
                                   _stream(xyz.device)),
           "ezsp_grid_subsample")
    return keep[:n_keep.value]


def edge_loss(emb: torch.Tensor, nbr: torch.Tensor, cls: torch.Tensor,
              word: torch.Tensor, tau: float, rho: float,
              want_affinity: bool = True, want_grad: bool = True,
              want_sampled: bool = True):
    """Affinity and contrastive edge loss over the kNN pairs.  Returns
    (stats dict, affinity [n,k] fp32 or None, grad [n,d] fp32 or None,
    sampled [n,k] uint8 or None)."""
    lib = load()
    emb = _dev_tensor(emb, torch.float32, "emb")
    n, d = emb.shape
    nbr = _dev_tensor(nbr, torch.int32, "nbr")
    if nbr.dim() != 2 or nbr.shape[0] != n:
        raise ValueError("nbr must have shape [n, k]")
    k = nbr.shape[1]
    cls = _dev_tensor(cls, torch.int32, "cls")
    if isinstance(word, torch.Tensor) and word.dtype == torch.uint32:
        word = word.view(torch.int32)
    word = _dev_tensor(word, torch.int32, "word (uint32 or its int32 bits)")
    if cls.shape != (n,) or word.shape != (n, k):
        raise ValueError("cls must be [n] and word [n, k]")
    dev = emb.device
    aff = torch.empty((n, k), dtype=torch.float32, device=dev) \
        if want_affinity else None
    grad = torch.empty((n, d), dtype=torch.float32, device=dev) \
        if want_grad else None
    smp = torch.empty((n, k), dtype=torch.uint8, device=dev) \
        if want_sampled else None
    out = LossStats()
    nbytes = lib.ezsp_edge_loss_workspace_size(n, k)
    ws = _workspace(nbytes, dev)
    _check(lib.ezsp_edge_loss(_ptr(emb), n, d, _ptr(nbr), k, _ptr(cls),
                              _ptr(word), float(tau), float(rho), _ptr(aff),
                              _ptr(grad), _ptr(smp), ctypes.byref(out),
                              _ptr(ws), nbytes, _stream(dev)),
           "ezsp_edge_loss")
    stats = {f: getattr(out, f) for f, _ in LossStats._fields_}
    return stats, aff, grad, smp


def purity(labels: torch.Tensor, n_comp: int, cls: torch.Tensor, n_cls: int):
    """Majority class per superpoint, per-class IoU, mIoU and purity.
    Returns (stats dict, majority [n_comp] int32, iou [n_cls] fp64)."""
    lib = load()
    labels = _dev_tensor(labels, torch.int32, "labels")
    cls = _dev_tensor(cls, torch.int32, "cls")
    n = labels.shape[0]
    if cls.shape != labels.shape:
        raise ValueError("labels and cls must have the same shape")
    dev = labels.device
    maj = torch.empty(int(n_comp), dtype=torch.int32, device=dev)
    iou = torch.empty(int(n_cls), dtype=torch.float64, device=dev)
    out = PurityStats()
    nbytes = lib.ezsp_purity_workspace_size(n, int(n_comp), int(n_cls))
    ws = _workspace(nbytes, dev)
    _check(lib.ezsp_purity(_ptr(labels), n, int(n_comp), _ptr(cls),
                           int(n_cls), _ptr(maj), _ptr(iou), ctypes.byref(out),
                           _ptr(ws), nbytes, _stream(dev)), "ezsp_purity")
    stats = {f: getattr(out, f) for f, _ in PurityStats._fields_}
    return stats, maj, iou


def embed_mlp(x_bits: torch.Tensor, w1, b1, w2, b2, w3, b3) -> torch.Tensor:
    """Per-point MLP d_in -> 32 -> 32 -> d_out on the matrix cores.  x_bits
    and the weights are bfloat16 tensors (or int16 tensors of their bits) on
    the device, weights as [fan_in, fan_out]; biases fp32.  Returns
    [n, d_out] fp32, computed in stream order (the call does not wait)."""
    lib = load()

    def bits(t, name):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
        if t.dtype == torch.bfloat16:
            t = t.view(torch.int16)
        if t.dtype != torch.int16:
            raise TypeError(f"{name} must be bfloat16 (or its int16 bits)")
        return t.contiguous()
    x = bits(x_bits, "x")
    w1, w2, w3 = bits(w1, "w1"), bits(w2, "w2"), bits(w3, "w3")
    b1 = _dev_tensor(b1, torch.float32, "b1")
    b2 = _dev_tensor(b2, torch.float32, "b2")
    b3 = _dev_tensor(b3, torch.float32, "b3")
    n, d_in = x.shape
    d_hid, d_out = w1.shape[1], w3.shape[1]
    if w1.shape[0] != d_in or w2.shape != (d_hid, d_hid) or \
            w3.shape[0] != d_hid:
        raise ValueError("weight shapes do not chain")
    out = torch.empty((n, d_out), dtype=torch.float32, device=x.device)
    _check(lib.ezsp_embed_mlp(_ptr(x), n, d_in, d_hid, d_out, _ptr(w1),
                              _ptr(b1), _ptr(w2), _ptr(b2), _ptr(w3),
                              _ptr(b3), _ptr(out), _stream(x.device)),
           "ezsp_embed_mlp")
    return out


# ---- dense operators of a trainable embedding network ---------------------
#
# Results lie outside torch's automatic differentiation, whether or not an
# input requires gradients: the gradients are those of the *_backward calls.

TYPE_CODES = {torch.bfloat16: 0, torch.float32: 1}
ACT_CODES = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _elsewhere(t, name, index):
    """Raises for a t that is not a tensor on device `index` (None: any)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    raise ValueError(f"{name} must be on device {index} as x, is on "
                     f"{t.get_device()}")


def _rows(t, name, index=None, shape=None, dtype=None):
    """A [n, d] tensor on a device (`index`, if given) whose rows are
    contiguous (columns of a wider table stay as they are, other orders are
    copied) and the distance between its rows."""
    if not isinstance(t, torch.Tensor) or \
            (not t.is_cuda if index is None else t.get_device() != index):
        _elsewhere(t, name, index)
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dtype not in TYPE_CODES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have shape [n, d]")
    n, d = t.shape
    if shape is not None and (n, d) != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got "
                         f"{list(t.shape)}")
    ld, one = t.stride()
    if (one != 1 and d > 1) or (ld < d and n > 1):
        t = t.contiguous()
        ld = d
    return t, max(ld, d)


def _vector(t, d, name, index):
    """A contiguous fp32 vector of d values on device `index`, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        _elsewhere(t, name, index)
    if t.dtype != torch.float32:
        raise TypeError(f"{name} must be torch.float32, got {t.dtype}")
    if t.shape != (d,):
        raise ValueError(f"{name} must have shape [{d}]")
    return t.contiguous()


def _at(t):
    return None if t is None else t.data_ptr()


# The calls below may take less time on the GPU than their arguments on the
# host, so their sizes are queried once each, the device and the stream are
# read without torch's objects, and what follows a call is in line.
@functools.lru_cache(maxsize=4096)
def _dense_bytes(name: str, *sizes) -> int:
    nbytes = getattr(load(), name)(*sizes)
    if nbytes == 0:
        raise EzspError(ERR_INVALID_ARG, "workspace size", "invalid sizes")
    return nbytes


def _dense_ws(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or \
    torch.cuda.current_device


def _on(index, fn):
    """fn, called with device `index` made the current one: a default stream
    is the current device's, whatever device it was asked of."""
    def call(*args):
        with torch.cuda.device(index):
            return fn(*args)
    return call


def layer_norm(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-5,
               out_dtype=None, want_stats: bool = False):
    """Layer norm over each row of x [n, d] (ezsp_layer_norm), bfloat16 or
    fp32, weight and bias [d] fp32 or None; y has out_dtype (x's by
    default).  Returns y, or with want_stats (y, mean [n], rstd [n]) for
    layer_norm_backward, which is where gradients come from: torch's own
    differentiation stops here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d = x.shape
    index = x.get_device()
    weight = _vector(weight, d, "weight", index)
    bias = _vector(bias, d, "bias", index)
    out_dtype = out_dtype or x.dtype
    if out_dtype not in TYPE_CODES:
        raise TypeError("out_dtype must be bfloat16 or float32")
    y = torch.empty((n, d), dtype=out_dtype, device=x.device)
    mean = rstd = None
    if want_stats:
        mean = torch.empty(n, dtype=torch.float32, device=x.device)
        rstd = torch.empty(n, dtype=torch.float32, device=x.device)
    fn = lib.ezsp_layer_norm if index == _current_device() else \
        _on(index, lib.ezsp_layer_norm)
    rc = fn(
        x.data_ptr(), ldx, TYPE_CODES[x.dtype], n, d, _at(weight), _at(bias),
        float(eps), y.data_ptr(), d, TYPE_CODES[out_dtype], _at(mean),
        _at(rstd), _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_layer_norm")
    return (y, mean, rstd) if want_stats else y


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor,
                        mean: torch.Tensor, rstd: torch.Tensor, weight=None,
                        dres=None, want_dx: bool = True,
                        want_sums: bool = True):
    """Gradients of layer_norm (ezsp_layer_norm_backward): (dx [n, d] of x's
    type, dweight [d], dbias [d] fp32), each None where it is not wanted.
    dres [n, d], of x's type, is added to dx."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d = x.shape
    index = x.get_device()
    dy, lddy = _rows(dy, "dy", index, (n, d))
    mean = _vector(mean, n, "mean", index)
    rstd = _vector(rstd, n, "rstd", index)
    weight = _vector(weight, d, "weight", index)
    lddres = 0
    if dres is not None:
        dres, lddres = _rows(dres, "dres", index, (n, d), x.dtype)
    dev = x.device
    dx = torch.empty((n, d), dtype=x.dtype, device=dev) if want_dx else None
    dw = db = None
    if want_sums:
        dw = torch.empty(d, dtype=torch.float32, device=dev)
        db = torch.empty(d, dtype=torch.float32, device=dev)
    nbytes = _dense_bytes("ezsp_layer_norm_backward_workspace_size", n, d)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_layer_norm_backward if index == _current_device() else \
        _on(index, lib.ezsp_layer_norm_backward)
    rc = fn(
        dy.data_ptr(), lddy, TYPE_CODES[dy.dtype], x.data_ptr(), ldx,
        TYPE_CODES[x.dtype], n, d, _at(weight), _at(mean), _at(rstd),
        _at(dres), lddres, _at(dx), d, _at(dw), _at(db), ws.data_ptr(),
        nbytes, _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_layer_norm_backward")
    return dx, dw, db


def _weight(t, d_in, dtype, name, index, d_out=None):
    """A contiguous matrix [d_in, d_out] of the given type on device
    `index`."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        _elsewhere(t, name, index)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or t.shape[0] != d_in or \
            (d_out is not None and t.shape[1] != d_out):
        raise ValueError(f"{name} must have shape [{d_in}, "
                         f"{'d_out' if d_out is None else d_out}]")
    return t.contiguous()


def _act(act):
    if act not in ACT_CODES:
        raise ValueError(f"act must be one of {sorted(ACT_CODES)}")
    return ACT_CODES[act]


def linear(x: torch.Tensor, w: torch.Tensor, bias=None, act: str = "none",
           residual=None, out_dtype=None, want_z: bool = False):
    """y = act(x w + bias) + residual (ezsp_linear): x [n, d_in] and
    w [d_in, d_out] bfloat16 or fp32, bias [d_out] fp32, residual [n, d_out]
    of y's type, which is out_dtype (x's by default, or fp32).  act: none,
    relu, gelu, silu.  Returns y, or with want_z (y, x w + bias) for
    linear_backward, which is where gradients come from: torch's own
    differentiation stops here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d_in = x.shape
    ty, dev, index = x.dtype, x.device, x.get_device()
    w = _weight(w, d_in, ty, "w", index)
    d_out = w.shape[1]
    code = _act(act)
    bias = _vector(bias, d_out, "bias", index)
    out_dtype = out_dtype or ty
    if out_dtype not in (ty, torch.float32):
        raise TypeError("out_dtype must be x's type or float32")
    ldr = 0
    if residual is not None:
        residual, ldr = _rows(residual, "residual", index, (n, d_out),
                              out_dtype)
    y = torch.empty((n, d_out), dtype=out_dtype, device=dev)
    z = torch.empty((n, d_out), dtype=ty, device=dev) if want_z else None
    nbytes = _dense_bytes("ezsp_linear_workspace_size", n, d_in, d_out)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_linear if index == _current_device() else \
        _on(index, lib.ezsp_linear)
    rc = fn(
        x.data_ptr(), ldx, n, d_in, d_out, TYPE_CODES[ty], w.data_ptr(),
        _at(bias), code, _at(residual), ldr, y.data_ptr(), d_out,
        TYPE_CODES[out_dtype], _at(z), d_out, ws.data_ptr(), nbytes,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_linear")
    return (y, z) if want_z else y


def linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor,
                    z=None, act: str = "none", want_dx: bool = True,
                    want_dw: bool = True, want_db: bool = True):
    """Gradients of linear (ezsp_linear_backward): (dx, dw of x's type,
    dbias fp32), each None where it is not wanted.  dy [n, d_out] has x's
    type or fp32; z is linear's second result (not needed without an
    activation).  With bfloat16, dx and dw take dy act'(z) rounded to it."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d_in = x.shape
    ty, dev, index = x.dtype, x.device, x.get_device()
    w = _weight(w, d_in, ty, "w", index)
    d_out = w.shape[1]
    code = _act(act)
    dy, lddy = _rows(dy, "dy", index, (n, d_out))
    ldz = 0
    if z is not None:
        z, ldz = _rows(z, "z", index, (n, d_out), ty)
    dx = torch.empty((n, d_in), dtype=ty, device=dev) if want_dx else None
    dw = torch.empty((d_in, d_out), dtype=ty, device=dev) if want_dw else None
    db = torch.empty(d_out, dtype=torch.float32, device=dev) \
        if want_db else None
    nbytes = _dense_bytes("ezsp_linear_backward_workspace_size", n, d_in,
                          d_out, TYPE_CODES[ty])
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_linear_backward if index == _current_device() else \
        _on(index, lib.ezsp_linear_backward)
    rc = fn(
        dy.data_ptr(), lddy, TYPE_CODES[dy.dtype], x.data_ptr(), ldx, n, d_in,
        d_out, TYPE_CODES[ty], w.data_ptr(), _at(z), ldz, code, _at(dx), d_in,
        _at(dw), _at(db), ws.data_ptr(), nbytes,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_linear_backward")
    return dx, dw, db


def gated_ff(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
             b_gate=None, b_up=None, act: str = "silu",
             want_saved: bool = False):
    """h = act(x w_gate + b_gate) * (x w_up + b_up) in one kernel
    (ezsp_gated_ff): x [n, d_in], weights [d_in, d_out], bfloat16 or fp32,
    biases [d_out] fp32 or None.  Returns h, or with want_saved (h, gate,
    up), the two sums that gated_ff_backward reads; gradients come from it,
    torch's own differentiation stops here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d_in = x.shape
    ty, dev, index = x.dtype, x.device, x.get_device()
    w_gate = _weight(w_gate, d_in, ty, "w_gate", index)
    d_out = w_gate.shape[1]
    w_up = _weight(w_up, d_in, ty, "w_up", index, d_out)
    code = _act(act)
    b_gate = _vector(b_gate, d_out, "b_gate", index)
    b_up = _vector(b_up, d_out, "b_up", index)
    h = torch.empty((n, d_out), dtype=ty, device=dev)
    gate = up = None
    if want_saved:
        gate, up = torch.empty_like(h), torch.empty_like(h)
    nbytes = _dense_bytes("ezsp_gated_ff_workspace_size", n, d_in, d_out)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_gated_ff if index == _current_device() else \
        _on(index, lib.ezsp_gated_ff)
    rc = fn(
        x.data_ptr(), ldx, n, d_in, d_out, TYPE_CODES[ty], w_gate.data_ptr(),
        _at(b_gate), w_up.data_ptr(), _at(b_up), code, h.data_ptr(), d_out,
        _at(gate), _at(up), d_out, ws.data_ptr(), nbytes,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_gated_ff")
    return (h, gate, up) if want_saved else h


def gated_ff_backward(dh: torch.Tensor, x: torch.Tensor,
                      w_gate: torch.Tensor, w_up: torch.Tensor,
                      gate: torch.Tensor, up: torch.Tensor,
                      act: str = "silu", want_dx: bool = True,
                      want_dw: bool = True, want_db: bool = True):
    """Gradients of gated_ff (ezsp_gated_ff_backward): (dx, dw_gate, dw_up of
    x's type, db_gate, db_up fp32), None where not wanted; gate and up are
    gated_ff's saved sums.  With bfloat16, dx, dw_gate and dw_up take the
    gradients of gate and up rounded to it."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d_in = x.shape
    ty, dev, index = x.dtype, x.device, x.get_device()
    w_gate = _weight(w_gate, d_in, ty, "w_gate", index)
    d_out = w_gate.shape[1]
    w_up = _weight(w_up, d_in, ty, "w_up", index, d_out)
    code = _act(act)
    dh, lddh = _rows(dh, "dh", index, (n, d_out), ty)
    gate, lds = _rows(gate, "gate", index, (n, d_out), ty)
    up, lds_up = _rows(up, "up", index, (n, d_out), ty)
    if lds != lds_up:
        gate, up, lds = gate.contiguous(), up.contiguous(), d_out
    dx = torch.empty((n, d_in), dtype=ty, device=dev) if want_dx else None
    dwg = dwu = dbg = dbu = None
    if want_dw:
        dwg, dwu = torch.empty_like(w_gate), torch.empty_like(w_up)
    if want_db:
        dbg = torch.empty(d_out, dtype=torch.float32, device=dev)
        dbu = torch.empty(d_out, dtype=torch.float32, device=dev)
    nbytes = _dense_bytes("ezsp_gated_ff_backward_workspace_size", n, d_in,
                          d_out, TYPE_CODES[ty])
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_gated_ff_backward if index == _current_device() else \
        _on(index, lib.ezsp_gated_ff_backward)
    rc = fn(
        dh.data_ptr(), lddh, x.data_ptr(), ldx, n, d_in, d_out,
        TYPE_CODES[ty], w_gate.data_ptr(), w_up.data_ptr(), gate.data_ptr(),
        up.data_ptr(), lds, code, _at(dx), d_in, _at(dwg), _at(dwu),
        _at(dbg), _at(dbu), ws.data_ptr(), nbytes,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_gated_ff_backward")
    return dx, dwg, dwu, dbg, dbu


# ---- operators of a trainable network of attention blocks ------------------

E4M3 = torch.float8_e4m3fn
RESULT_CODES = {**TYPE_CODES, E4M3: 2}


def rms_norm(x: torch.Tensor, weight=None, residual=None, eps: float = 1e-5,
             out_dtype=None, want_rstd: bool = False):
    """Root-mean-square norm over each row of x + residual (ezsp_rms_norm):
    x [n, d] bfloat16 or fp32, residual of the same shape in x's type or fp32
    or None, weight [d] fp32 or None; y has out_dtype (x's by default),
    bfloat16, fp32 or float8_e4m3fn.  Returns y, or a tuple of y and what the
    call asks for besides, in this order: with float8 the scale [n] of each
    row (y stands for y * scale), with a residual the sum x + residual [n, d]
    of the residual's type, with want_rstd rstd [n] for rms_norm_backward,
    which is where gradients come from: torch's own differentiation stops
    here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d = x.shape
    dev, index = x.device, x.get_device()
    weight = _vector(weight, d, "weight", index)
    out_dtype = out_dtype or x.dtype
    if out_dtype not in RESULT_CODES:
        raise TypeError("out_dtype must be bfloat16, float32 or float8_e4m3fn")
    stream = x.dtype
    total = None
    ldr = 0
    if residual is not None:
        residual, ldr = _rows(residual, "residual", index, (n, d))
        stream = residual.dtype
        if stream not in (x.dtype, torch.float32):
            raise TypeError("residual must have x's type or float32")
        total = torch.empty((n, d), dtype=stream, device=dev)
    y = torch.empty((n, d), dtype=out_dtype, device=dev)
    scale = torch.empty(n, dtype=torch.float32, device=dev) \
        if out_dtype == E4M3 else None
    rstd = torch.empty(n, dtype=torch.float32, device=dev) \
        if want_rstd else None
    fn = lib.ezsp_rms_norm if index == _current_device() else \
        _on(index, lib.ezsp_rms_norm)
    rc = fn(
        x.data_ptr(), ldx, TYPE_CODES[x.dtype], n, d, _at(residual), ldr,
        _at(total), d, TYPE_CODES[stream], _at(weight), float(eps),
        y.data_ptr(), d, RESULT_CODES[out_dtype], _at(scale), _at(rstd),
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_rms_norm")
    more = tuple(t for t in (scale, total, rstd) if t is not None)
    return (y, *more) if more else y


def rms_norm_backward(dy: torch.Tensor, x: torch.Tensor, rstd: torch.Tensor,
                      weight=None, dres=None, want_dx: bool = True,
                      want_dweight: bool = True):
    """Gradients of rms_norm (ezsp_rms_norm_backward): (dx [n, d] of x's type,
    dweight [d] fp32), each None where it is not wanted.  x is what was
    normalised: rms_norm's sum where it had a residual, whose gradient dx is
    too.  dres [n, d], of x's type, is added to dx."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d = x.shape
    index = x.get_device()
    dy, lddy = _rows(dy, "dy", index, (n, d))
    rstd = _vector(rstd, n, "rstd", index)
    weight = _vector(weight, d, "weight", index)
    lddres = 0
    if dres is not None:
        dres, lddres = _rows(dres, "dres", index, (n, d), x.dtype)
    dev = x.device
    dx = torch.empty((n, d), dtype=x.dtype, device=dev) if want_dx else None
    dw = torch.empty(d, dtype=torch.float32, device=dev) \
        if want_dweight else None
    nbytes = _dense_bytes("ezsp_rms_norm_backward_workspace_size", n, d)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_rms_norm_backward if index == _current_device() else \
        _on(index, lib.ezsp_rms_norm_backward)
    rc = fn(
        dy.data_ptr(), lddy, TYPE_CODES[dy.dtype], x.data_ptr(), ldx,
        TYPE_CODES[x.dtype], n, d, _at(weight), _at(rstd), _at(dres), lddres,
        _at(dx), d, _at(dw), ws.data_ptr(), nbytes, _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_rms_norm_backward")
    return dx, dw


def dropout(x: torch.Tensor, p: float, seed: int, offset=0, residual=None,
            out_dtype=None, step=None):
    """residual + dropout(x) (ezsp_dropout): each element of x [n, d],
    bfloat16 or fp32, is dropped with probability p (in steps of 2^-16) or
    scaled by 1 / (1 - p); the mask comes from (seed, offset, element) alone
    and is not stored.  seed and offset are whole numbers below 2^64; step,
    an int64 tensor of one element on the device, is added to offset when the
    kernel runs, so that replays of a captured graph can draw anew.  The
    result, and the residual [n, d], have out_dtype (x's by default, or
    fp32).  Gradients come from dropout_backward: torch's own differentiation
    stops here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, d = x.shape
    index = x.get_device()
    out_dtype = out_dtype or x.dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise TypeError("out_dtype must be x's type or float32")
    if not 0 <= seed < 1 << 64 or not 0 <= offset < 1 << 64:
        raise ValueError("seed and offset must be in [0, 2^64)")
    ldr = 0
    if residual is not None:
        residual, ldr = _rows(residual, "residual", index, (n, d), out_dtype)
    if step is not None:
        if not isinstance(step, torch.Tensor) or step.get_device() != index:
            _elsewhere(step, "step", index)
        if step.dtype != torch.int64 or step.numel() != 1:
            raise TypeError("step must be one torch.int64")
    y = torch.empty((n, d), dtype=out_dtype, device=x.device)
    fn = lib.ezsp_dropout if index == _current_device() else \
        _on(index, lib.ezsp_dropout)
    rc = fn(
        x.data_ptr(), ldx, TYPE_CODES[x.dtype], n, d, float(p), seed, offset,
        _at(step), _at(residual), ldr, y.data_ptr(), d, TYPE_CODES[out_dtype],
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_dropout")
    return y


def dropout_backward(dy: torch.Tensor, p: float, seed: int, offset=0,
                     out_dtype=None, step=None):
    """Gradient of dropout with respect to x: the mask of the same p, seed,
    offset and step, applied to dy.  (The residual's gradient is dy.)"""
    return dropout(dy, p, seed, offset, None, out_dtype, step)


def _ids(t, n, index):
    """A contiguous int32 vector of n classes on device `index`, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        _elsewhere(t, "ids", index)
    if t.dtype != torch.int32:
        raise TypeError(f"ids must be torch.int32, got {t.dtype}")
    if t.shape != (n,):
        raise ValueError(f"ids must have shape [{n}]")
    return t.contiguous()


def log_probs(x: torch.Tensor, ids=None, top: int = 0,
              want_entropy: bool = False):
    """Log probabilities under the softmax of each row of scores x [n, v],
    bfloat16 or fp32 (ezsp_log_probs).  Returns a tuple, all fp32 but the
    classes: with ids [n] int32 the log probability of each row's class (0
    where ids is outside [0, v)), always lse [n], with want_entropy the
    entropy [n], with top the classes [n, top] int32 of the largest scores
    and their log probabilities.  Gradients come from log_probs_backward:
    torch's own differentiation stops here.  Computed in stream order."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, v = x.shape
    dev, index = x.device, x.get_device()
    ids = _ids(ids, n, index)
    f32 = torch.float32
    logp = None if ids is None else torch.empty(n, dtype=f32, device=dev)
    lse = torch.empty(n, dtype=f32, device=dev)
    ent = torch.empty(n, dtype=f32, device=dev) if want_entropy else None
    top_ids = top_logp = None
    if top > 0:
        top_ids = torch.empty((n, top), dtype=torch.int32, device=dev)
        top_logp = torch.empty((n, top), dtype=f32, device=dev)
    nbytes = _dense_bytes("ezsp_log_probs_workspace_size", n, v, top)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_log_probs if index == _current_device() else \
        _on(index, lib.ezsp_log_probs)
    rc = fn(
        x.data_ptr(), ldx, TYPE_CODES[x.dtype], n, v, _at(ids), _at(logp),
        lse.data_ptr(), _at(ent), top, _at(top_ids), _at(top_logp),
        ws.data_ptr(), nbytes, _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_log_probs")
    return tuple(t for t in (logp, lse, ent, top_ids, top_logp)
                 if t is not None)


def log_probs_backward(dlogp, x: torch.Tensor, ids, lse: torch.Tensor,
                       entropy=None, dentropy=None):
    """Gradient of log_probs with respect to the scores
    (ezsp_log_probs_backward): dx [n, v] of x's type, from the gradients
    dlogp [n] of the classes' log probabilities and dentropy [n] of the
    entropy, fp32, either None; ids, lse and entropy as log_probs took and
    gave them."""
    lib = load()
    x, ldx = _rows(x, "x")
    n, v = x.shape
    index = x.get_device()
    dlogp = _vector(dlogp, n, "dlogp", index)
    ids = _ids(ids, n, index) if dlogp is not None else None
    lse = _vector(lse, n, "lse", index)
    dentropy = _vector(dentropy, n, "dentropy", index)
    entropy = _vector(entropy, n, "entropy", index) \
        if dentropy is not None else None
    dx = torch.empty((n, v), dtype=x.dtype, device=x.device)
    fn = lib.ezsp_log_probs_backward if index == _current_device() else \
        _on(index, lib.ezsp_log_probs_backward)
    rc = fn(
        _at(dlogp), _at(ids), x.data_ptr(), ldx, TYPE_CODES[x.dtype], n, v,
        _at(lse), _at(entropy), _at(dentropy), dx.data_ptr(), v,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_log_probs_backward")
    return dx


def _offsets(q_offsets, k_offsets, index):
    """Both arrays of a batch's offsets, int32 on device `index`, and the
    number of its clouds; (None, None, 0) without."""
    if q_offsets is None and k_offsets is None:
        return None, None, 0
    for t, name in ((q_offsets, "q_offsets"), (k_offsets, "k_offsets")):
        if not isinstance(t, torch.Tensor) or t.get_device() != index:
            _elsewhere(t, name, index)
        if t.dtype != torch.int32:
            raise TypeError(f"{name} must be torch.int32, got {t.dtype}")
    if q_offsets.dim() != 1 or q_offsets.shape != k_offsets.shape or \
            q_offsets.shape[0] < 2:
        raise ValueError("q_offsets and k_offsets must both have shape "
                         "[clouds + 1]")
    return q_offsets.contiguous(), k_offsets.contiguous(), \
        q_offsets.shape[0] - 1


def _attention_args(q, k, v, heads, kv_heads, scale):
    kv_heads = heads if kv_heads is None else kv_heads
    q, ldq = _rows(q, "q")
    index = q.get_device()
    nq, width = q.shape
    if heads < 1 or kv_heads < 1 or heads % kv_heads or width % heads:
        raise ValueError("q must have heads * d_head columns, heads a "
                         "multiple of kv_heads")
    dh = width // heads
    k, ldk = _rows(k, "k", index, dtype=q.dtype)
    if k.shape[1] != kv_heads * dh:
        raise ValueError(f"k must have {kv_heads * dh} columns")
    v, ldv = _rows(v, "v", index, tuple(k.shape), q.dtype)
    scale = dh ** -0.5 if scale is None else float(scale)
    return q, ldq, k, ldk, v, ldv, kv_heads, nq, k.shape[0], dh, index, scale


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                    heads: int, kv_heads=None, q_offsets=None, k_offsets=None,
                    key_bias=None, scale=None, want_lse: bool = False):
    """Attention of the rows of q [nq, heads * d] to those of k and v
    [nk, kv_heads * d], bfloat16 or fp32 (ezsp_cross_attention), d at most
    128; kv_heads is heads by default, else a divisor of it.  q_offsets and
    k_offsets [clouds + 1] int32, on the device, confine the rows of each
    cloud to its own keys; key_bias [nk] fp32 is added to the scores of each
    key, -inf masks it, and has no gradient; scale, from 2^-16 to 2^16, is
    d ** -0.5 by default.  Returns out
    [nq, heads * d], 0 for a row without keys, or with want_lse (out, lse
    [heads, nq] fp32) for cross_attention_backward, which is where gradients
    come from: torch's own differentiation stops here.  Computed in stream
    order."""
    lib = load()
    q, ldq, k, ldk, v, ldv, kv_heads, nq, nk, dh, index, scale = \
        _attention_args(q, k, v, heads, kv_heads, scale)
    q_offsets, k_offsets, clouds = _offsets(q_offsets, k_offsets, index)
    key_bias = _vector(key_bias, nk, "key_bias", index)
    dev = q.device
    out = torch.empty((nq, heads * dh), dtype=q.dtype, device=dev)
    lse = torch.empty((heads, nq), dtype=torch.float32, device=dev) \
        if want_lse else None
    nbytes = _dense_bytes("ezsp_cross_attention_workspace_size", nq, nk,
                          heads, kv_heads, dh)
    ws = _dense_ws(nbytes, dev)
    fn = lib.ezsp_cross_attention if index == _current_device() else \
        _on(index, lib.ezsp_cross_attention)
    rc = fn(
        q.data_ptr(), ldq, nq, k.data_ptr(), ldk, v.data_ptr(), ldv, nk,
        heads, kv_heads, dh, TYPE_CODES[q.dtype], _at(q_offsets),
        _at(k_offsets), clouds, _at(key_bias), scale, out.data_ptr(),
        heads * dh, _at(lse), ws.data_ptr(), nbytes, _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_cross_attention")
    return (out, lse) if want_lse else out


def cross_attention_backward(dout: torch.Tensor, q: torch.Tensor,
                             k: torch.Tensor, v: torch.Tensor,
                             out: torch.Tensor, lse: torch.Tensor, heads: int,
                             kv_heads=None, q_offsets=None, k_offsets=None,
                             key_bias=None, scale=None, want_dq: bool = True,
                             want_dkv: bool = True):
    """Gradients of cross_attention (ezsp_cross_attention_backward): (dq, dk,
    dv) of the inputs' type and shapes, None where not wanted; out and lse as
    cross_attention gave them, the other arguments as it took them."""
    lib = load()
    q, ldq, k, ldk, v, ldv, kv_heads, nq, nk, dh, index, scale = \
        _attention_args(q, k, v, heads, kv_heads, scale)
    q_offsets, k_offsets, clouds = _offsets(q_offsets, k_offsets, index)
    key_bias = _vector(key_bias, nk, "key_bias", index)
    dout, lddo = _rows(dout, "dout", index, tuple(q.shape), q.dtype)
    out, ldo = _rows(out, "out", index, tuple(q.shape), q.dtype)
    if not isinstance(lse, torch.Tensor) or lse.get_device() != index:
        _elsewhere(lse, "lse", index)
    if lse.dtype != torch.float32 or lse.shape != (heads, nq):
        raise ValueError(f"lse must be float32 of shape [{heads}, {nq}]")
    lse = lse.contiguous()
    dq = torch.empty((nq, heads * dh), dtype=q.dtype, device=q.device) \
        if want_dq else None
    dk = dv = None
    if want_dkv:
        dk = torch.empty((nk, kv_heads * dh), dtype=q.dtype, device=q.device)
        dv = torch.empty_like(dk)
    nbytes = _dense_bytes("ezsp_cross_attention_backward_workspace_size", nq,
                          nk, heads, kv_heads, dh)
    ws = _dense_ws(nbytes, q.device)
    fn = lib.ezsp_cross_attention_backward if index == _current_device() \
        else _on(index, lib.ezsp_cross_attention_backward)
    rc = fn(
        dout.data_ptr(), lddo, q.data_ptr(), ldq, nq, k.data_ptr(), ldk,
        v.data_ptr(), ldv, nk, out.data_ptr(), ldo, lse.data_ptr(), heads,
        kv_heads, dh, TYPE_CODES[q.dtype], _at(q_offsets), _at(k_offsets),
        clouds, _at(key_bias), scale, _at(dq), heads * dh, _at(dk),
        kv_heads * dh, _at(dv), kv_heads * dh, ws.data_ptr(), nbytes,
        _raw_stream(index))
    if rc != OK:
        _check(rc, "ezsp_cross_attention_backward")
    return dq, dk, dv
