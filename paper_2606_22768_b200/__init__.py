"""B200-native Factored Gossip DiLoCo outer round: thin ctypes binding of ``libfgd.so``.

Argument marshalling only -- every step of the round runs in the library's CUDA kernels.
PyTorch is used by callers for device memory and streams; this module only reads
``data_ptr()`` / ``cuda_stream`` from what it is given.  There is no CPU fallback: importing
works anywhere (the host helpers are pure CPU), but the shared library must exist, and
every GPU entry point fails loudly when there is no CUDA device.

Entry points carry the C names (``fgd_outer_grad``, ``fgd_mix``, ``fgd_outer_step``,
``fgd_consensus_distance`` and the host helpers); see ``include/fgd.h`` for the contract.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass, field
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfgd.so")

FGD_MAX_K = 64
FGD_MAX_D = 8

FGD_OK = 0
FGD_ERR_INVALID_ARG = -1
FGD_ERR_ALIGNMENT = -2
FGD_ERR_ALIAS = -3
FGD_ERR_UNSUPPORTED = -4
FGD_ERR_CUDA = -5
FGD_ERR_TIMEOUT = -6

FGD_MIX_IDENTITY, FGD_MIX_MEAN, FGD_MIX_SPARSE, FGD_MIX_DENSE = 0, 1, 2, 3
FGD_RENORM_NONE, FGD_RENORM_SELF_ABSORB, FGD_RENORM_METROPOLIS = 0, 1, 2
FGD_PATH_AUTO, FGD_PATH_REGISTER, FGD_PATH_TMA, FGD_PATH_TMA_FP32 = 0, 1, 2, 3


class FgdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"fgd status {status}: {message}")
        self.status = status
        self.message = message


class _CMixDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("K", ctypes.c_int32), ("D", ctypes.c_int32),
                ("renorm", ctypes.c_int32), ("nbr", ctypes.c_void_p), ("w", ctypes.c_void_p),
                ("w_self", ctypes.c_void_p), ("edge_mask", ctypes.c_void_p), ("W", ctypes.c_void_p)]


# fgd_attn_args, fgd_block_norm_args and fgd_qk_rope_args as they lie in memory (native alignment).  Small calls are bound by what the host does per
# call; one pack costs a fraction of filling nested ctypes structures.
_ATTN_ARGS = struct.Struct("@4i 12q Qd 3qQ 9q")
_NORM_ARGS = struct.Struct("@2i 2q i4x 2d 28q 2q")
_ROPE_ARGS = struct.Struct("@2i q 6i q d 37q 2q")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2606_22768_b200/build.py` "
                          "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, dbl = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double
    descp = ctypes.POINTER(_CMixDesc)
    sig = {
        "fgd_create": (i32, [ctypes.POINTER(vp), i32, i32, i64, i64]),
        "fgd_destroy": (i32, [vp]),
        "fgd_last_error": (ctypes.c_char_p, [vp]),
        "fgd_status_string": (ctypes.c_char_p, [i32]),
        "fgd_launch_count": (i64, [vp]),
        "fgd_set_path": (i32, [vp, i32]),
        "fgd_device_status": (i32, [vp, vp]),
        "fgd_debug_set": (i32, [vp, i32, i64]),
        "fgd_debug_stream_pattern": (i32, [vp, vp, vp, vp, vp, vp]),
        "fgd_outer_grad": (i32, [vp, vp, vp, vp, vp]),
        "fgd_mix": (i32, [vp, descp, vp, vp, i32, vp]),
        "fgd_outer_step": (i32, [vp, descp, descp, vp, i32, vp, vp, vp, vp, dbl, dbl, vp, vp]),
        "fgd_outer_step_ex": (i32, [vp, descp, descp, vp, i32, vp, vp, vp, vp, dbl, dbl, vp, vp, vp]),
        "fgd_outer_step_from_host": (i32, [vp, descp, descp, vp, i32, vp, vp, vp, vp, vp, dbl, dbl, vp, i32, vp]),
        "fgd_consensus_distance": (i32, [vp, vp, vp, vp]),
        "fgd_consensus_distance_noalloc": (i32, [i32, i32, i64, i64, vp, vp, vp]),
        "fgd_js_distance": (i32, [i32, i32, i64, i64, i32, vp, vp, vp, vp, vp, vp]),
        "fgd_attn_plan_create": (i32, [ctypes.POINTER(vp), i32, i32, vp]),
        "fgd_attn_plan_destroy": (i32, [vp]),
        "fgd_attn_forward": (i32, [vp, vp, vp]),
        "fgd_attn_backward": (i32, [vp, vp, vp]),
        "fgd_attn_status": (i32, [vp, vp]),
        "fgd_attn_debug_set": (i32, [vp, i32, i64]),
        "fgd_block_norm_forward": (i32, [i32, vp, vp]),
        "fgd_block_norm_backward": (i32, [i32, vp, vp]),
        "fgd_block_norm_workspace": (i64, [i32, i32, i32, i64, i64]),
        "fgd_act_save8": (i32, [i32, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp]),
        "fgd_act_load8": (i32, [i32, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp]),
        "fgd_swiglu8_forward": (i32, [i32, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp]),
        "fgd_swiglu8_backward": (i32, [i32, i32, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp]),
        "fgd_qk_rope_forward": (i32, [i32, vp, vp]),
        "fgd_qk_rope_backward": (i32, [i32, vp, vp]),
        "fgd_qk_rope_workspace": (i64, [i32, i32, i32]),
        "fgd_embed_forward": (i32, [i32, i32, i32, i64, i64, i64, vp, i32, i64, vp, i64, i64, dbl, vp, i64, vp]),
        "fgd_embed_backward": (i32, [i32, i32, i32, i64, i64, i64, vp, i32, i64, vp, i64, dbl, vp, i64, i64, vp, i64, vp]),
        "fgd_embed_workspace": (i64, [i32, i64, i64, i64]),
        "fgd_dropout": (i32, [i32, i32, i64, i64, vp, i64, vp, i64, dbl, u64, u64, vp, vp]),
        "fgd_topo_ring": (i32, [i32, vp, vp, vp]),
        "fgd_topo_onepeer_xor": (i32, [i32, i64, vp, vp, vp]),
        "fgd_topo_hypercube": (i32, [i32, vp, vp, vp]),
        "fgd_topo_random_matching": (i32, [i32, u64, i64, i32, vp, vp, vp]),
        "fgd_edge_mask": (i32, [u64, i64, i32, dbl, i32, i32, vp, vp]),
        "fgd_hash64": (u64, [u64, u64, u64, u64, u64]),
        "fgd_effective_weights": (i32, [descp, vp, vp]),
        "fgd_dense_matrix": (i32, [descp, vp]),
        "fgd_cd_finalize": (i32, [vp, i32, ctypes.POINTER(dbl), ctypes.POINTER(dbl)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib, tuple(sig)


_lib, EXPORTED_SYMBOLS = _load()


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data


@dataclass
class MixDesc:
    """Host-side description of one mixing operator (mirrors ``fgd_mix_desc``)."""
    kind: int
    K: int
    D: int = 0
    renorm: int = FGD_RENORM_NONE
    nbr: Optional[np.ndarray] = None        # int32 [K, D]
    w: Optional[np.ndarray] = None          # float32 [K, D]
    w_self: Optional[np.ndarray] = None     # float32 [K]
    edge_mask: Optional[np.ndarray] = None  # uint8 [K, D]
    W: Optional[np.ndarray] = None          # float32 [K, K]
    _c: Optional[_CMixDesc] = field(default=None, repr=False, compare=False)

    def c(self) -> _CMixDesc:
        conv = lambda a, dt: None if a is None else np.ascontiguousarray(a, dtype=dt)
        self.nbr, self.w = conv(self.nbr, np.int32), conv(self.w, np.float32)
        self.w_self, self.edge_mask = conv(self.w_self, np.float32), conv(self.edge_mask, np.uint8)
        self.W = conv(self.W, np.float32)
        self._c = _CMixDesc(self.kind, self.K, self.D, self.renorm, _np_ptr(self.nbr), _np_ptr(self.w),
                            _np_ptr(self.w_self), _np_ptr(self.edge_mask), _np_ptr(self.W))
        return self._c

    # -- constructors -----------------------------------------------------------------
    @staticmethod
    def identity(K: int) -> "MixDesc":
        return MixDesc(FGD_MIX_IDENTITY, K)

    @staticmethod
    def mean(K: int) -> "MixDesc":
        return MixDesc(FGD_MIX_MEAN, K)

    @staticmethod
    def dense(W) -> "MixDesc":
        W = np.ascontiguousarray(W, dtype=np.float32)
        return MixDesc(FGD_MIX_DENSE, W.shape[0], W=W)

    @staticmethod
    def sparse(nbr, w, w_self, edge_mask=None, renorm: int = FGD_RENORM_NONE) -> "MixDesc":
        nbr = np.ascontiguousarray(nbr, dtype=np.int32)
        K = nbr.shape[0]
        D = nbr.shape[1] if nbr.ndim == 2 else 0
        return MixDesc(FGD_MIX_SPARSE, K, D, renorm, nbr, np.asarray(w, dtype=np.float32),
                       np.asarray(w_self, dtype=np.float32),
                       None if edge_mask is None else np.asarray(edge_mask, dtype=np.uint8))

    @staticmethod
    def _topo(fn, K, D, *args) -> "MixDesc":
        nbr = np.full((K, max(D, 1)), -1, dtype=np.int32)
        w = np.zeros((K, max(D, 1)), dtype=np.float32)
        ws = np.zeros(K, dtype=np.float32)
        rc = fn(K, *args, nbr.ctypes.data, w.ctypes.data, ws.ctypes.data)
        if rc < 0:
            raise FgdError(rc, fgd_last_error(None))
        return MixDesc(FGD_MIX_SPARSE, K, rc, FGD_RENORM_NONE, nbr[:, :rc].copy(), w[:, :rc].copy(), ws)

    @staticmethod
    def ring(K: int) -> "MixDesc":
        return MixDesc._topo(_lib.fgd_topo_ring, K, 2)

    @staticmethod
    def onepeer_xor(K: int, rnd: int) -> "MixDesc":
        return MixDesc._topo(_lib.fgd_topo_onepeer_xor, K, 1, rnd)

    @staticmethod
    def hypercube(K: int) -> "MixDesc":
        return MixDesc._topo(_lib.fgd_topo_hypercube, K, max(1, K.bit_length() - 1))

    @staticmethod
    def random_matching(K: int, seed: int, rnd: int, mix_id: int) -> "MixDesc":
        return MixDesc._topo(_lib.fgd_topo_random_matching, K, 1, seed, rnd, mix_id)

    def with_failures(self, seed: int, rnd: int, mix_id: int, p_fail: float,
                      renorm: int = FGD_RENORM_METROPOLIS) -> "MixDesc":
        """Copy of a sparse descriptor with this round's Bernoulli edge mask attached."""
        mask = fgd_edge_mask(seed, rnd, mix_id, p_fail, self.nbr)
        return MixDesc(FGD_MIX_SPARSE, self.K, self.D, renorm, self.nbr, self.w, self.w_self, mask)


# ------------------------------------------------------------------------ host helpers
def fgd_last_error(ctx) -> str:
    h = ctx._h if isinstance(ctx, Context) else None
    return (_lib.fgd_last_error(h) or b"").decode()


def fgd_hash64(seed: int, rnd: int, tag: int, a: int, b: int) -> int:
    return int(_lib.fgd_hash64(seed, rnd, tag, a, b))


def fgd_edge_mask(seed: int, rnd: int, mix_id: int, p_fail: float, nbr) -> np.ndarray:
    nbr = np.ascontiguousarray(nbr, dtype=np.int32)
    K, D = nbr.shape
    mask = np.zeros((K, D), dtype=np.uint8)
    rc = _lib.fgd_edge_mask(seed, rnd, mix_id, float(p_fail), K, D, nbr.ctypes.data, mask.ctypes.data)
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))
    return mask


def fgd_effective_weights(desc: MixDesc):
    w_eff = np.zeros((desc.K, max(desc.D, 1)), dtype=np.float64)
    ws_eff = np.zeros(desc.K, dtype=np.float64)
    packed = np.zeros(desc.K * max(desc.D, 1), dtype=np.float64)
    rc = _lib.fgd_effective_weights(ctypes.byref(desc.c()), packed.ctypes.data, ws_eff.ctypes.data)
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))
    w_eff = packed[:desc.K * desc.D].reshape(desc.K, desc.D)
    return w_eff, ws_eff


def fgd_dense_matrix(desc: MixDesc) -> np.ndarray:
    W = np.zeros((desc.K, desc.K), dtype=np.float64)
    rc = _lib.fgd_dense_matrix(ctypes.byref(desc.c()), W.ctypes.data)
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))
    return W


def fgd_cd_finalize(sumsq):
    s = np.ascontiguousarray(sumsq, dtype=np.float64)
    a, b = ctypes.c_double(), ctypes.c_double()
    rc = _lib.fgd_cd_finalize(s.ctypes.data, s.shape[0], ctypes.byref(a), ctypes.byref(b))
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))
    return a.value, b.value


# ------------------------------------------------------------------------ GPU entry points
def _dev_ptr(t, name: str, dtype_name: str):
    if t is None:
        return None
    if not getattr(t, "is_cuda", False):
        raise TypeError(f"{name} must be a CUDA tensor")
    if str(t.dtype) != dtype_name:
        raise TypeError(f"{name} must be {dtype_name}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


class Context:
    """Owns one ``fgd_ctx``: fixed K, P, row stride ld and CUDA device."""

    def __init__(self, K: int, P: int, ld: Optional[int] = None, device: int = 0):
        self.K, self.P, self.ld, self.device = int(K), int(P), int(P if ld is None else ld), int(device)
        h = ctypes.c_void_p()
        rc = _lib.fgd_create(ctypes.byref(h), self.device, self.K, self.P, self.ld)
        if rc != 0:
            raise FgdError(rc, fgd_last_error(None))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            _lib.fgd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise FgdError(rc, fgd_last_error(self))

    @property
    def launch_count(self) -> int:
        return int(_lib.fgd_launch_count(self._h))


def fgd_set_path(ctx: Context, path: int) -> None:
    ctx._check(_lib.fgd_set_path(ctx._h, int(path)))


FGD_DEBUG_SPIN_LIMIT, FGD_DEBUG_SKIP_TILE, FGD_DEBUG_GOSSIP_PATH = 1, 2, 3


def fgd_debug_set(ctx: Context, key: int, value: int) -> None:
    """Test and measurement hooks: bounded device-side waits, fused-gossip kernel choice (see ``include/fgd.h``)."""
    ctx._check(_lib.fgd_debug_set(ctx._h, int(key), int(value)))


def fgd_debug_stream_pattern(ctx: Context, theta_local, theta_prev, momentum, theta_new, stream=None) -> None:
    """The fused step's HBM traffic without its arithmetic (a measurement aid, see ``include/fgd.h``)."""
    ctx._check(_lib.fgd_debug_stream_pattern(ctx._h, _dev_ptr(theta_local, "theta_local", "torch.float32"),
                                             _dev_ptr(theta_prev, "theta_prev", "torch.float32"),
                                             _dev_ptr(momentum, "momentum", "torch.float32"),
                                             _dev_ptr(theta_new, "theta_new", "torch.float32"), _stream(stream)))


def fgd_device_status(ctx: Context, stream=None) -> None:
    """Synchronises the stream; raises FgdError(FGD_ERR_TIMEOUT) if a device-side wait gave up."""
    ctx._check(_lib.fgd_device_status(ctx._h, _stream(stream)))


def fgd_outer_grad(ctx: Context, theta_prev, theta_local, g, stream=None) -> None:
    ctx._check(_lib.fgd_outer_grad(ctx._h, _dev_ptr(theta_prev, "theta_prev", "torch.float32"),
                                   _dev_ptr(theta_local, "theta_local", "torch.float32"),
                                   _dev_ptr(g, "g", "torch.float32"), _stream(stream)))


def fgd_mix(ctx: Context, desc: MixDesc, inp, out, out_is_vector: bool = False, stream=None) -> None:
    ctx._check(_lib.fgd_mix(ctx._h, ctypes.byref(desc.c()), _dev_ptr(inp, "in", "torch.float32"),
                            _dev_ptr(out, "out", "torch.float32"), int(bool(out_is_vector)), _stream(stream)))


def fgd_outer_step(ctx: Context, mix2: MixDesc, mix1_fused: Optional[MixDesc], x, x_is_vector: bool,
                   theta_local, theta_prev, momentum, theta_new, lr: float = 0.7, mu: float = 0.9,
                   cd_sumsq=None, stream=None) -> None:
    ctx._check(_lib.fgd_outer_step(
        ctx._h, ctypes.byref(mix2.c()), None if mix1_fused is None else ctypes.byref(mix1_fused.c()),
        _dev_ptr(x, "x", "torch.float32"), int(bool(x_is_vector)),
        _dev_ptr(theta_local, "theta_local", "torch.float32"),
        _dev_ptr(theta_prev, "theta_prev", "torch.float32"),
        _dev_ptr(momentum, "momentum", "torch.float32"),
        _dev_ptr(theta_new, "theta_new", "torch.float32"), float(lr), float(mu),
        _dev_ptr(cd_sumsq, "cd_sumsq", "torch.float64"), _stream(stream)))


class _CStepOptions(ctypes.Structure):
    _fields_ = [("mix2_ranges", ctypes.c_void_p), ("n_ranges", ctypes.c_int32), ("average_momentum", ctypes.c_int32),
                ("x_next", ctypes.c_void_p)]


def fgd_outer_step_ex(ctx: Context, mix2: MixDesc, mix1_fused: Optional[MixDesc], x, x_is_vector: bool,
                      theta_local, theta_prev, momentum, theta_new, lr: float = 0.7, mu: float = 0.9,
                      cd_sumsq=None, mix2_ranges=None, average_momentum: bool = False, x_next=None,
                      stream=None) -> None:
    """fgd_outer_step with the paper's two variants: Mix2 only inside the given (lo, hi) column
    ranges (the "-subset" configurations) and/or the momentum averaged first (GlobalM1S); with
    ``x_next`` ([P]) the kernel also writes the column mean of theta_new, i.e. next round's
    global-average Mix1 result."""
    ranges = None
    if mix2_ranges is not None:
        ranges = np.ascontiguousarray(np.asarray(mix2_ranges, dtype=np.int64).reshape(-1, 2))
    opts = _CStepOptions(None if ranges is None else ranges.ctypes.data, 0 if ranges is None else ranges.shape[0],
                         int(bool(average_momentum)), _dev_ptr(x_next, "x_next", "torch.float32"))
    ctx._check(_lib.fgd_outer_step_ex(
        ctx._h, ctypes.byref(mix2.c()), None if mix1_fused is None else ctypes.byref(mix1_fused.c()),
        _dev_ptr(x, "x", "torch.float32"), int(bool(x_is_vector)),
        _dev_ptr(theta_local, "theta_local", "torch.float32"),
        _dev_ptr(theta_prev, "theta_prev", "torch.float32"),
        _dev_ptr(momentum, "momentum", "torch.float32"),
        _dev_ptr(theta_new, "theta_new", "torch.float32"), float(lr), float(mu),
        _dev_ptr(cd_sumsq, "cd_sumsq", "torch.float64"), ctypes.byref(opts), _stream(stream)))


def fgd_outer_step_from_host(ctx: Context, mix2: MixDesc, mix1_fused: Optional[MixDesc], x, x_is_vector: bool,
                             theta_local_host, theta_local_dev, theta_prev, momentum, theta_new,
                             lr: float = 0.7, mu: float = 0.9, want_cd: bool = True, n_chunks: int = 8,
                             stream=None) -> Optional[np.ndarray]:
    """The outer step with theta_local arriving from HOST memory (a CPU tensor [K, ld], pinned for
    full copy bandwidth): copied chunk by chunk into ``theta_local_dev`` while the previous chunk's
    step runs.  With ``want_cd`` the call returns the consensus sums (float64 [K]) after the round
    has completed; without it returns None and is asynchronous."""
    if getattr(theta_local_host, "is_cuda", True) or str(theta_local_host.dtype) != "torch.float32":
        raise TypeError("theta_local_host must be a float32 CPU tensor")
    if theta_local_host.stride(-1) != 1 or (theta_local_host.dim() == 2 and theta_local_host.shape[0] > 1
                                             and theta_local_host.stride(0) != ctx.ld):
        raise ValueError("theta_local_host must be a [K, ld] matrix with the context's row stride")
    cd = np.empty(ctx.K, dtype=np.float64) if want_cd else None
    ctx._check(_lib.fgd_outer_step_from_host(
        ctx._h, ctypes.byref(mix2.c()), None if mix1_fused is None else ctypes.byref(mix1_fused.c()),
        _dev_ptr(x, "x", "torch.float32"), int(bool(x_is_vector)), theta_local_host.data_ptr(),
        _dev_ptr(theta_local_dev, "theta_local_dev", "torch.float32"),
        _dev_ptr(theta_prev, "theta_prev", "torch.float32"),
        _dev_ptr(momentum, "momentum", "torch.float32"),
        _dev_ptr(theta_new, "theta_new", "torch.float32"), float(lr), float(mu),
        None if cd is None else cd.ctypes.data, int(n_chunks), _stream(stream)))
    return cd


def fgd_consensus_distance(ctx: Context, theta, cd_sumsq, stream=None) -> None:
    ctx._check(_lib.fgd_consensus_distance(ctx._h, _dev_ptr(theta, "theta", "torch.float32"),
                                           _dev_ptr(cd_sumsq, "cd_sumsq", "torch.float64"), _stream(stream)))


def fgd_consensus_distance_noalloc(device: int, K: int, P: int, ld: int, theta, cd_sumsq, stream=None) -> None:
    """Consensus sums without a context and without any GPU allocation (for callers that may not
    allocate); partial sums go through a fixed array inside the library, shared by all calls, so
    calls on one GPU must not overlap.  See ``include/fgd.h``."""
    rc = _lib.fgd_consensus_distance_noalloc(int(device), int(K), int(P), int(ld),
                                             _dev_ptr(theta, "theta", "torch.float32"),
                                             _dev_ptr(cd_sumsq, "cd_sumsq", "torch.float64"), _stream(stream))
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))


def fgd_js_distance(worker_logits, avg_logits, top_idx, d_js, cd_worker, top_k: int = 100, device: int = 0,
                    stream=None) -> None:
    """JS functional disagreement of [K, U, V] worker logits against [U, V] averaged-model logits
    on the averaged model's top_k tokens; fills top_idx [U, top_k], d_js [K, U], cd_worker [K]."""
    K, U, V = worker_logits.shape
    rc = _lib.fgd_js_distance(int(device), int(K), int(U), int(V), int(top_k),
                              _dev_ptr(worker_logits, "worker_logits", "torch.float32"),
                              _dev_ptr(avg_logits, "avg_logits", "torch.float32"),
                              _dev_ptr(top_idx, "top_idx", "torch.int32"), _dev_ptr(d_js, "d_js", "torch.float64"),
                              _dev_ptr(cd_worker, "cd_worker", "torch.float64"), _stream(stream))
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))


# ------------------------------------------------------------------ operators of the inner step
FGD_F32, FGD_BF16, FGD_F16 = 0, 1, 2
FGD_GATE_NONE, FGD_GATE_CHANNEL, FGD_GATE_ELEMENT = 0, 1, 2
ACT8_GROUP = 32      # values that share one step in an 8-bit checkpoint


def _op_check(rc: int) -> None:
    if rc != 0:
        raise FgdError(rc, fgd_last_error(None))


def _types(torch):
    """Codes of the activation types, by torch type."""
    if not _types.codes:
        _types.codes = {torch.float32: FGD_F32, torch.bfloat16: FGD_BF16, torch.float16: FGD_F16}
    return _types.codes


_types.codes = {}


def _dtype_of(t, name: str) -> int:
    import torch
    code = _types(torch).get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _refuse(t, name: str, dtype, shape, device) -> None:
    """Why a tensor is not what it has to be."""
    if not getattr(t, "is_cuda", False):
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    raise ValueError(f"{name} must be contiguous along its last dimension")


def _stream_on(stream, device):
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the handle without a Stream object around it (2 us of a small call)
        return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _as_current(stream, handle, device):
    """Context in which torch allocates and works on the stream of a call: the argument as it was given (None: the current one), its handle."""
    import torch
    if stream is not None and not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _scratch(size: int, stream, handle, device):
    """Workspace of a call: from the memory of the stream that uses it.  A block of another stream's may have uses on that stream still to come before
    this call, and would need to be kept from others until after it."""
    import torch
    if stream is None:
        return torch.empty(max(size, 1), dtype=torch.uint8, device=device)
    with _as_current(stream, handle, device):
        return torch.empty(max(size, 1), dtype=torch.uint8, device=device)


def _device_of(t, name: str):
    if not getattr(t, "is_cuda", False):
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.device


class AttnPlan:
    """A packing of sequences: sequence i holds the tokens cu_seqlens[i] .. cu_seqlens[i+1] - 1 (host values).
    Create one per batch; every layer's forward and backward use it."""

    def __init__(self, cu_seqlens, device: int = 0):
        cu = np.ascontiguousarray(cu_seqlens, dtype=np.int64)
        if cu.ndim != 1 or cu.size < 1:
            raise ValueError("cu_seqlens must hold n_seqs + 1 values")
        h = ctypes.c_void_p()
        self._h = None
        _op_check(_lib.fgd_attn_plan_create(ctypes.byref(h), int(device), int(cu.size) - 1, cu.ctypes.data))
        self._h, self.device, self.tokens, self.n_seqs = h, int(device), int(cu[-1]), int(cu.size) - 1

    def close(self):
        if getattr(self, "_h", None):
            _lib.fgd_attn_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fgd_attn_status(plan: AttnPlan, stream=None) -> None:
    """Synchronises the stream (None: the current one of the plan's device); raises FgdError(FGD_ERR_TIMEOUT) if a device-side wait of a
    kernel of this plan gave up."""
    import torch
    _op_check(_lib.fgd_attn_status(plan._h, _stream_on(stream, torch.device("cuda", plan.device))))


def fgd_attn_debug_set(plan: AttnPlan, key: int, value: int) -> None:
    """Test hooks for the bounded device-side waits of the attention kernels (see ``include/fgd.h``)."""
    _op_check(_lib.fgd_attn_debug_set(plan._h, int(key), int(value)))


def _heads(t, name: str, dtype, shape, device):
    """(pointer, token stride, head stride)"""
    if t.dtype != dtype or t.shape != shape or t.device != device:
        _refuse(t, name, dtype, shape, device)
    token, head, last = t.stride()
    if last != 1 and shape[2] > 1:
        _refuse(t, name, dtype, shape, device)
    return t.data_ptr(), token, head


def _row_values(t, name: str, shape, device):
    """Pointer of a contiguous fp32 [heads, tokens] tensor."""
    import torch
    if t.dtype != torch.float32 or t.shape != shape or t.device != device:
        _refuse(t, name, torch.float32, shape, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


_NO_HEADS = (0, 0, 0)


def _attn_shapes(plan, q, k):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q and k must be [tokens, heads, width]")
    dev, qs, ks = _device_of(q, "q"), q.shape, k.shape
    if qs[0] != plan.tokens:
        raise ValueError(f"q has {qs[0]} tokens, the plan {plan.tokens}")
    if dev.index != plan.device:
        raise ValueError(f"q is on {dev}, the plan on cuda:{plan.device}")
    return dev, qs, (qs[0], ks[1], qs[2]), (qs[1], qs[0])


def fgd_attn_forward(plan: AttnPlan, q, k, v, o, lse, scale: Optional[float] = None, stream=None) -> None:
    """Causal attention over the plan's packed sequences: q [T, Hq, d], k and v [T, Hk, d] -> o [T, Hq, d], lse [Hq, T] (fp32).
    Any token and head strides (slices of a fused projection); ``scale`` defaults to d ** -0.5."""
    dev, qs, ks, rows = _attn_shapes(plan, q, k)
    dt, d = q.dtype, qs[2]
    args = _ATTN_ARGS.pack(_dtype_of(q, "q"), qs[1], ks[1], d, *_heads(q, "q", dt, qs, dev), *_heads(k, "k", dt, ks, dev), *_heads(v, "v", dt, ks, dev),
                           *_heads(o, "o", dt, qs, dev), _row_values(lse, "lse", rows, dev), d ** -0.5 if scale is None else scale,
                           *_NO_HEADS, 0, *_NO_HEADS, *_NO_HEADS, *_NO_HEADS)
    _op_check(_lib.fgd_attn_forward(plan._h, args, _stream_on(stream, dev)))


def fgd_attn_backward(plan: AttnPlan, q, k, v, o, dout, lse, delta, dq, dk, dv, scale: Optional[float] = None, stream=None) -> None:
    """Gradients of :func:`fgd_attn_forward` from its inputs, o and lse.  ``delta`` [Hq, T] (fp32) is scratch; dk and dv are summed
    over the query heads that share a key head."""
    dev, qs, ks, rows = _attn_shapes(plan, q, k)
    dt, d = q.dtype, qs[2]
    args = _ATTN_ARGS.pack(_dtype_of(q, "q"), qs[1], ks[1], d, *_heads(q, "q", dt, qs, dev), *_heads(k, "k", dt, ks, dev), *_heads(v, "v", dt, ks, dev),
                           *_heads(o, "o", dt, qs, dev), _row_values(lse, "lse", rows, dev), d ** -0.5 if scale is None else scale,
                           *_heads(dout, "dout", dt, qs, dev), _row_values(delta, "delta", rows, dev),
                           *_heads(dq, "dq", dt, qs, dev), *_heads(dk, "dk", dt, ks, dev), *_heads(dv, "dv", dt, ks, dev))
    _op_check(_lib.fgd_attn_backward(plan._h, args, _stream_on(stream, dev)))


_NO_MAT = (0, 0)


def _mat(t, name: str, dtype, rows: int, width: int, device):
    """(pointer, row stride); (0, 0) for None"""
    if t is None:
        return _NO_MAT
    if t.dtype != dtype or t.shape != (rows, width) or t.device != device:
        _refuse(t, name, dtype, (rows, width), device)
    ld, last = t.stride()
    if last != 1 and width > 1:
        _refuse(t, name, dtype, (rows, width), device)
    return t.data_ptr(), ld if rows > 1 else max(ld, width)


def _norm_shapes(first, gate, w_post, w_pre):
    """device, rows, width, workers, gate kind and the type of the gate"""
    import torch
    if first is None or first.dim() != 2:
        raise ValueError("activations must be [tokens, width]")
    dev, (T, H) = _device_of(first, "activations"), first.shape
    channel = w_pre if w_pre is not None else w_post
    if channel is None and gate is not None and gate.dtype == torch.float32 and (gate.shape != first.shape or first.dtype != torch.float32):
        channel = gate      # (of 16-bit activations an fp32 gate is always one per channel)
    K = 1 if channel is None else channel.shape[0]
    if K < 1 or T % K != 0:
        raise ValueError(f"{T} rows do not split over {K} workers")
    if gate is None:
        return dev, T, H, K, FGD_GATE_NONE, torch.float32
    # [K, width] is a gate per channel, [T, width] one per element (one row per worker: the fp32 one counts as per channel)
    if gate.shape[0] == K and (K != T or gate.dtype == torch.float32):
        return dev, T, H, K, FGD_GATE_CHANNEL, torch.float32
    return dev, T, H, K, FGD_GATE_ELEMENT, first.dtype


def fgd_block_norm_forward(x, y, gate, w_post, w_pre, x_new, n, eps: float = 1e-5, res_scale: float = 1.0, stream=None) -> None:
    """x_new = x + res_scale * gate * norm(y) * w_post and n = norm(x_new) * w_pre, in one pass.  Activations [T, H]; w_post, w_pre
    [K, H] fp32 for K workers with T / K rows each; gate None, [K, H] fp32 (per channel) or [T, H] (per element).  w_post, y, n (with
    w_pre), x_new and gate may be None, see ``include/fgd.h``; x_new may be x."""
    import torch
    dev, T, H, K, kind, gate_type = _norm_shapes(x, gate, w_post, w_pre)
    dt, f32, gate_rows = x.dtype, torch.float32, K if kind == FGD_GATE_CHANNEL else T
    mats = (_mat(x, "x", dt, T, H, dev) + _mat(y, "y", dt, T, H, dev) + _mat(gate, "gate", gate_type, gate_rows, H, dev)
            + _mat(w_post, "w_post", f32, K, H, dev) + _mat(w_pre, "w_pre", f32, K, H, dev) + _mat(x_new, "x_new", dt, T, H, dev) + _mat(n, "n", dt, T, H, dev))
    if T == 0:
        return
    args = _NORM_ARGS.pack(_dtype_of(x, "x"), K, T // K, H, kind, eps, res_scale, *mats, *_NO_MAT * 7, 0, 0)
    _op_check(_lib.fgd_block_norm_forward(dev.index, args, _stream_on(stream, dev)))


def fgd_block_norm_workspace(dtype: int, workers: int, rows: int, width: int, device: int = 0) -> int:
    """Bytes of scratch that :func:`fgd_block_norm_backward` needs for ``rows`` rows per worker."""
    n = int(_lib.fgd_block_norm_workspace(int(device), int(dtype), int(workers), int(rows), int(width)))
    if n < 0:
        raise FgdError(n, "fgd_block_norm_workspace: argument out of range")
    return n


def fgd_block_norm_backward(dn, dres, x_new, y, gate, w_post, w_pre, dx, dy, dgate, dw_post, dw_pre, eps: float = 1e-5, res_scale: float = 1.0,
                            workspace=None, stream=None) -> None:
    """Gradients of :func:`fgd_block_norm_forward` from x_new and y as stored; dn is the gradient of n, dres that of x_new from elsewhere
    (None: zero; without dn, dw_pre becomes zero), dx may be dres.  ``workspace``: a uint8 CUDA tensor of :func:`fgd_block_norm_workspace` bytes (None: allocated here)."""
    import torch
    first = dn if dn is not None else dres
    dev, T, H, K, kind, gate_type = _norm_shapes(first, gate, w_post, w_pre)
    dt, f32, gate_rows = first.dtype, torch.float32, K if kind == FGD_GATE_CHANNEL else T
    mats = (_NO_MAT + _mat(y, "y", dt, T, H, dev) + _mat(gate, "gate", gate_type, gate_rows, H, dev) + _mat(w_post, "w_post", f32, K, H, dev)
            + _mat(w_pre, "w_pre", f32, K, H, dev) + _mat(x_new, "x_new", dt, T, H, dev) + _NO_MAT + _mat(dn, "dn", dt, T, H, dev)
            + _mat(dres, "dres", dt, T, H, dev) + _mat(dx, "dx", dt, T, H, dev) + _mat(dy, "dy", dt, T, H, dev) + _mat(dgate, "dgate", gate_type, gate_rows, H, dev)
            + _mat(dw_post, "dw_post", f32, K, H, dev) + _mat(dw_pre, "dw_pre", f32, K, H, dev))
    code, handle = _dtype_of(first, "activations"), _stream_on(stream, dev)
    if T == 0:
        with _as_current(stream, handle, dev):
            for g in (dw_post, dw_pre, dgate):
                if g is not None:
                    g.zero_()
        return
    if workspace is None:
        workspace = _scratch(fgd_block_norm_workspace(code, K, T // K, H, dev.index), stream, handle, dev)
    args = _NORM_ARGS.pack(code, K, T // K, H, kind, eps, res_scale, *mats, _dev_ptr(workspace, "workspace", "torch.uint8"), workspace.numel())
    _op_check(_lib.fgd_block_norm_backward(dev.index, args, handle))


def fgd_act_save8(x, q8, e8, stream=None) -> None:
    """x [rows, width] -> its 8-bit checkpoint q8 (int8 [rows, width]) and e8 (uint8 [rows, ceil(width / 32)])."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must be [rows, width]")
    (R, W), dev = x.shape, _device_of(x, "x")
    _op_check(_lib.fgd_act_save8(dev.index, _dtype_of(x, "x"), R, W, *_mat(x, "x", x.dtype, R, W, dev), *_mat(q8, "q8", torch.int8, R, W, dev),
                                 *_mat(e8, "e8", torch.uint8, R, -(-W // ACT8_GROUP), dev), _stream_on(stream, dev)))


def fgd_act_load8(q8, e8, out, stream=None) -> None:
    """The values an 8-bit checkpoint stands for, in out's type."""
    import torch
    if out.dim() != 2:
        raise ValueError("out must be [rows, width]")
    (R, W), dev = out.shape, _device_of(out, "out")
    _op_check(_lib.fgd_act_load8(dev.index, _dtype_of(out, "out"), R, W, *_mat(q8, "q8", torch.int8, R, W, dev),
                                 *_mat(e8, "e8", torch.uint8, R, -(-W // ACT8_GROUP), dev), *_mat(out, "out", out.dtype, R, W, dev), _stream_on(stream, dev)))


def fgd_swiglu8_forward(gu, h, q8, e8, stream=None) -> None:
    """h = silu(g) * u for gu = [g | u] ([rows, 2 width]) and the checkpoint of gu: q8 int8 [rows, 2 width], e8 uint8 [rows, 2 ceil(width / 32)]."""
    import torch
    if h.dim() != 2:
        raise ValueError("h must be [rows, width]")
    (R, W), dev = h.shape, _device_of(h, "h")
    _op_check(_lib.fgd_swiglu8_forward(dev.index, _dtype_of(h, "h"), R, W, *_mat(gu, "gu", h.dtype, R, 2 * W, dev), *_mat(h, "h", h.dtype, R, W, dev),
                                       *_mat(q8, "q8", torch.int8, R, 2 * W, dev), *_mat(e8, "e8", torch.uint8, R, 2 * -(-W // ACT8_GROUP), dev),
                                       _stream_on(stream, dev)))


def fgd_swiglu8_backward(dh, q8, e8, dgu, h=None, stream=None) -> None:
    """Gradient of :func:`fgd_swiglu8_forward` from the checkpoint alone; ``h``, where given, receives the recomputed h."""
    import torch
    if dh.dim() != 2:
        raise ValueError("dh must be [rows, width]")
    (R, W), dev = dh.shape, _device_of(dh, "dh")
    _op_check(_lib.fgd_swiglu8_backward(dev.index, _dtype_of(dh, "dh"), R, W, *_mat(dh, "dh", dh.dtype, R, W, dev),
                                        *_mat(q8, "q8", torch.int8, R, 2 * W, dev), *_mat(e8, "e8", torch.uint8, R, 2 * -(-W // ACT8_GROUP), dev),
                                        *_mat(dgu, "dgu", dh.dtype, R, 2 * W, dev), *_mat(h, "h", dh.dtype, R, W, dev), _stream_on(stream, dev)))


def _whole_numbers(t, name: str, shape, device):
    """Pointer and bytes of a contiguous-rowed int64 or int32 tensor."""
    import torch
    if t.dtype != torch.int64 and t.dtype != torch.int32:
        raise TypeError(f"{name} must be int64 or int32, got {t.dtype}")
    if t.shape != shape or t.device != device or (t.stride(-1) != 1 and shape[-1] > 1):
        _refuse(t, name, t.dtype, shape, device)
    return t.data_ptr(), t.element_size()


def _rope_shapes(q, k, w_q, w_k, cos):
    """device, query and key shapes, workers, (rows of the tables, half of the rotated width)"""
    if q.dim() != 3 or (k is not None and k.dim() != 3):
        raise ValueError("q and k must be [tokens, heads, width]")
    if cos.dim() != 2:
        raise ValueError("cos and sin must be [rows, rotated width / 2]")
    dev, qs = _device_of(q, "q"), q.shape
    ks = (qs[0], 0 if k is None else k.shape[1], qs[2])
    w = w_q if w_q is not None else w_k
    K = 1 if w is None else w.shape[0]
    if K < 1 or qs[0] % K != 0:
        raise ValueError(f"{qs[0]} tokens do not split over {K} workers")
    return dev, qs, ks, K, cos.shape


def _rope_pack(q, cos, sin, positions, w_q, w_k, eps, interleaved, shapes, heads, dw, workspace):
    import torch
    dev, qs, ks, K, (N, half) = shapes
    f32, d = torch.float32, qs[2]
    pos, pos_bytes = (0, 0) if positions is None else _whole_numbers(positions, "positions", (qs[0],), dev)
    return _ROPE_ARGS.pack(_dtype_of(q, "q"), K, qs[0] // K, qs[1], ks[1], d, 2 * half, int(interleaved), pos_bytes, N, eps, *_mat(cos, "cos", f32, N, half, dev),
                           *_mat(sin, "sin", f32, N, half, dev), pos, *_mat(w_q, "w_q", f32, K, d, dev), *_mat(w_k, "w_k", f32, K, d, dev), *heads,
                           *_mat(dw[0], "dw_q", f32, K, d, dev), *_mat(dw[1], "dw_k", f32, K, d, dev), *workspace)


_NO_ROPE_GRADS, _NO_ROPE_OUTPUTS = (0,) * 18, (0,) * 6


def _rope_usual(q, k, q_to, k_to, w_q, w_k, cos, sin, positions, eps, interleaved, x_q=None, x_k=None, dw_q=None, dw_k=None):
    """The arguments of a call as they usually are, checked; None where anything is not as usual: then the checks one by one say what is wrong, if it is.
    (Small calls are bound by what the host does: written out, this takes about 6 us of it where the checks one by one take 9.)  q, k go in and q_to, k_to come out,
    gradients in a backward pass; x_q, x_k and dw_q, dw_k are then its q, k and the gradients of the weights.  Calls without positions, as the decoder's, with weights
    of one side, without keys, and backward passes without weights are not among them."""
    import torch
    if k is None or positions is None or (w_q is None) is not (w_k is None):
        return None
    f32, dt, dev, qs, ks, table, pt, code = torch.float32, q.dtype, q.device, q.shape, k.shape, cos.shape, positions.dtype, _types.codes.get(q.dtype)
    if len(qs) != 3 or len(ks) != 3 or len(table) != 2 or code is None or dev.type != "cuda":
        return None
    (T, hq, d), hk, (rows, half) = qs, ks[1], table
    if (ks[0] != T or ks[2] != d or k.dtype is not dt or q_to.dtype is not dt or k_to.dtype is not dt or q_to.shape != qs or k_to.shape != ks or k.device != dev
            or q_to.device != dev or k_to.device != dev or cos.dtype is not f32 or sin.dtype is not f32 or sin.shape != table or cos.device != dev or sin.device != dev
            or positions.shape != (T,) or positions.device != dev or (pt is not torch.int64 and pt is not torch.int32)):
        return None
    (q0, q1, q2), (k0, k1, k2), (y0, y1, y2), (z0, z1, z2) = q.stride(), k.stride(), q_to.stride(), k_to.stride()
    (c0, c1), (s0, s1), (p0,) = cos.stride(), sin.stride(), positions.stride()
    if not (q2 == k2 == y2 == z2 == c1 == s1 == p0 == 1 and c0 >= half and s0 >= half):
        return None
    K, weights, inputs, grads = 1, (0, 0, 0, 0), (0, 0, 0, 0, 0, 0), (0, 0, 0, 0)
    if w_q is not None:
        ws = w_q.shape
        K = ws[0]
        if K < 1 or T % K or ws != (K, d) or w_k.shape != ws or w_q.dtype is not f32 or w_k.dtype is not f32 or w_q.device != dev or w_k.device != dev:
            return None
        (g0, g1), (h0, h1) = w_q.stride(), w_k.stride()
        if not (g1 == h1 == 1 and g0 >= d and h0 >= d):
            return None
        weights = w_q.data_ptr(), g0, w_k.data_ptr(), h0
        if dw_q is not None:
            if (x_q.dtype is not dt or x_k.dtype is not dt or x_q.shape != qs or x_k.shape != ks or x_q.device != dev or x_k.device != dev or dw_q.dtype is not f32
                    or dw_k.dtype is not f32 or dw_q.shape != ws or dw_k.shape != ws or dw_q.device != dev or dw_k.device != dev):
                return None
            (a0, a1, a2), (b0, b1, b2), (g0, g1), (h0, h1) = x_q.stride(), x_k.stride(), dw_q.stride(), dw_k.stride()
            if not (a2 == b2 == g1 == h1 == 1 and g0 >= d and h0 >= d):
                return None
            inputs, grads = (x_q.data_ptr(), a0, a1, x_k.data_ptr(), b0, b1), (dw_q.data_ptr(), g0, dw_k.data_ptr(), h0)
    head = (code, K, T // K, hq, hk, d, 2 * half, int(interleaved), 8 if pt is torch.int64 else 4, rows, eps, cos.data_ptr(), c0, sin.data_ptr(), s0,
            positions.data_ptr(), *weights)
    return dev, K, d, head, inputs, (q.data_ptr(), q0, q1, k.data_ptr(), k0, k1), (q_to.data_ptr(), y0, y1, k_to.data_ptr(), z0, z1), grads


def _key_heads(t, name: str, dtype, shape, device):
    if shape[1] == 0 and t is None:
        return _NO_HEADS
    return _heads(t, name, dtype, shape, device)


def fgd_qk_rope_forward(q, k, w_q, w_k, cos, sin, positions, q_out, k_out, eps: float = 1e-5, interleaved: bool = False, stream=None) -> None:
    """Queries [T, Hq, d] and keys [T, Hk, d] (None: no keys) normalised per head with w_q, w_k ([K, d] fp32 for K workers with T / K tokens each; None: not
    normalised) and rotated by rows ``positions`` ([T] int64 or int32; None: row t) of the tables cos and sin ([N, r / 2] fp32; the first r channels turn).
    Any token and head strides; q_out may be q, k_out k.  See ``include/fgd.h``."""
    usual = _rope_usual(q, k, q_out, k_out, w_q, w_k, cos, sin, positions, eps, interleaved)
    if usual is not None:
        dev, _, _, head, _, source, target, _ = usual
        _op_check(_lib.fgd_qk_rope_forward(dev.index, _ROPE_ARGS.pack(*head, *source, *target, *_NO_ROPE_GRADS), _stream_on(stream, dev)))
        return
    shapes = dev, qs, ks, _, _ = _rope_shapes(q, k, w_q, w_k, cos)
    dt = q.dtype
    heads = (*_heads(q, "q", dt, qs, dev), *_key_heads(k, "k", dt, ks, dev), *_heads(q_out, "q_out", dt, qs, dev), *_key_heads(k_out, "k_out", dt, ks, dev),
             *_NO_HEADS, *_NO_HEADS, *_NO_HEADS, *_NO_HEADS)
    args = _rope_pack(q, cos, sin, positions, w_q, w_k, eps, interleaved, shapes, heads, (None, None), _NO_MAT)
    _op_check(_lib.fgd_qk_rope_forward(dev.index, args, _stream_on(stream, dev)))


def fgd_qk_rope_workspace(workers: int, head_dim: int, device: int = 0) -> int:
    """Bytes of scratch that :func:`fgd_qk_rope_backward` needs where there are weights."""
    n = int(_lib.fgd_qk_rope_workspace(int(device), int(workers), int(head_dim)))
    if n < 0:
        raise FgdError(n, "fgd_qk_rope_workspace: argument out of range")
    return n


def fgd_qk_rope_backward(dq_out, dk_out, q, k, w_q, w_k, cos, sin, positions, dq, dk, dw_q, dw_k, eps: float = 1e-5, interleaved: bool = False,
                         workspace=None, stream=None) -> None:
    """Gradients of :func:`fgd_qk_rope_forward` from its inputs (q and k may be None where neither is normalised); dq may be dq_out, dk dk_out.
    ``workspace``: a uint8 CUDA tensor of :func:`fgd_qk_rope_workspace` bytes (None: allocated here)."""
    usual = None
    if w_q is not None and q is not None and k is not None and dw_q is not None and dw_k is not None:
        usual = _rope_usual(dq_out, dk_out, dq, dk, w_q, w_k, cos, sin, positions, eps, interleaved, q, k, dw_q, dw_k)
    if usual is not None:
        dev, K, d, head, inputs, source, target, grads = usual
        handle = _stream_on(stream, dev)
        if workspace is None:
            workspace = _scratch(fgd_qk_rope_workspace(K, d, dev.index), stream, handle, dev)
        args = _ROPE_ARGS.pack(*head, *inputs, *_NO_ROPE_OUTPUTS, *source, *target, *grads, _dev_ptr(workspace, "workspace", "torch.uint8"), workspace.numel())
        _op_check(_lib.fgd_qk_rope_backward(dev.index, args, handle))
        return
    shapes = dev, qs, ks, K, _ = _rope_shapes(dq_out, dk_out, w_q, w_k, cos)
    dt = dq_out.dtype
    heads = (*(_NO_HEADS if w_q is None else _heads(q, "q", dt, qs, dev)), *(_NO_HEADS if w_k is None else _key_heads(k, "k", dt, ks, dev)), *_NO_HEADS, *_NO_HEADS,
             *_heads(dq_out, "dq_out", dt, qs, dev), *_key_heads(dk_out, "dk_out", dt, ks, dev), *_heads(dq, "dq", dt, qs, dev), *_key_heads(dk, "dk", dt, ks, dev))
    handle = _stream_on(stream, dev)
    if workspace is None and (w_q is not None or w_k is not None):
        workspace = _scratch(fgd_qk_rope_workspace(K, qs[2], dev.index), stream, handle, dev)
    room = _NO_MAT if workspace is None else (_dev_ptr(workspace, "workspace", "torch.uint8"), workspace.numel())
    args = _rope_pack(dq_out, cos, sin, positions, w_q, w_k, eps, interleaved, shapes, heads, (dw_q, dw_k), room)
    _op_check(_lib.fgd_qk_rope_backward(dev.index, args, handle))


def _table(t, name: str, device):
    """(pointer, worker stride, row stride) of an fp32 [workers, vocabulary, width] tensor"""
    import torch
    if t.dim() != 3:
        raise ValueError(f"{name} must be [workers, vocabulary, width]")
    if t.dtype != torch.float32 or t.device != device or (t.stride(2) != 1 and t.shape[2] > 1):
        _refuse(t, name, torch.float32, t.shape, device)
    K, V, W = t.shape
    row = t.stride(1) if V > 1 else W
    return t.data_ptr(), t.stride(0) if K > 1 else V * row, row


def _embed_tokens(tokens, K, device):
    if tokens.dim() != 2 or tokens.shape[0] != K:
        raise ValueError(f"tokens must be [{K}, rows], got {tuple(tokens.shape)}")
    ptr, size = _whole_numbers(tokens, "tokens", tokens.shape, device)
    return ptr, size, tokens.stride(0) if K > 1 else max(tokens.shape[1], 1)


def _embed_usual(tokens, table, x):
    """As :func:`_rope_usual`: tokens [K, R], table [K, V, W], x [K * R, W] and their pointers and strides."""
    import torch
    ks, ts, dev, tt, code = table.shape, tokens.shape, x.device, tokens.dtype, _types.codes.get(x.dtype)
    if (len(ks) != 3 or len(ts) != 2 or code is None or dev.type != "cuda" or ts[0] != ks[0] or x.shape != (ts[0] * ts[1], ks[2]) or table.dtype is not torch.float32
            or table.device != dev or tokens.device != dev or (tt is not torch.int64 and tt is not torch.int32)):
        return None
    (s0, s1, s2), (t0, t1), (x0, x1) = table.stride(), tokens.stride(), x.stride()
    if not (s2 == t1 == x1 == 1 and s1 >= ks[2] and t0 >= ts[1] and x0 >= ks[2]):
        return None
    return (dev, code, ks, ts[1], (tokens.data_ptr(), 8 if tt is torch.int64 else 4, t0), (table.data_ptr(), s0 if ks[0] > 1 else ks[1] * s1, s1),
            (x.data_ptr(), x0))


def fgd_embed_forward(tokens, table, out, scale: float = 1.0, stream=None) -> None:
    """out[m * rows + i] = scale * table[m, tokens[m, i]]: tokens [K, rows] int64 or int32, table [K, V, W] fp32 (e.g. a column range of the parameter
    matrix), out [K * rows, W].  A token below 0 is padding: its row is zero."""
    usual = _embed_usual(tokens, table, out)
    if usual is not None:
        dev, code, (K, V, W), R, tok, tab, mat = usual
        _op_check(_lib.fgd_embed_forward(dev.index, code, K, R, V, W, *tok, *tab, scale, *mat, _stream_on(stream, dev)))
        return
    dev = _device_of(out, "out")
    if out.dim() != 2:
        raise ValueError("out must be [tokens, width]")
    tab, (K, V, W) = _table(table, "table", dev), table.shape
    tok = _embed_tokens(tokens, K, dev)
    _op_check(_lib.fgd_embed_forward(dev.index, _dtype_of(out, "out"), K, tokens.shape[1], V, W, *tok, *tab, scale,
                                     *_mat(out, "out", out.dtype, K * tokens.shape[1], W, dev), _stream_on(stream, dev)))


def fgd_embed_workspace(workers: int, rows: int, vocab: int, width: int) -> int:
    """Bytes of scratch that :func:`fgd_embed_backward` needs for ``rows`` tokens per worker."""
    n = int(_lib.fgd_embed_workspace(int(workers), int(rows), int(vocab), int(width)))
    if n < 0:
        raise FgdError(n, "fgd_embed_workspace: argument out of range")
    return n


def fgd_embed_backward(tokens, dout, dtable, scale: float = 1.0, workspace=None, stream=None) -> None:
    """Gradient of :func:`fgd_embed_forward`: dtable [K, V, W] (fp32), all of it, from dout [K * rows, W].  ``workspace``: a uint8 CUDA tensor of
    :func:`fgd_embed_workspace` bytes (None: allocated here)."""
    usual = _embed_usual(tokens, dtable, dout)
    if usual is not None:
        dev, code, (K, V, W), rows, tok, tab, grad = usual
    else:
        dev = _device_of(dout, "dout")
        if dout.dim() != 2:
            raise ValueError("dout must be [tokens, width]")
        tab, (K, V, W) = _table(dtable, "dtable", dev), dtable.shape
        tok, rows = _embed_tokens(tokens, K, dev), tokens.shape[1]
        code, grad = _dtype_of(dout, "dout"), _mat(dout, "dout", dout.dtype, K * rows, W, dev)
    handle = _stream_on(stream, dev)
    room = 0, 0
    if workspace is None:
        size = fgd_embed_workspace(K, rows, V, W)
        if size:
            workspace = _scratch(size, stream, handle, dev)
    if workspace is not None:
        room = _dev_ptr(workspace, "workspace", "torch.uint8"), workspace.numel()
    _op_check(_lib.fgd_embed_backward(dev.index, code, K, rows, V, W, *tok, *grad, scale, *tab, *room, handle))


def fgd_dropout(x, out, p: float, seed: int, offset: int = 0, counter=None, stream=None) -> None:
    """out = x / (1 - p) where the generator of (seed, offset, row, column) keeps the value, else 0; the mask is never stored, and the backward pass is the
    same call on the gradient.  ``counter``: a CUDA int64 tensor of one value that is added to the offset when the kernel runs.  out may be x."""
    import torch
    xs, dt, dev, code = x.shape, x.dtype, x.device, _types.codes.get(x.dtype)
    if counter is None and len(xs) == 2 and code is not None and dev.type == "cuda" and out.dtype is dt and out.shape == xs and out.device == dev:
        (x0, x1), (o0, o1), (R, W) = x.stride(), out.stride(), xs
        if x1 == o1 == 1 and x0 >= W and o0 >= W:      # as it usually is; else the checks one by one
            _op_check(_lib.fgd_dropout(dev.index, code, R, W, x.data_ptr(), x0, out.data_ptr(), o0, p, seed, offset, 0, _stream_on(stream, dev)))
            return
    if x.dim() != 2:
        raise ValueError("x must be [rows, width]")
    (R, W), dev = x.shape, _device_of(x, "x")
    if counter is not None and (counter.dtype != torch.int64 or counter.numel() != 1 or counter.device != dev):
        raise ValueError("counter must be one int64 value on the device of x")
    _op_check(_lib.fgd_dropout(dev.index, _dtype_of(x, "x"), R, W, *_mat(x, "x", x.dtype, R, W, dev), *_mat(out, "out", x.dtype, R, W, dev), p, seed, offset,
                               0 if counter is None else counter.data_ptr(), _stream_on(stream, dev)))
