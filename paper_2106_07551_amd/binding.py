"""ctypes binding of libmalib.so (argument marshalling only).

Device buffers are torch CUDA (HIP) tensors; streams are torch streams.  Every
call goes straight to the C ABI of ``include/malib.h``; names follow it.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct
import sys
import os
from typing import Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmalib.so")

MALIB_OK, E_INVAL, E_NOMEM, E_HIP, E_UNSUPPORTED, E_DEVICE = 0, -1, -2, -3, -4, -5
POLICY_TABULAR, POLICY_MLP_F32, POLICY_MLP_BF16 = 0, 1, 2
ENV_MATRIX, ENV_ITER_MATRIX, ENV_PURSUIT, ENV_FEATURE = 0, 1, 2, 3
INIT_PER_ENV, INIT_SHARED = 0, 1
K_POLICY, K_SAMPLE, K_ENV, K_SETUP, K_PAYOFF = 0, 1, 2, 3, 4
DT_F32, DT_BF16 = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3

# every function declared in include/malib.h
EXPORTS = [
    "malib_pop_create", "malib_pop_destroy", "malib_rollout_batch", "malib_payoff_eval",
    "malib_meta_sample", "malib_last_error", "malib_profile_enable", "malib_profile_read",
    "malib_debug_tanh_ref", "malib_debug_bf16", "malib_debug_philox",
    "malib_payoff_matrix", "malib_solve_fp", "malib_meta_sample_device",
    "malib_pop_extend", "malib_expansion_pairs", "malib_aggregate", "malib_rollout_batch_traj",
    "malib_pop_policy_ids", "malib_rollout_batch_noalloc", "malib_pop_set_graph",
    "malib_solve_alpharank", "malib_solve_lp",
    "malib_linear", "malib_linear_backward", "malib_linear_work",
    "malib_policy_loss", "malib_distill_loss", "malib_loss_work",
    "malib_log_probs", "malib_log_probs_backward", "malib_log_probs_work", "malib_dropout",
    "malib_quantize_fp4", "malib_dequantize_fp4", "malib_linear_fp4",
]


class MalibError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"malib status {status}: {msg}")
        self.status = status


class ArgumentError(MalibError, ValueError):
    """An argument the binding rejects before calling the library (wrong
    dtype, size, layout or device of a buffer): status MALIB_E_INVAL, as the
    library itself reports invalid arguments."""

    def __init__(self, msg: str):
        super().__init__(E_INVAL, msg)


class PopDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("n_policies", C.c_int32), ("n_actions", C.c_int32),
                ("n_layers", C.c_int32), ("dims", C.POINTER(C.c_int32)),
                ("weights", C.POINTER(C.c_void_p)), ("biases", C.POINTER(C.c_void_p)),
                ("tab_logits", C.c_void_p), ("policy_ids", C.POINTER(C.c_int64))]


class EnvDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("n_agents", C.c_int32), ("n_actions", C.c_int32),
                ("grid", C.c_int32), ("team", C.POINTER(C.c_int8)), ("A", C.c_void_p),
                ("d", C.c_int32), ("init_mode", C.c_int32), ("W", C.c_void_p),
                ("emb", C.c_void_p), ("u", C.c_void_p)]


class TraceDesc(C.Structure):
    _fields_ = [("actions", C.c_void_p), ("n_snap", C.c_int32),
                ("snap_steps", C.POINTER(C.c_int32)), ("logits", C.c_void_p),
                ("states", C.c_void_p), ("perm", C.c_void_p), ("offsets", C.c_void_p)]


class TrajDesc(C.Structure):
    _fields_ = [("actions", C.c_void_p), ("rewards", C.c_void_p), ("flags", C.c_void_p),
                ("obs", C.c_void_p), ("capacity", C.c_int64), ("cursor", C.c_int64)]


class Mat(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("row_stride", C.c_int64), ("group_stride", C.c_int64)]


class LinearDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("groups", C.c_int64),
                ("rows", C.c_int64), ("inputs", C.c_int64), ("outputs", C.c_int64)]


class PolicyLossDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("action_bytes", C.c_int32), ("rows", C.c_int64),
                ("n_actions", C.c_int64), ("logits_stride", C.c_int64), ("ref_stride", C.c_int64),
                ("dlogits_stride", C.c_int64), ("mask_stride", C.c_int64),
                ("clip_low", C.c_float), ("clip_high", C.c_float), ("kl_coef", C.c_float),
                ("entropy_coef", C.c_float)]


class DistillDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("top", C.c_int32), ("rows", C.c_int64),
                ("n_actions", C.c_int64), ("logits_stride", C.c_int64),
                ("dlogits_stride", C.c_int64), ("mask_stride", C.c_int64),
                ("temperature", C.c_float)]


class LogProbsDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("action_bytes", C.c_int32), ("rows", C.c_int64),
                ("n_actions", C.c_int64), ("logits_stride", C.c_int64),
                ("dlogits_stride", C.c_int64), ("mask_stride", C.c_int64), ("top", C.c_int32),
                ("temperature", C.c_float)]


class DropoutDesc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("layer", C.c_uint32), ("rows", C.c_int64),
                ("cols", C.c_int64), ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("y_stride", C.c_int64), ("seed", C.c_uint64), ("step", C.c_uint64),
                ("p", C.c_double)]


class Fp4Desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("groups", C.c_int64),
                ("rows", C.c_int64), ("inputs", C.c_int64), ("outputs", C.c_int64),
                ("scale_group", C.c_int32), ("reserved", C.c_int32)]


class EvalStats(C.Structure):
    _fields_ = [("live_frames", C.c_int64), ("envs", C.c_int64), ("device_flags", C.c_int32)]


_lib = None


def lib():
    """Load libmalib.so; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                              "(hipcc, gfx950); there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        L.malib_pop_create.argtypes = [C.POINTER(PopDesc), vp, C.POINTER(vp)]
        L.malib_pop_create.restype = i32
        L.malib_pop_destroy.argtypes = [vp]
        L.malib_pop_destroy.restype = None
        L.malib_rollout_batch.argtypes = [vp, C.POINTER(EnvDesc), i64, vp, u64, i64, i32, vp,
                                          C.POINTER(TraceDesc), vp]
        L.malib_rollout_batch.restype = i32
        L.malib_payoff_eval.argtypes = [vp, vp, i32, vp, vp, vp, C.POINTER(EvalStats)]
        L.malib_payoff_eval.restype = i32
        L.malib_meta_sample.argtypes = [vp, i32, i32, i64, i32, u64, i64, vp, vp]
        L.malib_meta_sample.restype = i32
        L.malib_last_error.argtypes = []
        L.malib_last_error.restype = C.c_char_p
        L.malib_profile_enable.argtypes = [vp, i32, i32]
        L.malib_profile_enable.restype = i32
        L.malib_profile_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)]
        L.malib_profile_read.restype = i32
        L.malib_debug_tanh_ref.argtypes = [vp, vp, i64, vp]
        L.malib_debug_tanh_ref.restype = i32
        L.malib_debug_bf16.argtypes = [vp, vp, i64, vp]
        L.malib_debug_bf16.restype = i32
        L.malib_debug_philox.argtypes = [vp, u64, u64, vp, i64, vp]
        L.malib_debug_philox.restype = i32
        L.malib_payoff_matrix.argtypes = [vp, vp, vp]
        L.malib_payoff_matrix.restype = i32
        L.malib_solve_fp.argtypes = [vp, i32, i32, vp, vp, vp]
        L.malib_solve_fp.restype = i32
        L.malib_solve_alpharank.argtypes = [vp, i32, C.c_double, i32, vp, vp, vp, vp]
        L.malib_solve_alpharank.restype = i32
        L.malib_solve_lp.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp]
        L.malib_solve_lp.restype = i32
        L.malib_meta_sample_device.argtypes = [vp, i32, i32, i64, i32, vp, u64, i64, vp, vp]
        L.malib_meta_sample_device.restype = i32
        L.malib_rollout_batch_traj.argtypes = [vp, C.POINTER(EnvDesc), i64, vp, u64, i64, i32,
                                               vp, C.POINTER(TrajDesc), vp]
        L.malib_rollout_batch_traj.restype = i32
        L.malib_aggregate.argtypes = [vp, i32, vp, i32, i32, vp, vp]
        L.malib_aggregate.restype = i32
        L.malib_pop_extend.argtypes = [vp, vp, vp]
        L.malib_pop_extend.restype = i32
        L.malib_expansion_pairs.argtypes = [i32, i32, i32, i32, vp, vp, vp]
        L.malib_expansion_pairs.restype = i32
        L.malib_rollout_batch_noalloc.argtypes = [vp, C.POINTER(EnvDesc), i64, vp, u64, i64,
                                                  i32, vp, vp]
        L.malib_rollout_batch_noalloc.restype = i32
        L.malib_pop_set_graph.argtypes = [vp, i32]
        L.malib_pop_set_graph.restype = i32
        L.malib_pop_policy_ids.argtypes = [vp, vp, i32, C.POINTER(i32)]
        L.malib_pop_policy_ids.restype = i32
        # (descriptions as packed bytes or by reference)
        L.malib_linear.argtypes = [vp] * 8 + [i64, vp]
        L.malib_linear.restype = i32
        L.malib_linear_backward.argtypes = [vp] * 9 + [i64, vp]
        L.malib_linear_backward.restype = i32
        L.malib_linear_work.argtypes = [vp, i32, C.POINTER(i64)]
        L.malib_linear_work.restype = i32
        L.malib_policy_loss.argtypes = [vp] * 13 + [i64, vp]
        L.malib_policy_loss.restype = i32
        L.malib_distill_loss.argtypes = [vp] * 10 + [i64, vp]
        L.malib_distill_loss.restype = i32
        L.malib_loss_work.argtypes = [i32, i64, i64, C.POINTER(i64)]
        L.malib_loss_work.restype = i32
        L.malib_log_probs.argtypes = [vp] * 8 + [i64, vp]
        L.malib_log_probs.restype = i32
        L.malib_log_probs_backward.argtypes = [vp] * 9
        L.malib_log_probs_backward.restype = i32
        L.malib_log_probs_work.argtypes = [i32, i64, i64, i32, C.POINTER(i64)]
        L.malib_log_probs_work.restype = i32
        L.malib_dropout.argtypes = [vp] * 6
        L.malib_dropout.restype = i32
        L.malib_quantize_fp4.argtypes = [vp] * 5
        L.malib_quantize_fp4.restype = i32
        L.malib_dequantize_fp4.argtypes = [vp] * 5
        L.malib_dequantize_fp4.restype = i32
        L.malib_linear_fp4.argtypes = [vp] * 8
        L.malib_linear_fp4.restype = i32
        _lib = L
    return _lib


def _check(st: int):
    if st != MALIB_OK:
        raise MalibError(st, lib().malib_last_error().decode())


def _stream(stream):
    if stream is not None:
        return C.c_void_p(stream.cuda_stream)
    return C.c_void_p(_current_stream())


def _dptr(t, dtype=None, numel: Optional[int] = None, *, at_least: bool = False,
          what: str = "tensor") -> Optional[int]:
    """Device address of a contiguous device tensor (None passes through).

    The library's kernels read and write the buffers it is given with the
    sizes and element types the header states, so a tensor of another dtype
    or with fewer elements would be accessed out of bounds on the device:
    both are errors here (ArgumentError, raised, not asserted), as are host
    tensors and non-contiguous views.  `numel` is the exact count, or the minimum with
    `at_least`."""
    if t is None:
        return None
    _check_buf(t, dtype, numel, at_least, what)
    if not t.is_cuda:
        raise ArgumentError(f"{what}: expected a device tensor, got one on {t.device}")
    return t.data_ptr()


def _check_buf(t, dtype, numel, at_least, what):
    """dtype, element count and layout of a buffer (not its device)."""
    if t is None:
        return
    if dtype is not None and t.dtype != dtype:
        raise ArgumentError(f"{what}: expected dtype {dtype}, got {t.dtype}")
    if numel is not None:
        n = t.numel()
        if (n < numel) if at_least else (n != numel):
            raise ArgumentError(f"{what}: expected {'at least ' if at_least else ''}{numel} "
                                f"elements, got {n}")
    if not t.is_contiguous():
        raise ArgumentError(f"{what}: expected a contiguous tensor")


def _dptrs(*specs):
    """_dptr over several buffers (t, dtype, numel, at_least, what): every
    dtype, size and layout is checked before any device, so that the first
    error reported is the most specific one."""
    for sp in specs:
        _check_buf(*sp)
    return [_dptr(*sp[:3], at_least=sp[3], what=sp[4]) for sp in specs]


def _dbytes(t, nbytes: int, what: str) -> Optional[int]:
    """Like _dptr for buffers whose element type the caller chooses: at least
    `nbytes` bytes."""
    if t is None:
        return None
    if t.numel() * t.element_size() < nbytes:
        raise ArgumentError(f"{what}: expected at least {nbytes} bytes, got "
                         f"{t.numel() * t.element_size()}")
    return _dptr(t, what=what)


def _f32():
    import torch
    return torch.float32


def _pop_desc(kind, n_policies, n_actions, dims, weights, biases, tab_logits,
              policy_ids=None):
    """A malib_pop_desc over device tensors, with the ctypes arrays it points
    into (keep them alive until the call returns)."""
    d = PopDesc()
    d.kind, d.n_policies, d.n_actions = kind, n_policies, n_actions
    keep = []
    if policy_ids is not None:
        if len(policy_ids) != n_policies:
            raise ArgumentError(f"policy_ids: expected {n_policies} ids, got {len(policy_ids)}")
        ids = (C.c_int64 * n_policies)(*[int(x) for x in policy_ids])
        keep.append(ids)
        d.policy_ids = C.cast(ids, C.POINTER(C.c_int64))
    if kind == POLICY_TABULAR:
        d.n_layers = 0
        if tab_logits is None:
            raise ArgumentError("a tabular population needs tab_logits")
        d.tab_logits = _dptr(tab_logits, _f32(), n_policies * n_actions, what="tab_logits")
    else:
        if dims is None or len(dims) != 4 or len(weights) != 3:
            raise ArgumentError("an MLP population needs dims [in, h1, h2, A] and three weights")
        if biases is not None and len(biases) != 3:
            raise ArgumentError("biases: expected three entries (each a tensor or None)")
        d.n_layers = 3
        f32 = _f32()
        specs = [(w, f32, n_policies * dims[l + 1] * dims[l], False, f"weights[{l}]")
                 for l, w in enumerate(weights)]
        if biases is not None:
            specs += [(b, f32, n_policies * dims[l + 1], False, f"biases[{l}]")
                      for l, b in enumerate(biases)]
        ptrs = _dptrs(*specs)
        dd = (C.c_int32 * 4)(*dims)
        ww = (C.c_void_p * 3)(*ptrs[:3])
        keep += [dd, ww]
        d.dims = C.cast(dd, C.POINTER(C.c_int32))
        d.weights = C.cast(ww, C.POINTER(C.c_void_p))
        if biases is not None:
            bb = (C.c_void_p * 3)(*ptrs[3:])
            keep.append(bb)
            d.biases = C.cast(bb, C.POINTER(C.c_void_p))
    return d, keep


class Population:
    """A policy population handle (malib_pop_create / malib_pop_destroy) with its
    payoff table."""

    def __init__(self, kind: int, n_policies: int, n_actions: int, *, dims=None,
                 weights: Sequence = (), biases: Optional[Sequence] = None,
                 tab_logits=None, policy_ids: Optional[Sequence[int]] = None, stream=None):
        d, keep = _pop_desc(kind, n_policies, n_actions, dims, weights, biases, tab_logits,
                            policy_ids)
        h = C.c_void_p()
        self._destroy = lib().malib_pop_destroy
        self._finalizing = sys.is_finalizing
        _check(lib().malib_pop_create(C.byref(d), _stream(stream), C.byref(h)))
        del keep
        self.handle = h
        self.kind = kind
        self.dims = list(dims) if dims is not None else None
        self.P = n_policies
        self.A = n_actions

    def extend(self, n_new: int, *, weights: Sequence = (), biases: Optional[Sequence] = None,
               tab_logits=None, policy_ids: Optional[Sequence[int]] = None, stream=None):
        """malib_pop_extend: append n_new policies (indices P .. P + n_new - 1,
        caller ids ``policy_ids``, default the indices); the table keeps its
        cells and gains empty rows and columns."""
        d, keep = _pop_desc(self.kind, n_new, self.A, self.dims, weights, biases, tab_logits,
                            policy_ids)
        _check(lib().malib_pop_extend(self.handle, C.byref(d), _stream(stream)))
        del keep
        self.P += n_new

    def set_graph(self, enable: bool = True):
        """malib_pop_set_graph: replay each batch's launch sequence as one HIP graph."""
        _check(lib().malib_pop_set_graph(self.handle, int(bool(enable))))

    def policy_ids(self) -> np.ndarray:
        """malib_pop_policy_ids: the caller id of each index 0 .. P-1."""
        n = C.c_int32()
        out = np.zeros(self.P, np.int64)
        _check(lib().malib_pop_policy_ids(self.handle, out.ctypes.data, self.P, C.byref(n)))
        if n.value != self.P:
            raise RuntimeError(f"malib_pop_policy_ids returned {n.value} ids for P = {self.P}")
        return out

    def close(self):
        """malib_pop_destroy (also on garbage collection).  At interpreter exit
        the call is skipped: module globals and the HIP runtime may already be
        torn down, and the process's device memory is released with it; the
        functions used here are the ones captured when the handle was made."""
        h = getattr(self, "handle", None)
        if not h:
            return
        self.handle = None
        if self._finalizing():
            return
        self._destroy(h)

    __del__ = close

    def _batch_ptrs(self, env: "Env", n_envs: int, pair_assign, returns):
        """pair_assign int32 [n_envs][n_agents] and returns fp32 [n_agents][n_envs]
        (at least that many elements; counts the library rejects pass through
        to it)."""
        import torch
        ns = max(int(n_envs), 0) * env.n_agents
        return (_dptr(pair_assign, torch.int32, ns, at_least=True, what="pair_assign"),
                _dptr(returns, torch.float32, ns, at_least=True, what="returns"))

    def rollout(self, env: "Env", n_envs: int, pair_assign, seed: int, horizon: int, *,
                env_offset: int = 0, returns=None, trace: "Trace" = None, stream=None):
        pa, rp = self._batch_ptrs(env, n_envs, pair_assign, returns)
        tr = trace.checked(env, n_envs, horizon, self.P, self.A) if trace is not None else None
        _check(lib().malib_rollout_batch(
            self.handle, C.byref(env.desc), n_envs, pa, seed, env_offset,
            horizon, rp, C.byref(tr) if tr is not None else None,
            _stream(stream)))

    def rollout_noalloc(self, env: "Env", n_envs: int, pair_assign, seed: int, horizon: int,
                        *, env_offset: int = 0, returns=None, stream=None):
        """malib_rollout_batch_noalloc: the same batch on the library's static
        scratch (no device allocation; calls on one GPU must not overlap)."""
        pa, rp = self._batch_ptrs(env, n_envs, pair_assign, returns)
        _check(lib().malib_rollout_batch_noalloc(
            self.handle, C.byref(env.desc), n_envs, pa, seed, env_offset,
            horizon, rp, _stream(stream)))

    def rollout_traj(self, env: "Env", n_envs: int, pair_assign, seed: int, horizon: int,
                     traj: Traj, *, env_offset: int = 0, returns=None, stream=None):
        """malib_rollout_batch_traj: a rollout that also writes its per-step
        records into `traj` (advancing its cursor)."""
        pa, rp = self._batch_ptrs(env, n_envs, pair_assign, returns)
        traj.check(env)
        _check(lib().malib_rollout_batch_traj(
            self.handle, C.byref(env.desc), n_envs, pa, seed, env_offset,
            horizon, rp, C.byref(traj.desc), _stream(stream)))

    def payoff_matrix(self, out=None, stream=None):
        """malib_payoff_matrix: the table's means as a device fp64 [P][P] game
        (0 for empty cells)."""
        import torch
        if out is None:
            out = torch.empty((self.P, self.P), dtype=torch.float64, device="cuda")
        _check(lib().malib_payoff_matrix(
            self.handle, _dptr(out, torch.float64, self.P * self.P, what="out"),
            _stream(stream)))
        return out

    def payoff(self, reset: bool = False, stream=None, check: bool = True):
        P = self.P
        mean = np.zeros((P, P), np.float64)
        counts = np.zeros((P, P), np.int64)
        se = np.zeros((P, P), np.float64)
        st = EvalStats()
        rc = lib().malib_payoff_eval(self.handle, _stream(stream), int(reset),
                                     mean.ctypes.data, counts.ctypes.data, se.ctypes.data,
                                     C.byref(st))
        if check:
            _check(rc)
        out = {"mean": mean, "counts": counts, "stderr": se, "live_frames": st.live_frames,
               "envs": st.envs, "device_flags": st.device_flags, "status": rc}
        return out

    def profile_enable(self, on: bool = True, *, kernels=None, every: int = 1):
        """Time launches of the kernel classes in ``kernels`` (default: all when
        ``on``), one in ``every``."""
        mask = 0
        if on:
            ks = range(5) if kernels is None else kernels
            for k in ks:
                mask |= 1 << k
        _check(lib().malib_profile_enable(self.handle, mask, every))

    def profile_read(self, kernel: int):
        ms = C.c_double()
        n = C.c_int64()
        _check(lib().malib_profile_read(self.handle, kernel, C.byref(ms), C.byref(n)))
        return ms.value, n.value


class Env:
    """An environment description (malib_env_desc); keeps its device tensors alive."""

    def __init__(self, kind: int, n_agents: int, n_actions: int, *, team=None, A=None,
                 grid: int = 0, d: int = 0, W=None, emb=None, u=None,
                 init_mode: int = INIT_PER_ENV):
        e = EnvDesc()
        e.kind, e.n_agents, e.n_actions, e.grid, e.d, e.init_mode = (
            kind, n_agents, n_actions, grid, d, init_mode)
        self._keep = [A, W, emb, u]
        if team is not None:
            if len(team) != n_agents:
                raise ArgumentError(f"team: expected {n_agents} entries, got {len(team)}")
            tt = (C.c_int8 * n_agents)(*[int(x) for x in team])
            self._keep.append(tt)
            e.team = C.cast(tt, C.POINTER(C.c_int8))
        f32 = _f32()
        e.A, e.W, e.emb, e.u = _dptrs((A, f32, n_actions * n_actions, False, "A"),
                                      (W, f32, d * d, False, "W"),
                                      (emb, f32, n_agents * n_actions * d, False, "emb"),
                                      (u, f32, d, False, "u"))
        self.desc = e
        self.kind = kind
        self.n_agents = n_agents
        self.n_actions = n_actions
        self.d = d


class Traj:
    """A device ring of per-step records (malib_traj): actions [cap][n_agents]
    uint8, rewards [cap] fp32, flags [cap] uint8 and, optionally, obs in the
    environment's compact form (see malib.h)."""

    def __init__(self, capacity: int, n_agents: int, *, obs_shape=None, obs_dtype=None,
                 device="cuda"):
        import torch
        self.capacity = capacity
        self.actions = torch.empty((capacity, n_agents), dtype=torch.uint8, device=device)
        self.rewards = torch.empty(capacity, dtype=torch.float32, device=device)
        self.flags = torch.empty(capacity, dtype=torch.uint8, device=device)
        self.obs = None
        if obs_shape is not None:
            self.obs = torch.empty((capacity,) + tuple(obs_shape), dtype=obs_dtype,
                                   device=device)
        # its own tensors: the device is checked before each rollout (check)
        self.desc = TrajDesc(self.actions.data_ptr(), self.rewards.data_ptr(),
                             self.flags.data_ptr(),
                             None if self.obs is None else self.obs.data_ptr(), capacity, 0)

    @property
    def cursor(self) -> int:
        return self.desc.cursor

    def check(self, env: "Env"):
        """The ring's buffers against the environment's record layout."""
        if not 0 <= self.desc.capacity <= self.capacity:
            raise ArgumentError(f"traj: capacity {self.desc.capacity} is outside the ring's "
                             f"{self.capacity} records")
        if self.actions.shape[1] != env.n_agents:
            raise ArgumentError(f"traj: actions hold {self.actions.shape[1]} seats, the "
                             f"environment has {env.n_agents}")
        per = {ENV_ITER_MATRIX: 2, ENV_PURSUIT: 2, ENV_FEATURE: 2 * env.d}.get(env.kind, 0)
        if self.obs is not None and per:
            _dbytes(self.obs, self.capacity * per, "traj.obs")
        if not self.actions.is_cuda:
            raise ArgumentError(f"traj: expected device tensors, got ones on "
                                f"{self.actions.device}")


class Trace:
    """Parity trace buffers (malib_trace); any of them may be omitted."""

    def __init__(self, *, actions=None, snap_steps=(), logits=None, states=None, perm=None,
                 offsets=None):
        t = TraceDesc()
        t.actions = _dptr(actions)
        steps = list(snap_steps)
        t.n_snap = len(steps)
        ss = (C.c_int32 * max(1, len(steps)))(*steps)
        t.snap_steps = C.cast(ss, C.POINTER(C.c_int32))
        t.logits, t.states = _dptr(logits), _dptr(states)
        t.perm, t.offsets = _dptr(perm), _dptr(offsets)
        self._keep = [ss, actions, logits, states, perm, offsets]
        self.desc = t
        self.n_snap = len(steps)
        self.actions, self.logits, self.states = actions, logits, states
        self.perm, self.offsets = perm, offsets

    def checked(self, env: "Env", n_envs: int, horizon: int, P: int, A: int):
        """The descriptor, after checking each buffer against the batch that
        will write it (sizes as in malib.h's malib_trace)."""
        import torch
        ns = max(int(n_envs), 0) * env.n_agents
        h = max(int(horizon), 0)
        per = {ENV_ITER_MATRIX: 2, ENV_PURSUIT: 3, ENV_FEATURE: 4 * env.d}.get(env.kind, 0)
        st = self.states
        if st is not None and st.numel() * st.element_size() < self.n_snap * per * max(n_envs, 0):
            raise ArgumentError(f"trace.states: expected at least "
                                f"{self.n_snap * per * max(n_envs, 0)} bytes, got "
                                f"{st.numel() * st.element_size()}")
        _dptrs((self.actions, torch.uint8, h * ns, True, "trace.actions"),
               (self.logits, torch.float32, self.n_snap * ns * A, True, "trace.logits"),
               (st, None, None, True, "trace.states"),
               (self.perm, torch.int32, ns, True, "trace.perm"),
               (self.offsets, torch.int32, P + 1, True, "trace.offsets"))
        return self.desc


def meta_sample(sigma, n_policies: int, n_envs: int, n_agents: int, seed: int, *,
                env_offset: int = 0, out=None, stream=None):
    """malib_meta_sample: policy id per (env, seat) drawn from sigma [n_sigma][P]."""
    import torch
    s = np.ascontiguousarray(sigma, dtype=np.float32).reshape(-1, n_policies)
    if out is None:
        out = torch.empty((n_envs, n_agents), dtype=torch.int32, device="cuda")
    op = _dptr(out, torch.int32, max(n_envs, 0) * max(n_agents, 0), at_least=True, what="out")
    _check(lib().malib_meta_sample(s.ctypes.data, s.shape[0], n_policies, n_envs, n_agents,
                                   seed, env_offset, op, _stream(stream)))
    return out


def expansion_pairs(n_policies: int, first_new: int, per_pair: int, n_agents: int = 2,
                    team=None, *, out=None, stream=None):
    """malib_expansion_pairs: policy ids [(P^2 - first_new^2) * per_pair][n_agents]
    of the batch that simulates the cells of the new rows and columns."""
    import torch
    n = (n_policies * n_policies - first_new * first_new) * per_pair
    if out is None:
        out = torch.empty((max(n, 0), n_agents), dtype=torch.int32, device="cuda")
    tm = None
    if team is not None:
        tm = np.ascontiguousarray(team, dtype=np.int8)
        if tm.shape != (n_agents,):
            raise ArgumentError(f"team: expected shape ({n_agents},), got {tm.shape}")
    op = _dptr(out, torch.int32, max(n, 0) * max(n_agents, 0), at_least=True, what="out")
    _check(lib().malib_expansion_pairs(n_policies, first_new, per_pair, n_agents,
                                       None if tm is None else tm.ctypes.data, op,
                                       _stream(stream)))
    return out


def _game(M) -> int:
    """P of a device fp64 [P][P] game, checked."""
    import torch
    if M.dim() != 2 or M.shape[0] != M.shape[1]:
        raise ArgumentError(f"M: expected a square [P][P] game, got shape {tuple(M.shape)}")
    _dptr(M, torch.float64, what="M")
    return int(M.shape[0])


def solve_fp(M, iterations: int, *, sigma=None, gap=None, stream=None):
    """malib_solve_fp on a device fp64 [P][P] game: returns (sigma [2][P] play
    counts as fp32, gap [1] fp64), both device tensors."""
    import torch
    P = _game(M)
    if sigma is None:
        sigma = torch.empty((2, P), dtype=torch.float32, device=M.device)
    if gap is None:
        gap = torch.empty(1, dtype=torch.float64, device=M.device)
    _check(lib().malib_solve_fp(_dptr(M), P, iterations,
                                _dptr(sigma, torch.float32, 2 * P, what="sigma"),
                                _dptr(gap, torch.float64, 1, what="gap"), _stream(stream)))
    return sigma, gap


def solve_lp(M, *, work=None, stream=None):
    """malib_solve_lp on a device fp64 [P][P] game: returns (value [1] fp64,
    x [P] fp64, y [P] fp64, sigma [2][P] fp32, pivots [1] int32), device
    tensors; a workspace is allocated here when P > 96 and none is given."""
    import torch
    P = _game(M)
    dev = M.device
    value = torch.empty(1, dtype=torch.float64, device=dev)
    x = torch.empty(P, dtype=torch.float64, device=dev)
    y = torch.empty(P, dtype=torch.float64, device=dev)
    sigma = torch.empty((2, P), dtype=torch.float32, device=dev)
    pivots = torch.empty(1, dtype=torch.int32, device=dev)
    if work is None and P > 96:
        work = torch.empty((P + 1) * (2 * P + 1), dtype=torch.float64, device=dev)
    wp = _dptr(work, torch.float64, (P + 1) * (2 * P + 1), at_least=True, what="work")
    _check(lib().malib_solve_lp(_dptr(M), P, wp, _dptr(value), _dptr(x), _dptr(y),
                                _dptr(sigma), _dptr(pivots), _stream(stream)))
    return value, x, y, sigma, pivots


def solve_alpharank(M, alpha: float, m: int, *, pi=None, sigma=None, work=None, stream=None):
    """malib_solve_alpharank on a device fp64 [P][P] game: returns (pi [P]
    fp64, sigma [2][P] fp32 weight rows), device tensors; a [P][P] fp64
    workspace is allocated here when P > 128 and none is given."""
    import torch
    P = _game(M)
    if pi is None:
        pi = torch.empty(P, dtype=torch.float64, device=M.device)
    if sigma is None:
        sigma = torch.empty((2, P), dtype=torch.float32, device=M.device)
    if work is None and P > 128:
        work = torch.empty((P, P), dtype=torch.float64, device=M.device)
    _check(lib().malib_solve_alpharank(
        _dptr(M), P, float(alpha), int(m),
        _dptr(work, torch.float64, P * P, at_least=True, what="work"),
        _dptr(pi, torch.float64, P, what="pi"), _dptr(sigma, torch.float32, 2 * P, what="sigma"),
        _stream(stream)))
    return pi, sigma


def aggregate(M, sigma, br_row: int = -1, br_col: int = -1, *, out=None, stream=None):
    """malib_aggregate: device fp64 [5] = (nash payoff of the row side, of
    the column side, best-response payoff of br_row, of br_col, improvement)."""
    import torch
    P = _game(M)
    if out is None:
        out = torch.empty(5, dtype=torch.float64, device=M.device)
    _check(lib().malib_aggregate(_dptr(M), P, _dptr(sigma, torch.float32, 2 * P, what="sigma"),
                                 br_row, br_col, _dptr(out, torch.float64, 5, what="out"),
                                 _stream(stream)))
    return out


def meta_sample_device(sigma, n_policies: int, n_envs: int, n_agents: int, seed: int, *,
                       env_offset: int = 0, seat_row=None, out=None, stream=None):
    """malib_meta_sample_device: policy ids drawn from device weight rows
    sigma [n_sigma][P] (fp32); seat k uses row seat_row[k] (default: row 0
    for all seats when there is one row, else row k)."""
    import torch
    if n_policies < 1 or sigma.numel() % n_policies or sigma.numel() == 0:
        raise ArgumentError(f"sigma: expected [n_sigma][{n_policies}] weights, got "
                         f"{sigma.numel()} elements")
    n_sigma = sigma.numel() // n_policies
    sr = None
    if seat_row is not None:
        sr = np.ascontiguousarray(seat_row, dtype=np.int32)
        if sr.shape != (n_agents,):
            raise ArgumentError(f"seat_row: expected shape ({n_agents},), got {sr.shape}")
    if out is None:
        out = torch.empty((n_envs, n_agents), dtype=torch.int32, device=sigma.device)
    sp, op = _dptrs((sigma, torch.float32, None, False, "sigma"),
                    (out, torch.int32, max(n_envs, 0) * max(n_agents, 0), True, "out"))
    _check(lib().malib_meta_sample_device(sp, n_sigma, n_policies, n_envs, n_agents,
                                          None if sr is None else sr.ctypes.data, seed,
                                          env_offset, op, _stream(stream)))
    return out


# ------------------------------------------------------------ learner operators
#
# These are called once per layer and step, often on small batches where the host's
# share is the time: descriptions are packed into bytes (a tenth of a ctypes
# structure's time), and checks name what they found only once one has failed.
#
# torch's autograd does not see them: tensors that require gradients are taken for
# their values, outputs require none, and gradients are outputs of their own.

_MAT = struct.Struct("@Pqq")                  # malib_mat
_LINEAR = struct.Struct("@iiqqqq")            # malib_linear_desc
_POLICY_LOSS = struct.Struct("@iiqqqqqqffff")  # malib_policy_loss_desc
_DISTILL = struct.Struct("@iiqqqqqf4x")        # malib_distill_desc
_LOG_PROBS = struct.Struct("@iiqqqqqif")      # malib_log_probs_desc
_DROPOUT = struct.Struct("@iIqqqqqQQd")        # malib_dropout_desc
_FP4 = struct.Struct("@iiqqqqii")              # malib_fp4_desc


_calls = None


def _native():
    """The learner operators' calls in C++ (csrc/learner_calls.cpp): each takes the
    arguments of the function below that has its name, checks them, allocates and calls the
    library, or returns None where it does not take them.  Raises if they have not been
    built."""
    global _calls
    if _calls is None:
        lib()
        import torch  # noqa: F401  (the module's symbols)
        try:
            from . import _learner_calls as m
        except ImportError as e:
            raise ImportError(f"{e}: build it with __graft_entry__.build()") from e
        m.load(LIB_PATH)
        _calls = m
    return _calls


def _current_stream():
    import torch
    # (torch.cuda.current_stream() takes 8 us to make the object this is read from)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _empty(shape, dtype, device, stream):
    """A tensor from the memory pool of the stream the call runs on (the caching
    allocator hands memory out again in the order of one stream only)."""
    import torch
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


def _dtype_code(t, what):
    import torch
    dt = t.dtype
    if dt is torch.bfloat16:
        return DT_BF16
    if dt is torch.float32:
        return DT_F32
    raise ArgumentError(f"{what}: expected dtype float32 or bfloat16, got {dt}")


def _mat(t, dtype, G, rows, cols, what, out: bool = False):
    """A malib_mat (packed) over a tensor [rows][cols] or [groups][rows][cols]
    whose rows are contiguous; G is None without the group dimension.  An input
    without it is shared by the groups."""
    if t is None:
        return None
    shape = t.shape
    shared = G is not None and not out and len(shape) == 2
    want = (rows, cols) if G is None or shared else (G, rows, cols)
    if shape != want:
        raise ArgumentError(f"{what}: expected shape {want}, got {tuple(shape)}")
    if t.dtype is not dtype:
        raise ArgumentError(f"{what}: expected dtype {dtype}, got {t.dtype}")
    st = t.stride()
    if st[-1] != 1 and cols > 1:
        raise ArgumentError(f"{what}: expected contiguous rows, got column stride {st[-1]}")
    row = st[-2] if rows > 1 else cols
    group = 0 if G is None or shared else st[0] if G > 1 else rows * row
    return _MAT.pack(t.data_ptr(), row, group)


def _on_device(names, *tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            what = next(n for n, u in zip(names.split(), tensors) if u is t)
            raise ArgumentError(f"{what}: expected a device tensor, got one on {t.device}")


def _layer(x, w, act):
    """(groups or None, out, in) of a layer from its weight, and its checks."""
    shape, nx = w.shape, x.dim()
    n = len(shape)
    if n != 2 and n != 3:
        raise ArgumentError(f"w: expected [out][in] or [groups][out][in], got shape "
                            f"{tuple(shape)}")
    if nx != n and (nx != 2 or n != 3):
        raise ArgumentError(f"x: expected [rows][in] or, with weights per group, "
                            f"[groups][rows][in], got shape {tuple(x.shape)}")
    if act not in (ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU):
        raise ArgumentError(f"act: unknown activation {act!r}")
    return shape[0] if n == 3 else None, shape[-2], shape[-1]


@functools.lru_cache(maxsize=4096)
def _linear_work(desc, backward):
    need = C.c_int64()
    _check(lib().malib_linear_work(desc, backward, C.byref(need)))
    return need.value


@functools.lru_cache(maxsize=4096)
def _loss_work(code, n, a):
    need = C.c_int64()
    _check(lib().malib_loss_work(code, n, a, C.byref(need)))
    return need.value


def _workspace(need, work, device, stream):
    """(address, bytes, tensor) of a call's workspace, allocated unless the
    caller's is given."""
    import torch
    if work is not None:
        _dbytes(work, need, "work")
        return work.data_ptr(), work.numel() * work.element_size(), work
    if not need:
        return None, 0, None
    work = _empty((need,), torch.uint8, device, stream)
    return work.data_ptr(), need, work


def _ptr(t):
    return None if t is None else t.data_ptr()


def linear(x, w, bias=None, *, act: int = ACT_NONE, residual=None, pre=None, out=None, work=None,
           stream=None):
    """malib_linear: act(x w^T + bias) + residual for x [rows][in] and w
    [out][in], or [groups][rows][in] and [groups][out][in] (x without the
    group dimension is shared by the groups); float32 or bfloat16, bias
    float32.  `pre` receives the values before the activation, which
    linear_backward needs.  Returns [..][rows][out], outside torch's autograd
    graph: gradients are linear_backward's."""
    if stream is None and x.is_cuda:
        y = (_calls or _native()).linear(x, w, bias, act, residual, pre, out, work,
                                         _current_stream())
        if y is not None:
            return y
    code = _dtype_code(x, "x")
    G, n_out, n_in = _layer(x, w, act)
    rows, dt = x.shape[-2], x.dtype
    mx = _mat(x, dt, G, rows, n_in, "x")
    mw = _mat(w, dt, G, n_out, n_in, "w")
    mr = _mat(residual, dt, G, rows, n_out, "residual")
    mp = _mat(pre, dt, G, rows, n_out, "pre", True)
    if bias is not None:
        _check_buf(bias, _f32(), n_out * (G or 1), False, "bias")
    _on_device("x w bias residual pre out", x, w, bias, residual, pre, out)
    if out is None:
        out = _empty((rows, n_out) if G is None else (G, rows, n_out), dt, x.device, stream)
    my = _mat(out, dt, G, rows, n_out, "out", True)
    d = _LINEAR.pack(code, act, G or 1, rows, n_in, n_out)
    wp, nbytes, work = _workspace(_linear_work(d, 0), work, x.device, stream)
    _check(lib().malib_linear(d, mx, mw, _ptr(bias), mr, mp, my, wp, nbytes, _stream(stream)))
    return out


def linear_backward(dy, x, w, *, act: int = ACT_NONE, pre=None, want=(True, True, True), dx=None,
                    dw=None, dbias=None, work=None, stream=None):
    """malib_linear_backward: (dx, dw, dbias) of linear for the gradient dy of
    its output; `pre` is what linear wrote there (needed with an activation).
    `want` leaves outputs out (None is returned for them).  The residual's
    gradient is dy.  Outside torch's autograd graph, as linear."""
    if stream is None and dy.is_cuda:
        out = (_calls or _native()).linear_backward(dy, x, w, act, pre, want, dx, dw, dbias, work,
                                                    _current_stream())
        if out is not None:
            return out
    code = _dtype_code(dy, "dy")
    G, n_out, n_in = _layer(dy, w, act)
    rows, dt, dev = dy.shape[-2], dy.dtype, dy.device
    lead = () if G is None else (G,)
    mdy = _mat(dy, dt, G, rows, n_out, "dy")
    mx = _mat(x, dt, G, rows, n_in, "x")
    mw = _mat(w, dt, G, n_out, n_in, "w")
    if act == ACT_NONE:
        mp = None
    elif pre is None:
        raise ArgumentError("pre: the backward pass of an activation needs the values before it")
    else:
        mp = _mat(pre, dt, G, rows, n_out, "pre")
    _on_device("dy x w pre dx dw dbias", dy, x, w, pre, dx, dw, dbias)
    if not want[0]:
        dx = None
    elif dx is None:
        dx = _empty(lead + (rows, n_in), dt, dev, stream)
    if not want[1]:
        dw = None
    elif dw is None:
        dw = _empty(lead + (n_out, n_in), dt, dev, stream)
    if not want[2]:
        dbias = None
    elif dbias is None:
        dbias = _empty(lead + (n_out,), _f32(), dev, stream)
    else:
        _check_buf(dbias, _f32(), n_out * (G or 1), False, "dbias")
    mdx = _mat(dx, dt, G, rows, n_in, "dx", True)
    mdw = _mat(dw, dt, G, n_out, n_in, "dw", True)
    d = _LINEAR.pack(code, act, G or 1, rows, n_in, n_out)
    wp, nbytes, work = _workspace(_linear_work(d, 1), work, dev, stream)
    _check(lib().malib_linear_backward(d, mdy, mx, mw, mp, mdx, mdw, _ptr(dbias), wp, nbytes,
                                       _stream(stream)))
    return dx, dw, dbias


def _rows(t, dtypes, n, a, what) -> int:
    """Row stride of a tensor [n][a] whose rows are contiguous, checked."""
    if t is None:
        return 0
    if t.shape != (n, a):
        raise ArgumentError(f"{what}: expected shape {(n, a)}, got {tuple(t.shape)}")
    if t.dtype not in dtypes:
        raise ArgumentError(f"{what}: expected dtype {' or '.join(map(str, dtypes))}, got "
                            f"{t.dtype}")
    st = t.stride()
    if st[1] != 1 and a > 1:
        raise ArgumentError(f"{what}: expected contiguous rows, got column stride {st[1]}")
    return st[0] if n > 1 else a


def _loss_args(logits, mask, weight, dlogits):
    """What both losses check: (rows, n_actions, dtype code, strides of logits,
    dlogits and mask)."""
    import torch
    shape = logits.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ArgumentError(f"logits: expected [rows][n_actions], got shape {tuple(shape)}")
    code = _dtype_code(logits, "logits")
    n, a = shape
    dts = (logits.dtype,)
    sl = _rows(logits, dts, n, a, "logits")
    sm = _rows(mask, (torch.bool, torch.uint8), n, a, "mask")
    sd = _rows(dlogits, dts, n, a, "dlogits")
    if weight is not None:
        _check_buf(weight, torch.float32, n, False, "weight")
    return n, a, code, sl, sd, sm


def policy_loss(logits, actions, old_logp, advantage, *, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0,
                ref_logp=None, ref_logits=None, mask=None, weight=None, grad: bool = True,
                total=None, stats=None, dlogits=None, work=None, stream=None):
    """malib_policy_loss: the clipped policy loss with a divergence term over
    logits [rows][n_actions] (float32 or bfloat16) and its gradient.  actions:
    uint8, int32 or int64 [rows] (out of range: no action); mask: bool or uint8
    [rows][n_actions], legal entries.  Returns (total [1], stats [4][rows] =
    loss, log probability of the action, divergence and entropy of each row,
    dlogits or None without `grad`); total is outside torch's autograd graph,
    dlogits is its gradient."""
    if stream is None and logits.is_cuda:
        out = (_calls or _native()).policy_loss(
            logits, actions, old_logp, advantage, clip_low, clip_high, kl_coef, entropy_coef,
            ref_logp, ref_logits, mask, weight, grad, total, stats, dlogits, work,
            _current_stream())
        if out is not None:
            return out
    import torch
    n, a, code, sl, sd, sm = _loss_args(logits, mask, weight, dlogits)
    f32 = torch.float32
    if actions.dtype not in (torch.uint8, torch.int32, torch.int64):
        raise ArgumentError(f"actions: expected dtype uint8, int32 or int64, got {actions.dtype}")
    sr = _rows(ref_logits, (logits.dtype,), n, a, "ref_logits")
    _check_buf(actions, None, n, False, "actions")
    _check_buf(old_logp, f32, n, False, "old_logp")
    _check_buf(advantage, f32, n, False, "advantage")
    _check_buf(ref_logp, f32, n, False, "ref_logp")
    _check_buf(total, f32, 1, False, "total")
    _check_buf(stats, f32, 4 * n, False, "stats")
    _on_device("logits actions old_logp advantage ref_logp ref_logits mask weight total stats "
               "dlogits", logits, actions, old_logp, advantage, ref_logp, ref_logits, mask, weight,
               total, stats, dlogits)
    dev = logits.device
    if total is None:
        total = _empty((1,), f32, dev, stream)
    if stats is None:
        stats = _empty((4, n), f32, dev, stream)
    if not grad:
        dlogits = None
    elif dlogits is None:
        dlogits, sd = _empty((n, a), logits.dtype, dev, stream), a
    wp, nbytes, work = _workspace(_loss_work(code, n, a), work, dev, stream)
    d = _POLICY_LOSS.pack(code, actions.element_size(), n, a, sl, sr, sd, sm, clip_low, clip_high,
                          kl_coef, entropy_coef)
    _check(lib().malib_policy_loss(
        d, logits.data_ptr(), actions.data_ptr(), old_logp.data_ptr(), advantage.data_ptr(),
        _ptr(ref_logp), _ptr(ref_logits), _ptr(mask), _ptr(weight), total.data_ptr(),
        stats.data_ptr(), _ptr(dlogits), wp, nbytes, _stream(stream)))
    return total, stats, dlogits


def distill_loss(logits, teacher_idx, teacher_logits, *, temperature: float = 1.0, mask=None,
                 weight=None, grad: bool = True, total=None, loss=None, dlogits=None, work=None,
                 stream=None):
    """malib_distill_loss: distillation of teachers' top logits (teacher_idx
    int32 and teacher_logits float32 [rows][top], index -1 pads a list) into
    logits [rows][n_actions], and its gradient.  Returns (total [1], loss
    [rows], dlogits or None without `grad`); total is outside torch's autograd
    graph, dlogits is its gradient."""
    if stream is None and logits.is_cuda:
        out = (_calls or _native()).distill_loss(
            logits, teacher_idx, teacher_logits, temperature, mask, weight, grad, total, loss,
            dlogits, work, _current_stream())
        if out is not None:
            return out
    import torch
    n, a, code, sl, sd, sm = _loss_args(logits, mask, weight, dlogits)
    f32 = torch.float32
    if teacher_idx.dim() != 2:
        raise ArgumentError(f"teacher_idx: expected [rows][top], got shape "
                            f"{tuple(teacher_idx.shape)}")
    top = teacher_idx.shape[1]
    _check_buf(teacher_idx, torch.int32, n * top, False, "teacher_idx")
    _check_buf(teacher_logits, f32, n * top, False, "teacher_logits")
    _check_buf(total, f32, 1, False, "total")
    _check_buf(loss, f32, n, False, "loss")
    _on_device("logits teacher_idx teacher_logits mask weight total loss dlogits", logits,
               teacher_idx, teacher_logits, mask, weight, total, loss, dlogits)
    dev = logits.device
    if total is None:
        total = _empty((1,), f32, dev, stream)
    if loss is None:
        loss = _empty((n,), f32, dev, stream)
    if not grad:
        dlogits = None
    elif dlogits is None:
        dlogits, sd = _empty((n, a), logits.dtype, dev, stream), a
    wp, nbytes, work = _workspace(_loss_work(code, n, a), work, dev, stream)
    d = _DISTILL.pack(code, top, n, a, sl, sd, sm, temperature)
    _check(lib().malib_distill_loss(
        d, logits.data_ptr(), teacher_idx.data_ptr(), teacher_logits.data_ptr(), _ptr(mask),
        _ptr(weight), total.data_ptr(), loss.data_ptr(), _ptr(dlogits), wp, nbytes,
        _stream(stream)))
    return total, loss, dlogits


def _here(t):
    """The raw current stream of the device that is current where t lies on it (for the
    native calls), else None."""
    import torch
    d = torch._C._cuda_getDevice()
    return torch._C._cuda_getCurrentRawStream(d) if t.get_device() == d else None


def _guard(t, stream, names, *tensors):
    """Context of a launch over tensors that all have to lie on t's device, on a stream of
    that device."""
    import torch
    _on_device(names, *tensors)
    for u in tensors:
        if u is not None and u.device != t.device:
            what = next(n for n, v in zip(names.split(), tensors) if v is u)
            raise ArgumentError(f"{what}: expected a tensor on {t.device}, got one on {u.device}")
    if stream is not None and stream.device != t.device:
        raise ArgumentError(f"stream: expected one of {t.device}, got one of {stream.device}")
    return torch.cuda.device(t.device)


def _scored(logits, actions, mask, dlogits):
    """What both directions of log_probs check: (rows, n_actions, dtype code, bytes of an
    action, strides of logits, dlogits and mask)."""
    import torch
    n, a, code, sl, sd, sm = _loss_args(logits, mask, None, dlogits)
    if actions is None:
        return n, a, code, 0, sl, sd, sm
    if actions.dtype not in (torch.uint8, torch.int32, torch.int64):
        raise ArgumentError(f"actions: expected dtype uint8, int32 or int64, got {actions.dtype}")
    _check_buf(actions, None, n, False, "actions")
    return n, a, code, actions.element_size(), sl, sd, sm


def log_probs(logits, actions=None, *, temperature: float = 1.0, top: int = 0, mask=None,
              stats=None, top_idx=None, top_logp=None, work=None, stream=None):
    """malib_log_probs: log probabilities of `actions` (uint8, int32 or int64 [rows]; out of
    range: no action) under logits [rows][n_actions] (float32 or bfloat16) over
    `temperature`, the entropy of each row, and its `top` most likely entries.  Returns (stats
    [4][rows] = log probability of the action, entropy, largest legal logit m and the
    logarithm of the sum of e^((x - m) / temperature), top_idx int32 and top_logp
    float32 [rows][top], -1 and 0 behind the last entry, or None without `top`): stats[0] is
    policy_loss's old_logp or ref_logp, the lists are distill_loss's.  Outside torch's
    autograd graph: gradients are log_probs_backward's."""
    if stream is None and logits.is_cuda and (raw := _here(logits)) is not None:
        out = (_calls or _native()).log_probs(logits, actions, temperature, top, mask, stats,
                                              top_idx, top_logp, work, raw)
        if out is not None:
            return out
    import torch
    n, a, code, size, sl, _, sm = _scored(logits, actions, mask, None)
    if not 0 <= top <= 256:
        raise ArgumentError(f"top: expected 0 to 256, got {top}")
    f32 = torch.float32
    _check_buf(stats, f32, 4 * n, False, "stats")
    _check_buf(top_idx, torch.int32, n * top, False, "top_idx")
    _check_buf(top_logp, f32, n * top, False, "top_logp")
    with _guard(logits, stream, "logits actions mask stats top_idx top_logp work", logits,
                actions, mask, stats, top_idx, top_logp, work):
        dev = logits.device
        if stats is None:
            stats = _empty((4, n), f32, dev, stream)
        if top == 0:
            top_idx = top_logp = None
        if top and top_idx is None:
            top_idx = _empty((n, top), torch.int32, dev, stream)
        if top and top_logp is None:
            top_logp = _empty((n, top), f32, dev, stream)
        need = C.c_int64()
        _check(lib().malib_log_probs_work(code, n, a, top, C.byref(need)))
        wp, nbytes, work = _workspace(need.value, work, dev, stream)
        d = _LOG_PROBS.pack(code, size, n, a, sl, 0, sm, top, temperature)
        _check(lib().malib_log_probs(d, logits.data_ptr(), _ptr(actions), _ptr(mask),
                                     stats.data_ptr(), _ptr(top_idx), _ptr(top_logp), wp, nbytes,
                                     _stream(stream)))
    return stats, top_idx, top_logp


def log_probs_backward(logits, actions, stats, dlogp, dentropy=None, *, temperature: float = 1.0,
                       mask=None, dlogits=None, stream=None):
    """malib_log_probs_backward: the gradient of log_probs' logits for the gradients dlogp and
    dentropy (float32 [rows], either may be None) of its first two rows of stats, which
    are taken as log_probs returned them.  Returns dlogits (which may be logits
    itself).  Outside torch's autograd graph."""
    if stream is None and logits.is_cuda and (raw := _here(logits)) is not None:
        out = (_calls or _native()).log_probs_backward(logits, actions, stats, dlogp, dentropy,
                                                       temperature, mask, dlogits, raw)
        if out is not None:
            return out
    import torch
    n, a, code, size, sl, sd, sm = _scored(logits, actions, mask, dlogits)
    f32 = torch.float32
    _check_buf(stats, f32, 4 * n, False, "stats")
    _check_buf(dlogp, f32, n, False, "dlogp")
    _check_buf(dentropy, f32, n, False, "dentropy")
    with _guard(logits, stream, "logits actions mask stats dlogp dentropy dlogits", logits,
                actions, mask, stats, dlogp, dentropy, dlogits):
        if dlogits is None:
            dlogits, sd = _empty((n, a), logits.dtype, logits.device, stream), a
        d = _LOG_PROBS.pack(code, size, n, a, sl, sd, sm, 0, temperature)
        _check(lib().malib_log_probs_backward(
            d, logits.data_ptr(), _ptr(actions), _ptr(mask), stats.data_ptr(), _ptr(dlogp),
            _ptr(dentropy), dlogits.data_ptr(), _stream(stream)))
    return dlogits


def _flat_rows(t, like, what):
    """(rows, cols, row stride) of a tensor whose values are taken in its own order: any
    contiguous one, or [rows][cols] with contiguous rows."""
    if t is None:
        return 0, 0, 0
    if t.shape != like.shape:
        raise ArgumentError(f"{what}: expected shape {tuple(like.shape)}, got {tuple(t.shape)}")
    if t.dtype is not like.dtype:
        raise ArgumentError(f"{what}: expected dtype {like.dtype}, got {t.dtype}")
    cols = t.shape[-1] if t.dim() else 1
    rows = t.numel() // cols if cols else 0
    if t.is_contiguous():
        return rows, cols, cols
    if t.dim() != 2 or (t.stride(1) != 1 and cols > 1):
        raise ArgumentError(f"{what}: expected a contiguous tensor, or [rows][cols] with "
                            f"contiguous rows, got strides {t.stride()}")
    return rows, cols, t.stride(0) if rows > 1 else cols


def _u64(v, what, top=64):
    if not 0 <= v < 1 << top:
        raise ArgumentError(f"{what}: expected a number in [0, 2^{top}), got {v}")
    return v


def dropout(x, p: float, seed: int, step: int = 0, *, layer: int = 0, residual=None, out=None,
            device_step=None, stream=None):
    """malib_dropout: x k / q + residual, where a value stays (k = 1) with probability q = 1 - p
    (in steps of 2^-16) by the library's random stream, from its index, `seed`, `step`
    (plus the int64 in `device_step`, a device tensor of one number) and `layer`
    alone.  The index is that in x: parts of a batch in calls of their own need a layer or seed
    each.  float32 or bfloat16; contiguous tensors of any shape (the last dimension up to 2^24), or
    [rows][cols] with contiguous rows; `out` may be x or residual.  Outside torch's autograd
    graph: the gradient is dropout_backward's, the residual's is dy."""
    if stream is None and x.is_cuda and (raw := _here(x)) is not None:
        y = (_calls or _native()).dropout(x, p, seed, step, layer, residual, out, device_step,
                                          raw)
        if y is not None:
            return y
    import torch
    code = _dtype_code(x, "x")
    rows, cols, sx = _flat_rows(x, x, "x")
    _, _, sr = _flat_rows(residual, x, "residual")
    _, _, sy = _flat_rows(out, x, "out")
    _check_buf(device_step, torch.int64, 1, False, "device_step")
    for v, what, top in ((seed, "seed", 64), (step, "step", 64), (layer, "layer", 32)):
        _u64(v, what, top)
    if not 0.0 <= p <= 1.0:
        raise ArgumentError(f"p: expected a probability, got {p}")
    with _guard(x, stream, "x residual out device_step", x, residual, out, device_step):
        if out is None:
            out, sy = _empty((tuple(x.shape),), x.dtype, x.device, stream), cols
        if x.numel():
            d = _DROPOUT.pack(code, layer, rows, cols, sx, sr, sy, seed, step, p)
            _check(lib().malib_dropout(d, x.data_ptr(), _ptr(residual), _ptr(device_step),
                                       out.data_ptr(), _stream(stream)))
    return out


def dropout_backward(dy, p: float, seed: int, step: int = 0, *, layer: int = 0, dx=None,
                     device_step=None, stream=None):
    """The gradient of dropout's x for the gradient dy of its output: dy k / q, with the mask
    formed again from p, seed, step and layer.  dx may be dy itself."""
    return dropout(dy, p, seed, step, layer=layer, out=dx, device_step=device_step,
                   stream=stream)


def _fp4_shape(n_out, n_in, group):
    if group not in (32, 64, 128):
        raise ArgumentError(f"group: expected 32, 64 or 128, got {group}")
    tiles, blocks = (n_out + 15) // 16, (n_in + 127) // 128
    return (tiles, blocks, 64, 16), (tiles, blocks, 16, 128 // group)


def _fp4_held(codes, scales, G, n_out, n_in):
    """Checks codes and scales of a layer; returns their scale group."""
    import torch
    per = scales.shape[-1] if scales.dim() else 0
    if per not in (1, 2, 4):
        raise ArgumentError(f"scales: expected 1, 2 or 4 in the last dimension, got shape "
                            f"{tuple(scales.shape)}")
    lead = () if G is None else (G,)
    for t, shape, dt, align, what in zip(
            (codes, scales), _fp4_shape(n_out, n_in, 128 // per),
            (torch.uint8, torch.bfloat16), (16, 8), ("codes", "scales")):
        if t.shape != lead + shape:
            raise ArgumentError(f"{what}: expected shape {lead + shape}, got {tuple(t.shape)}")
        _check_buf(t, dt, None, False, what)
        if t.data_ptr() % align:
            raise ArgumentError(f"{what}: expected to start on {align} bytes")
    return 128 // per


def quantize_fp4(w, group: int = 32, *, codes=None, scales=None, stream=None):
    """malib_quantize_fp4: weights [out][in] or [groups][out][in] (float32 or bfloat16) in 4
    bits, `group` (32, 64 or 128) weights of a row sharing a scale.  Returns (codes uint8
    [..][ceil(out / 16)][ceil(in / 128)][64][16], scales bfloat16
    [..][ceil(out / 16)][ceil(in / 128)][16][128 / group]), in the order that linear_fp4
    takes."""
    if stream is None and w.is_cuda and (raw := _here(w)) is not None:
        out = (_calls or _native()).quantize_fp4(w, group, codes, scales, raw)
        if out is not None:
            return out
    import torch
    code = _dtype_code(w, "w")
    if w.dim() not in (2, 3):
        raise ArgumentError(f"w: expected [out][in] or [groups][out][in], got shape "
                            f"{tuple(w.shape)}")
    G, (n_out, n_in) = w.shape[0] if w.dim() == 3 else None, w.shape[-2:]
    mw = _mat(w, w.dtype, G, n_out, n_in, "w")
    sc, ss = _fp4_shape(n_out, n_in, group)
    lead = () if G is None else (G,)
    with _guard(w, stream, "w codes scales", w, codes, scales):
        if codes is None:
            codes = _empty((lead + sc,), torch.uint8, w.device, stream)
        if scales is None:
            scales = _empty((lead + ss,), torch.bfloat16, w.device, stream)
        if _fp4_held(codes, scales, G, n_out, n_in) != group:
            raise ArgumentError(f"scales: expected those of groups of {group}")
        d = _FP4.pack(code, ACT_NONE, 1 if G is None else G, 0, n_in, n_out, group, 0)
        _check(lib().malib_quantize_fp4(d, mw, codes.data_ptr(), scales.data_ptr(),
                                        _stream(stream)))
    return codes, scales


def dequantize_fp4(codes, scales, n_out: int, n_in: int, *, dtype=None, out=None, stream=None):
    """malib_dequantize_fp4: the weights [out][in] (or [groups][out][in]) that quantize_fp4's
    codes and scales stand for, in `dtype` (bfloat16 unless `out` has another; float32 is
    exact)."""
    if stream is None and codes.is_cuda and (raw := _here(codes)) is not None:
        w = (_calls or _native()).dequantize_fp4(codes, scales, n_out, n_in, dtype, out, raw)
        if w is not None:
            return w
    import torch
    G = codes.shape[0] if codes.dim() == 5 else None
    group = _fp4_held(codes, scales, G, n_out, n_in)
    if dtype is None:
        dtype = torch.bfloat16 if out is None else out.dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise ArgumentError(f"dtype: expected float32 or bfloat16, got {dtype}")
    with _guard(codes, stream, "codes scales out", codes, scales, out):
        if out is None:
            shape = (n_out, n_in) if G is None else (G, n_out, n_in)
            out = _empty((shape,), dtype, codes.device, stream)
        mw = _mat(out, dtype, G, n_out, n_in, "out", True)
        d = _FP4.pack(DT_BF16 if dtype is torch.bfloat16 else DT_F32, ACT_NONE,
                      1 if G is None else G, 0, n_in, n_out, group, 0)
        _check(lib().malib_dequantize_fp4(d, codes.data_ptr(), scales.data_ptr(), mw,
                                          _stream(stream)))
    return out


def linear_fp4(x, codes, scales, n_out: int, bias=None, *, act: int = ACT_NONE, residual=None,
               out=None, stream=None):
    """malib_linear_fp4: act(x w^T + bias) + residual with the weights of quantize_fp4, for
    x [rows][in], or with weights of several policies [groups][rows][in] (x without the
    group dimension is shared by the groups); float32 or bfloat16, bias float32.  For up to
    hundreds of bfloat16 rows (of all policies) of a wide layer, or thousands of a narrow one or in
    float32; for more linear on dequantize_fp4's weights takes less time.  Returns
    [..][rows][out]; nothing here has a gradient."""
    if stream is None and x.is_cuda and (raw := _here(x)) is not None:
        y = (_calls or _native()).linear_fp4(x, codes, scales, n_out, bias, act, residual, out,
                                             raw)
        if y is not None:
            return y
    code = _dtype_code(x, "x")
    G = codes.shape[0] if codes.dim() == 5 else None
    if x.dim() != 2 and (x.dim() != 3 or G is None):
        raise ArgumentError(f"x: expected [rows][in] or, with weights per group, "
                            f"[groups][rows][in], got shape {tuple(x.shape)}")
    if act not in (ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU):
        raise ArgumentError(f"act: unknown activation {act!r}")
    (rows, n_in), dt = x.shape[-2:], x.dtype
    group = _fp4_held(codes, scales, G, n_out, n_in)
    mx = _mat(x, dt, G, rows, n_in, "x")
    mr = _mat(residual, dt, G, rows, n_out, "residual")
    _check_buf(bias, _f32(), n_out * (1 if G is None else G), False, "bias")
    with _guard(x, stream, "x codes scales bias residual out", x, codes, scales, bias, residual,
                out):
        if out is None:
            out = _empty(((rows, n_out) if G is None else (G, rows, n_out),), dt, x.device,
                         stream)
        my = _mat(out, dt, G, rows, n_out, "out", True)
        d = _FP4.pack(code, act, 1 if G is None else G, rows, n_in, n_out, group, 0)
        _check(lib().malib_linear_fp4(d, mx, codes.data_ptr(), scales.data_ptr(), _ptr(bias), mr,
                                      my, _stream(stream)))
    return out


def debug_tanh_ref(x, y=None, stream=None):
    import torch
    if y is None:
        y = torch.empty_like(x)
    _check(lib().malib_debug_tanh_ref(_dptr(x, torch.float32, what="x"),
                                      _dptr(y, torch.float32, x.numel(), what="y"), x.numel(),
                                      _stream(stream)))
    return y


def debug_bf16(x, stream=None):
    """bf16 bit patterns (as int16) of an even-length fp32 device tensor."""
    import torch
    y = torch.empty(x.shape, dtype=torch.int16, device=x.device)
    _check(lib().malib_debug_bf16(_dptr(x, torch.float32, what="x"), _dptr(y), x.numel(),
                                  _stream(stream)))
    return y


def debug_philox(ctr, key0: int, key1: int, stream=None):
    import torch
    if ctr.dim() != 2 or ctr.shape[1] != 4:
        raise ArgumentError(f"ctr: expected [n][4] counters, got shape {tuple(ctr.shape)}")
    out = torch.empty_like(ctr)
    _check(lib().malib_debug_philox(_dptr(ctr, torch.int64, what="ctr"), key0, key1, _dptr(out),
                                    ctr.shape[0], _stream(stream)))
    return out
