"""Thin Python binding of libef21 (argument marshalling only).

PyTorch is used for device memory, streams and host<->device copies; every
step of the EF21 hot path runs inside the CUDA library.  There is no CPU or
PyTorch fallback: if ``libef21.so`` has not been built (``python -m
paper_2106_05203_b200.build``) importing this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.util
import os
import warnings
from typing import NamedTuple, Optional, Tuple

import numpy as np
import torch

from .build import call_built_for

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libef21.so")
CALL_PATH = os.path.join(_HERE, "_topk_call.so")
MODEL_CALL_PATH = os.path.join(_HERE, "_model_call.so")

EF21_OK = 0
STATUS_NAMES = {0: "EF21_OK", 1: "EF21_ERR_INVALID_ARG", 2: "EF21_ERR_STATE", 3: "EF21_ERR_WORKSPACE",
                4: "EF21_ERR_CUDA", 5: "EF21_ERR_TIMEOUT", 6: "EF21_ERR_NONFINITE", 7: "EF21_ERR_UNSUPPORTED"}
INIT_COMPRESSED, INIT_ZERO, INIT_GRADIENT = 0, 1, 2
PATH_AUTO, PATH_LAUNCHES, PATH_PERSISTENT = 0, 1, 2
VARIANT_EF21, VARIANT_EF21_PLUS, VARIANT_EF = 0, 1, 2
OBJECTIVE_LOGISTIC, OBJECTIVE_LEAST_SQUARES = 0, 1

# name -> (restype, argtypes); mirrors include/ef21.h
_i32, _i64, _f32, _f64, _sz, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_size_t, ctypes.c_void_p
_dp = ctypes.POINTER(ctypes.c_double)
SIGNATURES = {
    "ef21_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "ef21_workspace_bytes": (_sz, [_i32, _i64, _i32, _i64]),
    "ef21_create": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _f32, _f32, _i64, _vp, _sz, _vp]),
    "ef21_destroy": (None, [_vp]),
    "ef21_load_shards": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "ef21_load_shards_host": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "ef21_set_x": (ctypes.c_int, [_vp, _vp]),
    "ef21_init": (ctypes.c_int, [_vp, _i32]),
    "ef21_init_grads": (ctypes.c_int, [_vp, _vp, _i32]),
    "ef21_step": (ctypes.c_int, [_vp, _i32]),
    "ef21_step_grads": (ctypes.c_int, [_vp, _vp, _i32]),
    "ef21_step_minibatch": (ctypes.c_int, [_vp, _vp, _i32]),
    "ef21_step_minibatches": (ctypes.c_int, [_vp, _vp, _i32, _i32]),
    "ef21_step_randk": (ctypes.c_int, [_vp, _vp, _vp, _i32]),
    "ef21_local_grads": (ctypes.c_int, [_vp, _vp]),
    "ef21_topk_workspace_bytes": (_sz, [_i32, _i64, _i32]),
    "ef21_topk": (ctypes.c_int, [_vp, _i32, _i64, _i32, _vp, _vp, _vp, _sz, _vp]),
    "ef21_topk_static": (ctypes.c_int, [_vp, _i32, _i64, _i32, _vp, _vp, _vp]),
    "ef21_get_state": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp]),
    "ef21_get_state_host": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp]),
    "ef21_set_state": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "ef21_eval": (ctypes.c_int, [_vp, _dp, _dp, _dp]),
    "ef21_poll": (ctypes.c_int, [_vp]),
    "ef21_set_objective": (ctypes.c_int, [_vp, _i32]),
    "ef21_set_variant": (ctypes.c_int, [_vp, _i32]),
    "ef21_get_plus_choice": (ctypes.c_int, [_vp, _vp]),
    "ef21_set_topk_algorithm": (ctypes.c_int, [_vp, _i32]),
    "ef21_fallback_count": (ctypes.c_int, [_vp, ctypes.POINTER(_i64)]),
    "ef21_clear_status": (ctypes.c_int, [_vp]),
    "ef21_selftest_bounded_wait": (ctypes.c_int, [_vp, ctypes.c_uint32]),
    "ef21_selftest_exchange_floor": (ctypes.c_int, [_vp, ctypes.c_int32]),
    "ef21_set_persistent_body": (ctypes.c_int, [_vp, ctypes.c_int32]),
    "ef21_get_persistent_body": (ctypes.c_int32, [_vp]),
    "ef21_set_persistent_shape": (ctypes.c_int, [_vp, _i32, _i32, _i32]),
    "ef21_get_persistent_shape": (ctypes.c_int, [_vp, ctypes.POINTER(_i32), ctypes.POINTER(_i32), ctypes.POINTER(_i32)]),
    "ef21_get_persistent_form": (ctypes.c_int, [_vp, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]),
    "ef21_set_persistent_threads": (ctypes.c_int, [_vp, _i32]),
    "ef21_get_persistent_threads": (_i32, [_vp]),
    "ef21_set_path": (ctypes.c_int, [_vp, _i32]),
    "ef21_last_path": (_i32, [_vp]),
    "ef21_launch_count": (_i64, [_vp]),
    "ef21_token_logprobs_workspace_bytes": (_sz, [_i32, _i64, _i64, _i64]),
    "ef21_token_logprobs": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _i64, _i64, _vp, _i32, _i64, _f32, _i64, _vp, _vp, _vp, _sz, _vp]),
    "ef21_token_logprobs_grad": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _i64, _i64, _vp, _i32, _i64, _vp, _vp, _f32, _i64, _vp, _i64, _i64, _vp]),
    "ef21_preference_loss_workspace_bytes": (_sz, [_i64, _i64]),
    "ef21_preference_loss": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i64, _i64, _i64, _i64, _i64, _f64, _f64, _f64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "ef21_policy_loss_workspace_bytes": (_sz, [_i64, _i64]),
    "ef21_policy_loss": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _i32, _f64, _f64, _f64, _i32, _f64,
                                        _vp, _vp, _vp, _sz, _vp]),
    "ef21_balance_loss_workspace_bytes": (_sz, [_i64, _i64]),
    "ef21_balance_loss": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _vp, _i32, _i64, _i64, _vp, _f64, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "ef21_embedding": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _vp, _i32, _i64, _f32, _vp, _vp]),
    "ef21_embedding_grad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "ef21_embedding_grad": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _vp, _i32, _i64, _i64, _f32, _vp, _i32, _i64, _i32, _vp, _sz, _vp]),
}


class Ef21Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2106_05203_b200.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)          # AttributeError if the symbol is not exported
        fn.restype = res
        fn.argtypes = args
    return lib


def _load_module(name: str, path: str):
    spec = importlib.util.spec_from_file_location(name, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    if module.built_for != call_built_for():
        raise ImportError(f"{path} was built for {module.built_for}, this is {call_built_for()}")
    return module


def _address(entry) -> int:
    return ctypes.cast(entry, _vp).value


def _load_call(path: str = CALL_PATH):
    """The native form of topk() for the usual arguments (csrc/topk_call.cpp).  Where it is missing or does not fit this torch, every
    call of topk() is the general one, 4 us slower on short vectors."""
    try:
        module = _load_module("_topk_call", path)
    except (ImportError, OSError, AttributeError) as e:
        warnings.warn(f"topk() without its native call ({e}): build it with `python -m paper_2106_05203_b200.build`", RuntimeWarning, stacklevel=2)
        return lambda v, k: None
    module.set_entry(*(_address(f) for f in (_lib.ef21_topk_workspace_bytes, _lib.ef21_topk)))
    return module.topk


class _GeneralCalls:
    """In place of the native calls of a language model's worker: every call is the general one."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_model_calls(path: str = MODEL_CALL_PATH):
    """The native forms of token_logprobs() to embedding_grad() for the usual arguments (csrc/model_call.cpp).  Where they are missing or do not fit this
    torch, every call is the general one, some 10 us slower on small batches."""
    try:
        module = _load_module("_model_call", path)
        module.set_entries(*(_address(getattr(_lib, f)) for f in (
            "ef21_token_logprobs_workspace_bytes", "ef21_token_logprobs", "ef21_token_logprobs_grad", "ef21_preference_loss_workspace_bytes", "ef21_preference_loss", "ef21_policy_loss_workspace_bytes",
            "ef21_policy_loss", "ef21_balance_loss_workspace_bytes", "ef21_balance_loss", "ef21_embedding", "ef21_embedding_grad_workspace_bytes", "ef21_embedding_grad")))
    except (ImportError, OSError, AttributeError, TypeError) as e:
        warnings.warn(f"losses and embedding without their native calls ({e}): build them with `python -m paper_2106_05203_b200.build`", RuntimeWarning, stacklevel=2)
        return _GeneralCalls()
    return module


_lib = load_library()
_topk_call = _load_call()
_model_calls = _load_model_calls()


def _check(status: int, where: str) -> None:
    if status != EF21_OK:
        raise Ef21Error(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _stream_handle(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _dev_f32(t: torch.Tensor, shape=None) -> torch.Tensor:
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise TypeError("expected a contiguous float32 CUDA tensor")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def workspace_bytes(n: int, d: int, k: int, total_rows: int) -> int:
    return int(_lib.ef21_workspace_bytes(n, d, k, total_rows))


def status_string(status: int) -> str:
    return _lib.ef21_status_string(status).decode()


class EF21:
    """One EF21 problem resident on one GPU (names follow include/ef21.h)."""

    def __init__(self, n: int, d: int, k: int, gamma: float, lam: float = 0.0, total_rows: int = 0,
                 device: Optional[torch.device] = None, stream: Optional[torch.cuda.Stream] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("libef21 needs a CUDA device; there is no CPU path")
        self.device = torch.device(device if device is not None else "cuda:0")
        self.n, self.d, self.k, self.total_rows = int(n), int(d), int(k), int(total_rows)
        self.stream = stream
        nbytes = workspace_bytes(n, d, k, total_rows)
        if nbytes == 0:
            raise Ef21Error(1, "ef21_workspace_bytes")
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
            handle = _vp()
            _check(_lib.ef21_create(ctypes.byref(handle), n, d, k, gamma, lam, total_rows,
                                    ctypes.c_void_p(self._ws_ptr), nbytes, _stream_handle(stream)), "ef21_create")
        self._h = handle
        self._keep = []          # tensors that must outlive asynchronous calls

    def close(self) -> None:
        if getattr(self, "_h", None):
            _lib.ef21_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- data ---------------------------------------------------------------
    def load_shards(self, A: torch.Tensor, y: torch.Tensor, row_offsets) -> None:
        off = np.ascontiguousarray(np.asarray(row_offsets), dtype=np.int64)
        if off.shape != (self.n + 1,):
            raise ValueError("row_offsets must have n+1 entries")
        _dev_f32(A, (self.total_rows, self.d)); _dev_f32(y, (self.total_rows,))
        _check(_lib.ef21_load_shards(self._h, _ptr(A), _ptr(y), _np_ptr(off)), "ef21_load_shards")
        self._keep = [A, y]

    def load_shards_host(self, A: np.ndarray, y: np.ndarray, row_offsets) -> None:
        off = np.ascontiguousarray(np.asarray(row_offsets), dtype=np.int64)
        if off.shape != (self.n + 1,):
            raise ValueError("row_offsets must have n+1 entries")
        A = np.ascontiguousarray(A, dtype=np.float32); y = np.ascontiguousarray(y, dtype=np.float32)
        if A.shape != (self.total_rows, self.d) or y.shape != (self.total_rows,):
            raise ValueError("A must be [total_rows, d], y [total_rows]")
        _check(_lib.ef21_load_shards_host(self._h, _np_ptr(A), _np_ptr(y), _np_ptr(off)), "ef21_load_shards_host")
        self._keep = [A, y]

    def set_x(self, x0: torch.Tensor) -> None:
        _check(_lib.ef21_set_x(self._h, _ptr(_dev_f32(x0, (self.d,)))), "ef21_set_x")

    # -- algorithm ----------------------------------------------------------
    def init(self, mode: int = INIT_COMPRESSED) -> None:
        _check(_lib.ef21_init(self._h, mode), "ef21_init")

    def init_grads(self, V: Optional[torch.Tensor], mode: int = INIT_COMPRESSED) -> None:
        if V is not None:
            _dev_f32(V, (self.n, self.d))
        _check(_lib.ef21_init_grads(self._h, _ptr(V), mode), "ef21_init_grads")

    def step(self, steps: int = 1) -> None:
        _check(_lib.ef21_step(self._h, steps), "ef21_step")

    def step_grads(self, V: torch.Tensor, steps: int = 1) -> None:
        _check(_lib.ef21_step_grads(self._h, _ptr(_dev_f32(V, (self.n, self.d))), steps), "ef21_step_grads")

    def step_minibatch(self, batch: torch.Tensor) -> None:
        """One stochastic iteration; batch[n, tau] int32 row numbers inside each worker's shard."""
        if not (batch.is_cuda and batch.dtype == torch.int32 and batch.is_contiguous() and batch.dim() == 2
                and batch.shape[0] == self.n):
            raise TypeError("batch must be a contiguous int32 CUDA tensor of shape [n, tau]")
        _check(_lib.ef21_step_minibatch(self._h, _ptr(batch), int(batch.shape[1])), "ef21_step_minibatch")
        self._keep_batch = batch

    def step_minibatches(self, batches: torch.Tensor) -> None:
        """batches[steps, n, tau] int32 row numbers inside each worker's shard: that many stochastic iterations."""
        if not (batches.is_cuda and batches.dtype == torch.int32 and batches.is_contiguous() and batches.dim() == 3
                and batches.shape[1] == self.n):
            raise TypeError("batches must be a contiguous int32 CUDA tensor of shape [steps, n, tau]")
        _check(_lib.ef21_step_minibatches(self._h, _ptr(batches), int(batches.shape[2]), int(batches.shape[0])),
               "ef21_step_minibatches")
        self._keep_batch = batches

    def step_randk(self, sets: torch.Tensor, V: Optional[torch.Tensor] = None) -> None:
        """sets[steps, n, k] int32 (ascending, distinct coordinates per worker): that many iterations with the scaled
        Rand-k compressor; V[n, d] (optional) replaces the local gradients."""
        if not (sets.is_cuda and sets.dtype == torch.int32 and sets.is_contiguous() and sets.dim() == 3
                and sets.shape[1] == self.n and sets.shape[2] == self.k):
            raise TypeError("sets must be a contiguous int32 CUDA tensor of shape [steps, n, k]")
        if V is not None:
            _dev_f32(V, (self.n, self.d))
        _check(_lib.ef21_step_randk(self._h, _ptr(V), _ptr(sets), int(sets.shape[0])), "ef21_step_randk")
        self._keep_batch = (sets, V)

    def local_grads(self) -> torch.Tensor:
        out = torch.empty((self.n, self.d), dtype=torch.float32, device=self.device)
        _check(_lib.ef21_local_grads(self._h, _ptr(out)), "ef21_local_grads")
        return out

    # -- state --------------------------------------------------------------
    def get_state(self, messages: bool = True):
        """(x, g, gi, last_idx, last_val) as new device tensors."""
        dev = self.device
        x = torch.empty(self.d, dtype=torch.float32, device=dev)
        g = torch.empty(self.d, dtype=torch.float32, device=dev)
        gi = torch.empty((self.n, self.d), dtype=torch.float32, device=dev)
        li = torch.empty((self.n, self.k), dtype=torch.int32, device=dev) if messages else None
        lv = torch.empty((self.n, self.k), dtype=torch.float32, device=dev) if messages else None
        _check(_lib.ef21_get_state(self._h, _ptr(x), _ptr(g), _ptr(gi), _ptr(li), _ptr(lv)), "ef21_get_state")
        return x, g, gi, li, lv

    def get_state_host(self, want_gi: bool = True, messages: bool = True):
        """(x, g, gi, last_idx, last_val) as numpy arrays; synchronises."""
        x = np.empty(self.d, dtype=np.float32)
        g = np.empty(self.d, dtype=np.float32)
        gi = np.empty((self.n, self.d), dtype=np.float32) if want_gi else None
        li = np.empty((self.n, self.k), dtype=np.int32) if messages else None
        lv = np.empty((self.n, self.k), dtype=np.float32) if messages else None
        _check(_lib.ef21_get_state_host(self._h, _np_ptr(x), _np_ptr(g), _np_ptr(gi), _np_ptr(li), _np_ptr(lv)),
               "ef21_get_state_host")
        return x, g, gi, li, lv

    def set_state(self, x: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None,
                  gi: Optional[torch.Tensor] = None) -> None:
        if x is not None: _dev_f32(x, (self.d,))
        if g is not None: _dev_f32(g, (self.d,))
        if gi is not None: _dev_f32(gi, (self.n, self.d))
        _check(_lib.ef21_set_state(self._h, _ptr(x), _ptr(g), _ptr(gi)), "ef21_set_state")

    def eval(self) -> Tuple[float, float, float]:
        f, nrm, G = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        _check(_lib.ef21_eval(self._h, ctypes.byref(f), ctypes.byref(nrm), ctypes.byref(G)), "ef21_eval")
        return f.value, nrm.value, G.value

    def poll(self) -> int:
        return int(_lib.ef21_poll(self._h))

    def set_objective(self, objective: int) -> None:
        _check(_lib.ef21_set_objective(self._h, objective), "ef21_set_objective")

    def set_variant(self, variant: int) -> None:
        _check(_lib.ef21_set_variant(self._h, variant), "ef21_set_variant")

    def get_plus_choice(self) -> np.ndarray:
        out = np.zeros(self.n, dtype=np.int32)
        _check(_lib.ef21_get_plus_choice(self._h, _np_ptr(out)), "ef21_get_plus_choice")
        return out

    def set_topk_algorithm(self, algorithm: int) -> None:
        _check(_lib.ef21_set_topk_algorithm(self._h, algorithm), "ef21_set_topk_algorithm")

    def fallback_count(self) -> int:
        v = _i64()
        _check(_lib.ef21_fallback_count(self._h, ctypes.byref(v)), "ef21_fallback_count")
        return int(v.value)

    def clear_status(self) -> None:
        _check(_lib.ef21_clear_status(self._h), "ef21_clear_status")

    def selftest_bounded_wait(self, spin_limit: int) -> None:
        _check(_lib.ef21_selftest_bounded_wait(self._h, spin_limit), "ef21_selftest_bounded_wait")

    def set_persistent_body(self, body: int) -> None:
        _check(_lib.ef21_set_persistent_body(self._h, body), "ef21_set_persistent_body")

    def get_persistent_body(self) -> int:
        return int(_lib.ef21_get_persistent_body(self._h))

    def selftest_exchange_floor(self, steps: int) -> None:
        _check(_lib.ef21_selftest_exchange_floor(self._h, steps), "ef21_selftest_exchange_floor")

    def set_persistent_shape(self, cluster_blocks: int = 0, rows_per_batch: int = 0, row_source: int = -1) -> None:
        _check(_lib.ef21_set_persistent_shape(self._h, cluster_blocks, rows_per_batch, row_source),
               "ef21_set_persistent_shape")

    def get_persistent_shape(self):
        c, r, s = _i32(), _i32(), _i32()
        _check(_lib.ef21_get_persistent_shape(self._h, ctypes.byref(c), ctypes.byref(r), ctypes.byref(s)),
               "ef21_get_persistent_shape")
        return c.value, r.value, s.value

    def get_persistent_form(self):
        """(all workers in one cluster, ring stages per warp) of the last persistent launch."""
        one, stages = _i32(), _i32()
        _check(_lib.ef21_get_persistent_form(self._h, ctypes.byref(one), ctypes.byref(stages)), "ef21_get_persistent_form")
        return bool(one.value), stages.value

    def set_persistent_threads(self, threads_per_block: int) -> None:
        _check(_lib.ef21_set_persistent_threads(self._h, threads_per_block), "ef21_set_persistent_threads")

    def get_persistent_threads(self) -> int:
        return int(_lib.ef21_get_persistent_threads(self._h))

    def set_path(self, path: int) -> None:
        _check(_lib.ef21_set_path(self._h, path), "ef21_set_path")

    @property
    def last_path(self) -> int:
        return int(_lib.ef21_last_path(self._h))

    @property
    def launch_count(self) -> int:
        return int(_lib.ef21_launch_count(self._h))


_NO_SCRATCH = 256            # workspace size of shapes whose selection uses no scratch (the pointer still has to be valid)
_no_scratch_memory = {}      # device index -> one 512-byte tensor, never written


def _no_scratch(index: int) -> int:
    t = _no_scratch_memory.get(index)
    if t is None:
        t = _no_scratch_memory.setdefault(index, torch.empty(512, dtype=torch.uint8, device=torch.device("cuda", index)))
    return (t.data_ptr() + 255) // 256 * 256


def _current_raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):          # the same handle without a Stream object around it
    _current_raw_stream = torch._C._cuda_getCurrentRawStream


@functools.lru_cache(maxsize=1024)
def _topk_workspace_bytes(batch: int, d: int, k: int) -> int:
    nbytes = int(_lib.ef21_topk_workspace_bytes(batch, d, k))
    if nbytes == 0:
        raise Ef21Error(1, "ef21_topk_workspace_bytes")
    return nbytes


def topk(v: torch.Tensor, k: int, stream: Optional[torch.cuda.Stream] = None):
    """Top-k compressor on a batch of vectors v[batch, d] -> (idx[batch, k] int32, val[batch, k])."""
    if stream is None:
        out = _topk_call(v, k)                              # None: not one of the usual calls
        if out is not None:
            if type(out) is tuple:
                return out
            raise Ef21Error(out, "ef21_topk")
    if v.dim() == 1:
        v = v.unsqueeze(0)
    _dev_f32(v)
    batch, d = v.shape
    nbytes = _topk_workspace_bytes(batch, d, k)
    device = v.device
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return topk(v, k, stream)
    # No scratch is allocated where the library needs none, and nothing is recorded on the stream that everything was allocated on.
    idx = torch.empty_strided((batch, k), (k, 1), dtype=torch.int32, device=device)
    val = torch.empty_strided((batch, k), (k, 1), dtype=torch.float32, device=device)
    if nbytes <= _NO_SCRATCH:
        ws_ptr = _no_scratch(device.index)
    else:
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        ws_ptr = (ws.data_ptr() + 255) // 256 * 256
        if stream is not None:
            ws.record_stream(stream)
    handle = stream.cuda_stream if stream is not None else _current_raw_stream(device.index)
    status = _lib.ef21_topk(v.data_ptr(), batch, d, k, idx.data_ptr(), val.data_ptr(), ws_ptr, nbytes, handle)
    if status != EF21_OK:
        raise Ef21Error(status, "ef21_topk")
    return idx, val


def topk_static(v: torch.Tensor, k: int, idx: torch.Tensor, val: torch.Tensor,
                stream: Optional[torch.cuda.Stream] = None) -> None:
    """ef21_topk_static: Top-k into caller-provided outputs idx[batch, k] (int32) and val[batch, k]
    (float32) with no device scratch handed over and none allocated; for callers that must not
    touch the CUDA allocator.  Raises Ef21Error(EF21_ERR_UNSUPPORTED) beyond the built-in scratch
    (batch <= 64, batch * ceil(d / 4096) <= 16384)."""
    if v.dim() == 1:
        v = v.unsqueeze(0)
    _dev_f32(v)
    batch, d = v.shape
    if not (idx.is_cuda and idx.dtype == torch.int32 and idx.is_contiguous() and idx.numel() == batch * k):
        raise TypeError("idx must be a contiguous int32 CUDA tensor with batch*k entries")
    if not (val.is_cuda and val.dtype == torch.float32 and val.is_contiguous() and val.numel() == batch * k):
        raise TypeError("val must be a contiguous float32 CUDA tensor with batch*k entries")
    with torch.cuda.device(v.device):
        _check(_lib.ef21_topk_static(_ptr(v), batch, d, k, _ptr(idx), _ptr(val), _stream_handle(stream)),
               "ef21_topk_static")


# -- objectives of a language model's worker, and the sparse end of its gradient ------------------------------------------------------
# Every call works on the current stream of its tensors' device, or on `stream`: outputs and workspace then belong to that stream, and the
# caller orders it behind what made the inputs.  Results are constants to torch's autograd; a gradient goes on with tensor.backward(gradient).

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INDEX_TYPES = {torch.int32: 0, torch.int64: 1}
REDUCTIONS = {"token": 0, "sequence": 1}


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor          # fp32, one number
    rewards: torch.Tensor       # fp32 [2 P]: beta times every row's log ratio
    grad: torch.Tensor          # [2 P, T]: of logps, in its type


class PolicyLoss(NamedTuple):
    terms: torch.Tensor         # fp32 [4]: the loss, its policy term, the KL term before its weight, the share of clipped tokens
    grad: torch.Tensor          # [R, T]: of logps, in its type


class BalanceLoss(NamedTuple):
    loss: torch.Tensor          # fp32, one number
    counts: torch.Tensor        # int32 [E]: tokens per expert
    probs: torch.Tensor         # fp32 [E]: mean probabilities
    grad: torch.Tensor          # [R, E]: of the logits, in their type


def _native(out, where: str):
    """What a native call gave: its result, or the library's refusal."""
    if type(out) is int:
        raise Ef21Error(out, where)
    return out


def _type_of(t: torch.Tensor, name: str) -> int:
    code = DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _index_type_of(t: torch.Tensor, name: str) -> int:
    code = INDEX_TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be int32 or int64, not {t.dtype}")
    return code


def _last_contiguous(t: torch.Tensor, name: str) -> None:
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise TypeError(f"the last dimension of {name} must be contiguous")


def _matrix(t: torch.Tensor, name: str, shape, dtype=None) -> int:
    """The row stride of a matrix with contiguous rows."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be of shape {tuple(shape)}, not {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    _last_contiguous(t, name)
    return t.stride(0)


def _mask(t: Optional[torch.Tensor], shape) -> int:
    if t is None:
        return 0
    if t.dtype not in (torch.bool, torch.uint8):
        raise TypeError(f"mask must be bool or uint8, not {t.dtype}")
    return _matrix(t, "mask", shape)


def _same_device(*tensors: Optional[torch.Tensor]) -> torch.device:
    """The device of a call's tensors, whose memory has to hold their values."""
    if any(t is not None and t.is_neg() for t in tensors):
        raise TypeError("a view that takes the negative as it is read (resolve_neg() writes it out)")
    device = tensors[0].device
    if device.type != "cuda":
        raise TypeError("expected CUDA tensors; there is no CPU path")
    for t in tensors[1:]:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and on {t.device}")
    return device


def _elsewhere(device: torch.device, stream: Optional[torch.cuda.Stream]):
    """None where the call's stream and device are the current ones; else the context in which they are."""
    if stream is not None:
        if not isinstance(stream, torch.cuda.Stream):
            raise TypeError(f"stream must be a torch.cuda.Stream, not {type(stream).__name__}")
        if stream.device != device:
            raise ValueError(f"tensors on {device}, a stream of {stream.device}")
        return torch.cuda.stream(stream)
    return None if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _rows_apart(t: torch.Tensor, name: str) -> None:
    """Refuses a tensor some of whose rows lie on one another: every stride must step over all that the smaller ones reach."""
    reach = t.shape[-1]
    for size, stride in sorted(((n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n > 1), key=lambda p: p[1]):
        if stride < reach:
            raise ValueError(f"rows of {name} overlap")
        reach += (size - 1) * stride


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether the stretches of memory from the first to the last element of two tensors meet."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    (x, y), (u, v) = ((t.data_ptr(), t.data_ptr() + (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()) for t in (a, b))
    return x < v and u < y


def _workspace(nbytes: int, device: torch.device, where: str):
    """A workspace, and its 256-byte aligned address."""
    if nbytes == 0:
        raise Ef21Error(1, where)
    ws = torch.empty(nbytes + 255, dtype=torch.uint8, device=device)
    return ws, (ws.data_ptr() + 255) // 256 * 256


def _logit_rows(logits: torch.Tensor, name: str):
    """(batch, length, vocab, batch stride, row stride) of a matrix of rows, or of one per batch entry; a view such as x[:, :-1] is one too."""
    if logits.dim() == 2:
        _last_contiguous(logits, name)
        return 1, logits.shape[0], logits.shape[1], 0, logits.stride(0)
    if logits.dim() != 3:
        raise ValueError(f"{name} must be [rows, vocab] or [batch, length, vocab], not {tuple(logits.shape)}")
    _last_contiguous(logits, name)
    return (*logits.shape, logits.stride(0), logits.stride(1))


def _targets_fit(targets: torch.Tensor, logits: torch.Tensor) -> None:
    if targets.shape != logits.shape[:-1]:
        raise ValueError(f"targets must be of shape {tuple(logits.shape[:-1])}, not {tuple(targets.shape)}")


def _target_rows(targets: torch.Tensor):
    """targets and their stride between batch entries; copied where those of an entry do not follow one another (eight bytes a row)."""
    if targets.shape[-1] > 1 and targets.stride(-1) != 1:
        targets = targets.contiguous()
    return targets, targets.stride(0) if targets.dim() == 2 else 0


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, ignore: int = -100, stream: Optional[torch.cuda.Stream] = None):
    """Log-probabilities of targets[...] under softmax(scale * logits[..., vocab]) -> (logps, lse), fp32, of targets' shape.

    logits[rows, vocab] or [batch, length, vocab], with any strides between rows: score whole sequences as
    token_logprobs(logits[:, :-1], tokens[:, 1:]), no copy is made.  Where the target is `ignore`, the row is not read and both are 0.  The
    results are constants of autograd; token_logprobs_grad is the backward pass."""
    if stream is None:
        result = _model_calls.token_logprobs(logits, targets, scale, ignore)                        # None: not one of the usual calls
        if result is not None:
            return _native(result, "ef21_token_logprobs")
    dtype, index = _type_of(logits, "logits"), _index_type_of(targets, "targets")
    batch, length, vocab, batch_stride, row_stride = _logit_rows(logits, "logits")
    _targets_fit(targets, logits)
    device = _same_device(logits, targets)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return token_logprobs(logits, targets, scale, ignore)
    targets, target_stride = _target_rows(targets)
    nbytes = int(_lib.ef21_token_logprobs_workspace_bytes(dtype, batch, length, vocab))
    ws, ws_ptr = _workspace(nbytes, device, "ef21_token_logprobs_workspace_bytes")
    logps = torch.empty(targets.shape, dtype=torch.float32, device=device)
    lse = torch.empty(targets.shape, dtype=torch.float32, device=device)
    _check(_lib.ef21_token_logprobs(logits.data_ptr(), dtype, batch, length, vocab, batch_stride, row_stride, targets.data_ptr(), index, target_stride,
                                    scale, ignore, logps.data_ptr(), lse.data_ptr(), ws_ptr, nbytes, _current_raw_stream(device.index)), "ef21_token_logprobs")
    return logps, lse


def token_logprobs_grad(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, ignore: int = -100,
                        out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The logits' gradient, given that of the log-probabilities: grad[...] and lse[...] are contiguous fp32 of targets' shape, the other arguments as
    they were for token_logprobs.  out (of logits' shape and type) may be the logits themselves, which are then overwritten."""
    if stream is None and out is None:
        result = _model_calls.token_logprobs_grad(logits, targets, lse, grad, scale, ignore)                        # None: not one of the usual calls
        if result is not None:
            return _native(result, "ef21_token_logprobs_grad")
    dtype, index = _type_of(logits, "logits"), _index_type_of(targets, "targets")
    batch, length, vocab, batch_stride, row_stride = _logit_rows(logits, "logits")
    _targets_fit(targets, logits)
    for t, name in ((lse, "lse"), (grad, "grad")):
        if t.shape != targets.shape:
            raise ValueError(f"{name} must be of shape {tuple(targets.shape)}, not {tuple(t.shape)}")
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise TypeError(f"{name} must be contiguous float32")
    if out is not None:
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise ValueError("out must have the logits' shape and type")
        _rows_apart(out, "out")
        if not (out.data_ptr() == logits.data_ptr() and out.stride() == logits.stride()) and _overlap(out, logits):
            raise ValueError("out must be the logits, or apart from them")
        if any(_overlap(out, t) for t in (targets, lse, grad)):
            raise ValueError("out must be apart from targets, lse and grad")
    device = _same_device(logits, targets, lse, grad, out)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return token_logprobs_grad(logits, targets, lse, grad, scale, ignore, out)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=device)
    _, _, _, out_batch_stride, out_row_stride = _logit_rows(out, "out")
    targets, target_stride = _target_rows(targets)
    _check(_lib.ef21_token_logprobs_grad(logits.data_ptr(), dtype, batch, length, vocab, batch_stride, row_stride, targets.data_ptr(), index, target_stride,
                                         lse.data_ptr(), grad.data_ptr(), scale, ignore, out.data_ptr(), out_batch_stride, out_row_stride,
                                         _current_raw_stream(device.index)), "ef21_token_logprobs_grad")
    return out


def preference_loss(logps: torch.Tensor, ref_logps: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, beta: float = 0.1,
                    smoothing: float = 0.0, norm: Optional[float] = None, stream: Optional[torch.cuda.Stream] = None) -> PreferenceLoss:
    """Logistic loss of paired log ratios with its gradient: logps[2 P, T] are the log-probabilities of the chosen answers' tokens, then of the rejected
    ones', ref_logps those under the reference (None: 0), mask[2 P, T] the tokens that count (None: all).  The loss is the sum over pairs over `norm`
    (None: P).  The results are constants of autograd: logps.backward(result.grad) goes on from here."""
    if stream is None:
        result = _model_calls.preference_loss(logps, ref_logps, mask, beta, smoothing, norm)                        # None: not one of the usual calls
        if result is not None:
            return PreferenceLoss._make(_native(result, "ef21_preference_loss"))
    dtype = _type_of(logps, "logps")
    if logps.dim() != 2 or logps.shape[0] % 2 or logps.shape[0] == 0:
        raise ValueError(f"logps must be [2 pairs, length], not {tuple(logps.shape)}")
    shape = logps.shape
    logps_stride = _matrix(logps, "logps", shape)
    ref_stride = 0 if ref_logps is None else _matrix(ref_logps, "ref_logps", shape, logps.dtype)
    mask_stride = _mask(mask, shape)
    pairs, length = shape[0] // 2, shape[1]
    device = _same_device(logps, ref_logps, mask)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return preference_loss(logps, ref_logps, mask, beta, smoothing, norm)
    nbytes = int(_lib.ef21_preference_loss_workspace_bytes(pairs, length))
    ws, ws_ptr = _workspace(nbytes, device, "ef21_preference_loss_workspace_bytes")
    loss = torch.empty((), dtype=torch.float32, device=device)
    rewards = torch.empty(2 * pairs, dtype=torch.float32, device=device)
    grad = torch.empty(shape, dtype=logps.dtype, device=device)
    _check(_lib.ef21_preference_loss(logps.data_ptr(), _ptr(ref_logps), _ptr(mask), dtype, pairs, length, logps_stride, ref_stride, mask_stride, beta, smoothing,
                                     pairs if norm is None else norm, loss.data_ptr(), rewards.data_ptr(), grad.data_ptr(), ws_ptr, nbytes,
                                     _current_raw_stream(device.index)), "ef21_preference_loss")
    return PreferenceLoss(loss, rewards, grad)


def policy_loss(logps: torch.Tensor, old_logps: torch.Tensor, advantages: torch.Tensor, mask: Optional[torch.Tensor] = None,
                ref_logps: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0,
                reduction: str = "token", norm: Optional[float] = None, stream: Optional[torch.cuda.Stream] = None) -> PolicyLoss:
    """Clipped policy loss with a KL term, with its gradient: logps[R, T], old_logps and ref_logps of the tokens under the policy, the one that drew them, and
    the reference; advantages[R, T] per token, or [R] or [R, 1] per sequence; mask[R, T] the tokens that count (None: all).  reduction "token":
    all of these weigh the same; "sequence": every row that has any does.  `norm` replaces their number where a step comes in several calls.  The results are constants
    of autograd: logps.backward(result.grad) goes on from here."""
    if stream is None:
        result = _model_calls.policy_loss(logps, old_logps, advantages, mask, ref_logps, clip_low, clip_high, kl_weight, REDUCTIONS.get(reduction), norm)                        # None: not one of the usual calls
        if result is not None:
            return PolicyLoss._make(_native(result, "ef21_policy_loss"))
    dtype = _type_of(logps, "logps")
    if logps.dim() != 2:
        raise ValueError(f"logps must be [rows, length], not {tuple(logps.shape)}")
    if reduction not in REDUCTIONS:
        raise ValueError(f"reduction must be one of {tuple(REDUCTIONS)}, not {reduction!r}")
    if norm is not None and not norm > 0:
        raise ValueError("norm must be positive")
    shape = logps.shape
    rows, length = shape
    logps_stride = _matrix(logps, "logps", shape)
    old_stride = _matrix(old_logps, "old_logps", shape, logps.dtype)
    ref_stride = 0 if ref_logps is None else _matrix(ref_logps, "ref_logps", shape, logps.dtype)
    if ref_logps is None and kl_weight != 0:
        raise ValueError("a KL term needs ref_logps")
    if advantages.dtype != logps.dtype:
        raise TypeError(f"advantages must be {logps.dtype}, not {advantages.dtype}")
    per_token = 0
    if tuple(advantages.shape) == (rows,) or tuple(advantages.shape) == (rows, 1):
        adv_stride = advantages.stride(0)
    else:
        per_token = int(not (advantages.dim() == 2 and advantages.shape[1] > 1 and advantages.stride(1) == 0))
        if per_token:
            adv_stride = _matrix(advantages, "advantages", shape)
        elif tuple(advantages.shape) != tuple(shape):
            raise ValueError(f"advantages must be of shape {tuple(shape)} or {(rows,)}, not {tuple(advantages.shape)}")
        else:
            adv_stride = advantages.stride(0)
    mask_stride = _mask(mask, shape)
    device = _same_device(logps, old_logps, advantages, mask, ref_logps)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return policy_loss(logps, old_logps, advantages, mask, ref_logps, clip_low, clip_high, kl_weight, reduction, norm)
    nbytes = int(_lib.ef21_policy_loss_workspace_bytes(rows, length))
    ws, ws_ptr = _workspace(nbytes, device, "ef21_policy_loss_workspace_bytes")
    terms = torch.empty(4, dtype=torch.float32, device=device)
    grad = torch.empty(shape, dtype=logps.dtype, device=device)
    _check(_lib.ef21_policy_loss(logps.data_ptr(), old_logps.data_ptr(), _ptr(ref_logps), advantages.data_ptr(), _ptr(mask), dtype, rows, length, logps_stride,
                                 old_stride, ref_stride, adv_stride, mask_stride, per_token, clip_low, clip_high, kl_weight, REDUCTIONS[reduction],
                                 0.0 if norm is None else norm, terms.data_ptr(), grad.data_ptr(), ws_ptr, nbytes, _current_raw_stream(device.index)), "ef21_policy_loss")
    return PolicyLoss(terms, grad)


def balance_loss(logits: torch.Tensor, choices: torch.Tensor, mask: Optional[torch.Tensor] = None, weight: float = 1.0,
                 stream: Optional[torch.cuda.Stream] = None) -> BalanceLoss:
    """Balance loss of a router, tokens per expert, and the gradient of the router's logits[R, E]: choices[R, K] are the experts that each token goes to
    (one outside [0, E) counts for none), mask[R] the tokens that count (None: all).  The results are constants of autograd: logits.backward(result.grad) goes on from here."""
    if stream is None:
        result = _model_calls.balance_loss(logits, choices, mask, weight)                        # None: not one of the usual calls
        if result is not None:
            return BalanceLoss._make(_native(result, "ef21_balance_loss"))
    dtype, index = _type_of(logits, "logits"), _index_type_of(choices, "choices")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [rows, experts], not {tuple(logits.shape)}")
    rows, experts = logits.shape
    logits_stride = _matrix(logits, "logits", logits.shape)
    if choices.dim() != 2 or choices.shape[0] != rows:
        raise ValueError(f"choices must be [{rows}, chosen], not {tuple(choices.shape)}")
    choices_stride = _matrix(choices, "choices", choices.shape)
    if mask is not None and mask.dim() != 1:
        raise ValueError(f"mask must be of shape {(rows,)}, not {tuple(mask.shape)}")
    _mask(mask, (rows,))
    device = _same_device(logits, choices, mask)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return balance_loss(logits, choices, mask, weight)
    nbytes = int(_lib.ef21_balance_loss_workspace_bytes(rows, experts))
    ws, ws_ptr = _workspace(nbytes, device, "ef21_balance_loss_workspace_bytes")
    loss = torch.empty((), dtype=torch.float32, device=device)
    counts = torch.empty(experts, dtype=torch.int32, device=device)
    probs = torch.empty(experts, dtype=torch.float32, device=device)
    grad = torch.empty((rows, experts), dtype=logits.dtype, device=device)
    _check(_lib.ef21_balance_loss(logits.data_ptr(), dtype, rows, experts, logits_stride, choices.data_ptr(), index, choices.shape[1], choices_stride, _ptr(mask),
                                  weight, loss.data_ptr(), counts.data_ptr(), probs.data_ptr(), grad.data_ptr(), ws_ptr, nbytes,
                                  _current_raw_stream(device.index)), "ef21_balance_loss")
    return BalanceLoss(loss, counts, probs, grad)


def embedding(weight: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """scale * weight[tokens] -> [*tokens.shape, dim]; a token outside the table reads as zeros (as where a table is split by rows).  The
    result is a constant of autograd; embedding_grad is the backward pass."""
    if stream is None:
        result = _model_calls.embedding(weight, tokens, scale)                        # None: not one of the usual calls
        if result is not None:
            return _native(result, "ef21_embedding")
    dtype, index = _type_of(weight, "weight"), _index_type_of(tokens, "tokens")
    if weight.dim() != 2:
        raise ValueError(f"weight must be [vocab, dim], not {tuple(weight.shape)}")
    stride = _matrix(weight, "weight", weight.shape)
    device = _same_device(weight, tokens)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return embedding(weight, tokens, scale)
    tokens = tokens.contiguous()
    out = torch.empty((*tokens.shape, weight.shape[1]), dtype=weight.dtype, device=device)
    _check(_lib.ef21_embedding(weight.data_ptr(), dtype, weight.shape[0], weight.shape[1], stride, tokens.data_ptr(), index, tokens.numel(), scale,
                               out.data_ptr(), _current_raw_stream(device.index)), "ef21_embedding")
    return out


def embedding_grad(grad: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0, padding: int = -1, dtype: Optional[torch.dtype] = None,
                   out: Optional[torch.Tensor] = None, accumulate: bool = False, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The table's gradient [vocab, dim] from that of embedding(): for every token scale times the sum of grad[...] at its positions, in a fixed order.

    The result is of grad's type, or float32 (dtype=torch.float32, or an fp32 out).  accumulate adds to out; the token `padding` adds nothing."""
    if stream is None and out is None and not accumulate:
        result = _model_calls.embedding_grad(grad, tokens, vocab, scale, padding, dtype)                        # None: not one of the usual calls
        if result is not None:
            return _native(result, "ef21_embedding_grad")
    code, index = _type_of(grad, "grad"), _index_type_of(tokens, "tokens")
    if grad.dim() < 1 or tuple(grad.shape[:-1]) != tuple(tokens.shape):
        raise ValueError(f"grad must be of shape {(*tokens.shape, 'dim')}, not {tuple(grad.shape)}")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    dim, count = grad.shape[-1], tokens.numel()
    if grad.dim() == 2:
        stride = _matrix(grad, "grad", grad.shape)
    elif grad.is_contiguous():
        stride = dim
    else:
        raise TypeError("grad must be a matrix with contiguous rows, or contiguous")
    result = dtype or (grad.dtype if out is None else out.dtype)
    if result not in (grad.dtype, torch.float32) or (out is not None and out.dtype != result):
        raise TypeError(f"the result must be of grad's type or float32, not {result}")
    if out is not None:
        out_stride = _matrix(out, "out", (vocab, dim))
        _rows_apart(out, "out")
        if _overlap(out, grad) or _overlap(out, tokens):
            raise ValueError("out must be apart from grad and tokens")
    device = _same_device(grad, tokens, out)
    there = _elsewhere(device, stream)
    if there is not None:
        with there:
            return embedding_grad(grad, tokens, vocab, scale, padding, dtype, out, accumulate)
    tokens = tokens.contiguous()
    nbytes = int(_lib.ef21_embedding_grad_workspace_bytes(count, vocab, dim))
    ws, ws_ptr = _workspace(nbytes, device, "ef21_embedding_grad_workspace_bytes")
    if out is None:
        out, out_stride = torch.empty((vocab, dim), dtype=result, device=device), dim
    _check(_lib.ef21_embedding_grad(grad.data_ptr(), code, count, dim, stride, tokens.data_ptr(), index, vocab, padding, scale, out.data_ptr(), DTYPES[result],
                                    out_stride, int(accumulate), ws_ptr, nbytes, _current_raw_stream(device.index)), "ef21_embedding_grad")
    return out
