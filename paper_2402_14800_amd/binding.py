"""ctypes binding of libmoeprune.so: argument marshalling only.

Every function here has the name and meaning of the C entry point it calls (see
include/moeprune.h); torch supplies device memory and the stream, nothing else.
Importing this module raises if the library has not been built -- there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from ctypes import POINTER, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint32, c_void_p
from typing import Dict, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmoeprune.so")

MOEP_F32, MOEP_BF16 = 0, 1
_STATUS = {0: "MOEP_OK", 1: "MOEP_EINVAL", 2: "MOEP_EUNSUPPORTED", 3: "MOEP_EWORKSPACE", 4: "MOEP_EHIP"}

EXPORTS = (
    "moep_num_subsets", "moep_subset_unrank", "moep_subset_rank", "moep_last_error",
    "moe_expert_outputs_workspace", "moe_expert_outputs",
    "prune_enumerate_workspace", "prune_enumerate",
    "prune_enumerate_multi_workspace", "prune_enumerate_multi", "prune_enumerate_static",
    "prune_enumerate_direct_workspace", "prune_enumerate_direct",
    "moe_forward_skip_workspace", "moe_forward_skip", "moe_forward_pruned_skip",
    "moe_packed_weights_bytes", "moe_pack_weights", "moe_forward_pruned_skip_packed",
    "moe_expert_outputs_packed_workspace", "moe_expert_outputs_packed",
    "moe_forward_skip_topk_workspace", "moe_forward_skip_topk",
    "skip_calibrate_beta_workspace", "skip_calibrate_beta", "expert_selection_stats",
    "moe_expert_outputs_ranked_workspace", "moe_expert_outputs_ranked", "prune_enumerate_ranked",
    "moe_token_logprobs", "moe_distill_topk", "moe_distill_topk_backward",
    "expert_ffn_forward_workspace", "expert_ffn_forward", "expert_ffn_backward_workspace", "expert_ffn_backward",
    "moe_dispatch_rows_workspace", "moe_dispatch_rows", "moe_dispatch_rows_backward", "moe_combine_rows", "moe_combine_rows_backward",
    "moe_policy_loss", "moe_policy_loss_backward", "moe_preference_loss", "moe_preference_loss_backward",
    "moe_preference_loss_all_rows", "moe_preference_loss_backward_all_rows",
    "moep_timing_enable", "moep_timing_collect", "moep_timing_records", "moep_mfma_ceiling",
)


class MoepError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def library_path() -> str:
    return _LIB_PATH


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2402_14800_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    lib.moep_num_subsets.restype = c_int64
    lib.moep_num_subsets.argtypes = [c_int, c_int]
    lib.moep_subset_unrank.restype = c_int
    lib.moep_subset_unrank.argtypes = [c_int, c_int, c_int64, POINTER(c_uint32)]
    lib.moep_subset_rank.restype = c_int64
    lib.moep_subset_rank.argtypes = [c_int, c_int, c_uint32]
    lib.moep_last_error.restype = c_char_p
    lib.moep_last_error.argtypes = []
    lib.moe_expert_outputs_workspace.restype = c_size_t
    lib.moe_expert_outputs_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int]
    lib.moe_expert_outputs.restype = c_int
    lib.moe_expert_outputs.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_int,
                                                        c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.prune_enumerate_workspace.restype = c_size_t
    lib.prune_enumerate_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int, c_int]
    lib.prune_enumerate.restype = c_int
    lib.prune_enumerate.argtypes = [c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_int,
                                    c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.prune_enumerate_direct_workspace.restype = c_size_t
    lib.prune_enumerate_direct_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int, c_int]
    lib.prune_enumerate_direct.restype = c_int
    lib.prune_enumerate_direct.argtypes = lib.prune_enumerate.argtypes
    lib.prune_enumerate_static.restype = c_int
    lib.prune_enumerate_static.argtypes = [c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_int,
                                           c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.prune_enumerate_multi_workspace.restype = c_size_t
    lib.prune_enumerate_multi_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int, POINTER(c_int), c_int]
    lib.prune_enumerate_multi.restype = c_int
    lib.prune_enumerate_multi.argtypes = [c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_int,
                                          POINTER(c_int), c_void_p, c_void_p, c_void_p, c_void_p,
                                          c_void_p, c_size_t, c_void_p]
    lib.moe_forward_skip_workspace.restype = c_size_t
    lib.moe_forward_skip_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int]
    lib.moe_forward_skip.restype = c_int
    lib.moe_forward_skip.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_int, c_int, c_float,
                                                      c_void_p, c_void_p, c_void_p, c_void_p,
                                                      c_void_p, c_size_t, c_void_p]
    lib.moe_forward_pruned_skip.restype = c_int
    lib.moe_forward_pruned_skip.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_int, c_int, c_uint32,
                                                             c_float, c_void_p, c_void_p, c_void_p, c_void_p,
                                                             c_void_p, c_size_t, c_void_p]
    lib.moe_packed_weights_bytes.restype = c_size_t
    lib.moe_packed_weights_bytes.argtypes = [c_int, c_int, c_int, c_int]
    lib.moe_pack_weights.restype = c_int
    lib.moe_pack_weights.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p]
    lib.moe_expert_outputs_packed_workspace.restype = c_size_t
    lib.moe_expert_outputs_packed_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int]
    lib.moe_expert_outputs_packed.restype = c_int
    lib.moe_expert_outputs_packed.argtypes = [c_void_p] * 3 + [c_int64, c_int, c_int, c_int, c_int,
                                                               c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.moe_forward_pruned_skip_packed.restype = c_int
    lib.moe_forward_pruned_skip_packed.argtypes = [c_void_p] * 3 + [c_int64, c_int, c_int, c_int, c_int, c_int, c_uint32,
                                                                    c_float, c_void_p, c_void_p, c_void_p, c_void_p,
                                                                    c_void_p, c_size_t, c_void_p]
    lib.moe_forward_skip_topk_workspace.restype = c_size_t
    lib.moe_forward_skip_topk_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int, c_int]
    lib.moe_forward_skip_topk.restype = c_int
    lib.moe_forward_skip_topk.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_int, c_int, c_uint32,
                                                           c_float, c_void_p, c_void_p, c_void_p, c_void_p,
                                                           c_void_p, c_size_t, c_void_p]
    lib.skip_calibrate_beta_workspace.restype = c_size_t
    lib.skip_calibrate_beta_workspace.argtypes = [c_int64]
    lib.skip_calibrate_beta.restype = c_int
    lib.skip_calibrate_beta.argtypes = [c_void_p, c_int64, c_int, c_uint32, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.expert_selection_stats.restype = c_int
    lib.expert_selection_stats.argtypes = [c_void_p, c_int64, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p,
                                           c_void_p]
    lib.moe_expert_outputs_ranked_workspace.restype = c_size_t
    lib.moe_expert_outputs_ranked_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int, c_int]
    lib.moe_expert_outputs_ranked.restype = c_int
    lib.moe_expert_outputs_ranked.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_int, c_int,
                                                               c_void_p, c_void_p, c_void_p, c_void_p,
                                                               c_void_p, c_size_t, c_void_p]
    lib.prune_enumerate_ranked.restype = c_int
    lib.prune_enumerate_ranked.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int,
                                           c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                           c_void_p, c_size_t, c_void_p]
    lib.expert_ffn_forward_workspace.restype = c_size_t
    lib.expert_ffn_forward_workspace.argtypes = [c_int64, c_int, c_int, c_int, c_int]
    lib.expert_ffn_forward.restype = c_int
    lib.expert_ffn_forward.argtypes = [c_void_p] * 4 + [c_int64, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.expert_ffn_backward_workspace.restype = c_size_t
    lib.expert_ffn_backward_workspace.argtypes = [c_int64, c_int, c_int, c_int]
    lib.expert_ffn_backward.restype = c_int
    lib.expert_ffn_backward.argtypes = [c_void_p] * 6 + [c_int64, c_int, c_int, c_int] + [c_void_p] * 5 + [c_size_t, c_void_p]
    lib.moe_token_logprobs.restype = c_int
    lib.moe_token_logprobs.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int, c_int,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.moe_distill_topk.restype = c_int
    lib.moe_distill_topk.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int64, c_int, c_int, c_float,
                                     c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]
    lib.moe_distill_topk_backward.restype = c_int
    lib.moe_distill_topk_backward.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int64,
                                              c_int, c_int, c_float, c_void_p, c_int64, c_void_p]
    lib.moe_dispatch_rows_workspace.restype = c_size_t
    lib.moe_dispatch_rows_workspace.argtypes = [c_int64, c_int, c_int]
    lib.moe_dispatch_rows.restype = c_int
    lib.moe_dispatch_rows.argtypes = [c_void_p] * 3 + [c_int64, c_int, c_int, c_int, c_int] + [c_void_p] * 4 + [c_size_t, c_void_p]
    lib.moe_dispatch_rows_backward.restype = c_int
    lib.moe_dispatch_rows_backward.argtypes = [c_void_p] * 2 + [c_int64, c_int, c_int, c_int64, c_int, c_void_p, c_void_p]
    lib.moe_combine_rows.restype = c_int
    lib.moe_combine_rows.argtypes = [c_void_p] * 3 + [c_int64, c_int, c_int, c_int64, c_int, c_void_p, c_void_p]
    lib.moe_combine_rows_backward.restype = c_int
    lib.moe_combine_rows_backward.argtypes = [c_void_p] * 4 + [c_int64, c_int, c_int, c_int64, c_int] + [c_void_p] * 3
    lib.moe_policy_loss.restype = c_int
    lib.moe_policy_loss.argtypes = [c_void_p, c_int64] + [c_void_p] * 4 + [c_int64, c_int64, c_int] + [c_float] * 4 + \
        [c_void_p] * 5 + [c_int64, c_void_p]
    lib.moe_policy_loss_backward.restype = c_int
    lib.moe_policy_loss_backward.argtypes = [c_void_p, c_int64] + [c_void_p] * 3 + [c_int64, c_int64, c_int, c_float, c_void_p, c_int64, c_void_p]
    lib.moe_preference_loss.restype = c_int
    lib.moe_preference_loss.argtypes = [c_void_p, c_int64] + [c_void_p] * 3 + [c_int64, c_int64, c_int64, c_int, c_float, c_float, c_int] + \
        [c_void_p] * 6 + [c_int64, c_void_p]
    lib.moe_preference_loss_backward.restype = c_int
    lib.moe_preference_loss_backward.argtypes = [c_void_p, c_int64] + [c_void_p] * 4 + [c_int64, c_int64, c_int64, c_int, c_void_p, c_int64,
                                                                                         c_void_p]
    for whole, like in ((lib.moe_preference_loss_all_rows, lib.moe_preference_loss),
                        (lib.moe_preference_loss_backward_all_rows, lib.moe_preference_loss_backward)):
        whole.restype, whole.argtypes = like.restype, like.argtypes
    lib.moep_timing_enable.restype = c_int
    lib.moep_timing_enable.argtypes = [c_int]
    lib.moep_timing_collect.restype = c_int
    lib.moep_timing_collect.argtypes = [POINTER(c_char_p), POINTER(c_double), POINTER(c_int64), c_int]
    lib.moep_timing_records.restype = c_int
    lib.moep_timing_records.argtypes = [POINTER(c_char_p), POINTER(c_float), c_int]
    lib.moep_mfma_ceiling.restype = c_int
    lib.moep_mfma_ceiling.argtypes = [c_void_p, c_void_p, c_size_t, c_int, c_void_p, c_size_t, POINTER(c_double),
                                      c_void_p]
    return lib


_lib = _load()


def _check(status: int) -> None:
    if status != 0:
        raise MoepError(status, _lib.moep_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MOEP_F32
    if t.dtype == torch.bfloat16:
        return MOEP_BF16
    raise TypeError(f"unsupported storage dtype {t.dtype}: use float32 or bfloat16")


def _dev(*tensors: torch.Tensor) -> torch.device:
    index = tensors[0].get_device()                      # (an int, -1 on the host: device objects cost 0.2 us each)
    for t in tensors:
        if t.get_device() != index or not t.is_cuda:
            raise ValueError("all tensors must live on the same GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous (row-major)")
    return tensors[0].device


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()           # (every such parameter is declared c_void_p, which takes an int)


# The current stream's handle; a Stream object of torch.cuda.current_stream takes 2 us, and is what a torch without the other has.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream(dev: torch.device):
    return _raw_stream(dev.index)


def _workspace(nbytes: int, dev: torch.device, ws: Optional[torch.Tensor]) -> torch.Tensor:
    if ws is not None:
        if ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on the same GPU")
        return ws
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=dev)


# ---------------------------------------------------------------- host helpers
def num_subsets(E: int, r: int) -> int:
    return int(_lib.moep_num_subsets(E, r))


def subset_unrank(E: int, r: int, idx: int) -> int:
    m = c_uint32(0)
    _check(_lib.moep_subset_unrank(E, r, idx, ctypes.byref(m)))
    return int(m.value)


def subset_rank(E: int, r: int, mask: int) -> int:
    return int(_lib.moep_subset_rank(E, r, mask))


# ---------------------------------------------------------------- entry points
def moe_expert_outputs_workspace(T: int, E: int, H: int, F: int, dtype_code: int) -> int:
    return int(_lib.moe_expert_outputs_workspace(T, E, H, F, dtype_code))


def moe_expert_outputs(x, Wgate, W1, W3, W2, logits=None, Y=None, workspace=None):
    """logits [T,E] fp32 and Y [E,T,H] for every expert and token (asynchronous on the current stream)."""
    dev = _dev(x, Wgate, W1, W3, W2)
    dt = _dtype_code(x)
    T, H = x.shape
    E, F, _ = W1.shape
    assert Wgate.shape == (E, H) and W3.shape == (E, F, H) and W2.shape == (E, H, F)
    assert all(_dtype_code(t) == dt for t in (Wgate, W1, W3, W2))
    if logits is None:
        logits = torch.empty((T, E), dtype=torch.float32, device=dev)
    if Y is None:
        Y = torch.empty((E, T, H), dtype=x.dtype, device=dev)
    need = _lib.moe_expert_outputs_workspace(T, E, H, F, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.moe_expert_outputs(_ptr(x), _ptr(Wgate), _ptr(W1), _ptr(W3), _ptr(W2), T, E, H, F, dt,
                                   _ptr(logits), _ptr(Y), _ptr(ws), ws.numel(), _stream(dev)))
    return logits, Y


def prune_enumerate_workspace(T: int, E: int, H: int, k: int, r: int, dtype_code: int) -> int:
    return int(_lib.prune_enumerate_workspace(T, E, H, k, r, dtype_code))


def prune_enumerate(logits, Y, k: int, r: int, workspace=None, count_unaffected: bool = True):
    """loss [C(E,r)] fp32, argmin [1] int32, argmin_mask [1] (int32 view of the uint32 mask),
    unaffected_pairs [1] int64 (or None).  Device tensors; asynchronous on the current stream."""
    dev = _dev(logits, Y)
    dt = _dtype_code(Y)
    E, T, H = Y.shape
    assert logits.shape == (T, E) and logits.dtype == torch.float32
    n = num_subsets(E, r)
    if n < 0:
        raise MoepError(1, f"r={r} out of range [1, E={E}]")
    loss = torch.empty((n,), dtype=torch.float32, device=dev)
    argmin = torch.empty((1,), dtype=torch.int32, device=dev)
    amask = torch.empty((1,), dtype=torch.int32, device=dev)
    unaffected = torch.empty((1,), dtype=torch.int64, device=dev) if count_unaffected else None
    need = _lib.prune_enumerate_workspace(T, E, H, k, r, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.prune_enumerate(_ptr(logits), _ptr(Y), T, E, H, dt, k, r, _ptr(loss), _ptr(argmin),
                                _ptr(amask), _ptr(unaffected), _ptr(ws), ws.numel(), _stream(dev)))
    return loss, argmin, amask, unaffected


def prune_enumerate_direct(logits, Y, k: int, r: int, workspace=None, count_unaffected: bool = True):
    """prune_enumerate's outputs from Eq. 3 as written (no Gram matrices); at most 128 subsets, k <= 4."""
    dev = _dev(logits, Y)
    dt = _dtype_code(Y)
    E, T, H = Y.shape
    assert logits.shape == (T, E) and logits.dtype == torch.float32
    n = num_subsets(E, r)
    if n < 0:
        raise MoepError(1, f"r={r} out of range [1, E={E}]")
    loss = torch.empty((n,), dtype=torch.float32, device=dev)
    argmin = torch.empty((1,), dtype=torch.int32, device=dev)
    amask = torch.empty((1,), dtype=torch.int32, device=dev)
    unaffected = torch.empty((1,), dtype=torch.int64, device=dev) if count_unaffected else None
    need = _lib.prune_enumerate_direct_workspace(T, E, H, k, r, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.prune_enumerate_direct(_ptr(logits), _ptr(Y), T, E, H, dt, k, r, _ptr(loss), _ptr(argmin),
                                       _ptr(amask), _ptr(unaffected), _ptr(ws), ws.numel(), _stream(dev)))
    return loss, argmin, amask, unaffected


STATIC_SCRATCH_BYTES = 32 << 20      # MOEP_STATIC_SCRATCH_BYTES of include/moeprune.h


def prune_enumerate_static(logits, Y, k: int, r: int, out=None, count_unaffected: bool = True):
    """prune_enumerate on the library's built-in scratch array: no workspace, nothing allocated by the call
    when `out` carries the four output tensors (loss, argmin, argmin_mask, unaffected_pairs)."""
    dev = _dev(logits, Y)
    dt = _dtype_code(Y)
    E, T, H = Y.shape
    assert logits.shape == (T, E) and logits.dtype == torch.float32
    if out is None:
        n = num_subsets(E, r)
        if n < 0:
            raise MoepError(1, f"r={r} out of range [1, E={E}]")
        out = (torch.empty((n,), dtype=torch.float32, device=dev), torch.empty((1,), dtype=torch.int32, device=dev),
               torch.empty((1,), dtype=torch.int32, device=dev),
               torch.empty((1,), dtype=torch.int64, device=dev) if count_unaffected else None)
    loss, argmin, amask, unaffected = out
    _check(_lib.prune_enumerate_static(_ptr(logits), _ptr(Y), T, E, H, dt, k, r, _ptr(loss), _ptr(argmin),
                                       _ptr(amask), _ptr(unaffected), _stream(dev)))
    return loss, argmin, amask, unaffected


def prune_enumerate_multi_workspace(T: int, E: int, H: int, k: int, rs, dtype_code: int) -> int:
    arr = (c_int * len(rs))(*rs)
    return int(_lib.prune_enumerate_multi_workspace(T, E, H, k, len(rs), arr, dtype_code))


def prune_enumerate_multi(logits, Y, k: int, rs, workspace=None, count_unaffected: bool = True):
    """prune_enumerate for every r of `rs` with one pass over Y.  Returns a list of
    (loss [C(E,r)], argmin [1], argmin_mask [1], unaffected_pairs [1] or None), one per r (views)."""
    dev = _dev(logits, Y)
    dt = _dtype_code(Y)
    E, T, H = Y.shape
    assert logits.shape == (T, E) and logits.dtype == torch.float32
    rs = [int(r) for r in rs]
    ns = [num_subsets(E, r) for r in rs]
    if not rs or min(ns) < 0:
        raise MoepError(1, f"rs={rs}: every r must lie in [1, E={E}]")
    loss = torch.empty((sum(ns),), dtype=torch.float32, device=dev)
    argmin = torch.empty((len(rs),), dtype=torch.int32, device=dev)
    amask = torch.empty((len(rs),), dtype=torch.int32, device=dev)
    unaffected = torch.empty((len(rs),), dtype=torch.int64, device=dev) if count_unaffected else None
    arr = (c_int * len(rs))(*rs)
    need = _lib.prune_enumerate_multi_workspace(T, E, H, k, len(rs), arr, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.prune_enumerate_multi(_ptr(logits), _ptr(Y), T, E, H, dt, k, len(rs), arr, _ptr(loss), _ptr(argmin),
                                      _ptr(amask), _ptr(unaffected), _ptr(ws), ws.numel(), _stream(dev)))
    out, off = [], 0
    for i, n in enumerate(ns):                           # (slices: autograd lets a caller write into them, unlike the views of split)
        out.append((loss[off:off + n], argmin[i:i + 1], amask[i:i + 1],
                    unaffected[i:i + 1] if unaffected is not None else None))
        off += n
    return out


def moe_expert_outputs_ranked(x, Wgate, W1, W3, W2, n_rank: int, workspace=None, out=None):
    """logits [T,E] fp32, ranked_experts [T,n_rank] int32, slot_of [T,n_rank] int32, Yr [T*n_rank,H].
    `out` may carry a previous call's (logits, ranked_experts, slot_of, Yr) to be overwritten."""
    dev = _dev(x, Wgate, W1, W3, W2)
    dt = _dtype_code(x)
    T, H = x.shape
    E, F, _ = W1.shape
    assert Wgate.shape == (E, H) and W3.shape == (E, F, H) and W2.shape == (E, H, F)
    if out is None:
        logits = torch.empty((T, E), dtype=torch.float32, device=dev)
        experts = torch.empty((T, max(n_rank, 1)), dtype=torch.int32, device=dev)
        slot_of = torch.empty((T, max(n_rank, 1)), dtype=torch.int32, device=dev)
        Yr = torch.empty((T * max(n_rank, 1), H), dtype=x.dtype, device=dev)
    else:
        logits, experts, slot_of, Yr = out
    need = _lib.moe_expert_outputs_ranked_workspace(T, E, H, F, dt, n_rank)
    ws = _workspace(need, dev, workspace)
    _check(_lib.moe_expert_outputs_ranked(_ptr(x), _ptr(Wgate), _ptr(W1), _ptr(W3), _ptr(W2), T, E, H, F, dt,
                                          n_rank, _ptr(logits), _ptr(experts), _ptr(slot_of), _ptr(Yr),
                                          _ptr(ws), ws.numel(), _stream(dev)))
    return logits, experts, slot_of, Yr


def prune_enumerate_ranked(logits, experts, slot_of, Yr, k: int, r: int, workspace=None,
                           count_unaffected: bool = True):
    """As prune_enumerate, from the outputs of moe_expert_outputs_ranked."""
    dev = _dev(logits, Yr)
    dt = _dtype_code(Yr)
    T, E = logits.shape
    n_rank = experts.shape[1]
    H = Yr.shape[1]
    n_sub = num_subsets(E, r)
    if n_sub < 0:
        raise MoepError(1, f"r={r} out of range for E={E}")
    loss = torch.empty((n_sub,), dtype=torch.float32, device=dev)
    argmin = torch.empty((1,), dtype=torch.int32, device=dev)
    amask = torch.empty((1,), dtype=torch.int32, device=dev)
    unaff = torch.empty((1,), dtype=torch.int64, device=dev) if count_unaffected else None
    need = _lib.prune_enumerate_workspace(T, E, H, k, r, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.prune_enumerate_ranked(_ptr(logits), _ptr(experts), _ptr(slot_of), _ptr(Yr), T, E, H, dt, n_rank,
                                       k, r, _ptr(loss), _ptr(argmin), _ptr(amask), _ptr(unaff), _ptr(ws),
                                       ws.numel(), _stream(dev)))
    return loss, argmin, amask, unaff


def moe_forward_skip_workspace(T: int, E: int, H: int, F: int, dtype_code: int) -> int:
    return int(_lib.moe_forward_skip_workspace(T, E, H, F, dtype_code))


def moe_forward_skip(x, Wgate, W1, W3, W2, beta: float, k: int = 2, workspace=None,
                     want_logits: bool = True, want_top2: bool = True, kept_mask: Optional[int] = None):
    """out [T,H], skip_mask [T] uint8, logits [T,E] fp32 (or None), top2 [T,2] int32 (or None).
    With `kept_mask` the call goes to moe_forward_pruned_skip (top-2 among the kept experts)."""
    dev = _dev(x, Wgate, W1, W3, W2)
    dt = _dtype_code(x)
    T, H = x.shape
    E, F, _ = W1.shape
    assert Wgate.shape == (E, H) and W3.shape == (E, F, H) and W2.shape == (E, H, F)
    out = torch.empty((T, H), dtype=x.dtype, device=dev)
    skip = torch.empty((T,), dtype=torch.uint8, device=dev)
    logits = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
    top2 = torch.empty((T, 2), dtype=torch.int32, device=dev) if want_top2 else None
    need = _lib.moe_forward_skip_workspace(T, E, H, F, dt)
    ws = _workspace(need, dev, workspace)
    if kept_mask is None:
        _check(_lib.moe_forward_skip(_ptr(x), _ptr(Wgate), _ptr(W1), _ptr(W3), _ptr(W2), T, E, H, F, dt, k,
                                     c_float(beta), _ptr(out), _ptr(skip), _ptr(logits), _ptr(top2),
                                     _ptr(ws), ws.numel(), _stream(dev)))
    else:
        _check(_lib.moe_forward_pruned_skip(_ptr(x), _ptr(Wgate), _ptr(W1), _ptr(W3), _ptr(W2), T, E, H, F, dt, k,
                                            c_uint32(kept_mask), c_float(beta), _ptr(out), _ptr(skip),
                                            _ptr(logits), _ptr(top2), _ptr(ws), ws.numel(), _stream(dev)))
    return out, skip, logits, top2


def moe_forward_pruned_skip(x, Wgate, W1, W3, W2, kept_mask: int, beta: float, **kw):
    return moe_forward_skip(x, Wgate, W1, W3, W2, beta, kept_mask=kept_mask, **kw)


def moe_pack_weights(W1, W3, W2) -> torch.Tensor:
    """The layer's expert weights in the layout the bf16 GEMMs read (uint8 tensor, for *_packed calls)."""
    dev = _dev(W1, W3, W2)
    dt = _dtype_code(W1)
    E, F, H = W1.shape
    assert W3.shape == (E, F, H) and W2.shape == (E, H, F)
    need = int(_lib.moe_packed_weights_bytes(E, H, F, dt))
    if need == 0:
        raise MoepError(2, "moe_pack_weights: bf16 weights with H and F multiples of 64 only")
    packed = torch.empty((need,), dtype=torch.uint8, device=dev)
    _check(_lib.moe_pack_weights(_ptr(W1), _ptr(W3), _ptr(W2), E, H, F, dt, _ptr(packed), _stream(dev)))
    return packed


def moe_expert_outputs_packed(x, Wgate, packed, F: int, logits=None, Y=None, workspace=None):
    """moe_expert_outputs on weights packed once by moe_pack_weights."""
    dev = _dev(x, Wgate, packed)
    dt = _dtype_code(x)
    T, H = x.shape
    E = Wgate.shape[0]
    assert Wgate.shape == (E, H) and packed.numel() == int(_lib.moe_packed_weights_bytes(E, H, F, dt))
    if logits is None:
        logits = torch.empty((T, E), dtype=torch.float32, device=dev)
    if Y is None:
        Y = torch.empty((E, T, H), dtype=x.dtype, device=dev)
    need = _lib.moe_expert_outputs_packed_workspace(T, E, H, F, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.moe_expert_outputs_packed(_ptr(x), _ptr(Wgate), _ptr(packed), T, E, H, F, dt, _ptr(logits), _ptr(Y),
                                          _ptr(ws), ws.numel(), _stream(dev)))
    return logits, Y


def moe_forward_pruned_skip_packed(x, Wgate, packed, F: int, beta: float, kept_mask: Optional[int] = None,
                                   k: int = 2, workspace=None, want_logits: bool = True, want_top2: bool = True):
    """moe_forward_pruned_skip on weights packed once by moe_pack_weights."""
    dev = _dev(x, Wgate, packed)
    dt = _dtype_code(x)
    T, H = x.shape
    E = Wgate.shape[0]
    assert Wgate.shape == (E, H) and packed.numel() == int(_lib.moe_packed_weights_bytes(E, H, F, dt))
    if kept_mask is None:
        kept_mask = (1 << E) - 1
    out = torch.empty((T, H), dtype=x.dtype, device=dev)
    skip = torch.empty((T,), dtype=torch.uint8, device=dev)
    logits = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
    top2 = torch.empty((T, 2), dtype=torch.int32, device=dev) if want_top2 else None
    need = _lib.moe_forward_skip_workspace(T, E, H, F, dt)
    ws = _workspace(need, dev, workspace)
    _check(_lib.moe_forward_pruned_skip_packed(_ptr(x), _ptr(Wgate), _ptr(packed), T, E, H, F, dt, k,
                                               c_uint32(kept_mask), c_float(beta), _ptr(out), _ptr(skip),
                                               _ptr(logits), _ptr(top2), _ptr(ws), ws.numel(), _stream(dev)))
    return out, skip, logits, top2


def moe_forward_skip_topk(x, Wgate, W1, W3, W2, k: int, beta: float, kept_mask: Optional[int] = None,
                          workspace=None, want_logits: bool = True, want_topk: bool = True):
    """out [T,H], n_used [T] int32 (i* per token), logits [T,E] fp32 (or None), topk [T,k] int32 (or None)."""
    dev = _dev(x, Wgate, W1, W3, W2)
    dt = _dtype_code(x)
    T, H = x.shape
    E, F, _ = W1.shape
    assert Wgate.shape == (E, H) and W3.shape == (E, F, H) and W2.shape == (E, H, F)
    if kept_mask is None:
        kept_mask = (1 << E) - 1
    out = torch.empty((T, H), dtype=x.dtype, device=dev)
    n_used = torch.empty((T,), dtype=torch.int32, device=dev)
    logits = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
    topk = torch.empty((T, max(k, 1)), dtype=torch.int32, device=dev) if want_topk else None
    need = _lib.moe_forward_skip_topk_workspace(T, E, H, F, dt, k)
    ws = _workspace(need, dev, workspace)
    _check(_lib.moe_forward_skip_topk(_ptr(x), _ptr(Wgate), _ptr(W1), _ptr(W3), _ptr(W2), T, E, H, F, dt, k,
                                      c_uint32(kept_mask), c_float(beta), _ptr(out), _ptr(n_used),
                                      _ptr(logits), _ptr(topk), _ptr(ws), ws.numel(), _stream(dev)))
    return out, n_used, logits, topk


def skip_calibrate_beta(logits, kept_mask: Optional[int] = None, workspace=None) -> torch.Tensor:
    """beta [1] fp32 on the device: the median of w_e1 / w_e0 over the rows of logits [T,E]."""
    dev = _dev(logits)
    assert logits.dtype == torch.float32 and logits.dim() == 2
    T, E = logits.shape
    if kept_mask is None:
        kept_mask = (1 << E) - 1
    beta = torch.empty((1,), dtype=torch.float32, device=dev)
    need = _lib.skip_calibrate_beta_workspace(T)
    ws = _workspace(need, dev, workspace)
    _check(_lib.skip_calibrate_beta(_ptr(logits), T, E, c_uint32(kept_mask), _ptr(beta), _ptr(ws), ws.numel(),
                                    _stream(dev)))
    return beta


def expert_selection_stats(logits, k: int, r: Optional[int] = None):
    """count [E] int64, coselect [E,E] int64, frequency_mask (int32 view of the uint32 mask, [1]) or None."""
    dev = _dev(logits)
    assert logits.dtype == torch.float32 and logits.dim() == 2
    T, E = logits.shape
    count = torch.empty((E,), dtype=torch.int64, device=dev)
    co = torch.empty((E, E), dtype=torch.int64, device=dev)
    fmask = torch.empty((1,), dtype=torch.int32, device=dev) if r is not None else None
    _check(_lib.expert_selection_stats(_ptr(logits), T, E, k, r if r is not None else 0, _ptr(count), _ptr(co),
                                       _ptr(fmask), _stream(dev)))
    return count, co, fmask


# ---------------------------------------------------------------- one expert's block
def _ffn_shapes(x, W1, W3, W2, what: str):
    dt = _dtype_code(x)
    if x.dim() != 2 or W1.dim() != 2:
        raise ValueError(f"{what}: x must be [T, H] and W1 [F, H]")
    T, H = x.shape
    F = W1.shape[0]
    if W1.shape != (F, H) or W3.shape != (F, H) or W2.shape != (H, F) or any(w.dtype != x.dtype for w in (W1, W3, W2)):
        raise ValueError(f"{what}: W1, W3 must be [F, H] and W2 [H, F], of x's type")
    return T, H, F, dt


def expert_ffn_forward_workspace(T: int, H: int, F: int, dtype_code: int, save: bool = False) -> int:
    return int(_lib.expert_ffn_forward_workspace(T, H, F, dtype_code, 1 if save else 0))


def expert_ffn_forward(x, W1, W3, W2, save: bool = False, workspace=None):
    """y [T,H] of one expert's block on the rows of x [T,H]; with `save` also gate_up [2,T,F] fp32 for the backward call."""
    dev = _dev(x, W1, W3, W2)
    T, H, F, dt = _ffn_shapes(x, W1, W3, W2, "expert_ffn_forward")
    y = torch.empty((T, H), dtype=x.dtype, device=dev)
    gate_up = torch.empty((2, T, F), dtype=torch.float32, device=dev) if save else None
    ws = _workspace(_lib.expert_ffn_forward_workspace(T, H, F, dt, 1 if save else 0), dev, workspace)
    _check(_lib.expert_ffn_forward(_ptr(x), _ptr(W1), _ptr(W3), _ptr(W2), T, H, F, dt, _ptr(y), _ptr(gate_up),
                                   _ptr(ws), ws.numel(), _stream(dev)))
    return (y, gate_up) if save else y


def expert_ffn_backward_workspace(T: int, H: int, F: int, dtype_code: int) -> int:
    return int(_lib.expert_ffn_backward_workspace(T, H, F, dtype_code))


def expert_ffn_backward(dy, x, W1, W3, W2, gate_up, input_gradient: bool = True, weight_gradients: bool = True, workspace=None):
    """dx [T,H], dW1, dW3 [F,H], dW2 [H,F] from dy [T,H] and the forward call's gate_up; None for what is not asked for."""
    dev = _dev(dy, x, W1, W3, W2, gate_up)
    T, H, F, dt = _ffn_shapes(x, W1, W3, W2, "expert_ffn_backward")
    if dy.shape != x.shape or dy.dtype != x.dtype or gate_up.shape != (2, T, F) or gate_up.dtype != torch.float32:
        raise ValueError("expert_ffn_backward: dy must be like x, and gate_up [2, T, F] in float32")
    dx = torch.empty_like(x) if input_gradient else None
    dW1, dW3, dW2 = (torch.empty_like(w) if weight_gradients else None for w in (W1, W3, W2))
    ws = _workspace(_lib.expert_ffn_backward_workspace(T, H, F, dt), dev, workspace)
    _check(_lib.expert_ffn_backward(_ptr(dy), _ptr(x), _ptr(W1), _ptr(W3), _ptr(W2), _ptr(gate_up), T, H, F, dt, _ptr(dx),
                                    _ptr(dW1), _ptr(dW3), _ptr(dW2), _ptr(ws), ws.numel(), _stream(dev)))
    return dx, dW1, dW3, dW2


# ---------------------------------------------------------------- rows to the experts and back
# (sizes as plain numbers: torch.empty takes 0.4 us longer for a tuple, and these calls allocate several small tensors)
_empty = torch.empty

# Kernels go to the current device; where the tensors lie on another one, that is made current for the call.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call_on(dev: torch.device, call, *args) -> None:
    """call(*args, stream) with `dev` the current device, and its status checked."""
    if _current_device() == dev.index:
        _check(call(*args, _raw_stream(dev.index)))
    else:
        with torch.cuda.device(dev):
            _check(call(*args, _raw_stream(dev.index)))


def _given(*tensors):
    return [t for t in tensors if t is not None]


def _slot_rows(rows, slot_of, what: str):
    """T, k, H, R and the type code of rows [R,H] named by slot_of [T,k]."""
    if rows.dim() != 2 or slot_of.dim() != 2 or slot_of.dtype != torch.int32:
        raise ValueError(f"{what}: rows must be [R, H] and slot_of [T, k] in int32")
    return slot_of.shape[0], slot_of.shape[1], rows.shape[1], rows.shape[0], _dtype_code(rows)


def _slot_weights(weights, slot_of, what: str):
    if weights is not None and (weights.shape != slot_of.shape or weights.dtype != torch.float32):
        raise ValueError(f"{what}: weights must be [T, k] in float32, as slot_of is")


@functools.lru_cache(maxsize=256)
def moe_dispatch_rows_workspace(T: int, k: int, E: int) -> int:
    return int(_lib.moe_dispatch_rows_workspace(T, k, E))


def moe_dispatch_rows(x, experts, num_experts: int, used=None, rows=None, workspace=None):
    """rows [T*k,H], slot_of [T,k] int32 and offsets [num_experts+1] int32: every token's row of x [T,H] copied to the experts [T,k] int32
    that it goes to, sorted by expert.  `used` [T] int32: how many of a token's slots are used (None: all).  `rows`, if given, is written
    in place; what lies behind the last used row stays as it was (without it: is not initialised)."""
    if x.dim() != 2 or experts.dim() != 2 or experts.shape[0] != x.shape[0] or experts.dtype != torch.int32:
        raise ValueError("moe_dispatch_rows: x must be [T, H] and experts [T, k] in int32")
    T, H = x.shape
    k = experts.shape[1]
    dt = _dtype_code(x)
    if used is not None and (used.shape != (T,) or used.dtype != torch.int32):
        raise ValueError("moe_dispatch_rows: used must be [T] in int32")
    if rows is not None and (rows.shape != (T * k, H) or rows.dtype != x.dtype):
        raise ValueError("moe_dispatch_rows: rows must be [T * k, H], of x's type")
    dev = _dev(x, experts, *_given(used, rows))
    if rows is None:
        rows = _empty(T * k, H, dtype=x.dtype, device=dev)
    slot_of = torch.empty_like(experts)
    offsets = _empty(max(num_experts, 0) + 1, dtype=torch.int32, device=dev)
    need = moe_dispatch_rows_workspace(T, k, num_experts)
    ws = _workspace(need, dev, workspace) if need or workspace is not None else None
    _call_on(dev, _lib.moe_dispatch_rows, _ptr(x), _ptr(experts), _ptr(used), T, k, num_experts, H, dt, _ptr(rows), _ptr(slot_of),
             _ptr(offsets), _ptr(ws), ws.numel() if ws is not None else 0)
    return rows, slot_of, offsets


def moe_dispatch_rows_backward(drows, slot_of):
    """dx [T,H]: the gradients of a token's rows added up, from drows [R,H] and moe_dispatch_rows's slot_of [T,k]."""
    T, k, H, R, dt = _slot_rows(drows, slot_of, "moe_dispatch_rows_backward")
    dev = _dev(drows, slot_of)
    dx = _empty(T, H, dtype=drows.dtype, device=dev)
    _call_on(dev, _lib.moe_dispatch_rows_backward, _ptr(drows), _ptr(slot_of), T, k, H, R, dt, _ptr(dx))
    return dx


def moe_combine_rows(y, slot_of, weights=None):
    """out [T,H]: the experts' output rows y [R,H] weighted (weights [T,k] fp32, None: 1) and added up by token."""
    T, k, H, R, dt = _slot_rows(y, slot_of, "moe_combine_rows")
    _slot_weights(weights, slot_of, "moe_combine_rows")
    dev = _dev(y, slot_of) if weights is None else _dev(y, slot_of, weights)
    out = _empty(T, H, dtype=y.dtype, device=dev)
    _call_on(dev, _lib.moe_combine_rows, _ptr(y), _ptr(slot_of), _ptr(weights), T, k, H, R, dt, _ptr(out))
    return out


def moe_combine_rows_backward(dout, y, slot_of, weights=None, weight_gradient: bool = True, dy=None):
    """dy [R,H] and dweights [T,k] fp32 (None without `weight_gradient`) from dout [T,H].  `dy`, if given, is written in place (it may be y);
    rows that no slot names stay as they were (without it: are not initialised)."""
    T, k, H, R, dt = _slot_rows(y, slot_of, "moe_combine_rows_backward")
    _slot_weights(weights, slot_of, "moe_combine_rows_backward")
    if dout.shape != (T, H) or dout.dtype != y.dtype or (dy is not None and (dy.shape != y.shape or dy.dtype != y.dtype)):
        raise ValueError("moe_combine_rows_backward: dout must be [T, H] and dy like y, of y's type")
    dev = _dev(y, dout, slot_of, *_given(weights, dy))
    if dy is None:
        dy = _empty(R, H, dtype=y.dtype, device=dev)
    dweights = _empty(T, k, dtype=torch.float32, device=dev) if weight_gradient else None
    _call_on(dev, _lib.moe_combine_rows_backward, _ptr(dout), _ptr(y), _ptr(slot_of), _ptr(weights), T, k, H, R, dt, _ptr(dy), _ptr(dweights))
    return dy, dweights


# ---------------------------------------------------------------- logits
def _logit_rows(logits):
    """T, V and the distance between rows of a 2-D tensor whose rows may lie further apart than they are long."""
    if logits.dim() != 2:
        raise ValueError("logits must be [T, V]")
    T, V = logits.shape
    step, unit = logits.stride()
    if not logits.is_cuda:
        raise ValueError("all tensors must live on the same GPU")
    if (unit != 1 and V > 1) or (step < V and T > 1):
        raise ValueError("rows of logits must be contiguous and must not overlap")
    return T, V, max(step, V) if T > 1 else V


def _beside(t, shape, dtype, index: int, what: str):
    """Checks an operand that goes with the logits on GPU `index`."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}, not {t.dtype} of {tuple(t.shape)}")
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous and on the logits' GPU")


def moe_token_logprobs(logits, tokens, top: int = 0):
    """logprob [T], entropy [T], top_logprob [T,top] (fp32) and top_ids [T,top] int32 of logits [T,V] at tokens [T] int64
    (negative: none given).  Rows of logits may be views into longer rows."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    _beside(tokens, (T,), torch.int64, dev.index, "tokens")
    columns = max(top, 0)
    logprob, entropy = _empty(T, dtype=torch.float32, device=dev), _empty(T, dtype=torch.float32, device=dev)
    top_logprob = _empty(T, columns, dtype=torch.float32, device=dev)
    top_ids = _empty(T, columns, dtype=torch.int32, device=dev)
    _check(_lib.moe_token_logprobs(logits.data_ptr(), ld, tokens.data_ptr(), T, V, dt, top, logprob.data_ptr(), entropy.data_ptr(),
                                   top_logprob.data_ptr(), top_ids.data_ptr(), _raw_stream(dev.index)))
    return logprob, entropy, top_logprob, top_ids


def _gradient_rows(logits, grad, T: int, V: int):
    if grad is None:
        return _empty(T, V, dtype=logits.dtype, device=logits.device), V
    if grad.shape != logits.shape or grad.dtype != logits.dtype or grad.get_device() != logits.get_device():
        raise ValueError("the gradient must be like the logits")
    return grad, _logit_rows(grad)[2]


def _alternatives(ids, teacher, T: int, index: int) -> int:
    if ids.dim() != 2:
        raise ValueError("ids must be [T, K]")
    K = ids.shape[1]
    _beside(ids, (T, K), torch.int32, index, "ids")
    _beside(teacher, (T, K), torch.float32, index, "teacher")
    return K


def moe_distill_topk(logits, ids, teacher, temperature: float = 1.0, weights=None, gradient: bool = False, out=None):
    """loss [T] and stats [T,2] (fp32) of the student's logits [T,V] against the teacher's alternatives, ids [T,K] int32 and
    teacher [T,K] fp32; with `gradient` also the gradient of (weights * loss).sum() by the logits, in the same pass, into
    `out` if given (which may be `logits` itself), else into rows of V elements.  Of logits that are views into longer rows of
    which not all start alike within 16 bytes the gradient is written fastest into an `out` of the same layout."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    K = _alternatives(ids, teacher, T, dev.index)
    if weights is not None:
        _beside(weights, (T,), torch.float32, dev.index, "weights")
    loss, stats = _empty(T, dtype=torch.float32, device=dev), _empty(T, 2, dtype=torch.float32, device=dev)
    grad, ld_grad = _gradient_rows(logits, out, T, V) if gradient else (None, 0)
    _check(_lib.moe_distill_topk(logits.data_ptr(), ld, ids.data_ptr(), teacher.data_ptr(), T, V, K, dt, temperature, _ptr(weights),
                                 loss.data_ptr(), stats.data_ptr(), _ptr(grad), ld_grad, _raw_stream(dev.index)))
    return (loss, stats, grad) if gradient else (loss, stats)


def moe_distill_topk_backward(logits, ids, teacher, stats, grad_loss, temperature: float = 1.0, out=None):
    """The gradient [T,V] by the logits, from moe_distill_topk's stats and the upstream gradient [T] fp32 of its loss."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    K = _alternatives(ids, teacher, T, dev.index)
    _beside(stats, (T, 2), torch.float32, dev.index, "stats")
    _beside(grad_loss, (T,), torch.float32, dev.index, "grad_loss")
    grad, ld_grad = _gradient_rows(logits, out, T, V)
    _check(_lib.moe_distill_topk_backward(logits.data_ptr(), ld, ids.data_ptr(), teacher.data_ptr(), stats.data_ptr(),
                                          grad_loss.data_ptr(), T, V, K, dt, temperature, grad.data_ptr(), ld_grad,
                                          _raw_stream(dev.index)))
    return grad


# ---------------------------------------------------------------- losses on given answers
def moe_policy_loss(logits, tokens, old_logprob, advantages, ref_logprob=None, clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0,
                    temperature: float = 1.0, weights=None, gradient: bool = False, out=None):
    """loss [T], logprob [T] and stats [T,3] (fp32) of sampled tokens [T] int64 (negative: left out) under logits [T,V], from the log
    probabilities with which they were sampled, their advantages and, with `kl`, a reference's log probabilities (all [T] fp32); with
    `gradient` also the gradient of (weights * loss).sum() by the logits, in the same pass, into `out` if given (which may be `logits`).  A row of
    weight 0 is left out as one without a token is: its loss and log probability are 0 too.  Of logits that are views into longer rows the
    gradient is written fastest into an `out` of the same layout, as in moe_distill_topk."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    _beside(tokens, (T,), torch.int64, dev.index, "tokens")
    _beside(old_logprob, (T,), torch.float32, dev.index, "old_logprob")
    _beside(advantages, (T,), torch.float32, dev.index, "advantages")
    if ref_logprob is not None:
        _beside(ref_logprob, (T,), torch.float32, dev.index, "ref_logprob")
    if weights is not None:
        _beside(weights, (T,), torch.float32, dev.index, "weights")
    loss, logprob = _empty(T, dtype=torch.float32, device=dev), _empty(T, dtype=torch.float32, device=dev)
    stats = _empty(T, 3, dtype=torch.float32, device=dev)
    grad, ld_grad = _gradient_rows(logits, out, T, V) if gradient else (None, 0)
    _call_on(dev, _lib.moe_policy_loss, logits.data_ptr(), ld, tokens.data_ptr(), old_logprob.data_ptr(), advantages.data_ptr(), _ptr(ref_logprob),
             T, V, dt, clip_low, clip_high, kl, temperature, _ptr(weights), loss.data_ptr(), logprob.data_ptr(), stats.data_ptr(), _ptr(grad), ld_grad)
    return (loss, logprob, stats, grad) if gradient else (loss, logprob, stats)


def moe_policy_loss_backward(logits, tokens, stats, grad_loss, temperature: float = 1.0, out=None):
    """The gradient [T,V] by the logits, from moe_policy_loss's stats and the upstream gradient [T] fp32 of its loss."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    _beside(tokens, (T,), torch.int64, dev.index, "tokens")
    _beside(stats, (T, 3), torch.float32, dev.index, "stats")
    _beside(grad_loss, (T,), torch.float32, dev.index, "grad_loss")
    grad, ld_grad = _gradient_rows(logits, out, T, V)
    _call_on(dev, _lib.moe_policy_loss_backward, logits.data_ptr(), ld, tokens.data_ptr(), stats.data_ptr(), grad_loss.data_ptr(), T, V, dt,
             temperature, grad.data_ptr(), ld_grad)
    return grad


def _pairs(offsets, index: int) -> int:
    if offsets.dim() != 1 or offsets.shape[0] % 2 == 0:
        raise ValueError("offsets must be [2 * pairs + 1]")
    _beside(offsets, offsets.shape, torch.int64, index, "offsets")
    return offsets.shape[0] // 2


def moe_preference_loss(logits, tokens, offsets, ref_logprob, beta: float = 0.1, smoothing: float = 0.0, average: bool = False, weights=None,
                        gradient: bool = False, out=None):
    """loss [P], rewards [2,P], logprob [T] and stats [T,3] (fp32) of P pairs of answers: answer a is rows offsets[a] .. offsets[a+1] - 1 of
    logits [T,V], offsets [2 P + 1] int64; pair i is answers i (chosen) and P + i (rejected); tokens [T] int64 (negative: none), ref_logprob
    [T] fp32.  With `gradient` also the gradient of (weights * loss).sum(), weights [P] (one of 0 leaves its pair's loss), by the logits, into
    `out` if given (which may be `logits`): its rows outside all answers stay as they were in `out`, and are 0 without it."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    P = _pairs(offsets, dev.index)
    _beside(tokens, (T,), torch.int64, dev.index, "tokens")
    _beside(ref_logprob, (T,), torch.float32, dev.index, "ref_logprob")
    if weights is not None:
        _beside(weights, (P,), torch.float32, dev.index, "weights")
    loss, rewards = _empty(P, dtype=torch.float32, device=dev), _empty(2, P, dtype=torch.float32, device=dev)
    logprob, stats = _empty(T, dtype=torch.float32, device=dev), _empty(T, 3, dtype=torch.float32, device=dev)
    grad, ld_grad = _gradient_rows(logits, out, T, V) if gradient else (None, 0)
    call = _lib.moe_preference_loss_all_rows if gradient and out is None else _lib.moe_preference_loss
    _call_on(dev, call, logits.data_ptr(), ld, tokens.data_ptr(), offsets.data_ptr(), ref_logprob.data_ptr(), T, V, P, dt, beta,
             smoothing, 1 if average else 0, _ptr(weights), loss.data_ptr(), rewards.data_ptr(), logprob.data_ptr(), stats.data_ptr(), _ptr(grad),
             ld_grad)
    return (loss, rewards, logprob, stats, grad) if gradient else (loss, rewards, logprob, stats)


def moe_preference_loss_backward(logits, tokens, offsets, stats, grad_loss, out=None):
    """The gradient [T,V] by the logits, from moe_preference_loss's stats and the upstream gradient [P] fp32 of its loss.  Rows outside all
    answers stay as they were in `out`, and are 0 without it."""
    T, V, ld = _logit_rows(logits)
    dt = _dtype_code(logits)
    dev = logits.device
    P = _pairs(offsets, dev.index)
    _beside(tokens, (T,), torch.int64, dev.index, "tokens")
    _beside(stats, (T, 3), torch.float32, dev.index, "stats")
    _beside(grad_loss, (P,), torch.float32, dev.index, "grad_loss")
    grad, ld_grad = _gradient_rows(logits, out, T, V)
    call = _lib.moe_preference_loss_backward_all_rows if out is None else _lib.moe_preference_loss_backward
    _call_on(dev, call, logits.data_ptr(), ld, tokens.data_ptr(), offsets.data_ptr(), stats.data_ptr(),
             grad_loss.data_ptr(), T, V, P, dt, grad.data_ptr(), ld_grad)
    return grad


# ---------------------------------------------------------------- kernel timing
def kernel_timing_enable(on: bool = True) -> None:
    _check(_lib.moep_timing_enable(1 if on else 0))


def kernel_timing_collect() -> Dict[str, Tuple[float, int]]:
    """{kernel name: (total milliseconds, launches)} since the last collect; waits for the GPU."""
    cap = 64
    names = (c_char_p * cap)()
    ms = (c_double * cap)()
    cnt = (c_int64 * cap)()
    n = _lib.moep_timing_collect(names, ms, cnt, cap)
    if n < 0:
        raise MoepError(4, _lib.moep_last_error().decode())
    return {names[i].decode(): (float(ms[i]), int(cnt[i])) for i in range(n)}


def kernel_timing_records():
    """[(kernel name, milliseconds)] launch by launch since the last collect; waits for the GPU."""
    cap = 8192
    names = (c_char_p * cap)()
    ms = (c_float * cap)()
    n = _lib.moep_timing_records(names, ms, cap)
    if n < 0:
        raise MoepError(4, _lib.moep_last_error().decode())
    return [(names[i].decode(), float(ms[i])) for i in range(n)]


def mfma_ceiling(a_src: torch.Tensor, b_src: torch.Tensor, steps: int, sink: Optional[torch.Tensor] = None) -> float:
    """Enqueues the MFMA-only launch (operand bits from the two bf16 tensors) and returns its flop count."""
    dev = _dev(a_src, b_src)
    if sink is None:
        sink = torch.empty((1 << 17,), dtype=torch.float32, device=dev)
    flop = c_double(0.0)
    nbytes = min(a_src.numel() * a_src.element_size(), b_src.numel() * b_src.element_size())
    _check(_lib.moep_mfma_ceiling(_ptr(a_src), _ptr(b_src), nbytes, steps, _ptr(sink), sink.numel(),
                                  ctypes.byref(flop), _stream(dev)))
    return float(flop.value)


def kernel_timing_reset() -> None:
    kernel_timing_collect()
