"""Thin Python binding over the C-ABI library (include/tslt.h): argument marshalling only.

Every function takes torch tensors that live on the GPU, allocates the outputs and the workspace
with torch (device memory and streams are torch's job here, nothing else), passes raw device
pointers and the current HIP stream to the library and returns the output tensors.  There is no
fallback: if the library is missing, or a tensor is not on a GPU, the call raises.

The calls of a serving loop (with the caller's outputs and workspace; pack and unpack) go through `_binding`
(csrc/binding.cpp), which makes the same checks natively; where one does not hold it returns None and the
function here goes through them one by one and says which.  Without a `_binding` built for this torch and this
Python every call takes the functions here, which cost the host 7 us more.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence

import torch

from .build import built_for

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtslt.so")

F32, BF16, F16 = 0, 1, 2
OP_TRUNCATE, OP_SAMPLE, OP_VERIFY, OP_VERIFY_TREE, OP_VERIFY_TREE_PATH, OP_TRUNCATE_SHARED = 0, 1, 2, 3, 4, 5
ROW_NONFINITE, ROW_EMPTY, ROW_TOKEN_NOT_IN_SET, ROW_BAD_SET, ROW_EXACT_PATH = 1, 2, 4, 8, 256
ROW_BAD_PAGE, ROW_BAD_INDEX = 16, 32
PAGE_TOKENS = 64
MAX_TOP = 32
MAX_AXES = 4
MAX_K_CAP = 1024
PAYLOAD = {"f32": 0, "bf16": 1, "f16": 2}       # tslt_dtype codes of the formats a payload can travel in

EXPORTS = ("tslt_version", "tslt_last_error", "tslt_workspace_bytes", "tslt_truncate", "tslt_truncate_sample", "tslt_sample",
           "tslt_pack_bound_words", "tslt_pack", "tslt_pack_cleared", "tslt_unpack",
           "tslt_verify", "tslt_verify_accept", "tslt_verify_resample", "tslt_verify_staged", "tslt_verify_accept_staged",
           "tslt_verify_static", "tslt_truncation_stats", "tslt_multicandidate_stats", "tslt_calibrate_read", "tslt_verify_tree",
           "tslt_cache_append", "tslt_cache_attend", "tslt_cache_attend_workspace_bytes", "tslt_cache_weigh", "tslt_cache_evict",
           "tslt_rotate", "tslt_rotate_backward", "tslt_rotate_backward_workspace_bytes",
           "tslt_logprob", "tslt_logprob_workspace_bytes", "tslt_logprob_backward",
           "tslt_adapt", "tslt_adapt_workspace_bytes")

class _Cache(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Rotation(ctypes.Structure):
    _fields_ = [("position", ctypes.c_void_p), ("position_seq_stride", ctypes.c_int64), ("base", ctypes.c_void_p), ("freq", ctypes.c_void_p),
                ("axis", ctypes.c_void_p), ("axes", ctypes.c_int32), ("rotary", ctypes.c_int32), ("adjacent", ctypes.c_int32), ("eps", ctypes.c_float),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p)]


_lib = None
_fast = None                                    # the module _binding, bound to the library that is loaded (None: there is none to use)


class TsltError(RuntimeError):
    pass


def load(path: Optional[str] = None):
    """Open the library; raises if it has not been built (python -m paper_2512_16273_amd.build)."""
    global _lib, _fast
    if _lib is not None and path is None:
        return _lib
    path = path or os.environ.get("TSLT_LIBRARY") or LIB_PATH      # TSLT_LIBRARY: another build of the same ABI
    if not os.path.exists(path):
        raise TsltError(f"{path} not found: build it with `python -m paper_2512_16273_amd.build` "
                        "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    c = ctypes
    vp, i32, i64, f32, sz = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
    lib.tslt_version.restype = c.c_int
    lib.tslt_version.argtypes = []
    lib.tslt_last_error.restype = c.c_char_p
    lib.tslt_last_error.argtypes = []
    lib.tslt_workspace_bytes.restype = sz
    lib.tslt_workspace_bytes.argtypes = [c.c_int, i64, i64, i64, i32]
    lib.tslt_truncate.restype = c.c_int
    lib.tslt_truncate.argtypes = [vp, c.c_int, i64, i64, i64, f32, i32, f32, i32, c.c_int, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tslt_pack_bound_words.restype = i64
    lib.tslt_pack_bound_words.argtypes = [i64, i32, i64]
    for fn in (lib.tslt_pack, lib.tslt_pack_cleared):
        fn.restype = c.c_int
        fn.argtypes = [vp, vp, vp, i64, i32, i64, c.c_int, vp, i64, vp, vp]
    lib.tslt_unpack.restype = c.c_int
    lib.tslt_unpack.argtypes = [vp, vp, i64, i32, i64, c.c_int, vp, vp, vp, vp]
    lib.tslt_truncate_sample.restype = c.c_int
    lib.tslt_truncate_sample.argtypes = [vp, c.c_int, i64, i64, i64, f32, i32, f32, i32, c.c_int, vp, vp, vp, vp, vp, vp,
                                         vp, i32, i32, vp, vp, vp, sz, vp]
    lib.tslt_sample.restype = c.c_int
    lib.tslt_sample.argtypes = [vp, vp, vp, i64, i32, vp, i32, i32, vp, vp, vp]
    for fn in (lib.tslt_verify, lib.tslt_verify_accept, lib.tslt_verify_resample):
        fn.restype = c.c_int
        fn.argtypes = [vp, c.c_int, i64, i32, i64, i64, f32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    for fn in (lib.tslt_verify_staged, lib.tslt_verify_accept_staged):
        fn.restype = c.c_int
        fn.argtypes = [vp, c.c_int, i64, i32, i64, i64, f32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, i32]
    lib.tslt_verify_static.restype = c.c_int
    lib.tslt_verify_static.argtypes = [vp, c.c_int, i64, i32, i64, i64, f32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.tslt_calibrate_read.restype = c.c_int
    lib.tslt_calibrate_read.argtypes = [vp, sz, i32, vp, vp]
    lib.tslt_truncation_stats.restype = c.c_int
    lib.tslt_truncation_stats.argtypes = [vp, c.c_int, i64, i64, i64, f32, vp, vp, vp, i32, c.POINTER(i32), i32, vp, vp, vp, vp]
    lib.tslt_multicandidate_stats.restype = c.c_int
    lib.tslt_multicandidate_stats.argtypes = [vp, c.c_int, i64, i64, i64, f32, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.tslt_verify_tree.restype = c.c_int
    lib.tslt_verify_tree.argtypes = [vp, c.c_int, i64, i64, i64, f32, i32, c.POINTER(i32), vp, vp, vp, i32, vp, vp,
                                     vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    cache, rows = c.POINTER(_Cache), c.POINTER(_Rows)
    lib.tslt_cache_append.restype = c.c_int
    lib.tslt_cache_append.argtypes = [cache, vp, i64, vp, i64, i32, rows, rows, c.c_int, vp, i32, vp, vp, vp, vp]
    lib.tslt_cache_attend_workspace_bytes.restype = sz
    lib.tslt_cache_attend_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64]
    lib.tslt_cache_attend.restype = c.c_int
    lib.tslt_cache_attend.argtypes = [cache, vp, i64, vp, i64, i32, i32, rows, rows, rows, c.c_int, vp, i64, vp, f32, vp, vp, vp, vp, sz, vp]
    lib.tslt_cache_weigh.restype = c.c_int
    lib.tslt_cache_weigh.argtypes = [cache, vp, i64, vp, i64, i32, i32, rows, c.c_int, vp, vp, f32, vp, f32, vp, vp, vp]
    lib.tslt_cache_evict.restype = c.c_int
    lib.tslt_cache_evict.argtypes = [cache, vp, i64, vp, i64, vp, i32, i32, vp, i64, vp, vp, vp, vp, vp]
    how = c.POINTER(_Rotation)
    lib.tslt_rotate.restype = c.c_int
    lib.tslt_rotate.argtypes = [rows, rows, c.c_int, i64, i32, i32, i32, i32, how, vp, rows, rows, vp, vp]
    lib.tslt_rotate_backward_workspace_bytes.restype = sz
    lib.tslt_rotate_backward_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    lib.tslt_rotate_backward.restype = c.c_int
    lib.tslt_rotate_backward.argtypes = [rows, rows, rows, rows, c.c_int, i64, i32, i32, i32, i32, how, vp, rows, rows, vp, vp, vp, vp, sz, vp]
    lib.tslt_logprob_workspace_bytes.restype = sz
    lib.tslt_logprob_workspace_bytes.argtypes = [i64, i32, i64, i32]
    lib.tslt_logprob.restype = c.c_int
    lib.tslt_logprob.argtypes = [vp, c.c_int, i64, i32, i64, i64, i64, f32, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tslt_logprob_backward.restype = c.c_int
    lib.tslt_logprob_backward.argtypes = [vp, c.c_int, i64, i32, i64, i64, i64, f32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, i64, i64, vp]
    lib.tslt_adapt_workspace_bytes.restype = sz
    lib.tslt_adapt_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    lib.tslt_adapt.restype = c.c_int
    lib.tslt_adapt.argtypes = [rows, i32, rows, rows, i32, c.c_int, i64, i32, vp, vp, i64, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    _fast = _native_binding()
    if _fast is not None:
        _fast.bind(*[c.cast(getattr(lib, fn), vp).value for fn in (
            "tslt_workspace_bytes", "tslt_truncate_sample", "tslt_verify", "tslt_verify_accept", "tslt_verify_resample", "tslt_verify_tree",
            "tslt_pack_bound_words", "tslt_pack_cleared", "tslt_unpack",
            "tslt_cache_append", "tslt_cache_attend", "tslt_cache_weigh", "tslt_cache_evict",
            "tslt_rotate", "tslt_rotate_backward", "tslt_logprob", "tslt_logprob_backward", "tslt_adapt")])
    _lib = lib
    return lib


def _native_binding():
    """The module `_binding` where it is there, imports, and was built for this torch and this Python; else None."""
    try:
        from . import _binding
    except ImportError:
        return None
    return _binding if getattr(_binding, "built_for", "") == built_for() else None


def _check(code: int):
    if code != 0:
        raise TsltError(f"tslt error {code}: {load().tslt_last_error().decode()}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float16:
        return F16
    raise TsltError(f"unsupported logits dtype {t.dtype}")


def _dev(t: torch.Tensor, dtype=None, name="tensor", contiguous=True) -> torch.Tensor:
    if t.is_cuda and (dtype is None or t.dtype is dtype) and (not contiguous or t.is_contiguous()):
        return t
    if not t.is_cuda:
        raise TsltError(f"{name} must live on the GPU (there is no CPU path)")
    if dtype is not None and t.dtype != dtype:
        raise TsltError(f"{name} must be {dtype}, got {t.dtype}")
    if contiguous and not t.is_contiguous():
        raise TsltError(f"{name} must be contiguous")
    return t


# (Pointers and streams go to ctypes as plain integers, without a c_void_p for each of the twenty arguments of a call.)
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    """The current device's current stream; what torch.cuda.current_stream().cuda_stream gives, without the object."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _rows_2d(logits: torch.Tensor):
    """[..., V] view as rows with a common stride (the last dimension must be dense)."""
    if logits.stride(-1) != 1:
        raise TsltError("logits must be dense along the vocabulary")
    V = logits.shape[-1]
    if logits.dim() == 1:
        return 1, V, V
    flat = logits.reshape(-1, V) if logits.is_contiguous() else logits
    if flat.dim() != 2:
        raise TsltError("non-contiguous logits must be 2-D [rows, V]")
    return flat.shape[0], V, flat.stride(0)


def workspace_bytes(op: int, n_outer: int, n_inner: int, V: int, k_cap: int) -> int:
    return int(load().tslt_workspace_bytes(op, n_outer, n_inner, V, k_cap))


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)   # torch aligns to >= 256 bytes


def _truncate_workspace_bytes(rows: int, V: int, k_cap: int) -> int:
    return _memoised_workspace_bytes(load(), torch.cuda.current_device(), OP_TRUNCATE_SHARED, rows, V, k_cap)


@functools.lru_cache(maxsize=256)               # (the device: how many rows are shared goes by its compute units)
def _memoised_workspace_bytes(lib, device: int, op: int, rows: int, V: int, k_cap: int) -> int:
    return int(lib.tslt_workspace_bytes(op, rows, 0, V, k_cap))


def truncate(logits: torch.Tensor, temperature: float, top_k: int, top_p: float, k_cap: int,
             want_prob: bool = True, out: Optional[dict] = None, u: Optional[torch.Tensor] = None,
             payload: str = "f32", without_replacement: bool = False) -> dict:
    """tslt_truncate over logits [..., V].  Returns idx, logit, prob, count, mass, status ([rows, k_cap] /
    [rows]).  With uniforms u [rows, n] it is tslt_truncate_sample: the result also holds token, slot
    [rows, n], n draws from each row's q_hat (i.i.d., or without replacement).  payload = "bf16" / "f16" rounds the kept values to the
    format in which they will travel before q_hat and the draws are computed."""
    lib = load()
    if _fast is not None and out is not None and u is not None and logits.is_cuda:
        code = _fast.truncate(logits, float(temperature), int(top_k), float(top_p), int(k_cap), PAYLOAD[payload], without_replacement,
                              out, u, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    _dev(logits, name="logits", contiguous=False)
    rows, V, stride = _rows_2d(logits)
    dev = logits.device
    if out is None:
        out = {
            "idx": torch.empty(rows, k_cap, dtype=torch.int32, device=dev),
            "logit": torch.empty(rows, k_cap, dtype=torch.float32, device=dev),
            "prob": torch.empty(rows, k_cap, dtype=torch.float32, device=dev) if want_prob else None,
            "count": torch.empty(rows, dtype=torch.int32, device=dev),
            "mass": torch.empty(rows, dtype=torch.float32, device=dev),
            "status": torch.empty(rows, dtype=torch.int32, device=dev),
        }
    # (a few long rows: memory in which the workgroups that share each of them hand over what they have found)
    ws_bytes = _truncate_workspace_bytes(rows, V, int(k_cap)) if rows else 0
    held = torch.empty(ws_bytes, dtype=torch.uint8, device=dev) if ws_bytes else None
    ws = _ptr(held)
    if u is None:
        _check(lib.tslt_truncate(_ptr(logits), _dtype_code(logits), rows, V, stride, float(temperature), int(top_k),
                                 float(top_p), int(k_cap), PAYLOAD[payload], _ptr(out["idx"]), _ptr(out["logit"]), _ptr(out.get("prob")),
                                 _ptr(out["count"]), _ptr(out.get("mass")), _ptr(out.get("status")), ws, ws_bytes, _stream()))
        return out
    _dev(u, torch.float32, "u")
    u2 = u.reshape(rows, -1)
    n = u2.shape[1]
    if "token" not in out:
        out["token"] = torch.empty(rows, n, dtype=torch.int32, device=dev)
        out["slot"] = torch.empty(rows, n, dtype=torch.int32, device=dev)
    _check(lib.tslt_truncate_sample(_ptr(logits), _dtype_code(logits), rows, V, stride, float(temperature), int(top_k),
                                    float(top_p), int(k_cap), PAYLOAD[payload], _ptr(out["idx"]), _ptr(out["logit"]),
                                    _ptr(out.get("prob")), _ptr(out["count"]), _ptr(out.get("mass")),
                                    _ptr(out.get("status")), _ptr(u2), n, 1 if without_replacement else 0,
                                    _ptr(out["token"]), _ptr(out.get("slot")),
                                    ws, ws_bytes, _stream()))
    return out


def pack(idx: torch.Tensor, logit: torch.Tensor, count: torch.Tensor, V: int, payload: str) -> dict:
    """tslt_pack: truncated sets [rows, k_cap] -> words (uint32, as int32 storage), row_offset [rows + 1] int64."""
    lib = load()
    if _fast is not None and idx.is_cuda:
        made = _fast.pack(idx, logit, count, int(V), PAYLOAD[payload], _stream())
        if made is not None:
            if made[0]:
                _check(made[0])
            return made[1]
    _dev(idx, torch.int32, "idx"); _dev(logit, torch.float32, "logit"); _dev(count, torch.int32, "count")
    rows, k_cap = idx.shape
    cap = int(lib.tslt_pack_bound_words(rows, k_cap, V))
    # (the library clears what lies behind the stream; without rows, or with arguments that it refuses, there is none)
    words = torch.empty(cap, dtype=torch.int32, device=idx.device) if cap > 0 else torch.zeros(1, dtype=torch.int32, device=idx.device)
    offs = torch.empty(rows + 1, dtype=torch.int64, device=idx.device)
    _check(lib.tslt_pack_cleared(idx.data_ptr(), logit.data_ptr(), count.data_ptr(), rows, k_cap, int(V), PAYLOAD[payload],
                                 words.data_ptr(), cap, offs.data_ptr(), _stream()))
    return {"words": words, "row_offset": offs}


def unpack(words: torch.Tensor, row_offset: torch.Tensor, rows: int, k_cap: int, V: int, payload: str) -> dict:
    """tslt_unpack: the inverse of pack -> idx, logit [rows, k_cap], count [rows]."""
    lib = load()
    if _fast is not None and words.is_cuda:
        made = _fast.unpack(words, row_offset, rows, k_cap, int(V), PAYLOAD[payload], _stream())
        if made is not None:
            if made[0]:
                _check(made[0])
            return made[1]
    _dev(words, torch.int32, "words"); _dev(row_offset, torch.int64, "row_offset")
    dev = words.device
    out = {"idx": torch.empty(rows, k_cap, dtype=torch.int32, device=dev),
           "logit": torch.empty(rows, k_cap, dtype=torch.float32, device=dev),
           "count": torch.empty(rows, dtype=torch.int32, device=dev)}
    _check(lib.tslt_unpack(words.data_ptr(), row_offset.data_ptr(), rows, k_cap, int(V), PAYLOAD[payload], out["idx"].data_ptr(),
                           out["logit"].data_ptr(), out["count"].data_ptr(), _stream()))
    return out


def sample(idx: torch.Tensor, logit: torch.Tensor, count: torch.Tensor, u: torch.Tensor,
           without_replacement: bool = False, out: Optional[dict] = None) -> dict:
    """tslt_sample: idx/logit [rows, k_cap], count [rows], u [rows, n] -> token, slot [rows, n]."""
    lib = load()
    _dev(idx, torch.int32, "idx"); _dev(logit, torch.float32, "logit"); _dev(count, torch.int32, "count")
    _dev(u, torch.float32, "u")
    rows, k_cap = idx.shape
    u2 = u.reshape(rows, -1)
    n = u2.shape[1]
    if out is None:
        out = {"token": torch.empty(rows, n, dtype=torch.int32, device=idx.device),
               "slot": torch.empty(rows, n, dtype=torch.int32, device=idx.device)}
    _check(lib.tslt_sample(_ptr(idx), _ptr(logit), _ptr(count), rows, k_cap, _ptr(u2), n,
                           1 if without_replacement else 0, _ptr(out["token"]), _ptr(out.get("slot")), _stream()))
    return out


_PHASES = {"both": 0, "accept": 1, "resample": 2}


def verify(target: torch.Tensor, temperature: float, q_idx: torch.Tensor, q_logit: torch.Tensor,
           q_count: torch.Tensor, draft_tokens: torch.Tensor, u_accept: torch.Tensor, u_resample: torch.Tensor,
           out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None, phase: str = "both",
           first_stage: int = 0) -> dict:
    """tslt_verify: target [B, gamma+1, V]; sparse sets [B, gamma, k_cap]; returns accept_len [B],
    tokens [B, gamma+1], ratio, beta [B, gamma], status [B].  phase = "accept" / "resample" calls
    tslt_verify_accept / tslt_verify_resample (then `out` and `workspace` must be passed to both).
    first_stage > 0 calls tslt_verify_staged / tslt_verify_accept_staged."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and not first_stage and target.is_cuda:
        code = _fast.verify(_PHASES[phase], target, float(temperature), q_idx, q_logit, q_count, draft_tokens, u_accept, u_resample, out,
                            workspace, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    fn = {"both": lib.tslt_verify, "accept": lib.tslt_verify_accept, "resample": lib.tslt_verify_resample}[phase]
    extra = ()
    if first_stage and phase != "resample":
        fn = {"both": lib.tslt_verify_staged, "accept": lib.tslt_verify_accept_staged}[phase]
        extra = (int(first_stage),)
    _dev(target, name="target")
    if target.dim() != 3:
        raise TsltError("target must be [B, gamma+1, V]")
    B, g1, V = target.shape
    gamma = g1 - 1
    _dev(q_idx, torch.int32, "q_idx"); _dev(q_logit, torch.float32, "q_logit"); _dev(q_count, torch.int32, "q_count")
    _dev(draft_tokens, torch.int32, "draft_tokens"); _dev(u_accept, torch.float32, "u_accept")
    _dev(u_resample, torch.float32, "u_resample")
    k_cap = q_idx.shape[-1]
    if q_idx.numel() != B * gamma * k_cap or u_resample.numel() != B * g1 or u_accept.numel() != B * gamma:
        raise TsltError("verify: shapes do not agree")
    dev = target.device
    if out is None:
        out = {"accept_len": torch.empty(B, dtype=torch.int32, device=dev),
               "tokens": torch.empty(B, g1, dtype=torch.int32, device=dev),
               "ratio": torch.empty(B, gamma, dtype=torch.float32, device=dev),
               "beta": torch.empty(B, gamma, dtype=torch.float32, device=dev),
               "status": torch.empty(B, dtype=torch.int32, device=dev)}
    ws = workspace if workspace is not None else _workspace(workspace_bytes(OP_VERIFY, B, gamma, V, k_cap), dev)
    _check(fn(target.data_ptr(), _dtype_code(target), B, gamma, V, target.stride(1), float(temperature),
              q_idx.data_ptr(), q_logit.data_ptr(), q_count.data_ptr(), k_cap, draft_tokens.data_ptr(), u_accept.data_ptr(),
              u_resample.data_ptr(), _ptr(out["accept_len"]), _ptr(out["tokens"]), _ptr(out.get("ratio")),
              _ptr(out.get("beta")), _ptr(out.get("status")), _ptr(ws), ws.numel() if ws is not None else 0,
              _stream(), *extra))
    return out


STATIC_MAX_POSITIONS = 262144


def verify_static(target: torch.Tensor, temperature: float, q_idx: torch.Tensor, q_logit: torch.Tensor,
                  q_count: torch.Tensor, draft_tokens: torch.Tensor, u_accept: torch.Tensor, u_resample: torch.Tensor,
                  out: dict) -> dict:
    """tslt_verify_static: tslt_verify without a workspace (the library's own static device array holds the
    per-position decisions).  `out` must hold preallocated accept_len, tokens, ratio, beta, status tensors: this
    wrapper allocates nothing either."""
    lib = load()
    _dev(target, name="target")
    if target.dim() != 3:
        raise TsltError("target must be [B, gamma+1, V]")
    B, g1, V = target.shape
    gamma = g1 - 1
    _dev(q_idx, torch.int32, "q_idx"); _dev(q_logit, torch.float32, "q_logit"); _dev(q_count, torch.int32, "q_count")
    _dev(draft_tokens, torch.int32, "draft_tokens"); _dev(u_accept, torch.float32, "u_accept")
    _dev(u_resample, torch.float32, "u_resample")
    k_cap = q_idx.shape[-1]
    if q_idx.numel() != B * gamma * k_cap or u_resample.numel() != B * g1 or u_accept.numel() != B * gamma:
        raise TsltError("verify_static: shapes do not agree")
    if out["accept_len"].numel() != B or out["tokens"].numel() != B * g1:
        raise TsltError("verify_static: output shapes do not agree")
    _check(lib.tslt_verify_static(_ptr(target), _dtype_code(target), B, gamma, V, target.stride(1), float(temperature),
                                  _ptr(q_idx), _ptr(q_logit), _ptr(q_count), k_cap, _ptr(draft_tokens), _ptr(u_accept),
                                  _ptr(u_resample), _ptr(out["accept_len"]), _ptr(out["tokens"]), _ptr(out.get("ratio")),
                                  _ptr(out.get("beta")), _ptr(out.get("status")), _stream()))
    return out


def calibrate_read(src: torch.Tensor, n_blocks: int, sink: torch.Tensor) -> None:
    """tslt_calibrate_read: one read-only streaming launch over the whole of `src` (time it from outside)."""
    _dev(src, name="src"); _dev(sink, name="sink")
    _check(load().tslt_calibrate_read(_ptr(src), src.numel() * src.element_size(), int(n_blocks), _ptr(sink), _stream()))


def truncation_stats(target: torch.Tensor, temperature: float, q_idx: torch.Tensor, q_logit: torch.Tensor,
                     q_count: torch.Tensor, k_list: Sequence[int]) -> dict:
    """tslt_truncation_stats: target [rows, V]; sets [rows, k_cap]; returns keep, beta [rows, len(k_list)] and
    status [rows]."""
    lib = load()
    _dev(target, name="target")
    if target.dim() != 2:
        raise TsltError("target must be [rows, V]")
    rows, V = target.shape
    _dev(q_idx, torch.int32, "q_idx"); _dev(q_logit, torch.float32, "q_logit"); _dev(q_count, torch.int32, "q_count")
    k_cap = q_idx.shape[-1]
    if q_idx.numel() != rows * k_cap or q_logit.numel() != rows * k_cap or q_count.numel() != rows:
        raise TsltError("truncation_stats: shapes do not agree")
    ks = (ctypes.c_int32 * len(k_list))(*[int(k) for k in k_list])
    dev = target.device
    out = {"keep": torch.empty(rows, len(k_list), dtype=torch.float32, device=dev),
           "beta": torch.empty(rows, len(k_list), dtype=torch.float32, device=dev),
           "status": torch.empty(rows, dtype=torch.int32, device=dev)}
    _check(lib.tslt_truncation_stats(_ptr(target), _dtype_code(target), rows, V, target.stride(0), float(temperature),
                                     _ptr(q_idx), _ptr(q_logit), _ptr(q_count), k_cap, ks, len(k_list),
                                     _ptr(out["keep"]), _ptr(out["beta"]), _ptr(out["status"]), _stream()))
    return out


def multicandidate_stats(target: torch.Tensor, temperature: float, q_idx: torch.Tensor, q_logit: torch.Tensor,
                         q_count: torch.Tensor, k: int) -> dict:
    """tslt_multicandidate_stats: target [rows, V]; sets [rows, k_cap]; returns beta [rows, k], theta [rows] and
    status [rows]."""
    lib = load()
    _dev(target, name="target")
    if target.dim() != 2:
        raise TsltError("target must be [rows, V]")
    rows, V = target.shape
    _dev(q_idx, torch.int32, "q_idx"); _dev(q_logit, torch.float32, "q_logit"); _dev(q_count, torch.int32, "q_count")
    k_cap = q_idx.shape[-1]
    if q_idx.numel() != rows * k_cap or q_logit.numel() != rows * k_cap or q_count.numel() != rows:
        raise TsltError("multicandidate_stats: shapes do not agree")
    dev = target.device
    out = {"beta": torch.empty(rows, int(k), dtype=torch.float32, device=dev),
           "theta": torch.empty(rows, dtype=torch.float32, device=dev),
           "status": torch.empty(rows, dtype=torch.int32, device=dev)}
    _check(lib.tslt_multicandidate_stats(_ptr(target), _dtype_code(target), rows, V, target.stride(0), float(temperature),
                                         _ptr(q_idx), _ptr(q_logit), _ptr(q_count), k_cap, int(k), _ptr(out["beta"]),
                                         _ptr(out["theta"]), _ptr(out["status"]), _stream()))
    return out


def verify_tree(target: torch.Tensor, temperature: float, expansion: Sequence[int], q_idx: torch.Tensor,
                q_logit: torch.Tensor, q_count: torch.Tensor, cand_tokens: torch.Tensor, u_accept: torch.Tensor,
                u_resample: torch.Tensor, all_nodes: bool = True, out: Optional[dict] = None,
                workspace: Optional[torch.Tensor] = None, without_replacement: bool = False) -> dict:
    """tslt_verify_tree: target [B, N_nodes, V]; sparse sets [B, N_int, k_cap]; cand_tokens, u_accept
    [B, N_nodes-1]; u_resample [B, N_nodes].  Returns seq [B, depth+1], len [B], node_token / node_slot
    [B, N_nodes] (when all_nodes), ratio and beta [B, N_nodes-1], status [B].  without_replacement selects the rule
    for candidates that were drawn without replacement."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and target.is_cuda:
        code = _fast.verify_tree(target, float(temperature), expansion, q_idx, q_logit, q_count, cand_tokens, u_accept, u_resample,
                                 without_replacement, out, workspace, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    _dev(target, name="target")
    if target.dim() != 3:
        raise TsltError("target must be [B, N_nodes, V]")
    B, n_nodes, V = target.shape
    depth = len(expansion)
    _dev(q_idx, torch.int32, "q_idx"); _dev(q_logit, torch.float32, "q_logit"); _dev(q_count, torch.int32, "q_count")
    _dev(cand_tokens, torch.int32, "cand_tokens"); _dev(u_accept, torch.float32, "u_accept")
    _dev(u_resample, torch.float32, "u_resample")
    k_cap = q_idx.shape[-1]
    dev = target.device
    if out is None:
        out = {"seq": torch.empty(B, depth + 1, dtype=torch.int32, device=dev),
               "len": torch.empty(B, dtype=torch.int32, device=dev),
               "node_token": torch.empty(B, n_nodes, dtype=torch.int32, device=dev) if all_nodes else None,
               "node_slot": torch.empty(B, n_nodes, dtype=torch.int32, device=dev) if all_nodes else None,
               "ratio": torch.empty(B, max(n_nodes - 1, 1), dtype=torch.float32, device=dev),
               "beta": torch.empty(B, max(n_nodes - 1, 1), dtype=torch.float32, device=dev),
               "status": torch.empty(B, dtype=torch.int32, device=dev)}
    ws = workspace if workspace is not None else _workspace(
        workspace_bytes(OP_VERIFY_TREE if all_nodes else OP_VERIFY_TREE_PATH, B, n_nodes, V, k_cap), dev)
    exp_arr = (ctypes.c_int32 * depth)(*[int(k) for k in expansion])
    _check(lib.tslt_verify_tree(_ptr(target), _dtype_code(target), B, V, target.stride(1), float(temperature), depth,
                                exp_arr, _ptr(q_idx), _ptr(q_logit), _ptr(q_count), k_cap, _ptr(cand_tokens),
                                _ptr(u_accept), _ptr(u_resample), 1 if without_replacement else 0,
                                _ptr(out.get("node_token")),
                                _ptr(out.get("node_slot")), _ptr(out["seq"]), _ptr(out["len"]), _ptr(out.get("ratio")),
                                _ptr(out.get("beta")), _ptr(out.get("status")), _ptr(ws), ws.numel() if ws is not None else 0, _stream()))
    return out


# ---- keys and values in 8 bits -----------------------------------------------------------------------------------

def cache_create(n_pages: int, heads: int, head_dim: int, device="cuda") -> dict:
    """An empty cache: codes [n_pages, heads, 2, 64 * head_dim] uint8 and scale [n_pages, heads, 2] fp32 (see include/tslt.h for
    their layout)."""
    return {"codes": torch.zeros(n_pages, heads, 2, PAGE_TOKENS * head_dim, dtype=torch.uint8, device=device),
            "scale": torch.ones(n_pages, heads, 2, dtype=torch.float32, device=device)}


def tree_mask(expansion: Sequence[int], device="cuda") -> torch.Tensor:
    """The mask of cache_attend for a token tree stored breadth-first, as verify_tree takes it: [1, N_nodes, ceil(N_nodes / 32)]
    int32, of every node its ancestors and itself."""
    rows, layer = [1], [0]
    for k in expansion:
        layer = [parent for parent in layer for _ in range(int(k))]
        rows += [0] * len(layer)
        first = len(rows) - len(layer)
        for i, parent in enumerate(layer):
            rows[first + i] = rows[parent] | 1 << (first + i)
        layer = list(range(first, len(rows)))
    words = (len(rows) + 31) // 32
    bits = b"".join(r.to_bytes(4 * words, "little") for r in rows)
    return torch.frombuffer(bytearray(bits), dtype=torch.int32).view(1, len(rows), words).to(device)


def _cache_of(cache: dict):
    codes, scale = cache["codes"], cache["scale"]
    _dev(codes, torch.uint8, "codes"); _dev(scale, torch.float32, "scale")
    if codes.dim() != 4 or codes.shape[2] != 2 or codes.shape[3] % PAGE_TOKENS or scale.shape != codes.shape[:3]:
        raise TsltError("a cache is codes [n_pages, heads, 2, 64 * head_dim] and scale [n_pages, heads, 2]")
    n_pages, heads, _, size = codes.shape
    return _Cache(codes.data_ptr(), scale.data_ptr(), n_pages, heads, size // PAGE_TOKENS), heads, size // PAGE_TOKENS


def _sequences(pages: torch.Tensor, length: torch.Tensor):
    _dev(pages, torch.int32, "pages"); _dev(length, torch.int32, "length")
    if pages.dim() != 2 or length.numel() != pages.shape[0]:
        raise TsltError("pages must be [B, width], length [B]")
    return pages.shape


def _rows_of(t: torch.Tensor, name: str, shape, dtype) -> _Rows:
    _dev(t, dtype, name, contiguous=False)
    if tuple(t.shape) != tuple(shape):
        raise TsltError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise TsltError(f"{name} must be dense along its last dimension")
    seq, token, head = (s if n > 1 else 0 for s, n in zip(t.stride()[:3], t.shape[:3]))      # (what no second row uses may be anything)
    return _Rows(t.data_ptr(), seq, token, head)


def _counted(t: Optional[torch.Tensor], name: str, numel: int) -> Optional[int]:
    if t is None:
        return None
    _dev(t, torch.int32, name)
    if t.numel() != numel:
        raise TsltError(f"{name} has {t.numel()} entries, {numel} are needed")
    return t.data_ptr()


def _sized(out: dict, name: str, dtype, numel: int, optional=False) -> Optional[int]:
    t = out.get(name)
    if t is None and optional:
        return None
    if t is None:
        raise TsltError(f"out holds no {name}")
    _dev(t, dtype, name)
    if t.numel() != numel:
        raise TsltError(f"{name} has {t.numel()} entries, {numel} are needed")
    return t.data_ptr()


def cache_append(cache: dict, pages: torch.Tensor, length: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 count: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None, out: Optional[dict] = None) -> dict:
    """tslt_cache_append: k, v [B, n, heads, D] (any of the three types, any strides that keep rows 16-byte aligned) to the end of
    the sequences pages [B, width], length [B] of the cache, which changes in place.  index [B, m]: which of
    the n tokens, in order; count [B]: how many of them.  Returns length, the new one, and status [B]."""
    lib = load()
    if _fast is not None and out is not None and k.is_cuda:
        code = _fast.cache_append(cache, pages, length, k, v, count, index, out, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    c, heads, D = _cache_of(cache)
    B, width = _sequences(pages, length)
    if k.dim() != 4:
        raise TsltError("k must be [B, n, heads, D]")
    n = k.shape[1]
    kr, vr = _rows_of(k, "k", (B, n, heads, D), k.dtype), _rows_of(v, "v", (B, n, heads, D), k.dtype)
    if index is not None and index.dim() != 2:
        raise TsltError("index must be [B, m]")
    most = 0 if index is None else index.shape[1]
    if out is None:
        out = {"length": torch.empty(B, dtype=torch.int32, device=k.device), "status": torch.empty(B, dtype=torch.int32, device=k.device)}
    _check(lib.tslt_cache_append(c, pages.data_ptr(), width, length.data_ptr(), B, n, kr, vr, _dtype_code(k),
                                 _counted(index, "index", B * most), most, _counted(count, "count", B), _sized(out, "length", torch.int32, B),
                                 _sized(out, "status", torch.int32, B, optional=True), _stream()))
    return out


def cache_attend_workspace_bytes(B: int, n: int, heads_q: int, heads: int, head_dim: int, width: int) -> int:
    return int(load().tslt_cache_attend_workspace_bytes(B, n, heads_q, heads, head_dim, width))


def cache_attend(q: torch.Tensor, cache: dict, pages: torch.Tensor, length: torch.Tensor, k: Optional[torch.Tensor] = None,
                 v: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                 scale: Optional[float] = None, out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """tslt_cache_attend: q [B, n, heads_q, D] over the sequences' cached tokens and, where k, v [B, n, heads, D] are given, over the new
    tokens that `mask` shows ([B or 1, n, ceil(n / 32)] int32, see tree_mask; None: a chain).  scale: 1 / sqrt(D).  Returns out
    [B, n, heads_q, D], lse [B, n, heads_q] and status [B]."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and q.is_cuda:
        code = _fast.cache_attend(q, cache, pages, length, k, v, mask, count, scale, out, workspace, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    c, heads, D = _cache_of(cache)
    B, width = _sequences(pages, length)
    if q.dim() != 4:
        raise TsltError("q must be [B, n, heads_q, D]")
    _, n, heads_q, _ = q.shape
    qr = _rows_of(q, "q", (B, n, heads_q, D), q.dtype)
    if (k is None) != (v is None):
        raise TsltError("k and v come together")
    kr = None if k is None else _rows_of(k, "k", (B, n, heads, D), q.dtype)
    vr = None if v is None else _rows_of(v, "v", (B, n, heads, D), q.dtype)
    mask_ptr, mask_seq = None, 0
    if mask is not None:
        _dev(mask, torch.int32, "mask")
        words = (n + 31) // 32
        if mask.dim() != 3 or mask.shape[0] not in (1, B) or tuple(mask.shape[1:]) != (n, words):
            raise TsltError(f"mask must be [B or 1, {n}, {words}], got {list(mask.shape)}")
        mask_ptr, mask_seq = mask.data_ptr(), n * words if mask.shape[0] > 1 else 0
    if out is None:
        out = {"out": torch.empty(B, n, heads_q, D, dtype=q.dtype, device=q.device),
               "lse": torch.empty(B, n, heads_q, dtype=torch.float32, device=q.device),
               "status": torch.empty(B, dtype=torch.int32, device=q.device)}
    ws = workspace if workspace is not None else _workspace(cache_attend_workspace_bytes(B, n, heads_q, heads, D, width), q.device)
    _check(lib.tslt_cache_attend(c, pages.data_ptr(), width, length.data_ptr(), B, n, heads_q, qr, kr, vr, _dtype_code(q), mask_ptr, mask_seq,
                                 _counted(count, "count", B), float(D ** -0.5 if scale is None else scale),
                                 _sized(out, "out", q.dtype, B * n * heads_q * D), _sized(out, "lse", torch.float32, B * n * heads_q),
                                 _sized(out, "status", torch.int32, B, optional=True), _ptr(ws), ws.numel() if ws is not None else 0, _stream()))
    return out


def cache_weigh(q: torch.Tensor, lse: torch.Tensor, cache: dict, pages: torch.Tensor, length: torch.Tensor, weight: torch.Tensor,
                decay: float = 1.0, count: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[dict] = None) -> dict:
    """tslt_cache_weigh: weight [B, heads, width * 64] times decay, and what cache_attend's rows q with its lse gave each cached token.
    Returns weight (out may hold the same array) and status [B]."""
    lib = load()
    if _fast is not None and out is not None and q.is_cuda:
        code = _fast.cache_weigh(q, lse, cache, pages, length, weight, float(decay), count, scale, out, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    c, heads, D = _cache_of(cache)
    B, width = _sequences(pages, length)
    if q.dim() != 4:
        raise TsltError("q must be [B, n, heads_q, D]")
    _, n, heads_q, _ = q.shape
    qr = _rows_of(q, "q", (B, n, heads_q, D), q.dtype)
    _dev(lse, torch.float32, "lse"); _dev(weight, torch.float32, "weight")
    if lse.numel() != B * n * heads_q or weight.numel() != B * heads * width * PAGE_TOKENS:
        raise TsltError("cache_weigh: shapes do not agree")
    if out is None:
        out = {"weight": torch.empty_like(weight), "status": torch.empty(B, dtype=torch.int32, device=q.device)}
    _check(lib.tslt_cache_weigh(c, pages.data_ptr(), width, length.data_ptr(), B, n, heads_q, qr, _dtype_code(q), lse.data_ptr(),
                                _counted(count, "count", B), float(D ** -0.5 if scale is None else scale), weight.data_ptr(), float(decay),
                                _sized(out, "weight", torch.float32, weight.numel()), _sized(out, "status", torch.int32, B, optional=True),
                                _stream()))
    return out


def cache_evict(cache: dict, pages: torch.Tensor, length: torch.Tensor, weight: torch.Tensor, keep: int, recent: int,
                new_pages: torch.Tensor, out: Optional[dict] = None) -> dict:
    """tslt_cache_evict: of every head the `recent` last tokens and those of most weight, `keep` in all, copied to the pages
    new_pages [B, new_width] of the same cache.  Returns length [B], kept [B, heads, keep], weight [B, heads, new_width * 64] and status [B]."""
    keep, recent = int(keep), int(recent)
    if not all(-(1 << 31) <= x < 1 << 31 for x in (keep, recent)):         # (ctypes would cut them)
        raise TsltError(f"keep and recent must fit 32 bits (got {keep}, {recent})")
    lib = load()
    if _fast is not None and out is not None and weight.is_cuda:
        code = _fast.cache_evict(cache, pages, length, weight, keep, recent, new_pages, out, _stream())
        if code is not None:
            if code:
                _check(code)
            return out
    c, heads, D = _cache_of(cache)
    B, width = _sequences(pages, length)
    _dev(weight, torch.float32, "weight"); _dev(new_pages, torch.int32, "new_pages")
    if weight.numel() != B * heads * width * PAGE_TOKENS or new_pages.dim() != 2 or new_pages.shape[0] != B:
        raise TsltError("cache_evict: shapes do not agree")
    new_width = new_pages.shape[1]
    if out is None:
        out = {"length": torch.empty(B, dtype=torch.int32, device=weight.device),
               "kept": torch.empty(B, heads, max(keep, 0), dtype=torch.int32, device=weight.device),
               "weight": torch.empty(B, heads, new_width * PAGE_TOKENS, dtype=torch.float32, device=weight.device),
               "status": torch.empty(B, dtype=torch.int32, device=weight.device)}
    _check(lib.tslt_cache_evict(c, pages.data_ptr(), width, length.data_ptr(), B, weight.data_ptr(), keep, recent, new_pages.data_ptr(),
                                new_width, _sized(out, "length", torch.int32, B), _sized(out, "kept", torch.int32, B * heads * max(keep, 0)),
                                _sized(out, "weight", torch.float32, B * heads * new_width * PAGE_TOKENS),
                                _sized(out, "status", torch.int32, B, optional=True), _stream()))
    return out


# ---- around attention and verification ---------------------------------------------------------------------------
#
# Results are no part of a graph of autograd's, also of tensors that ask for a gradient: the gradients are the calls rotate_backward and logprob_backward.

def _here(made: dict, names, **given) -> int:
    """The current stream; the tensors of the call, those of `made` that are named among them, have to live on its device."""
    device = torch.cuda.current_device()
    for name, t in (*given.items(), *((f"out {name}", made.get(name)) for name in names)):
        if t is not None and t.device.index != device:
            raise TsltError(f"{name} lives on {t.device}, the current device is cuda:{device}")
    return torch._C._cuda_getCurrentRawStream(device)


def _told(out: dict, *names: str) -> dict:
    """out, with torch told that those of its tensors were written to (one that a gradient needs as it was is an error then)."""
    torch.autograd.graph.increment_version([t for t in map(out.get, names) if t is not None])
    return out


def _current():
    """The current device and its current stream."""
    device = torch.cuda.current_device()
    return device, torch._C._cuda_getCurrentRawStream(device)


def _optional(t: Optional[torch.Tensor], name: str, dtype, shape) -> Optional[int]:
    if t is None:
        return None
    _dev(t, dtype, name)
    if tuple(t.shape) != tuple(shape):
        raise TsltError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _fits(call: str, *sizes: int) -> None:
    """Sizes that the library takes in 32 bits (ctypes would cut them)."""
    if max(sizes) >= 1 << 31:
        raise TsltError(f"{call}: a size of {max(sizes)} does not fit 31 bits")


def _given(out: dict, name: str) -> torch.Tensor:
    if out.get(name) is None:
        raise TsltError(f"out holds no {name}")
    return out[name]


def _rotation(B: int, n: int, D: int, position, freq, axis, base, q_weight, k_weight, eps, adjacent) -> _Rotation:
    pairs = 0
    if freq is not None:
        _dev(freq, torch.float32, "freq")
        if freq.dim() != 1:
            raise TsltError("freq must be [rotary / 2]")
        pairs = freq.numel()
    axes, seq = MAX_AXES, 0                     # (without positions a token is at the same place on every axis)
    if position is not None:
        _dev(position, torch.int32, "position")
        if position.dim() != 3 or position.shape[0] not in (1, B) or position.shape[1] != n:
            raise TsltError(f"position must be [B or 1, {n}, axes], got {list(position.shape)}")
        axes, seq = position.shape[2], n * position.shape[2] if position.shape[0] > 1 else 0
    eps = -1.0 if eps is None else float(eps)
    if eps < 0 and (q_weight is not None or k_weight is not None):
        raise TsltError("weights belong to a norm: eps is needed")
    return _Rotation(_ptr(position), seq, _counted(base, "base", B), _ptr(freq), _counted(axis, "axis", pairs), axes, 2 * pairs, 1 if adjacent else 0, eps,
                     _optional(q_weight, "q_weight", torch.float32, (D,)), _optional(k_weight, "k_weight", torch.float32, (D,)))


def rotate(q: torch.Tensor, k: Optional[torch.Tensor], position: Optional[torch.Tensor], freq: Optional[torch.Tensor],
           axis: Optional[torch.Tensor] = None, base: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
           k_weight: Optional[torch.Tensor] = None, eps: Optional[float] = None, adjacent: bool = False, count: Optional[torch.Tensor] = None,
           out: Optional[dict] = None) -> dict:
    """tslt_rotate: q [B, n, heads_q, D] and k [B, n, heads, D] (or None; any strides that keep rows 16-byte aligned) normed where eps is given, with
    the weights q_weight, k_weight [D], and rotated by the angles (base [B] + position [B or 1, n, axes]) * freq [rotary / 2].  axis [rotary / 2]:
    which axis each pair goes by; position None: token i is at i.  Returns q, k and status [B]; out may hold q and k themselves."""
    lib = load()
    if _fast is not None and out is not None and q.is_cuda:
        code = _fast.rotate(q, k, position, freq, axis, base, q_weight, k_weight, eps, adjacent, count, out, *_current())
        if code is not None:
            if code:
                _check(code)
            return out
    _dev(q, name="q", contiguous=False)
    if q.dim() != 4:
        raise TsltError("q must be [B, n, heads_q, D]")
    B, n, heads_q, D = q.shape
    heads = 0
    if k is not None:
        if k.dim() != 4:
            raise TsltError("k must be [B, n, heads, D]")
        heads = k.shape[2]
    _fits("rotate", n, heads_q, heads, D)
    qr, kr = _rows_of(q, "q", q.shape, q.dtype), None if k is None else _rows_of(k, "k", (B, n, heads, D), q.dtype)
    how = _rotation(B, n, D, position, freq, axis, base, q_weight, k_weight, eps, adjacent)
    if out is None:
        out = {"q": torch.empty(B, n, heads_q, D, dtype=q.dtype, device=q.device),
               "k": None if k is None else torch.empty(B, n, heads, D, dtype=q.dtype, device=q.device),
               "status": torch.empty(B, dtype=torch.int32, device=q.device)}
    _check(lib.tslt_rotate(qr, kr, _dtype_code(q), B, n, heads_q, heads, D, how, _counted(count, "count", B),
                           _rows_of(_given(out, "q"), "out q", q.shape, q.dtype),
                           None if k is None else _rows_of(_given(out, "k"), "out k", k.shape, q.dtype),
                           _sized(out, "status", torch.int32, B, optional=True),
                           _here(out, ("q", "status") if k is None else ("q", "k", "status"), q=q, k=k, position=position, freq=freq, axis=axis, base=base,
                                 q_weight=q_weight, k_weight=k_weight, count=count)))
    return _told(out, "q", "status") if k is None else _told(out, "q", "k", "status")


def rotate_backward_workspace_bytes(B: int, n: int, heads_q: int, heads: int, head_dim: int) -> int:
    return int(load().tslt_rotate_backward_workspace_bytes(B, n, heads_q, heads, head_dim))


def rotate_backward(grad_q: torch.Tensor, grad_k: Optional[torch.Tensor], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                    position: Optional[torch.Tensor], freq: Optional[torch.Tensor], axis: Optional[torch.Tensor] = None,
                    base: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                    eps: Optional[float] = None, adjacent: bool = False, count: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                    workspace: Optional[torch.Tensor] = None) -> dict:
    """tslt_rotate_backward: the gradients q and k of rotate's inputs from those of its results, and of the weights that were given (q_weight, k_weight [D]
    fp32); q and k as rotate was given them (None without a norm).  Returns q, k, q_weight, k_weight and status [B]; out may hold grad_q and grad_k
    themselves."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and grad_q.is_cuda:
        code = _fast.rotate_backward(grad_q, grad_k, q, k, position, freq, axis, base, q_weight, k_weight, eps, adjacent, count, out, workspace, *_current())
        if code is not None:
            if code:
                _check(code)
            return out
    _dev(grad_q, name="grad_q", contiguous=False)
    if grad_q.dim() != 4:
        raise TsltError("grad_q must be [B, n, heads_q, D]")
    B, n, heads_q, D = grad_q.shape
    dtype, dev, heads = grad_q.dtype, grad_q.device, 0
    if grad_k is not None:
        if grad_k.dim() != 4:
            raise TsltError("grad_k must be [B, n, heads, D]")
        heads = grad_k.shape[2]
    _fits("rotate_backward", n, heads_q, heads, D)
    gq = _rows_of(grad_q, "grad_q", grad_q.shape, dtype)
    gk = None if grad_k is None else _rows_of(grad_k, "grad_k", (B, n, heads, D), dtype)
    qr = None if q is None or eps is None else _rows_of(q, "q", grad_q.shape, dtype)
    kr = None if k is None or eps is None or grad_k is None else _rows_of(k, "k", grad_k.shape, dtype)
    how = _rotation(B, n, D, position, freq, axis, base, q_weight, k_weight, eps, adjacent)
    if out is None:
        out = {"q": torch.empty(B, n, heads_q, D, dtype=dtype, device=dev),
               "k": None if grad_k is None else torch.empty(B, n, heads, D, dtype=dtype, device=dev),
               "q_weight": None if q_weight is None else torch.empty(D, dtype=torch.float32, device=dev),
               "k_weight": None if k_weight is None or grad_k is None else torch.empty(D, dtype=torch.float32, device=dev),
               "status": torch.empty(B, dtype=torch.int32, device=dev)}
    dq, dk = _sized(out, "q_weight", torch.float32, D, optional=True), _sized(out, "k_weight", torch.float32, D, optional=True)
    ws = workspace
    if ws is None and (dq or dk):
        ws = _workspace(rotate_backward_workspace_bytes(B, n, heads_q, heads, D), dev)
    _check(lib.tslt_rotate_backward(gq, gk, qr, kr, _dtype_code(grad_q), B, n, heads_q, heads, D, how, _counted(count, "count", B),
                                    _rows_of(_given(out, "q"), "out q", grad_q.shape, dtype),
                                    None if grad_k is None else _rows_of(_given(out, "k"), "out k", grad_k.shape, dtype), dq, dk,
                                    _sized(out, "status", torch.int32, B, optional=True), _ptr(ws), ws.numel() if ws is not None else 0,
                                    _here(out, ("q", "q_weight", "k_weight", "status") if grad_k is None else ("q", "k", "q_weight", "k_weight", "status"),
                                          grad_q=grad_q, grad_k=grad_k, q=q if qr else None, k=k if kr else None, position=position, freq=freq, axis=axis, base=base,
                                          q_weight=q_weight, k_weight=k_weight, count=count, workspace=ws)))
    return _told(out, *(("q",) if grad_k is None else ("q", "k")), "q_weight", "k_weight", "status")


def _logits(t: torch.Tensor, name: str):
    """[B, n, V], dense along V; strides of sequences and rows."""
    _dev(t, name=name, contiguous=False)
    if t.dim() != 3:
        raise TsltError(f"{name} must be [B, n, V]")
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise TsltError(f"{name} must be dense along the vocabulary")
    return tuple(s if n > 1 else 0 for s, n in zip(t.stride()[:2], t.shape[:2]))


def logprob_workspace_bytes(B: int, m: int, V: int, top: int) -> int:
    return int(load().tslt_logprob_workspace_bytes(B, m, V, top))


def logprob(logits: torch.Tensor, temperature: float, tokens: Optional[torch.Tensor] = None, top: int = 0, index: Optional[torch.Tensor] = None,
            count: Optional[torch.Tensor] = None, out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """tslt_logprob: logits [B, n, V] (any strides, dense along V); of the rows index [B, m] (None: all n), the first count [B] of them, the log probability
    of tokens [B, m] (-1: none), the entropy and the normaliser, and the `top` likeliest tokens with theirs.  Returns logp, entropy, lse, status [B, m] and, with
    top, top_idx and top_logp [B, m, top]; of a given out what it holds."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and logits.is_cuda:
        code = _fast.logprob(logits, temperature, tokens, top, index, count, out, workspace, *_current())
        if code is not None:
            if code:
                _check(code)
            return out
    seq, row = _logits(logits, "logits")
    B, n, V = logits.shape
    top = int(top)
    if index is not None and index.dim() != 2:
        raise TsltError("index must be [B, m]")
    m = n if index is None else index.shape[1]
    if not -(1 << 31) <= top < 1 << 31:
        raise TsltError(f"top must be 0 to {MAX_TOP} (got {top})")
    _fits("logprob", n, m)
    dev = logits.device
    if out is None:
        out = {name: torch.empty(B, m, dtype=torch.float32, device=dev) for name in ("logp", "entropy", "lse")}
        out["status"] = torch.empty(B, m, dtype=torch.int32, device=dev)
        if top > 0:
            out["top_idx"] = torch.empty(B, m, top, dtype=torch.int32, device=dev)
            out["top_logp"] = torch.empty(B, m, top, dtype=torch.float32, device=dev)
    ws = workspace
    if ws is None:
        ws = _workspace(logprob_workspace_bytes(B, m, V, top) if B else 0, dev)
    results = [_sized(out, name, torch.float32, B * m, optional=True) for name in ("logp", "entropy", "lse")]
    _check(lib.tslt_logprob(logits.data_ptr(), _dtype_code(logits), B, n, V, seq, row, float(temperature), _counted(index, "index", B * m), m,
                            _counted(count, "count", B), _counted(tokens, "tokens", B * m), top, *results,
                            _sized(out, "top_idx", torch.int32, B * m * top) if top > 0 else None,
                            _sized(out, "top_logp", torch.float32, B * m * top) if top > 0 else None,
                            _sized(out, "status", torch.int32, B * m, optional=True), _ptr(ws), ws.numel() if ws is not None else 0,
                            _here(out, ("logp", "entropy", "lse", "status", "top_idx", "top_logp")[:6 if top > 0 else 4], logits=logits, tokens=tokens, index=index,
                                  count=count, workspace=ws)))
    return _told(out, "logp", "entropy", "lse", "status", *(("top_idx", "top_logp") if top > 0 else ()))


def logprob_backward(logits: torch.Tensor, temperature: float, tokens: Optional[torch.Tensor], lse: torch.Tensor, entropy: Optional[torch.Tensor] = None,
                     grad_logp: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None, grad_lse: Optional[torch.Tensor] = None,
                     top_idx: Optional[torch.Tensor] = None, grad_top: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                     out: Optional[dict] = None) -> dict:
    """tslt_logprob_backward: the gradient `logits` [B, n, V] of what logprob was given, without an index, from those of its results (None: 0); tokens, lse,
    entropy, top_idx as it was given them and gave them.  out may hold the logits themselves."""
    lib = load()
    if _fast is not None and out is not None and logits.is_cuda:
        code = _fast.logprob_backward(logits, temperature, tokens, lse, entropy, grad_logp, grad_entropy, grad_lse, top_idx, grad_top, count, out, *_current())
        if code is not None:
            if code:
                _check(code)
            return out
    seq, row = _logits(logits, "logits")
    B, n, V = logits.shape
    top = 0
    if grad_top is not None:
        if grad_top.dim() != 3:
            raise TsltError("grad_top must be [B, n, top]")
        top = grad_top.shape[2]
        if not 1 <= top <= MAX_TOP:
            raise TsltError(f"grad_top must be [B, n, top] with top from 1 to {MAX_TOP}")
    _fits("logprob_backward", n)
    if out is None:
        out = {"logits": torch.empty(B, n, V, dtype=logits.dtype, device=logits.device)}
    made = _given(out, "logits")
    out_seq, out_row = _logits(made, "out logits")
    if made.shape != logits.shape or made.dtype != logits.dtype:
        raise TsltError(f"out logits must be {list(logits.shape)} of {logits.dtype}")
    if lse is None:
        raise TsltError("lse is needed")

    def given(t, name):
        return _optional(t, name, torch.float32, (B, n))
    _check(lib.tslt_logprob_backward(logits.data_ptr(), _dtype_code(logits), B, n, V, seq, row, float(temperature), _counted(count, "count", B),
                                     _counted(tokens, "tokens", B * n), given(lse, "lse"), given(entropy, "entropy"),
                                     _counted(top_idx, "top_idx", B * n * top) if top else None, top, given(grad_logp, "grad_logp"),
                                     given(grad_entropy, "grad_entropy"), given(grad_lse, "grad_lse"),
                                     _optional(grad_top, "grad_top", torch.float32, (B, n, top)), made.data_ptr(), out_seq, out_row,
                                     _here(out, ("logits",), logits=logits, tokens=tokens, lse=lse, entropy=entropy, grad_logp=grad_logp, grad_entropy=grad_entropy,
                                           grad_lse=grad_lse, top_idx=top_idx if top else None, grad_top=grad_top, count=count)))
    return _told(out, "logits")


def _token_rows(t: torch.Tensor, name: str, shape, dtype) -> _Rows:
    """[B, n, width], dense along the width."""
    _dev(t, dtype, name, contiguous=False)
    if tuple(t.shape) != tuple(shape):
        raise TsltError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise TsltError(f"{name} must be dense along its last dimension")
    seq, token = (s if n > 1 else 0 for s, n in zip(t.stride()[:2], t.shape[:2]))
    return _Rows(t.data_ptr(), seq, token, 0)


def adapt_workspace_bytes(B: int, n: int, K: int, N: int, R: int) -> int:
    return int(load().tslt_adapt_workspace_bytes(B, n, K, N, R))


def adapt(x: torch.Tensor, base: torch.Tensor, a: torch.Tensor, b: torch.Tensor, adapter: torch.Tensor, scale: Optional[torch.Tensor] = None,
          rank: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None, out: Optional[dict] = None,
          workspace: Optional[torch.Tensor] = None) -> dict:
    """tslt_adapt: to base [B, n, N], what a projection gave for x [B, n, K], scale (x a^T) b^T of each sequence's adapter [B] (-1: none), of a
    [adapters, R, K] and b [adapters, N, R], R a multiple of 16, the first rank [adapters] of which count; scale [adapters] fp32.  x: any strides that keep rows
    16-byte aligned; base and out: any.  Returns out [B, n, N] and status [B]; out may hold base itself."""
    lib = load()
    if _fast is not None and out is not None and workspace is not None and x.is_cuda:
        code = _fast.adapt(x, base, a, b, adapter, scale, rank, count, out, workspace, *_current())
        if code is not None:
            if code:
                _check(code)
            return out
    _dev(x, name="x", contiguous=False); _dev(base, name="base", contiguous=False)
    if x.dim() != 3 or base.dim() != 3 or a.dim() != 3 or b.dim() != 3:
        raise TsltError("adapt: x must be [B, n, K], base [B, n, N], a [adapters, R, K], b [adapters, N, R]")
    B, n, K = x.shape
    N, adapters, R = base.shape[2], a.shape[0], a.shape[1]
    _fits("adapt", n, K, N, R)
    xr, br = _token_rows(x, "x", x.shape, x.dtype), _token_rows(base, "base", (B, n, N), x.dtype)
    if out is None:
        out = {"out": torch.empty(B, n, N, dtype=x.dtype, device=x.device), "status": torch.empty(B, dtype=torch.int32, device=x.device)}
    ws = workspace if workspace is not None else _workspace(adapt_workspace_bytes(B, n, K, N, R) if B else 0, x.device)
    _check(lib.tslt_adapt(xr, K, br, _token_rows(_given(out, "out"), "out", (B, n, N), x.dtype), N, _dtype_code(x), B, n,
                          _optional(a, "a", x.dtype, (adapters, R, K)), _optional(b, "b", x.dtype, (adapters, N, R)), adapters, R,
                          _counted(adapter, "adapter", B), _optional(scale, "scale", torch.float32, (adapters,)), _counted(rank, "rank", adapters),
                          _counted(count, "count", B), _sized(out, "status", torch.int32, B, optional=True), _ptr(ws), ws.numel() if ws is not None else 0,
                          _here(out, ("out", "status"), x=x, base=base, a=a, b=b, adapter=adapter, scale=scale, rank=rank, count=count, workspace=ws)))
    return _told(out, "out", "status")
