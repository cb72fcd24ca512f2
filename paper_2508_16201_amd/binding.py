"""ctypes binding of ``libspecvlm.so``: argument marshalling only.

Every function has the name of the C entry point it calls (``include/specvlm.h``)
and takes torch tensors that live on the GPU; torch provides device memory and
the current stream, nothing else.  There is no CPU fallback: if the HIP
library is missing or a call fails, an exception is raised.

The plain calls of the short functions are marshalled by ``_calls.so``
(``csrc/calls.cpp``); what it does not take goes through the code here, which
is also what decides what is refused.
"""
from __future__ import annotations

import ctypes as C
import os
import warnings
from typing import Optional, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# SPECVLM_LIB names another build of the same library (the host-sanitized one the CPU tests make)
LIB_PATH = os.environ.get("SPECVLM_LIB") or os.path.join(_HERE, "libspecvlm.so")
_lib = None
_calls = None

EXPORTS = (
    "specvlm_status_string", "specvlm_version",
    "specvlm_score_workspace_bytes", "specvlm_score",
    "specvlm_score_layers_workspace_bytes", "specvlm_score_layers",
    "specvlm_select_workspace_bytes", "specvlm_select",
    "specvlm_top_p_count_workspace_bytes", "specvlm_top_p_count",
    "specvlm_gather_kv",
    "specvlm_decode_attn_workspace_bytes", "specvlm_decode_attn",
    "specvlm_decode_attn_static_scratch_bytes", "specvlm_decode_attn_static",
    "specvlm_accept_workspace_bytes", "specvlm_accept",
    "specvlm_tree_attn", "specvlm_accept_tree_workspace_bytes", "specvlm_accept_tree",
    "specvlm_baseline_count", "specvlm_baseline_workspace_bytes", "specvlm_baseline_keep",
    "specvlm_probe_read",
    "specvlm_paged_attn_workspace_bytes", "specvlm_paged_attn",
    "specvlm_rope_turns", "specvlm_rope_append",
    "specvlm_pages_assign_workspace_bytes", "specvlm_pages_assign", "specvlm_pages_copy",
    "specvlm_pages_shared_workspace_bytes", "specvlm_pages_shared", "specvlm_shared_attn_workspace_bytes", "specvlm_shared_attn",
    "specvlm_cross_attn_workspace_bytes", "specvlm_cross_attn",
)


class _RopeSpec(C.Structure):
    _fields_ = [("kind", C.c_int), ("base", C.c_double), ("factor", C.c_double), ("original_len", C.c_double),
                ("beta_fast", C.c_double), ("beta_slow", C.c_double)]


class SpecVLMError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {status_string(status)} ({status})")


def lib() -> C.CDLL:
    """Load the HIP library (built by ``paper_2508_16201_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2508_16201_amd.build` "
                "(there is no fallback path)")
        l = C.CDLL(LIB_PATH)
        l.specvlm_status_string.restype = C.c_char_p
        l.specvlm_status_string.argtypes = [C.c_int]
        l.specvlm_version.restype = C.c_int
        for name in EXPORTS:
            if name.endswith("_workspace_bytes") or name.endswith("_scratch_bytes"):
                getattr(l, name).restype = C.c_size_t
        i64, i32, f32, vp, sz = C.c_int64, C.c_int, C.c_float, C.c_void_p, C.c_size_t
        l.specvlm_score_workspace_bytes.argtypes = [i32] * 8
        l.specvlm_score.argtypes = [vp, i64, i64, vp, i64, i64, vp, vp, vp, i32,
                                    i32, i32, i32, i32, i32, i32, i32, i32, f32,
                                    i32, vp, f32, vp, vp, sz, vp]
        l.specvlm_score_layers_workspace_bytes.argtypes = [i32] * 9
        l.specvlm_score_layers.argtypes = [vp, i64, i64, i64, vp, i64, i64, i64, i32, vp, vp, vp, i32,
                                           i32, i32, i32, i32, i32, i32, i32, i32, f32,
                                           i32, vp, i64, f32, vp, vp, sz, vp]
        l.specvlm_select_workspace_bytes.argtypes = [i32, i32]
        l.specvlm_select.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        l.specvlm_top_p_count_workspace_bytes.argtypes = [i32, i32]
        l.specvlm_top_p_count.argtypes = [vp, vp, i32, i32, f32, vp, vp, vp, sz, vp]
        l.specvlm_gather_kv.argtypes = [vp, vp, i64, i64, i64, vp, vp, i64, i64, i64,
                                        i32, i32, i32, i32, vp, i32, vp, vp, vp, i32, vp, i32, i32, vp]
        l.specvlm_decode_attn_workspace_bytes.argtypes = [i32] * 7
        l.specvlm_decode_attn.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i32, i32,
                                          i32, i32, i32, f32, vp, vp, i32, vp, sz, vp]
        l.specvlm_decode_attn_static_scratch_bytes.argtypes = []
        l.specvlm_decode_attn_static.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i32, i32,
                                                 i32, i32, i32, f32, vp, vp, i32, vp]
        l.specvlm_tree_attn.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i32, i32,
                                        i32, i32, i32, f32, vp, vp, vp, i32, vp, sz, vp]
        l.specvlm_accept_tree_workspace_bytes.argtypes = [i32] * 3
        l.specvlm_accept_tree.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        l.specvlm_baseline_count.argtypes = [i32] * 8
        l.specvlm_baseline_count.restype = C.c_int
        l.specvlm_baseline_workspace_bytes.argtypes = [i32] * 2
        l.specvlm_baseline_keep.argtypes = [i32] * 8 + [C.c_uint64, vp, vp, sz, vp]
        l.specvlm_baseline_keep.restype = C.c_int
        l.specvlm_probe_read.argtypes = [vp, sz, vp, sz, vp, vp]
        l.specvlm_probe_read.restype = C.c_int
        l.specvlm_accept_workspace_bytes.argtypes = [i32] * 4
        l.specvlm_accept.argtypes = [vp, vp, vp, vp, i32, i32, i32, f32, vp, vp, vp, sz, vp]
        for name in ("specvlm_score", "specvlm_select", "specvlm_top_p_count", "specvlm_gather_kv",
                     "specvlm_decode_attn", "specvlm_decode_attn_static", "specvlm_accept", "specvlm_tree_attn",
                     "specvlm_accept_tree", "specvlm_paged_attn", "specvlm_rope_turns", "specvlm_rope_append", "specvlm_pages_assign",
                     "specvlm_pages_copy", "specvlm_pages_shared", "specvlm_shared_attn", "specvlm_cross_attn"):
            getattr(l, name).restype = C.c_int
        l.specvlm_paged_attn_workspace_bytes.argtypes = [i32] * 5
        l.specvlm_paged_attn.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, i32, i32, vp, i64, i32, vp, vp, i32, i32, i32,
                                         i32, i32, i32, f32, i32, i32, vp, vp, vp, vp, sz, vp]
        l.specvlm_rope_turns.argtypes = [i32, C.POINTER(_RopeSpec), vp]
        l.specvlm_rope_append.argtypes = [vp, i64, i64, vp, i64, i64, vp, vp, i64, i64, vp, vp, i64, i64, i64, i32, i32, vp, i64, i32,
                                          vp, vp, i32, i32, vp, vp, i32, i32, f32, i32, i32, i32, vp]
        l.specvlm_pages_assign_workspace_bytes.argtypes = [i32] * 2
        l.specvlm_pages_assign.argtypes = [vp, i64, i32, i32, vp, vp, vp, i32, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        l.specvlm_pages_copy.argtypes = [vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, i32, i32, vp, vp, i64, i64, i64, i64, i32, i32,
                                         vp, i64, i32, i32, i32, vp, i32, vp, vp, vp, vp, i64, vp, i32, i32, vp]
        l.specvlm_pages_shared_workspace_bytes.argtypes = [i32]
        l.specvlm_pages_shared.argtypes = [vp, i64, i32, i32, i32, vp, vp, i32, i32, i32, vp, vp, sz, vp]
        l.specvlm_shared_attn_workspace_bytes.argtypes = [i32] * 5
        l.specvlm_shared_attn.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, i32, i32, vp, i64, i32, vp, vp, vp, i32, i32, i32, i32,
                                          i32, i32, i32, f32, vp, vp, vp, vp, sz, vp]
        l.specvlm_cross_attn_workspace_bytes.argtypes = [i32] * 5
        l.specvlm_cross_attn.argtypes = [vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp, vp, sz, vp]
        _lib = l
    return _lib


class _NoCalls:
    """Stands in for _calls where that is not to be had: every call is left to the general code."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_calls():
    """The native marshalling, connected to the library; the first call of a short function asks for it.  Without it (a build without it,
    or for another torch) the general code makes every call, in more host time."""
    global _calls
    if _raw_stream is None:
        _calls = _NoCalls()
    else:
        try:
            from . import _calls as native
            compiled_for = getattr(native, "torch_version", None)             # (an older _calls.so does not say)
            if compiled_for != torch.__version__.split("+")[0]:             # (it reads torch's objects in place)
                raise ImportError(f"compiled for torch {compiled_for}, this is {torch.__version__}")
            native.connect(version(), {name: C.cast(getattr(lib(), name), C.c_void_p).value for name in native.functions})
            _calls = native
        except ImportError as e:
            warnings.warn(f"{os.path.join(_HERE, '_calls.so')} is missing or does not fit this torch, so calls take longer on the host (build it "
                          f"with `python -m paper_2508_16201_amd.build`): {e}", RuntimeWarning, stacklevel=3)
            _calls = _NoCalls()
    return _calls


def status_string(status: int) -> str:
    return lib().specvlm_status_string(int(status)).decode()


def version() -> int:
    return lib().specvlm_version()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors must live on the GPU")
    return t.data_ptr()          # (an int: the argtypes make the pointer of it)


# (None on a torch without GPU support, which can still import this module: a call there finds no tensor on a GPU)
_raw_stream, _current_device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream() -> int:
    """The hipStream_t of torch's current stream on the current device, without a Stream object around it: what is
    not marshalled by _calls.so takes its host time here, and every call asks."""
    return _raw_stream(_current_device())


def _check(fn: str, rc: int):
    if rc != 0:
        raise SpecVLMError(fn, rc)


def _contiguous_ptrs(what: str, *tensors: Optional[torch.Tensor]):
    """The device addresses of tensors (None stays None) that have to be contiguous."""
    for t in tensors:
        if t is not None and not t.is_contiguous():
            raise ValueError(what + " inputs must be contiguous")
    return [None if t is None else _ptr(t) for t in tensors]


def new_workspace(nbytes: int, device=None) -> torch.Tensor:
    """A 256-byte aligned device buffer (torch's caching allocator aligns to 512)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device or "cuda")


def _thd(t: torch.Tensor) -> Tuple[int, int]:
    """(token stride, head stride) in elements of a [tokens, heads, d] view."""
    st = t.stride()
    if len(st) != 3 or st[2] != 1:
        raise ValueError("expected a [tokens, heads, d] view with contiguous d")
    return st[0], st[1]


# --------------------------------------------------------------------------- score
def score_workspace_bytes(n_text, n_keys, n_video, n_q_heads, n_kv_heads, head_dim,
                          have_row_lse=False, batch=1) -> int:
    return lib().specvlm_score_workspace_bytes(batch, n_text, n_keys, n_video, n_q_heads, n_kv_heads,
                                               head_dim, int(have_row_lse))


def score_layers_workspace_bytes(n_layers, n_text, n_keys, n_video, n_q_heads, n_kv_heads, head_dim,
                                 have_row_lse=False, batch=1) -> int:
    return lib().specvlm_score_layers_workspace_bytes(n_layers, batch, n_text, n_keys, n_video, n_q_heads,
                                                      n_kv_heads, head_dim, int(have_row_lse))


def _dev_i32(a, device):
    """Device int32 prefix offsets; a host sequence is uploaded (and its maxima returned)."""
    if isinstance(a, torch.Tensor):
        return a, None
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return torch.from_numpy(arr).to(device), arr


def _batch_sizes(device, cu_text, cu_keys, cu_video, n_text, n_keys, n_video, max_n_text, max_n_keys,
                 max_n_video, total_video):
    """(batch, device offset arrays, maxima, total video tokens) of a score call; one request without offsets."""
    if cu_text is None:
        return 1, (None, None, None), n_text, n_keys, n_video, n_video
    dev = [_dev_i32(a, device) for a in (cu_text, cu_keys, cu_video)]
    ptrs = tuple(x[0] for x in dev)
    batch = ptrs[0].numel() - 1
    hosts = [x[1] for x in dev]
    if all(h is not None for h in hosts):
        n_text = int(np.diff(hosts[0]).max()) if batch else 0
        n_keys = int(np.diff(hosts[1]).max()) if batch else 0
        n_video = int(np.diff(hosts[2]).max()) if batch else 0
        total_video = int(hosts[2][-1])
    else:
        if None in (max_n_text, max_n_keys, max_n_video, total_video):
            raise ValueError("device cu arrays need max_n_text, max_n_keys, max_n_video and total_video")
        n_text, n_keys, n_video = max_n_text, max_n_keys, max_n_video
    return batch, ptrs, n_text, n_keys, n_video, total_video


def score_layers(q_text: torch.Tensor, k_cache: torch.Tensor, video_start: int, n_video: int,
                 text_pos0: int, softmax_scale: float, *, norm_mode: int = 0,
                 row_lse: Optional[torch.Tensor] = None, beta: float = 0.0,
                 scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 cu_text=None, cu_keys=None, cu_video=None, max_n_text: Optional[int] = None,
                 max_n_keys: Optional[int] = None, max_n_video: Optional[int] = None,
                 total_video: Optional[int] = None) -> torch.Tensor:
    """q_text [layers,L,H_q,d] bf16, k_cache [layers,n_keys,H_kv,d] bf16 (any layer / token / head strides with
    contiguous d), row_lse [layers,L,H_q] fp32 or None -> scores fp32 [n_video] summed over the layers.
    A batch is given as for score(): requests concatenated along the token axis of every layer."""
    n_layers, n_text, hq, d = q_text.shape
    _, n_keys, hkv, _ = k_cache.shape
    if k_cache.shape[0] != n_layers:
        raise ValueError("q_text and k_cache must have the same number of layers")
    if q_text.stride(3) != 1 or k_cache.stride(3) != 1:
        raise ValueError("the head dimension must be contiguous")
    if row_lse is not None and (row_lse.shape != (n_layers, n_text, hq) or not row_lse[0].is_contiguous()):
        raise ValueError("row_lse must be [layers, n_text, H_q] with contiguous layers")
    batch, ptrs, n_text, n_keys, n_video, total_video = _batch_sizes(
        q_text.device, cu_text, cu_keys, cu_video, n_text, n_keys, n_video, max_n_text, max_n_keys, max_n_video,
        total_video)
    if scores is None:
        scores = torch.empty(total_video, dtype=torch.float32, device=q_text.device)
        if beta != 0.0:
            raise ValueError("beta != 0 needs an existing scores tensor")
    if workspace is None:
        workspace = new_workspace(score_layers_workspace_bytes(n_layers, n_text, n_keys, n_video, hq, hkv, d,
                                                               row_lse is not None, batch=max(batch, 1)), q_text.device)
    qs, ks = q_text.stride(), k_cache.stride()
    rc = lib().specvlm_score_layers(_ptr(q_text), qs[0], qs[1], qs[2], _ptr(k_cache), ks[0], ks[1], ks[2], n_layers,
                                    _ptr(ptrs[0]), _ptr(ptrs[1]), _ptr(ptrs[2]), batch, n_text, n_keys, video_start,
                                    n_video, text_pos0, hq, hkv, d,
                                    float(softmax_scale), norm_mode, _ptr(row_lse),
                                    0 if row_lse is None else row_lse.stride(0), float(beta), _ptr(scores),
                                    _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_score_layers", rc)
    return scores


def score(q_text: torch.Tensor, k_cache: torch.Tensor, video_start: int, n_video: int,
          text_pos0: int, softmax_scale: float, *, norm_mode: int = 0,
          row_lse: Optional[torch.Tensor] = None, beta: float = 0.0,
          scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
          cu_text=None, cu_keys=None, cu_video=None, max_n_text: Optional[int] = None,
          max_n_keys: Optional[int] = None, max_n_video: Optional[int] = None,
          total_video: Optional[int] = None) -> torch.Tensor:
    """q_text [L,H_q,d] bf16, k_cache [n_keys,H_kv,d] bf16 -> scores fp32 [n_video].

    A batch: requests concatenated along the token axis, cu_text / cu_keys / cu_video = int32 prefix
    offsets [batch+1] on the device (host sequences are uploaded); n_video is then ignored and
    text_pos0 = -1 places every request's text queries on its last keys.  With device tensors the
    maxima over the batch and the total number of video tokens must be given."""
    if cu_text is None:
        got = (_calls or _load_calls()).score(q_text, k_cache, video_start, n_video, text_pos0, softmax_scale, norm_mode, row_lse, beta, scores,
                                              workspace)
        if got is not None:
            if type(got) is int:
                _check("specvlm_score", got)
            return got
    n_text, hq, d = q_text.shape
    n_keys, hkv, _ = k_cache.shape
    if cu_text is None:
        batch, p_text, p_keys, p_video, total_video = 1, None, None, None, n_video
    else:
        batch, cu, n_text, n_keys, n_video, total_video = _batch_sizes(
            q_text.device, cu_text, cu_keys, cu_video, n_text, n_keys, n_video, max_n_text, max_n_keys, max_n_video,
            total_video)
        p_text, p_keys, p_video = _ptr(cu[0]), _ptr(cu[1]), _ptr(cu[2])
    if scores is None:
        if beta != 0.0:
            raise ValueError("beta != 0 needs an existing scores tensor")
        scores = q_text.new_empty(total_video, dtype=torch.float32)
    if workspace is None:
        workspace = new_workspace(score_workspace_bytes(n_text, n_keys, n_video, hq, hkv, d, row_lse is not None,
                                                        batch=max(batch, 1)), q_text.device)
    (q_tok, q_head, q_one), (k_tok, k_head, k_one) = q_text.stride(), k_cache.stride()
    if q_one != 1 or k_one != 1:
        raise ValueError("expected a [tokens, heads, d] view with contiguous d")
    rc = lib().specvlm_score(_ptr(q_text), q_tok, q_head, _ptr(k_cache), k_tok, k_head, p_text, p_keys, p_video,
                             batch, n_text, n_keys, video_start, n_video, text_pos0, hq, hkv, d, softmax_scale, norm_mode,
                             None if row_lse is None else _ptr(row_lse), beta, _ptr(scores), _ptr(workspace),
                             workspace.numel(), _raw_stream(_current_device()))
    if rc:
        _check("specvlm_score", rc)
    return scores


# -------------------------------------------------------------------------- select
def select(scores: torch.Tensor, k_top: torch.Tensor, keep_budget: torch.Tensor, total_keep: int,
           *, cu_video: Optional[torch.Tensor] = None, cu_keep: Optional[torch.Tensor] = None,
           max_n_video: Optional[int] = None, want_flags: bool = True, want_status: bool = False,
           keep_idx: Optional[torch.Tensor] = None):
    """scores fp32 [sum V_b]; k_top/keep_budget device int32 [batch] -> keep_idx int32 [total_keep]."""
    if not want_status:
        got = (_calls or _load_calls()).select(scores, k_top, keep_budget, total_keep, cu_video, cu_keep, max_n_video, want_flags, keep_idx)
        if got is not None:
            if type(got) is int:
                _check("specvlm_select", got)
            return got
    batch = k_top.numel()
    if max_n_video is None:
        if cu_video is not None:
            raise ValueError("max_n_video is required with cu_video")
        max_n_video = scores.numel()
    dev = scores.device
    if keep_idx is None:
        keep_idx = torch.empty(total_keep, dtype=torch.int32, device=dev)
    flags = torch.empty(total_keep, dtype=torch.uint8, device=dev) if want_flags else None
    status = torch.empty(batch, dtype=torch.int32, device=dev) if want_status else None
    rc = lib().specvlm_select(_ptr(scores), _ptr(cu_video), _ptr(k_top), _ptr(keep_budget),
                              _ptr(cu_keep), batch, max_n_video, total_keep, _ptr(keep_idx),
                              _ptr(flags), _ptr(status), None, 0, _stream())
    _check("specvlm_select", rc)
    out = (keep_idx, flags)
    return out + (status,) if want_status else out


def top_p_count(scores: torch.Tensor, lam: float, *, cu_video: Optional[torch.Tensor] = None,
                max_n_video: Optional[int] = None, max_count: Optional[torch.Tensor] = None,
                count: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scores fp32 [sum V_b] -> count int32 [batch]: Eq. 6's retention size per request."""
    got = (_calls or _load_calls()).top_p_count(scores, lam, cu_video, max_n_video, max_count, count)
    if got is not None:
        if type(got) is int:
            _check("specvlm_top_p_count", got)
        return got
    batch = 1 if cu_video is None else cu_video.numel() - 1
    if max_n_video is None:
        if cu_video is not None:
            raise ValueError("max_n_video is required with cu_video")
        max_n_video = scores.numel()
    if count is None:
        count = torch.empty(batch, dtype=torch.int32, device=scores.device)
    rc = lib().specvlm_top_p_count(_ptr(scores), _ptr(cu_video), batch, max_n_video, float(lam),
                                   _ptr(max_count), _ptr(count), None, 0, _stream())
    _check("specvlm_top_p_count", rc)
    return count


# ----------------------------------------------------------------------- gather_kv
def gather_kv(k_src: torch.Tensor, v_src: Optional[torch.Tensor], video_start: int, n_video: int,
              keep_idx: torch.Tensor, k_dst: Optional[torch.Tensor] = None,
              v_dst: Optional[torch.Tensor] = None, *, cu_keys: Optional[torch.Tensor] = None,
              cu_video: Optional[torch.Tensor] = None, cu_keep: Optional[torch.Tensor] = None,
              want_status: bool = False):
    """k_src/v_src bf16 [layers, n_keys, H_kv, d] (any layer/token/head strides, d contiguous).

    A batch: requests concatenated along the token axis, cu_keys / cu_video / cu_keep device int32
    [batch+1]; n_video is then the total over the batch."""
    if not want_status:
        got = (_calls or _load_calls()).gather_kv(k_src, v_src, video_start, n_video, keep_idx, k_dst, v_dst, cu_keys, cu_video, cu_keep)
        if got is not None:
            if type(got) is int:
                _check("specvlm_gather_kv", got)
            return got
    if k_src.dim() != 4 or k_src.stride(3) != 1:
        raise ValueError("expected [layers, tokens, heads, d] with contiguous d")
    n_layers, n_keys, hkv, d = k_src.shape
    n_keep = keep_idx.numel()
    n_dst = n_keys - n_video + n_keep
    batch = 1 if cu_keys is None else cu_keys.numel() - 1
    if k_dst is None:
        k_dst = torch.empty((n_layers, n_dst, hkv, d), dtype=k_src.dtype, device=k_src.device)
    if v_src is not None and v_dst is None:
        v_dst = torch.empty_like(k_dst)
    if v_src is not None and v_src.stride() != k_src.stride():
        raise ValueError("K and V must share strides")
    if v_dst is not None and v_dst.stride() != k_dst.stride():
        raise ValueError("K and V destinations must share strides")
    status = torch.empty(1, dtype=torch.int32, device=k_src.device) if want_status else None
    src, dst = k_src.stride(), k_dst.stride()
    rc = lib().specvlm_gather_kv(_ptr(k_src), _ptr(v_src), src[0], src[1], src[2], _ptr(k_dst), _ptr(v_dst),
                                 dst[0], dst[1], dst[2], n_layers, n_keys, video_start,
                                 n_video, _ptr(keep_idx), n_keep, _ptr(cu_keys), _ptr(cu_video),
                                 _ptr(cu_keep), batch, _ptr(status), hkv, d, _stream())
    _check("specvlm_gather_kv", rc)
    return (k_dst, v_dst, status) if want_status else (k_dst, v_dst)


# --------------------------------------------------------------------- decode_attn
def decode_attn_workspace_bytes(batch, q_len, kv_len, n_q_heads, n_kv_heads, head_dim,
                                num_splits=0) -> int:
    return lib().specvlm_decode_attn_workspace_bytes(batch, q_len, kv_len, n_q_heads, n_kv_heads,
                                                     head_dim, num_splits)


def decode_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, softmax_scale: float, *,
                cu_q: Optional[torch.Tensor] = None, cu_kv: Optional[torch.Tensor] = None,
                max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
                out: Optional[torch.Tensor] = None, want_lse: bool = False, num_splits: int = 0,
                workspace: Optional[torch.Tensor] = None, ancestor_mask: Optional[torch.Tensor] = None):
    """q [sum q_len,H_q,d], k/v [sum kv_len,H_kv,d] bf16 views -> out like q (and lse fp32)."""
    got = (_calls or _load_calls()).decode_attn(q, k, v, softmax_scale, cu_q, cu_kv, max_q_len, max_kv_len, out, want_lse, num_splits, workspace,
                                                ancestor_mask)
    if got is not None:
        if type(got) is int:
            _check("specvlm_decode_attn" if ancestor_mask is None else "specvlm_tree_attn", got)
        return got
    tq, hq, d = q.shape
    tk, hkv, _ = k.shape
    if cu_q is None:
        batch, q_len, kv_len = 1, tq, tk
    else:
        batch = cu_q.numel() - 1
        if max_q_len is None or max_kv_len is None:
            raise ValueError("max_q_len and max_kv_len are required with cu_q/cu_kv")
        q_len, kv_len = max_q_len, max_kv_len
    if out is None:
        out = torch.empty_like(q)
    if out.stride() != q.stride():
        raise ValueError("out must share q's strides")
    if v.stride() != k.stride():
        raise ValueError("K and V must share strides")
    lse = torch.empty((tq, hq), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        workspace = new_workspace(decode_attn_workspace_bytes(batch, q_len, kv_len, hq, hkv, d, num_splits), q.device)
    qs, ks = _thd(q), _thd(k)
    if ancestor_mask is None:
        rc = lib().specvlm_decode_attn(_ptr(q), qs[0], qs[1], _ptr(k), _ptr(v), ks[0], ks[1],
                                       _ptr(cu_q), _ptr(cu_kv), batch, q_len, kv_len, hq, hkv, d,
                                       float(softmax_scale), _ptr(out), _ptr(lse), num_splits,
                                       _ptr(workspace), workspace.numel(), _stream())
        _check("specvlm_decode_attn", rc)
    else:
        rc = lib().specvlm_tree_attn(_ptr(q), qs[0], qs[1], _ptr(k), _ptr(v), ks[0], ks[1],
                                     _ptr(cu_q), _ptr(cu_kv), batch, q_len, kv_len, hq, hkv, d,
                                     float(softmax_scale), _ptr(ancestor_mask), _ptr(out), _ptr(lse),
                                     num_splits, _ptr(workspace), workspace.numel(), _stream())
        _check("specvlm_tree_attn", rc)
    return (out, lse) if want_lse else out


def decode_attn_static(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, softmax_scale: float, *,
                       out: torch.Tensor, lse: Optional[torch.Tensor] = None,
                       cu_q: Optional[torch.Tensor] = None, cu_kv: Optional[torch.Tensor] = None,
                       max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
                       num_splits: int = 0) -> torch.Tensor:
    """decode_attn through the entry point that takes no workspace; the caller supplies every output
    (this wrapper allocates nothing either)."""
    tq, hq, d = q.shape
    tk, hkv, _ = k.shape
    if cu_q is None:
        batch, q_len, kv_len = 1, tq, tk
    else:
        batch = cu_q.numel() - 1
        if max_q_len is None or max_kv_len is None:
            raise ValueError("max_q_len and max_kv_len are required with cu_q/cu_kv")
        q_len, kv_len = max_q_len, max_kv_len
    if out.stride() != q.stride() or v.stride() != k.stride():
        raise ValueError("out must share q's strides, V must share K's")
    qs, ks = _thd(q), _thd(k)
    rc = lib().specvlm_decode_attn_static(_ptr(q), qs[0], qs[1], _ptr(k), _ptr(v), ks[0], ks[1],
                                          _ptr(cu_q), _ptr(cu_kv), batch, q_len, kv_len, hq, hkv, d,
                                          float(softmax_scale), _ptr(out), _ptr(lse), num_splits, _stream())
    _check("specvlm_decode_attn_static", rc)
    return out


def tree_attn(q, k, v, softmax_scale, ancestor_mask: torch.Tensor, **kw):
    """decode_attn for a block of draft-tree nodes; ancestor_mask int64/uint64 [sum q_len]."""
    return decode_attn(q, k, v, softmax_scale, ancestor_mask=ancestor_mask, **kw)


# ------------------------------------------------------------------- paged caches
def _on_device(**tensors: Optional[torch.Tensor]):
    """Tensors of one call lie on the current device, whose stream the call goes to."""
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.device.index != _current_device()):
            raise ValueError(f"{name} must live on the current GPU")


def _typed(dtype: torch.dtype, **tensors: Optional[torch.Tensor]):
    for name, t in tensors.items():
        if t is not None and t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, not {t.dtype}")


def _int32s(n: Optional[int], **tensors: Optional[torch.Tensor]):
    """Contiguous int32 vectors, of n entries."""
    _typed(torch.int32, **tensors)
    for name, t in tensors.items():
        if t is not None and (t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n)):
            raise ValueError(f"{name} must be a contiguous vector" + ("" if n is None else f" of {n} entries"))


def _table(name: str, t: torch.Tensor):
    """(row stride, entries a row) of a page table."""
    _typed(torch.int32, **{name: t})
    if t.dim() != 2 or (t.numel() > 0 and t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be [requests, pages] with contiguous rows")
    return t.stride(0), t.shape[1]


def _pool(k: torch.Tensor, v: Optional[torch.Tensor], dims: int, what: str = "pools"):
    """Strides of a pool [(layers,) pages, page_size, heads, d] that K and V share."""
    _typed(torch.bfloat16, k_pages=k, v_pages=v)
    if k.dim() != dims or k.stride(dims - 1) != 1:
        raise ValueError(f"{what} must be {'[layers, ' if dims == 5 else '['}pages, page_size, heads, d] with contiguous d")
    if v is not None and (v.shape != k.shape or v.stride() != k.stride()):
        raise ValueError("K and V must share shape and strides")
    return k.stride()


def paged_attn_workspace_bytes(batch, q_len, n_q_heads, n_kv_heads, head_dim) -> int:
    return lib().specvlm_paged_attn_workspace_bytes(batch, q_len, n_q_heads, n_kv_heads, head_dim)


def paged_attn(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, kv_lens: torch.Tensor,
               softmax_scale: float, *, cu_q: Optional[torch.Tensor] = None, max_q_len: Optional[int] = None,
               max_kv_len: Optional[int] = None, window: int = 0, n_sinks: int = 0, ancestor_mask: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """Attention of every request's block of new tokens, q [sum q_len, H_q, d] bf16, over its cache in pages
    [pages, page_size, H_kv, d] bf16 -> out like q (and lse fp32).

    page_table int32 [batch, max_pages], kv_lens int32 [batch] (the block included); without cu_q every request has
    q.shape[0] / batch queries, with it max_q_len says the most.  max_kv_len: the most that kv_lens may hold (the whole
    table's worth by default).  window > 0: a query sees that many tokens up to its own, and the first n_sinks.
    ancestor_mask int64/uint64 [sum q_len]: a draft tree's, as in tree_attn.  out may be q."""
    got = (_calls or _load_calls()).paged_attn(q, k_pages, v_pages, page_table, kv_lens, softmax_scale, cu_q, max_q_len, max_kv_len, window, n_sinks,
                                               ancestor_mask, out, want_lse, workspace)
    if got is not None:
        if type(got) is int:
            _check("specvlm_paged_attn", got)
        return got
    _on_device(q=q, k_pages=k_pages, v_pages=v_pages, page_table=page_table, kv_lens=kv_lens, cu_q=cu_q,
               ancestor_mask=ancestor_mask, out=out, workspace=workspace)
    _typed(torch.bfloat16, q=q, out=out)
    (page, tok, head, _), (row, max_pages) = _pool(k_pages, v_pages, 4), _table("page_table", page_table)
    batch, (tq, hq, d), (n_pages, page_size, hkv, kd) = page_table.shape[0], q.shape, k_pages.shape
    if kd != d:
        raise ValueError("q and the pages must have one head dimension")
    _int32s(batch, kv_lens=kv_lens)
    if cu_q is None:
        if batch and tq % batch:
            raise ValueError("without cu_q every request has as many queries")
        q_len = tq // batch if batch else 0
    else:
        _int32s(batch + 1, cu_q=cu_q)
        if max_q_len is None:
            raise ValueError("max_q_len is required with cu_q")
        q_len = max_q_len
    kv_len = max_pages * page_size if max_kv_len is None else max_kv_len
    if ancestor_mask is not None and (ancestor_mask.dtype not in (torch.int64, torch.uint64) or not ancestor_mask.is_contiguous()
                                      or ancestor_mask.numel() < tq):
        raise ValueError("ancestor_mask must be a contiguous int64 or uint64 value for every query")
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.stride() != q.stride():
        raise ValueError("out must share q's shape and strides")
    lse = torch.empty((tq, hq), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        workspace = new_workspace(paged_attn_workspace_bytes(batch, q_len, hq, hkv, d), q.device)
    q_tok, q_head = _thd(q)
    rc = lib().specvlm_paged_attn(_ptr(q), q_tok, q_head, _ptr(k_pages), _ptr(v_pages), page, tok, head, n_pages, page_size,
                                  _ptr(page_table), row, max_pages, _ptr(kv_lens), _ptr(cu_q), batch, q_len, kv_len, hq, hkv, d,
                                  float(softmax_scale), window, n_sinks, _ptr(ancestor_mask), _ptr(out), _ptr(lse),
                                  _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_paged_attn", rc)
    return (out, lse) if want_lse else out


def pages_shared_workspace_bytes(batch) -> int:
    return lib().specvlm_pages_shared_workspace_bytes(batch)


def pages_shared(page_table: torch.Tensor, kv_lens: torch.Tensor, n_pages: int, page_size: int, q_len: int, *, cu_q: Optional[torch.Tensor] = None,
                 min_tokens: int = 256, groups: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Which neighbouring requests share how many tokens of their first pages -> groups int32 [3, batch] for shared_attn: each
    one's first neighbour of its group, for that one the number of them (0 for the others), the tokens that they share.

    page_table int32 [batch, max_pages], kv_lens int32 [batch], the block of q_len tokens (cu_q: of their own numbers) included.
    min_tokens: fewer common tokens are not worth a group.  (For a few requests about a video of some thousand tokens paged_attn is the faster
    call whatever the groups: the header has the line between it and shared_attn.)"""
    got = (_calls or _load_calls()).pages_shared(page_table, kv_lens, n_pages, page_size, q_len, cu_q, min_tokens, groups, workspace)
    if got is not None:
        if type(got) is int:
            _check("specvlm_pages_shared", got)
        return got
    _on_device(page_table=page_table, kv_lens=kv_lens, cu_q=cu_q, groups=groups, workspace=workspace)
    row, max_pages = _table("page_table", page_table)
    batch = page_table.shape[0]
    _int32s(batch, kv_lens=kv_lens)
    _int32s(batch + 1, cu_q=cu_q)
    if groups is None:
        groups = torch.empty((3, batch), dtype=torch.int32, device=page_table.device)
    _groups(batch, groups)
    if workspace is None:
        workspace = new_workspace(pages_shared_workspace_bytes(batch), page_table.device)
    rc = lib().specvlm_pages_shared(_ptr(page_table), row, max_pages, n_pages, page_size, _ptr(kv_lens), _ptr(cu_q), batch, q_len, min_tokens,
                                    _ptr(groups), _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_pages_shared", rc)
    return groups


def _groups(batch: int, groups: torch.Tensor):
    _typed(torch.int32, groups=groups)
    if groups.shape != (3, batch) or not groups.is_contiguous():
        raise ValueError("groups must be contiguous [3, requests]")


def shared_attn_workspace_bytes(batch, n_queries, n_q_heads, n_kv_heads, head_dim) -> int:
    return lib().specvlm_shared_attn_workspace_bytes(batch, n_queries, n_q_heads, n_kv_heads, head_dim)


def shared_attn(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, kv_lens: torch.Tensor,
                softmax_scale: float, groups: torch.Tensor, *, cu_q: Optional[torch.Tensor] = None, max_q_len: Optional[int] = None,
                max_kv_len: Optional[int] = None, ancestor_mask: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """paged_attn for a batch whose neighbouring requests share their first pages, which are read and computed once for all of a
    group; groups int32 [3, batch] from pages_shared.  Blocks may be of any length (with ancestor_mask up to 64).

    The other arguments are paged_attn's; without cu_q every request has q.shape[0] / batch queries."""
    got = (_calls or _load_calls()).shared_attn(q, k_pages, v_pages, page_table, kv_lens, softmax_scale, groups, cu_q, max_q_len, max_kv_len,
                                                ancestor_mask, out, want_lse, workspace)
    if got is not None:
        if type(got) is int:
            _check("specvlm_shared_attn", got)
        return got
    _on_device(q=q, k_pages=k_pages, v_pages=v_pages, page_table=page_table, kv_lens=kv_lens, groups=groups, cu_q=cu_q,
               ancestor_mask=ancestor_mask, out=out, workspace=workspace)
    _typed(torch.bfloat16, q=q, out=out)
    (page, tok, head, _), (row, max_pages) = _pool(k_pages, v_pages, 4), _table("page_table", page_table)
    batch, (tq, hq, d), (n_pages, page_size, hkv, kd) = page_table.shape[0], q.shape, k_pages.shape
    if kd != d:
        raise ValueError("q and the pages must have one head dimension")
    _int32s(batch, kv_lens=kv_lens)
    _groups(batch, groups)
    if cu_q is None:
        if batch and tq % batch:
            raise ValueError("without cu_q every request has as many queries")
        q_len = tq // batch if batch else 0
    else:
        _int32s(batch + 1, cu_q=cu_q)
        if max_q_len is None:
            raise ValueError("max_q_len is required with cu_q")
        q_len = max_q_len
    kv_len = max_pages * page_size if max_kv_len is None else max_kv_len
    if ancestor_mask is not None and (ancestor_mask.dtype not in (torch.int64, torch.uint64) or not ancestor_mask.is_contiguous()
                                      or ancestor_mask.numel() < tq):
        raise ValueError("ancestor_mask must be a contiguous int64 or uint64 value for every query")
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.stride() != q.stride():
        raise ValueError("out must share q's shape and strides")
    lse = torch.empty((tq, hq), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        workspace = new_workspace(shared_attn_workspace_bytes(batch, tq, hq, hkv, d), q.device)
    q_tok, q_head = _thd(q)
    rc = lib().specvlm_shared_attn(_ptr(q), q_tok, q_head, _ptr(k_pages), _ptr(v_pages), page, tok, head, n_pages, page_size,
                                   _ptr(page_table), row, max_pages, _ptr(kv_lens), _ptr(groups), _ptr(cu_q), batch, tq, q_len, kv_len, hq, hkv, d,
                                   float(softmax_scale), _ptr(ancestor_mask), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_shared_attn", rc)
    return (out, lse) if want_lse else out


def cross_attn_workspace_bytes(batch, n_queries, n_q_heads, n_kv_heads, head_dim) -> int:
    return lib().specvlm_cross_attn_workspace_bytes(batch, n_queries, n_q_heads, n_kv_heads, head_dim)


def cross_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, softmax_scale: float, *, cu_q: Optional[torch.Tensor] = None,
               cu_kv: Optional[torch.Tensor] = None, key_ranges: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """Attention of texts, q [queries, H_q, d] bf16, over encoders' states, k and v [states, H_kv, d] bf16 -> out like q (and lse fp32).

    cu_q and cu_kv int32 [batch + 1], prefix offsets of each entry's queries and states, of any lengths; None: all look at all.
    key_ranges int32 [queries, 2]: the states [from, to) of its entry that a query sees.  out may be q."""
    got = (_calls or _load_calls()).cross_attn(q, k, v, softmax_scale, cu_q, cu_kv, key_ranges, out, want_lse, workspace)
    if got is not None:
        if type(got) is int:
            _check("specvlm_cross_attn", got)
        return got
    _on_device(q=q, k=k, v=v, cu_q=cu_q, cu_kv=cu_kv, key_ranges=key_ranges, out=out, workspace=workspace)
    _typed(torch.bfloat16, q=q, k=k, v=v, out=out)
    (tq, hq, d), (tk, hkv, kd) = q.shape, k.shape
    if kd != d:
        raise ValueError("q and the states must have one head dimension")
    if v.shape != k.shape or v.stride() != k.stride():
        raise ValueError("K and V must share shape and strides")
    if (cu_q is None) != (cu_kv is None):
        raise ValueError("cu_q and cu_kv go together")
    batch = 1
    if cu_q is not None:
        batch = cu_q.numel() - 1
        if batch < 0:
            raise ValueError("cu_q has an entry more than there are entries")
        _int32s(batch + 1, cu_q=cu_q, cu_kv=cu_kv)
    if key_ranges is not None:
        _typed(torch.int32, key_ranges=key_ranges)
        if key_ranges.shape != (tq, 2) or not key_ranges.is_contiguous():
            raise ValueError("key_ranges must be contiguous [queries, 2]")
    if out is None:
        out = torch.empty_like(q)
    if out.shape != q.shape or out.stride() != q.stride():
        raise ValueError("out must share q's shape and strides")
    lse = torch.empty((tq, hq), dtype=torch.float32, device=q.device) if want_lse else None
    if workspace is None:
        workspace = new_workspace(cross_attn_workspace_bytes(batch, tq, hq, hkv, d), q.device)
    (q_tok, q_head), (k_tok, k_head) = _thd(q), _thd(k)
    rc = lib().specvlm_cross_attn(_ptr(q), q_tok, q_head, _ptr(k), _ptr(v), k_tok, k_head, _ptr(cu_q), _ptr(cu_kv), batch, tq, tk, hq, hkv, d,
                                  float(softmax_scale), _ptr(key_ranges), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_cross_attn", rc)
    return (out, lse) if want_lse else out


ROPE_SCALINGS = {None: 0, "linear": 1, "base": 2, "by-parts": 3}


def rope_turns(rot_dim: int, base: float, *, scaling: Optional[str] = None, factor: float = 1.0, original_len: float = 0.0,
               beta_fast: float = 32.0, beta_slow: float = 1.0, device=None) -> torch.Tensor:
    """The frequencies of rotary positions for rope_append: int64 [rot_dim / 2], turns a position in units of 2^-64."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {list(ROPE_SCALINGS)}")
    turns = np.zeros(max(rot_dim, 0) // 2, dtype=np.uint64)
    spec = _RopeSpec(ROPE_SCALINGS[scaling], base, factor, original_len, beta_fast, beta_slow)
    _check("specvlm_rope_turns", lib().specvlm_rope_turns(rot_dim, C.byref(spec), turns.ctypes.data))
    return torch.from_numpy(turns.view(np.int64)).to(device or "cuda")


def rope_append(k: Optional[torch.Tensor], v: Optional[torch.Tensor], k_pages: Optional[torch.Tensor], v_pages: Optional[torch.Tensor],
                page_table: Optional[torch.Tensor], kv_lens: Optional[torch.Tensor], *, q: Optional[torch.Tensor] = None,
                q_out: Optional[torch.Tensor] = None, turns: Optional[torch.Tensor] = None, interleaved: bool = False,
                magnitude: float = 1.0, positions: Optional[torch.Tensor] = None, cu_q: Optional[torch.Tensor] = None):
    """The new tokens of every request: q [tokens, H_q, d] and k [tokens, H_kv, d] turned to their positions (turns: from
    rope_turns, int64 [rot_dim / 2]; None turns nothing), k and v written to the last rows of the requests' caches -> q_out.

    kv_lens counts the new tokens.  positions int32 [tokens] where they are not the places in the cache.  q_out may be q.
    With k, v and the pages None only q is turned."""
    got = (_calls or _load_calls()).rope_append(k, v, k_pages, v_pages, page_table, kv_lens, q, q_out, turns, interleaved, magnitude, positions, cu_q)
    if got is not None:
        if type(got) is int:
            _check("specvlm_rope_append", got)
        return None if got is True else got
    one = q if k is None else k
    if one is None:
        raise ValueError("neither q nor k")
    if (k is None) != (v is None):
        raise ValueError("k and v go together")
    _on_device(q=q, q_out=q_out, k=k, v=v, turns=turns, positions=positions, cu_q=cu_q, kv_lens=kv_lens, page_table=page_table)
    _typed(torch.bfloat16, q=q, q_out=q_out, k=k, v=v)
    n, _, d = one.shape
    batch = kv_lens.numel() if kv_lens is not None else cu_q.numel() - 1 if cu_q is not None else 1
    _int32s(batch, kv_lens=kv_lens)
    _int32s(batch + 1, cu_q=cu_q)
    _int32s(n, positions=positions)
    if turns is not None and (turns.dtype not in (torch.int64, torch.uint64) or turns.dim() != 1 or not turns.is_contiguous()):
        raise ValueError("turns must be a contiguous int64 or uint64 vector")
    qs = os_ = ks = (0, 0)
    hq = hkv = 0
    if q is not None:
        if q_out is None:
            q_out = torch.empty_like(q)
        if q.shape[0] != n or q.shape[2] != d or q_out.shape != q.shape:
            raise ValueError("q, q_out and k must agree in tokens and head dimension")
        qs, os_, hq = _thd(q), _thd(q_out), q.shape[1]
    page = tok = head = row = n_pages = page_size = max_pages = 0
    if k is not None:
        if k_pages is None or v_pages is None or page_table is None or kv_lens is None:
            raise ValueError("k and v need pages, a page table and kv_lens")
        if v.shape != k.shape or v.stride() != k.stride():
            raise ValueError("K and V must share shape and strides")
        _on_device(k_pages=k_pages, v_pages=v_pages)
        (page, tok, head, _), (row, max_pages) = _pool(k_pages, v_pages, 4), _table("page_table", page_table)
        n_pages, page_size, hkv, pd = k_pages.shape
        if pd != d or hkv != k.shape[1] or page_table.shape[0] != batch:
            raise ValueError("k, the pages and the page table must agree in heads, head dimension and requests")
        ks = _thd(k)
    rc = lib().specvlm_rope_append(_ptr(q), *qs, _ptr(q_out), *os_, _ptr(k), _ptr(v), *ks, _ptr(k_pages), _ptr(v_pages), page, tok, head,
                                   n_pages, page_size, _ptr(page_table), row, max_pages, _ptr(kv_lens), _ptr(cu_q), batch, n,
                                   _ptr(positions), _ptr(turns), 0 if turns is None else 2 * turns.numel(), int(interleaved),
                                   float(magnitude), hq, hkv, d, _stream())
    _check("specvlm_rope_append", rc)
    return q_out


def pages_assign(page_table: torch.Tensor, parent: torch.Tensor, keep_len: torch.Tensor, new_len: torch.Tensor, n_pages: int,
                 page_size: int, *, max_pages: Optional[int] = None, window: int = 0, n_sinks: int = 0,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """The next page table: row b goes on from row parent[b] of page_table (-1: from nothing), keeps keep_len[b] tokens and has
    room for new_len[b]; int32 vectors on the device.
    -> (table [batch, max_pages], copy_start [batch], copy_rows [batch], ref_counts [n_pages], status [batch]), all int32:
    copy_rows[b] tokens from copy_start[b] on are to be copied from row parent[b] of the old table to row b of the new one
    (pages_copy), ref_counts says how many rows hold each page, status is 0, -1 (the row does not fit together) or -5 (too
    few pages are free: the row is without those, and without the page that its kept tokens end in where another row goes on in
    that; assign again from page_table for fewer rows, or go on later from the row's whole pages)."""
    got = (_calls or _load_calls()).pages_assign(page_table, parent, keep_len, new_len, n_pages, page_size, max_pages, window, n_sinks, out, workspace)
    if got is not None:
        if type(got) is int:
            _check("specvlm_pages_assign", got)
        return got
    _on_device(page_table=page_table, parent=parent, keep_len=keep_len, new_len=new_len, out=out, workspace=workspace)
    old_row, old_pages = _table("page_table", page_table)
    batch = parent.numel()
    _int32s(batch, parent=parent, keep_len=keep_len, new_len=new_len)
    if max_pages is None:
        max_pages = old_pages if out is None else out.shape[1]
    if out is None:
        out = page_table.new_empty((batch, max_pages))
    row, width = _table("out", out)
    if out.shape[0] != batch or width != max_pages:
        raise ValueError("out must be [batch, max_pages]")
    if n_pages < 0:
        raise ValueError("n_pages must not be negative")
    copies = page_table.new_empty((3, batch))
    refs = page_table.new_empty(n_pages)
    if workspace is None:
        workspace = new_workspace(lib().specvlm_pages_assign_workspace_bytes(batch, n_pages), page_table.device)
    at = copies.data_ptr()
    rc = lib().specvlm_pages_assign(_ptr(page_table), old_row, page_table.shape[0], old_pages, _ptr(parent), _ptr(keep_len), _ptr(new_len),
                                    batch, _ptr(out), row, max_pages, n_pages, page_size, window, n_sinks, at, at + 4 * batch,
                                    _ptr(refs), at + 8 * batch, _ptr(workspace), workspace.numel(), _stream())
    _check("specvlm_pages_assign", rc)
    return out, copies[0], copies[1], refs, copies[2]


def pages_copy(k_src: torch.Tensor, v_src: Optional[torch.Tensor], src_table: torch.Tensor, k_dst: torch.Tensor, v_dst: Optional[torch.Tensor],
               dst_table: torch.Tensor, n_rows: Optional[torch.Tensor], max_rows: int, *, src_row: Optional[torch.Tensor] = None,
               src_start: Optional[torch.Tensor] = None, dst_start: Optional[torch.Tensor] = None,
               row_idx: Optional[torch.Tensor] = None, cu_idx: Optional[torch.Tensor] = None) -> None:
    """Rows between pools [layers, pages, page_size, H_kv, d] bf16, in every layer: for request b (a row of dst_table) and
    i < n_rows[b] (at most max_rows) token src_start[b] + (row_idx's i-th of the request, or i) of row src_row[b] (b) of
    src_table goes to token dst_start[b] + i of row b of dst_table.  Vectors are int32 [batch]; row_idx is [batch, entries],
    or one list cut by cu_idx [batch + 1] (n_rows may then be None).  Source and destination may be one pool if no row moves up."""
    got = (_calls or _load_calls()).pages_copy(k_src, v_src, src_table, k_dst, v_dst, dst_table, n_rows, max_rows, src_row, src_start, dst_start,
                                               row_idx, cu_idx)
    if got is not None:
        if type(got) is int:
            _check("specvlm_pages_copy", got)
        return
    _on_device(k_src=k_src, v_src=v_src, src_table=src_table, k_dst=k_dst, v_dst=v_dst, dst_table=dst_table, n_rows=n_rows, src_row=src_row,
               src_start=src_start, dst_start=dst_start, row_idx=row_idx, cu_idx=cu_idx)
    if (v_src is None) != (v_dst is None):
        raise ValueError("v_src and v_dst go together")
    src, dst = _pool(k_src, v_src, 5, "source pools"), _pool(k_dst, v_dst, 5, "destination pools")
    (src_stride, src_pages), (dst_stride, dst_pages) = _table("src_table", src_table), _table("dst_table", dst_table)
    layers, _, _, hkv, d = k_src.shape
    if k_dst.shape[0] != layers or k_dst.shape[3:] != k_src.shape[3:]:
        raise ValueError("the pools must agree in layers, heads and head dimension")
    batch = dst_table.shape[0]
    _int32s(batch, n_rows=n_rows, src_row=src_row, src_start=src_start, dst_start=dst_start)
    _typed(torch.int32, row_idx=row_idx)
    idx_stride = 0
    if cu_idx is not None:
        _int32s(batch + 1, cu_idx=cu_idx)
        _int32s(None, row_idx=row_idx)
        if row_idx is not None and row_idx.numel() == 0:        # (lists of which each is empty)
            return
    elif row_idx is not None:
        if row_idx.dim() != 2 or row_idx.shape[0] != batch or row_idx.shape[1] < max_rows or (row_idx.shape[1] > 1 and row_idx.stride(1) != 1):
            raise ValueError("row_idx must be [batch, at least max_rows] with contiguous rows")
        idx_stride = row_idx.stride(0)
    rc = lib().specvlm_pages_copy(_ptr(k_src), _ptr(v_src), *src[:4], k_src.shape[1], k_src.shape[2], _ptr(src_table), src_stride,
                                  src_table.shape[0], src_pages, _ptr(k_dst), _ptr(v_dst), *dst[:4], k_dst.shape[1], k_dst.shape[2],
                                  _ptr(dst_table), dst_stride, dst_pages, layers, batch, _ptr(n_rows), max_rows, _ptr(src_row),
                                  _ptr(src_start), _ptr(dst_start), _ptr(row_idx), idx_stride, _ptr(cu_idx), hkv, d, _stream())
    _check("specvlm_pages_copy", rc)


# -------------------------------------------------------------------------- accept
def accept_workspace_bytes(batch, gamma, vocab, sampling) -> int:
    return lib().specvlm_accept_workspace_bytes(batch, gamma, vocab, int(sampling))


def accept(target_logits: torch.Tensor, draft_tokens: torch.Tensor, *,
           draft_logits: Optional[torch.Tensor] = None, uniforms: Optional[torch.Tensor] = None,
           temperature: float = 1.0, workspace: Optional[torch.Tensor] = None,
           n_accepted: Optional[torch.Tensor] = None, out_tokens: Optional[torch.Tensor] = None):
    """target_logits fp32 [batch, gamma+1, vocab] -> (n_accepted int32 [batch], out_tokens int32 [batch, gamma+1])."""
    got = (_calls or _load_calls()).accept(target_logits, draft_tokens, draft_logits, uniforms, temperature, workspace, n_accepted, out_tokens)
    if got is not None:
        if type(got) is int:
            _check("specvlm_accept", got)
        return got
    batch, g1, vocab = target_logits.shape
    gamma = g1 - 1
    if n_accepted is None:
        n_accepted = torch.empty(batch, dtype=torch.int32, device=target_logits.device)
    if out_tokens is None:
        out_tokens = torch.empty((batch, g1), dtype=torch.int32, device=target_logits.device)
    if workspace is None:
        workspace = new_workspace(accept_workspace_bytes(batch, gamma, vocab, uniforms is not None), target_logits.device)
    target, draft, tokens, u = _contiguous_ptrs("accept", target_logits, draft_logits, draft_tokens, uniforms)
    rc = lib().specvlm_accept(target, draft, tokens, u, batch, gamma, vocab, temperature, _ptr(n_accepted),
                              _ptr(out_tokens), _ptr(workspace), workspace.numel(), _raw_stream(_current_device()))
    if rc:
        _check("specvlm_accept", rc)
    return n_accepted, out_tokens


def accept_tree(target_logits: torch.Tensor, node_tokens: torch.Tensor, parent: torch.Tensor, *,
                workspace: Optional[torch.Tensor] = None):
    """target_logits fp32 [batch, n_nodes, vocab], node_tokens int32 [batch, n_nodes], parent int32 [n_nodes]
    -> (n_accepted [batch], accepted_nodes [batch, n_nodes], out_tokens [batch, n_nodes])."""
    batch, n_nodes, vocab = target_logits.shape
    dev = target_logits.device
    n_acc = torch.empty(batch, dtype=torch.int32, device=dev)
    nodes = torch.empty((batch, n_nodes), dtype=torch.int32, device=dev)
    out = torch.empty((batch, n_nodes), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = new_workspace(lib().specvlm_accept_tree_workspace_bytes(batch, n_nodes, vocab), dev)
    for t in (target_logits, node_tokens, parent):
        if not t.is_contiguous():
            raise ValueError("accept_tree inputs must be contiguous")
    rc = lib().specvlm_accept_tree(_ptr(target_logits), _ptr(node_tokens), _ptr(parent), batch, n_nodes,
                                   vocab, _ptr(n_acc), _ptr(nodes), _ptr(out), _ptr(workspace),
                                   workspace.numel(), _stream())
    _check("specvlm_accept_tree", rc)
    return n_acc, nodes, out


# ------------------------------------------------------------------- baseline pruners
BASELINE_MODES = {"window-front": 0, "window-middle": 1, "window-end": 2, "uniform": 3,
                  "frame-drop": 4, "lattice": 5, "random": 6, "uniform-per-frame": 7}


def baseline_keep(mode: str, n_video: int, keep_budget: int, *, n_frames: int = 0, grid_h: int = 0,
                  grid_w: int = 0, stride_h: int = 1, stride_w: int = 1, seed: int = 0,
                  device=None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Retention set of the named attention-agnostic pruner -> ascending int32 indices on the device."""
    m = BASELINE_MODES[mode]
    count = lib().specvlm_baseline_count(m, n_video, n_frames, grid_h, grid_w, keep_budget, stride_h, stride_w)
    if count < 0:
        raise SpecVLMError("specvlm_baseline_count", count)
    keep_idx = torch.empty(count, dtype=torch.int32, device=device or "cuda")
    need = lib().specvlm_baseline_workspace_bytes(m, n_video)
    if need and workspace is None:
        workspace = new_workspace(need, keep_idx.device)
    rc = lib().specvlm_baseline_keep(m, n_video, n_frames, grid_h, grid_w, keep_budget, stride_h, stride_w,
                                     seed, _ptr(keep_idx), _ptr(workspace),
                                     workspace.numel() if workspace is not None else 0, _stream())
    _check("specvlm_baseline_keep", rc)
    return keep_idx


# ------------------------------------------------------------------------ diagnostics
def probe_read(a: torch.Tensor, b: Optional[torch.Tensor] = None) -> None:
    """One launch that merely reads the bytes of `a` (and `b`): the bare-read yardstick of the benchmark.
    Both must be dense in memory (any dimension order)."""
    def span(t):
        if t is None:
            return None, 0
        return t.data_ptr(), t.numel() * t.element_size()
    pa, na = span(a)
    pb, nb = span(b)
    _check("specvlm_probe_read", lib().specvlm_probe_read(pa, na, pb, nb, None, _stream()))
