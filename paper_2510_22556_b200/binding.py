"""Thin binding of libsablock.so (include/sablock.h), argument marshalling only: by ctypes, the entry points that
enqueue work through the C module csrc/fastcall.c where it is built.

Every function takes torch CUDA tensors (or raw pointers), passes their device pointers
through the C ABI and enqueues on torch's current stream.  No step of the pass runs in
Python or torch; if the library is missing the import of `lib()` fails loudly.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional, Sequence

import torch

try:
    from . import _fastcall
except ImportError:                        # not built: ctypes marshals
    _fastcall = None

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsablock.so")

OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "WORKSPACE_TOO_SMALL", 4: "CUDA", 5: "TIMEOUT",
                6: "INTERNAL"}
F32, BF16 = 0, 1
SCORE_AUTO, SCORE_SIMT, SCORE_TENSOR, SCORE_FUSED = 0, 1, 2, 3

EXPORTS = [
    "sablock_params_default", "sablock_status_string", "sablock_version", "sablock_workspace_bytes",
    "sablock_read_status", "sablock_segment", "sablock_score", "sablock_select", "sablock_compact",
    "sablock_compress", "sablock_compress_layers", "sablock_compress_layers_host", "sablock_last_launch_count",
    "sablock_params_sizeof", "sablock_workspace_region", "sablock_profile_enable", "sablock_profile_read",
    "sablock_profile_stage_name", "sablock_segment_static", "sablock_last_cuda_error", "sablock_read_status_detail",
    "sablock_decode_workspace_bytes", "sablock_decode_attention",
    "sablock_pages_sizeof", "sablock_paged_append", "sablock_paged_workspace_bytes", "sablock_paged_attention",
    "sablock_page_select", "sablock_paged_sparse_attention",
]


class Params(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int), ("window", C.c_int),
        ("dtype", C.c_int),
        ("k_stride_token", C.c_longlong), ("k_stride_head", C.c_longlong), ("k_stride_layer", C.c_longlong),
        ("v_stride_token", C.c_longlong), ("v_stride_head", C.c_longlong), ("v_stride_layer", C.c_longlong),
        ("alpha", C.c_float), ("eta", C.c_float), ("eps", C.c_float), ("tau", C.c_float),
        ("pool_kernel", C.c_int), ("pool_mode", C.c_int), ("budget_includes_window", C.c_int),
        ("delim_bitmap", C.c_void_p), ("vocab_size", C.c_int),
        ("score_impl", C.c_int), ("debug_sync", C.c_int), ("row_lse", C.c_void_p), ("reproducible", C.c_int), ("reserved", C.c_int * 5),
    ]


class Pages(C.Structure):
    """Description of a paged cache (sablock_pages_t); make_pages fills one from its tensors."""
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p), ("bounds", C.c_void_p), ("table", C.c_void_p), ("seq_lens", C.c_void_p),
        ("table_stride", C.c_longlong),
        ("k_stride_page", C.c_longlong), ("k_stride_row", C.c_longlong), ("k_stride_head", C.c_longlong),
        ("v_stride_page", C.c_longlong), ("v_stride_row", C.c_longlong), ("v_stride_head", C.c_longlong),
        ("n_seqs", C.c_int), ("n_pages", C.c_int), ("page_size", C.c_int), ("max_pages", C.c_int), ("reserved", C.c_int * 4),
    ]


class SablockError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = lib().sablock_last_cuda_error().decode() if code == 4 else ""
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)} ({lib().sablock_status_string(code).decode()})"
                         + (f" [{detail}]" if detail else ""))


_lib = None


def _load(path: str):
    """dlopens one build of the library and declares the argument types of its entry points."""
    if not os.path.exists(path):
        raise ImportError(f"{path} not found: build it with `python -m paper_2510_22556_b200.build` "
                          "or __graft_entry__.build()")
    l = C.CDLL(path)
    l.sablock_status_string.restype = C.c_char_p
    l.sablock_last_cuda_error.restype = C.c_char_p
    l.sablock_params_sizeof.restype = C.c_size_t
    if l.sablock_params_sizeof() != C.sizeof(Params):
        raise ImportError("sablock_params_t layout mismatch between the library and the binding")
    l.sablock_pages_sizeof.restype = C.c_size_t
    if l.sablock_pages_sizeof() != C.sizeof(Pages):
        raise ImportError("sablock_pages_t layout mismatch between the library and the binding")
    l.sablock_workspace_bytes.restype = C.c_size_t
    l.sablock_workspace_bytes.argtypes = [C.c_void_p, C.c_longlong, C.c_int, C.c_int, C.c_int]
    vp, ci, sz = C.c_void_p, C.c_int, C.c_size_t
    l.sablock_read_status.argtypes = [vp, vp, vp]
    l.sablock_read_status_detail.argtypes = [vp, vp, vp]
    l.sablock_workspace_region.argtypes = [vp, C.c_longlong, ci, ci, ci, C.c_char_p, vp, vp]
    l.sablock_params_default.argtypes = [vp]
    l.sablock_profile_read.argtypes = [ci, vp, ci]
    l.sablock_profile_stage_name.restype = C.c_char_p
    l.sablock_segment.argtypes = [vp, vp, ci, vp, vp, vp, vp, sz, vp]
    l.sablock_segment_static.argtypes = [vp, vp, ci, vp, vp, vp, vp, vp]
    l.sablock_score.argtypes = [vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    l.sablock_select.argtypes = [vp, vp, ci, vp, vp, ci, vp, ci, vp, vp, vp, vp, sz, vp]
    l.sablock_compact.argtypes = [vp, vp, vp, ci, vp, ci, vp, vp, vp]
    l.sablock_compress.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, ci, vp, vp, vp, vp, vp, sz, vp]
    l.sablock_compress_layers.argtypes = [vp, ci, ci, vp, vp, vp, vp, vp, ci, vp, ci, vp, vp, vp, vp, vp, sz, vp]
    l.sablock_compress_layers_host.argtypes = [vp, ci, ci, vp, vp, vp, vp, vp, ci, vp, ci, vp, vp, vp, vp,
                                               vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    ll = C.c_longlong
    l.sablock_paged_append.argtypes = [vp, vp, ci, vp, vp, ll, vp, ll, vp, ll, vp, vp, vp, ci, ci, vp]
    l.sablock_paged_workspace_bytes.restype = sz
    l.sablock_paged_workspace_bytes.argtypes = [vp, vp, ci]
    l.sablock_paged_attention.argtypes = [vp, vp, vp, vp, ci, vp, vp, vp, sz, vp]
    l.sablock_page_select.argtypes = [vp, vp, vp, ci, ci, ci, vp, vp]
    l.sablock_paged_sparse_attention.argtypes = [vp, vp, vp, ci, ci, ci, vp, vp, vp, vp, sz, vp]
    # The entry points that enqueue work, by their short names: through the C module where it is built.  A
    # sequence argument is a tuple or list there and a ctypes array here.
    for name in ("segment", "segment_static", "score", "select", "compact", "compress", "compress_layers", "compress_layers_host",
                 "decode_attention", "paged_append", "paged_attention", "page_select", "paged_sparse_attention"):
        fn = getattr(l, "sablock_" + name)
        setattr(l, name, _fastcall.bind(C.cast(fn, C.c_void_p).value) if _fastcall else fn)
    l.decode_step = _fastcall.bind_decode(C.cast(l.sablock_decode_attention, C.c_void_p).value) if _fastcall else None
    l.append_step = (_fastcall.bind_append(C.cast(l.sablock_paged_append, C.c_void_p).value) if hasattr(_fastcall, "bind_append") else None)
    l.sablock_decode_workspace_bytes.restype = C.c_size_t
    l.sablock_decode_workspace_bytes.argtypes = [vp, ci, ci]
    l.sablock_decode_attention.argtypes = [vp, ci, vp, vp, vp, ci, vp, vp, vp, vp, sz, vp]
    return l


def lib():
    """The CUDA library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        _lib = _load(LIB_PATH)
    return _lib


@contextlib.contextmanager
def use_library(path: str):
    """Routes every call of this module through another build of the library (the tests of the
    give-up paths use one with shortened waits) for the duration of the block."""
    global _lib
    saved = _lib
    _lib = _load(path)
    try:
        yield _lib
    finally:
        _lib = saved


def _ptr(t: Optional[torch.Tensor]):
    """Device address as an integer: the argument types declared in _load() make a pointer of it."""
    return None if t is None else t.data_ptr()


def _stream() -> int:
    """Handle of torch's current stream on the current device (the stream object that
    torch.cuda.current_stream() builds around it costs more than the launch of a kernel)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(code: int, where: str):
    if code != OK:
        raise SablockError(code, where)


def _iarr(xs: Sequence[int]):
    """A sequence of ints as an argument of an entry point."""
    if _fastcall is not None:
        return xs if type(xs) is tuple or type(xs) is list else [int(x) for x in xs]
    return (C.c_int * len(xs))(*[int(x) for x in xs])


def make_params(n_q_heads: int, n_kv_heads: int, head_dim: int, window: int, dtype: torch.dtype,
                delim_bitmap: Optional[torch.Tensor] = None, vocab_size: int = 0, **kw) -> Params:
    p = Params()
    lib().sablock_params_default(C.addressof(p))
    p.n_q_heads, p.n_kv_heads, p.head_dim, p.window = n_q_heads, n_kv_heads, head_dim, window
    p.dtype = {torch.float32: F32, torch.bfloat16: BF16}[dtype]
    if delim_bitmap is not None:
        p.delim_bitmap = delim_bitmap.data_ptr()
        p.vocab_size = vocab_size
        p._bitmap_ref = delim_bitmap          # keep the device buffer alive as long as the block
    for k, v in kw.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        if k == "row_lse" and isinstance(v, torch.Tensor):
            if v.dtype != torch.float32 or not v.is_contiguous():
                raise TypeError("row_lse must be a contiguous float32 tensor")
            p._row_lse_ref = v                # keep the device buffer alive as long as the block
            v = v.data_ptr()
        setattr(p, k, v)
    return p


def workspace_bytes(p: Params, total_tokens: int, max_L: int, n_seqs: int = 1, n_layers: int = 1) -> int:
    n = lib().sablock_workspace_bytes(C.addressof(p), total_tokens, max_L, n_seqs, n_layers)
    if n == 0:
        raise SablockError(1, "sablock_workspace_bytes")
    return int(n)


def workspace_view(p: Params, ws: torch.Tensor, name: str, total_tokens: int, max_L: int, n_seqs: int = 1,
                   n_layers: int = 1) -> torch.Tensor:
    """A typed view of one of the fused call's intermediate arrays inside the workspace."""
    off, nb = C.c_size_t(0), C.c_size_t(0)
    _check(lib().sablock_workspace_region(C.addressof(p), total_tokens, max_L, n_seqs, n_layers, name.encode(),
                                          C.addressof(off), C.addressof(nb)), "sablock_workspace_region")
    raw = ws[off.value: off.value + nb.value]
    dt = torch.float32 if name in ("s", "e", "s_refined") else torch.int32
    v = raw.view(dt)
    return v.view(n_layers, total_tokens) if dt == torch.float32 else v


def alloc_workspace(p: Params, total_tokens: int, max_L: int, n_seqs: int = 1, n_layers: int = 1,
                    device="cuda") -> torch.Tensor:
    return torch.empty(workspace_bytes(p, total_tokens, max_L, n_seqs, n_layers), dtype=torch.uint8, device=device)


def read_status(ws: torch.Tensor) -> int:
    raw = C.c_int(0)
    code = lib().sablock_read_status(_ptr(ws), _stream(), C.addressof(raw))
    return code


def read_status_detail(ws: torch.Tensor):
    """(status code, raw status word, code | CTA << 8 | warp << 20 of the first wait that gave up)."""
    raw = (C.c_int * 2)()
    code = lib().sablock_read_status_detail(_ptr(ws), _stream(), C.addressof(raw))
    return code, int(raw[0]), int(raw[1])


def profile_enable(slots: int) -> None:
    _check(lib().sablock_profile_enable(int(slots)), "sablock_profile_enable")


def profile_read(slot: int):
    """Stage name -> milliseconds for the fused call that used event slot `slot`."""
    buf = (C.c_float * 16)()
    n = lib().sablock_profile_read(slot, C.addressof(buf), 16)
    return {lib().sablock_profile_stage_name(i).decode(): float(buf[i]) for i in range(n)}


def last_launch_count() -> int:
    return int(lib().sablock_last_launch_count())


def segment(p: Params, token_ids: torch.Tensor, ws: torch.Tensor):
    L = token_ids.numel()
    T = L - p.window
    seg_id = torch.empty(max(T, 1), dtype=torch.int32, device=token_ids.device)
    seg_start = torch.empty(max(T, 1) + 1, dtype=torch.int32, device=token_ids.device)
    n_seg = torch.empty(1, dtype=torch.int32, device=token_ids.device)   # always written
    _check(lib().segment(C.addressof(p), _ptr(token_ids), L, _ptr(seg_id), _ptr(seg_start), _ptr(n_seg),
                                 _ptr(ws), ws.numel(), _stream()), "sablock_segment")
    return seg_id, seg_start, n_seg


SEGMENT_STATIC_MAX_T = 1024 * 2048


def segment_static(p: Params, token_ids: torch.Tensor, seg_id: torch.Tensor, seg_start: torch.Tensor,
                   n_seg: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
    """sablock_segment without a workspace: the caller supplies every buffer (outputs included), and the
    kernel's CTAs exchange their counts on chip.  Nothing is allocated here."""
    _check(lib().segment_static(C.addressof(p), _ptr(token_ids), token_ids.numel(), _ptr(seg_id),
                                        _ptr(seg_start), _ptr(n_seg), _ptr(status), _stream()),
           "sablock_segment_static")


def score(p: Params, q_win: torch.Tensor, k: torch.Tensor, seg_start: torch.Tensor, n_seg: torch.Tensor,
          ws: torch.Tensor, want_stats: bool = False):
    L = k.shape[0]
    T = L - p.window
    dev = k.device
    s = torch.empty(T, dtype=torch.float32, device=dev)
    e = torch.empty(T, dtype=torch.float32, device=dev)
    sr = torch.empty(T, dtype=torch.float32, device=dev)
    stats = torch.zeros(3 * T, dtype=torch.float32, device=dev) if want_stats else None
    _check(lib().score(C.addressof(p), _ptr(q_win), _ptr(k), L, _ptr(seg_start), _ptr(n_seg), _ptr(s), _ptr(e),
                               _ptr(sr), _ptr(stats), _ptr(ws), ws.numel(), _stream()), "sablock_score")
    return s, e, sr, (stats.view(3, T) if want_stats else None)


def rows_out(p: Params, budget: int, L: int) -> int:
    n = budget if p.budget_includes_window else budget + p.window
    return L if n >= L else n


def select(p: Params, s_refined: torch.Tensor, L: int, seg_start: torch.Tensor, n_seg: torch.Tensor, budget: int,
           candidates: Sequence[int], ws: torch.Tensor, want_segments: bool = False):
    dev = s_refined.device
    T = L - p.window
    out_idx = torch.empty(rows_out(p, budget, L), dtype=torch.int32, device=dev)
    seg_g = torch.zeros(max(T, 1), dtype=torch.int32, device=dev) if want_segments else None
    seg_b = torch.zeros(max(T, 1), dtype=torch.int32, device=dev) if want_segments else None
    cand = _iarr(candidates)
    _check(lib().select(C.addressof(p), _ptr(s_refined), L, _ptr(seg_start), _ptr(n_seg), budget, cand,
                                len(candidates), _ptr(out_idx), _ptr(seg_g), _ptr(seg_b), _ptr(ws), ws.numel(),
                                _stream()), "sablock_select")
    return out_idx, seg_g, seg_b


def compact(p: Params, k: torch.Tensor, v: torch.Tensor, out_idx: torch.Tensor):
    n = out_idx.numel()
    out_k = torch.empty((n,) + tuple(k.shape[1:]), dtype=k.dtype, device=k.device)
    out_v = torch.empty_like(out_k)
    _check(lib().compact(C.addressof(p), _ptr(k), _ptr(v), k.shape[0], _ptr(out_idx), n, _ptr(out_k),
                                 _ptr(out_v), _stream()), "sablock_compact")
    return out_k, out_v


def compress(p: Params, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor, token_ids: torch.Tensor, budget: int,
             candidates: Sequence[int], ws: torch.Tensor):
    """One layer of one sequence.  Returns (out_k, out_v, out_idx, n_keep tensor)."""
    L = k.shape[0]
    n = rows_out(p, budget, L)
    out_k = torch.empty((n,) + tuple(k.shape[1:]), dtype=k.dtype, device=k.device)
    out_v = torch.empty_like(out_k)
    out_idx = torch.empty(n, dtype=torch.int32, device=k.device)
    n_keep = torch.empty(1, dtype=torch.int32, device=k.device)          # always written
    cand = _iarr(candidates)
    _check(lib().compress(C.addressof(p), _ptr(q_win), _ptr(k), _ptr(v), _ptr(token_ids), L, budget, cand,
                                  len(candidates), _ptr(out_k), _ptr(out_v), _ptr(out_idx), _ptr(n_keep), _ptr(ws),
                                  ws.numel(), _stream()), "sablock_compress")
    return out_k, out_v, out_idx, n_keep


class LayersOut:
    """Pre-allocated outputs of compress_layers: out_k/out_v [layers, seqs, n_out, Hkv, D], out_idx, n_keep."""

    def __init__(self, p: Params, n_layers: int, n_seqs: int, budget: int, dtype, device="cuda", pinned_host=False):
        n_out = budget if p.budget_includes_window else budget + p.window
        kw = dict(device="cpu", pin_memory=True) if pinned_host else dict(device=device)
        self.n_out = n_out
        self.out_k = torch.empty(n_layers, n_seqs, n_out, p.n_kv_heads, p.head_dim, dtype=dtype, **kw)
        self.out_v = torch.empty(n_layers, n_seqs, n_out, p.n_kv_heads, p.head_dim, dtype=dtype, **kw)
        self.out_idx = torch.empty(n_layers, n_seqs, n_out, dtype=torch.int32, **kw)
        self.n_keep = torch.zeros(n_layers, n_seqs, dtype=torch.int32, **kw)


def compress_layers(p: Params, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor, token_ids: torch.Tensor,
                    cu_seqlens: Sequence[int], budget: int, candidates: Sequence[int], ws: torch.Tensor,
                    out: Optional[LayersOut] = None) -> LayersOut:
    n_layers, n_seqs = q_win.shape[0], q_win.shape[1]
    if out is None:
        out = LayersOut(p, n_layers, n_seqs, budget, k.dtype, k.device)
    cu = _iarr(cu_seqlens)
    cand = _iarr(candidates)
    _check(lib().compress_layers(C.addressof(p), n_layers, n_seqs, _ptr(q_win), _ptr(k), _ptr(v),
                                         _ptr(token_ids), cu, budget, cand, len(candidates), _ptr(out.out_k),
                                         _ptr(out.out_v), _ptr(out.out_idx), _ptr(out.n_keep), _ptr(ws), ws.numel(),
                                         _stream()), "sablock_compress_layers")
    return out


def compress_layers_host(p: Params, h_q, h_k, h_v, h_ids, cu_seqlens, budget, candidates, h_out: LayersOut,
                         d_q, d_k, d_v, d_ids, d_out: LayersOut, ws: torch.Tensor) -> LayersOut:
    """End-to-end variant: host (ideally pinned) inputs and outputs, device staging supplied by the caller."""
    n_layers, n_seqs = h_q.shape[0], h_q.shape[1]
    cu = _iarr(cu_seqlens)
    cand = _iarr(candidates)
    _check(lib().compress_layers_host(
        C.addressof(p), n_layers, n_seqs, _ptr(h_q), _ptr(h_k), _ptr(h_v), _ptr(h_ids), cu, budget, cand,
        len(candidates), _ptr(h_out.out_k), _ptr(h_out.out_v), _ptr(h_out.out_idx), _ptr(h_out.n_keep),
        _ptr(d_q), _ptr(d_k), _ptr(d_v), _ptr(d_ids), _ptr(d_out.out_k), _ptr(d_out.out_v), _ptr(d_out.out_idx),
        _ptr(d_out.n_keep), _ptr(ws), ws.numel(), _stream()), "sablock_compress_layers_host")
    return h_out


def decode_attention(p: Params, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     n_valid: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                     want_lse: bool = False):
    """One decode step's attention over a cache.  q [n_prob, H, D]; k_cache, v_cache
    [n_prob, n_rows, Hkv, D] (contiguous).  Returns out f32 [n_prob, H, D] (and lse [n_prob, H])."""
    if ws is None:
        n_prob, n_rows = q.shape[0], k_cache.shape[1]
        nb = int(lib().sablock_decode_workspace_bytes(C.addressof(p), n_prob, n_rows))
        if nb == 0:
            raise SablockError(2, "sablock_decode_workspace_bytes")
        ws = torch.empty(nb, dtype=torch.uint8, device=q.device)
    # (empty_like is the cheaper call; it keeps the strides of a dense input, so it is for contiguous ones)
    out = (torch.empty_like(q, dtype=torch.float32) if q.is_contiguous()
           else torch.empty(q.shape, dtype=torch.float32, device=q.device))
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
    l = lib()
    if l.decode_step is not None:
        code = l.decode_step(C.addressof(p), q, k_cache, v_cache, n_valid, out, lse, ws, _stream())
    else:
        n_prob, H, D = q.shape
        code = l.decode_attention(C.addressof(p), n_prob, _ptr(q), _ptr(k_cache), _ptr(v_cache), k_cache.shape[1], _ptr(n_valid),
                                  _ptr(out), _ptr(lse), _ptr(ws), ws.numel(), _stream())
    if code != OK:
        raise SablockError(code, "sablock_decode_attention")
    return (out, lse) if want_lse else out


# ---- paged cache ------------------------------------------------------------------------------------------
def _refuse(name: str, t, dtype: torch.dtype, device, shape: Sequence[Optional[int]], how: str) -> None:
    """Says what is wrong with a tensor that an entry point could not tell from an address."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor expected, got {type(t).__name__}")
    if t.dtype != dtype or t.device != device:
        raise TypeError(f"{name}: {dtype} on {device} expected, got {t.dtype} on {t.device}")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{name}: shape {tuple(shape)} expected, got {tuple(t.shape)}")
    raise ValueError(f"{name}: {how}")


def _fits(t: torch.Tensor, dtype: torch.dtype, device, shape) -> bool:
    return t.dtype == dtype and t.device == device and t.shape == shape and t.is_contiguous()


def _token_stride(t: torch.Tensor, dtype: torch.dtype, device, n: int, heads: int, d: int) -> int:
    """Elements from token to token of a [n, heads, d] tensor whose heads are contiguous, -1 where it is none."""
    if t.dtype != dtype or t.device != device or t.shape != (n, heads, d):
        return -1
    if n and ((d > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != d) or (n > 1 and t.stride(0) == 0)):
        return -1                                  # (one token repeated: to the entry points a stride of 0 says contiguous)
    return t.stride(0) if n > 1 else 0


if hasattr(_fastcall, "token_stride"):     # (not in a module that was built before it; a build makes it anew)
    _fits, _token_stride = _fastcall.fits, _fastcall.token_stride


def _contiguous(name: str, t: torch.Tensor, dtype: torch.dtype, device, shape) -> int:
    """Address of a contiguous tensor of that type, device and shape; refuses others."""
    if not (isinstance(t, torch.Tensor) and _fits(t, dtype, device, shape)):
        _refuse(name, t, dtype, device, shape, "must be contiguous")
    return t.data_ptr()


def _scratch(pages: Pages, ws: Optional[torch.Tensor]):
    """Address and bytes of a caller's scratch (one without a storage of that size, or elsewhere, is refused), none for None."""
    if ws is None:
        return None, 0
    if not isinstance(ws, torch.Tensor):
        raise TypeError(f"ws: a tensor expected, got {type(ws).__name__}")
    if ws.device != pages._device or not ws.is_contiguous():
        raise ValueError(f"ws: a contiguous tensor on {pages._device} expected")
    return ws.data_ptr(), ws.numel()


def _tokens(name: str, t: torch.Tensor, dtype: torch.dtype, device, n: int, heads: int, d: int) -> int:
    """Token stride of a [n, heads, d] tensor whose heads are contiguous; refuses others."""
    s = _token_stride(t, dtype, device, n, heads, d) if isinstance(t, torch.Tensor) else -1
    if s < 0:
        _refuse(name, t, dtype, device, (n, heads, d), "the heads of a token must be contiguous, and tokens lie apart")
    return s


def make_pages(p: Params, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, seq_lens: torch.Tensor,
               bounds: Optional[torch.Tensor] = None) -> Pages:
    """Description of a paged cache: pools [n_pages, page_size, Hkv, D] (any strides with contiguous channels), table int32
    [n_seqs, max_pages], seq_lens int32 [n_seqs], bounds [n_pages, Hkv, 2, D] where pages are to be selected.  It refers to the
    tensors: what they hold at the time of a call counts, and they live as long as it does.  Its own fields stay as they are: other
    tensors or sizes are another description."""
    dt, dev, hkv, d = {F32: torch.float32, BF16: torch.bfloat16}[p.dtype], k_pages.device, p.n_kv_heads, p.head_dim
    for name, t, shape in (("k_pages", k_pages, (None, None, hkv, d)), ("v_pages", v_pages, (*k_pages.shape[:2], hkv, d))):
        if t.dtype != dt or t.device != dev or t.dim() != 4 or t.shape[2:] != (hkv, d) or t.shape != k_pages.shape or (d > 1 and t.stride(3) != 1):
            _refuse(name, t, dt, dev, shape, "channels must be contiguous")
        if any(t.stride(i) == 0 and t.shape[i] > 1 for i in range(3)):
            raise ValueError(f"{name}: pages, rows and heads must lie apart")       # (to the entry points a stride of 0 says contiguous)
    if table.dtype != torch.int32 or table.device != dev or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        _refuse("table", table, torch.int32, dev, (None, None), "the entries of a sequence must be contiguous")
    if table.shape[0] > 1 and table.stride(0) < table.shape[1]:
        raise ValueError("table: the sequences' entries must lie apart")
    g = Pages()
    for name, t in (("k", k_pages), ("v", v_pages)):
        setattr(g, name, t.data_ptr())
        for i, what in enumerate(("page", "row", "head")):
            setattr(g, f"{name}_stride_{what}", t.stride(i) if t.shape[i] > 1 else 0)
    g.n_pages, g.page_size = k_pages.shape[:2]
    g.n_seqs, g.max_pages = table.shape
    g.table, g.table_stride = table.data_ptr(), table.stride(0) if g.n_seqs > 1 else 0
    g.seq_lens = _contiguous("seq_lens", seq_lens, torch.int32, dev, (g.n_seqs,))
    if bounds is not None:
        g.bounds = _contiguous("bounds", bounds, dt, dev, (g.n_pages, hkv, 2, d))
    g._refs = k_pages, v_pages, table, seq_lens, bounds
    g._sizes = (p.n_q_heads, p.n_kv_heads, p.head_dim, p.dtype)
    g._dtype, g._device, g._index, g._q_shape = dt, dev, -1 if dev.index is None else dev.index, (g.n_seqs, p.n_q_heads, d)
    # what the calls' outputs and scratch look like: empty_like of a tensor costs half of an empty
    g._lse_like = torch.empty(1, device=dev).expand(g.n_seqs, p.n_q_heads)
    g._like = {}
    # what the marshalling module checks an append against (there is no stream to enqueue on without a GPU)
    g._fast = (dt, dev, g.n_seqs, hkv, p.n_q_heads, d, torch.int32, torch.float32, torch.empty_like) if dev.type == "cuda" else None
    return g


def paged_workspace_bytes(p: Params, pages: Pages, n_selected: int = -1) -> int:
    """Scratch of a call over all rows (0), of paged_sparse_attention with n_selected pages, of any call (-1)."""
    n = int(lib().sablock_paged_workspace_bytes(C.addressof(p), C.addressof(pages), n_selected))
    if n == 0:
        raise SablockError(2, "sablock_paged_workspace_bytes")
    return n


def _pages_stream(p: Params, pages: Pages) -> int:
    """torch's current stream; the parameter block has to be that of the cache and the current device the cache's (a launch goes
    to the current one)."""
    if (p.n_q_heads, p.n_kv_heads, p.head_dim, p.dtype) != pages._sizes:         # (the cache's own block too: its fields may have changed)
        raise ValueError("the parameter block is of other sizes than the one that the cache was described with")
    dev = torch._C._cuda_getDevice()
    if dev != pages._index:
        raise ValueError(f"the cache is on {pages._device}, the current device is cuda:{dev}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _check_choice(pages: Pages, n_selected: int, n_first: int, n_last: int, where: str) -> None:
    """Refuses what the entry point would, before a list of that size is allocated and the numbers are cut to 32 bits."""
    if n_selected < 1 or n_first < 0 or n_last < 0 or n_first + n_last > n_selected:
        raise SablockError(1, where)
    if n_selected * pages.page_size > 1 << 30:                                     # (rows that a sequence can have)
        raise SablockError(2, where)


def _like(p: Params, pages: Pages, n_selected: int):
    """What the scratch (None where a call needs none) and the page list of such a call look like; kept with the handle, so the block
    has been found to be the cache's (_pages_stream) before."""
    like = pages._like.get(n_selected)
    if like is None:
        n, dev = paged_workspace_bytes(p, pages, n_selected), pages._device
        like = pages._like[n_selected] = (
            torch.empty(1, dtype=torch.uint8, device=dev).expand(n) if n > 16 else None,
            torch.empty(1, dtype=torch.int32, device=dev).expand(pages.n_seqs, p.n_kv_heads, max(int(n_selected), 0)))
    return like


def paged_append(p: Params, pages: Pages, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, interleaved: bool = False,
                 cu_new: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """New tokens k, v [n, Hkv, D] become the last rows of their sequences (cu_new int32 [n_seqs + 1]: whose they are; None: one
    each), keys and queries q [n, H, D] rotated by positions * inv_freq on the way.  Returns the rotated queries; the rows of tokens that
    have no place (behind the last sequence, of an empty one, past the table) are not written, in a result made here as in q_out."""
    l, fast = lib(), pages._fast
    if l.append_step is not None and fast is not None:
        done = l.append_step(C.addressof(p), C.addressof(pages), fast, k, v, q, q_out, positions, inv_freq, interleaved, cu_new, _pages_stream(p, pages))
        if done is not NotImplemented:
            if type(done) is int:
                raise SablockError(done, "sablock_paged_append")
            return done
    # (something does not fit, or the module is not there: the same again, step by step)
    dt, dev, hkv, H, d = pages._dtype, pages._device, p.n_kv_heads, p.n_q_heads, p.head_dim
    n = k.shape[0]
    ks, vs, qs, q_at, out_at = _tokens("k", k, dt, dev, n, hkv, d), _tokens("v", v, dt, dev, n, hkv, d), 0, None, None
    if q is not None:
        qs, q_at = _tokens("q", q, dt, dev, n, H, d), q.data_ptr()
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            out_at = q_out.data_ptr()
        else:
            out_at = _contiguous("q_out", q_out, dt, dev, (n, H, d))
    elif q_out is not None:
        raise ValueError("q_out without q")
    pos_at = None if positions is None else _contiguous("positions", positions, torch.int32, dev, (n,))
    freq_at, rotary = None, 0
    if inv_freq is not None:
        rotary = 2 * inv_freq.shape[0]
        freq_at = _contiguous("inv_freq", inv_freq, torch.float32, dev, (rotary // 2,))
    cu_at = None if cu_new is None else _contiguous("cu_new", cu_new, torch.int32, dev, (pages.n_seqs + 1,))
    code = l.paged_append(C.addressof(p), C.addressof(pages), n, cu_at, k.data_ptr(), ks, v.data_ptr(), vs, q_at, qs, out_at, pos_at,
                              freq_at, rotary, 1 if interleaved else 0, _pages_stream(p, pages))
    if code != OK:
        raise SablockError(code, "sablock_paged_append")
    return q_out


def paged_attention(p: Params, pages: Pages, q: torch.Tensor, selected: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, want_lse: bool = False):
    """Attention of one new token per sequence, q [n_seqs, H, D], over the rows of its pages, or over the pages selected int32
    [n_seqs, Hkv, n], n > 0.  Returns out f32 [n_seqs, H, D] (and lse [n_seqs, H])."""
    q_at = _contiguous("q", q, pages._dtype, pages._device, pages._q_shape)
    sel_at, n = None, 0
    if selected is not None:
        n = selected.shape[-1]
        sel_at = _contiguous("selected", selected, torch.int32, pages._device, (pages.n_seqs, p.n_kv_heads, n))
        if n == 0:                                 # (without an address it would say all rows)
            raise SablockError(1, "sablock_paged_attention")
    stream = _pages_stream(p, pages)
    out = torch.empty_like(q, dtype=torch.float32)
    lse = torch.empty_like(pages._lse_like) if want_lse else None
    if ws is None:
        like = _like(p, pages, 0 if selected is None else -1)[0]
        ws = None if like is None else torch.empty_like(like)
    ws_at, ws_bytes = _scratch(pages, ws)
    code = lib().paged_attention(C.addressof(p), C.addressof(pages), q_at, sel_at, n, out.data_ptr(), lse.data_ptr() if want_lse else None,
                                 ws_at, ws_bytes, stream)
    if code != OK:
        raise SablockError(code, "sablock_paged_attention")
    return (out, lse) if want_lse else out


def page_select(p: Params, pages: Pages, q: torch.Tensor, n_selected: int, n_first: int = 1, n_last: int = 1) -> torch.Tensor:
    """The pages whose bounds promise the largest logits, per KV head: int32 [n_seqs, Hkv, n_selected], ascending, then -1."""
    q_at = _contiguous("q", q, pages._dtype, pages._device, pages._q_shape)
    _check_choice(pages, n_selected, n_first, n_last, "sablock_page_select")
    stream = _pages_stream(p, pages)
    selected = torch.empty_like(_like(p, pages, n_selected)[1])
    _check(lib().page_select(C.addressof(p), C.addressof(pages), q_at, n_selected, n_first, n_last, _ptr(selected), stream),
           "sablock_page_select")
    return selected


def paged_sparse_attention(p: Params, pages: Pages, q: torch.Tensor, n_selected: int, n_first: int = 1, n_last: int = 1,
                           ws: Optional[torch.Tensor] = None, want_lse: bool = False):
    """page_select and paged_attention over what it selects.  Returns (out, selected), and lse behind them."""
    q_at = _contiguous("q", q, pages._dtype, pages._device, pages._q_shape)
    _check_choice(pages, n_selected, n_first, n_last, "sablock_paged_sparse_attention")
    stream = _pages_stream(p, pages)
    out = torch.empty_like(q, dtype=torch.float32)
    lse = torch.empty_like(pages._lse_like) if want_lse else None
    ws_like, sel_like = _like(p, pages, n_selected)
    selected = torch.empty_like(sel_like)
    if ws is None and ws_like is not None:
        ws = torch.empty_like(ws_like)
    ws_at, ws_bytes = _scratch(pages, ws)
    code = lib().paged_sparse_attention(C.addressof(p), C.addressof(pages), q_at, n_selected, n_first, n_last, selected.data_ptr(),
                                        out.data_ptr(), lse.data_ptr() if want_lse else None, ws_at, ws_bytes, stream)
    if code != OK:
        raise SablockError(code, "sablock_paged_sparse_attention")
    return (out, selected, lse) if want_lse else (out, selected)
