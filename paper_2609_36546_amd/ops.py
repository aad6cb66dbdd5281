"""Thin ctypes binding of libipdv.so (argument marshalling only).

Every function takes device tensors, checks dtype / device / contiguity /
shape, passes raw pointers and the current HIP stream to the C ABI of the
same name, and raises RuntimeError with the library's message on a non-OK
status.  All arithmetic runs in the library's gfx950 kernels; there is no
other path.  Outputs and workspaces can be passed in (to keep a call free of
allocations) or are allocated here with torch.  No call is recorded by
autograd, whether its inputs require gradients or not: a gradient is a call of
its own (rope_window's with inverse=True).
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libipdv.so")

IPDV_F32 = 0
IPDV_BF16 = 1
MAX_K = 32

_lib = None


class IpdvError(RuntimeError):
    def __init__(self, func: str, status: int, msg: str):
        super().__init__(f"{func} failed with status {status}: {msg}")
        self.status = status


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2609_36546_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, u8p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        ci, cf, cs = ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.ipdv_attn_workspace_size.argtypes = [ci] * 7
        L.ipdv_attn_workspace_size.restype = cs
        L.verify_attn_paged.argtypes = [vp, vp, vp, vp, vp, i32p, ci, i32p, i32p, i32p, ci, ci, vp,
                                        ci, ci, ci, ci, ci, cf, ci, vp, cs, vp]
        L.verify_attn_paged.restype = ci
        L.ipdv_lmhead_workspace_size.argtypes = [ci] * 4
        L.ipdv_lmhead_workspace_size.restype = cs
        L.ipdv_workspace_size.argtypes = [ci, ctypes.POINTER(ctypes.c_int32), ci]
        L.ipdv_workspace_size.restype = cs
        L.ipdv_check_page_table.argtypes = [vp, ci, ci, vp, vp, vp, ci, ci, ci, ci,
                                            ctypes.POINTER(ctypes.c_int32)]
        L.ipdv_check_page_table.restype = ci
        L.verify_attn_paged_noalloc.argtypes = [vp, vp, vp, vp, vp, i32p, ci, i32p, i32p, i32p, ci,
                                                ci, vp, ci, ci, ci, ci, ci, cf, ci, vp]
        L.verify_attn_paged_noalloc.restype = ci
        L.lmhead_logsoftmax_verify.argtypes = [vp, vp, i32p, i32p, ci, ci, ci, ci, f32p, f32p, i32p,
                                               i32p, f32p, f32p, ci, vp, cs, vp]
        L.lmhead_logsoftmax_verify.restype = ci
        L.accept_scan.argtypes = [i32p, i32p, i32p, ci, u8p, i32p, i32p, ctypes.c_int32,
                                  ctypes.c_int32, ci, i32p, i32p, u8p, u8p, i32p, u8p, vp]
        L.accept_scan.restype = ci
        L.accept_scan_rule.argtypes = [i32p, i32p, i32p, ci, u8p, i32p, i32p, ctypes.c_int32,
                                       ctypes.c_int32, ci, ci, ci, f32p, ctypes.c_float,
                                       ctypes.c_float, i32p, i32p, u8p, u8p, i32p, u8p, vp]
        L.accept_scan_rule.restype = ci
        L.lmhead_sample.argtypes = [vp, vp, ci, ci, ci, ci, vp, cs, f32p, i32p, ci, vp]
        L.lmhead_sample.restype = ci
        L.ipdv_lmhead_packed_w_size.argtypes = [ci, ci]
        L.ipdv_lmhead_packed_w_size.restype = cs
        L.lmhead_pack_w.argtypes = [vp, ci, ci, vp, ci, vp]
        L.lmhead_pack_w.restype = ci
        L.lmhead_logp_gather.argtypes = [vp, vp, ci, ci, ci, f32p, i32p, ci, f32p, ci, vp]
        L.lmhead_logp_gather.restype = ci
        L.source_split_kl.argtypes = [ci, ci, i32p, f32p, f32p, i32p, f32p, f32p, u8p, ci, ci,
                                      f32p, f32p, f32p, f32p, i32p, ci, f32p, f32p, vp]
        L.source_split_kl.restype = ci
        L.sample_takeover.argtypes = [vp, vp, ci, ci, ci, ci, vp, cs, i32p, ci, i32p, u8p, i32p,
                                      i32p, f32p, ctypes.c_int32, i32p, u8p, ci, vp]
        L.sample_takeover.restype = ci
        i64, cd = ctypes.c_int64, ctypes.c_double
        L.ipdv_rope_inv_freq.argtypes = [ci, cd, ci, cd, ci, cd, cd, vp, ctypes.POINTER(cf)]
        L.ipdv_rope_inv_freq.restype = ci
        L.rope_window.argtypes = ([vp, i64] * 4 + [f32p, i32p, i32p, i32p] + [ci] * 7 +
                                  [cf, ci, ci, vp])
        L.rope_window.restype = ci
        L.kv_append_q8.argtypes = [vp, i64, vp, i64, vp, vp, vp, i32p, ci, i32p, i32p, i32p,
                                   ci, ci, ci, ci, ci, ci, ci, vp]
        L.kv_append_q8.restype = ci
        L.kv_read_q8.argtypes = [vp, vp, vp, i32p, ci, i32p, i32p, i32p, ci, ci, vp, vp,
                                 ci, ci, ci, ci, ci, vp]
        L.kv_read_q8.restype = ci
        L.ipdv_attn_q8_workspace_size.argtypes = [ci] * 5
        L.ipdv_attn_q8_workspace_size.restype = cs
        L.verify_attn_q8.argtypes = [vp, i64, vp, vp, vp, i32p, ci, i32p, i32p, i32p, ci, ci, vp,
                                     ci, ci, ci, ci, ci, cf, ci, vp, cs, vp]
        L.verify_attn_q8.restype = ci
        L.ipdv_sample_logits_workspace_size.argtypes = [ci, ci]
        L.ipdv_sample_logits_workspace_size.restype = cs
        L.sample_logits.argtypes = [vp, i64, ci, ci, f32p, f32p, i32p, f32p, f32p, i32p, f32p, ci,
                                    vp, cs, vp]
        L.sample_logits.restype = ci
        L.ipdv_attn_masked_workspace_size.argtypes = [ci] * 9
        L.ipdv_attn_masked_workspace_size.restype = cs
        L.verify_attn_masked.argtypes = [vp, i64, vp, vp, vp, vp, i32p, ci, i32p, i32p, i32p, ci, ci,
                                         cf, ci, f32p, i32p, i32p, vp, f32p, ci, ci, ci, ci, ci, cf,
                                         ci, vp, cs, vp]
        L.verify_attn_masked.restype = ci
        L.attn_mass.argtypes = [vp, i64, vp, f32p, i32p, ci, i32p, i32p, i32p, ci, ci, cf, ci, f32p,
                                i32p, i32p, f32p, cf, f32p, ci, ci, ci, ci, ci, cf, ci, vp]
        L.attn_mass.restype = ci
        L.kv_evict.argtypes = [vp, vp, f32p, i32p, ci, i32p, ci, i32p, i32p, i32p, ci, ci, ci, i32p,
                               i32p, ci, ci, ci, ci, ci, vp]
        L.kv_evict.restype = ci
        L.ipdv_verify_drafts_workspace_size.argtypes = [ci] * 5
        L.ipdv_verify_drafts_workspace_size.restype = cs
        L.verify_drafts.argtypes = ([vp, i64, vp, i64, ci, ci, i32p, i32p, ci, f32p, f32p] +
                                    [f32p, i32p, f32p, f32p] * 2 +
                                    [ctypes.c_int32, i32p, i32p, u8p, f32p, f32p, ci, vp, cs, vp])
        L.verify_drafts.restype = ci
        L.ipdv_trace_events.argtypes = [ctypes.c_void_p, ci]
        L.ipdv_trace_events.restype = ci
        L.ipdv_trace_count.restype = ci
        L.ipdv_last_error.restype = ctypes.c_char_p
        L.ipdv_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(func: str, status: int):
    if status != 0:
        raise IpdvError(func, status, lib().ipdv_last_error().decode())


# The calls below take 5-10 us on the device at their smallest, so their host
# side counts: pointers go to ctypes as plain integers, the stream handle comes
# without a Stream object, a tensor that passes every check does so in one
# expression, and the workspace size is queried only to allocate one (the
# library checks what it is given).  Host time of one attention call 17.7 us
# before, 12.8 after; of the smallest verify step 72.7 and 55.8.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: torch.device):
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _need(t: torch.Tensor, name: str, dtype=None, device=None, ndim=None):
    try:
        if (t.is_cuda and t.dtype is dtype and t.device == device and t.dim() == ndim
                and t.is_contiguous() and isinstance(t, torch.Tensor)):
            return
    except AttributeError:
        pass                      # not a tensor: named below
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device} (is on {t.device})")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (is {t.dtype})")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims (has {t.dim()})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return IPDV_BF16
    if dt == torch.float32:
        return IPDV_F32
    raise ValueError(f"unsupported dtype {dt}")


def trace_events(events) -> None:
    """Bracket every kernel the library launches with these torch.cuda.Event
    objects (in order; see ipdv_trace_events).  None turns tracing off."""
    global _trace_keep
    if not events:
        lib().ipdv_trace_events(None, 0)
        _trace_keep = None
        return
    for e in events:            # torch creates the HIP event on first record
        if e.cuda_event == 0:
            e.record()
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _trace_keep = arr
    lib().ipdv_trace_events(ctypes.cast(arr, ctypes.c_void_p), len(events))


def trace_count() -> int:
    return int(lib().ipdv_trace_count())


_trace_keep = None


def version() -> str:
    return lib().ipdv_version().decode()


# ---------------------------------------------------------------------------

def attn_workspace_size(n_seq, Hq, Hkv, D, max_q, max_pages, page_size) -> int:
    return int(lib().ipdv_attn_workspace_size(n_seq, Hq, Hkv, D, max_q, max_pages, page_size))


def check_page_table(page_table, ctx_lens, cu_q, max_q: int, page_size: int, num_pages: int,
                     seq_ids=None, n_seq: Optional[int] = None, rows: Optional[int] = None,
                     writes: bool = True):
    """ipdv_check_page_table on host copies of the arrays (tensors on any
    device, or numpy arrays).  Raises IpdvError naming the first contract
    violation; returns None when the table is valid.  rows: the rows that the
    window tensors hold, which the handled windows must not pass.  writes=False
    is for calls that only read the pages: windows may share them."""
    import numpy as np

    def host(x):
        if isinstance(x, torch.Tensor):
            x = x.detach().cpu().numpy()
        return np.ascontiguousarray(np.asarray(x, np.int32))

    pt, ctx, cu = host(page_table), host(ctx_lens), host(cu_q)
    sid = None if seq_ids is None else host(seq_ids)
    B = ctx.shape[0]
    if pt.ndim != 2 or pt.shape[0] != B or cu.shape[0] != B + 1:
        raise ValueError("page_table must be [B, maxp] and cu_q [B+1]")
    if n_seq is None:
        n_seq = B if sid is None else sid.shape[0]
    ids = np.arange(n_seq) if sid is None else sid[:n_seq]
    ids = ids[(ids >= 0) & (ids < B)]               # others are named by the library
    k = np.diff(cu.astype(np.int64))
    if not writes and B > 0 and cu[0] == 0 and (k >= 0).all() and (ctx[ids] >= 0).all() and (k[ids] <= max_q).all():
        # the same positions with no window among them
        end = ctx.astype(np.int64) + k
        ctx = np.ascontiguousarray(np.minimum(end, 2 ** 31 - 1).astype(np.int32))
        cu_read = np.zeros(B + 1, np.int32)
    else:
        cu_read = cu
    p = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)
    bad = ctypes.c_int32(-1)
    st = lib().ipdv_check_page_table(p(pt), B, pt.shape[1], p(ctx), p(cu_read), p(sid), n_seq, max_q,
                                     page_size, num_pages, ctypes.byref(bad))
    _check("ipdv_check_page_table", st)
    if rows is not None:
        for b in ids:
            if k[b] > 0 and cu[b + 1] > rows:
                raise IpdvError("check_page_table", -1, f"sequence {b}: rows {cu[b]} .. {cu[b + 1] - 1} of {rows}")


def verify_attn_paged(q, k_new, v_new, k_cache, v_cache, page_table, ctx_lens, cu_q,
                      max_q: int, seq_ids=None, n_seq: Optional[int] = None,
                      scale: Optional[float] = None, out=None, workspace=None,
                      validate: bool = False):
    """Append the window to the paged cache and attend (see include/ipdv.h).

    q [T,Hq,D], k_new/v_new [T,Hkv,D], k_cache [P,Hkv,D/32,ps,32], v_cache [P,Hkv,D,ps]
    (bf16 or fp32), page_table [B,maxp] int32, ctx_lens [B] int32, cu_q [B+1]
    int32, seq_ids [n] int32 or None.  Returns out [T,Hq,D].  validate=True
    first runs check_page_table on host copies (a device-to-host copy and a
    synchronisation; for debugging).
    """
    dev = q.device
    dt = q.dtype
    _need(q, "q", dt, dev, 3)
    T, Hq, D = q.shape
    _need(k_new, "k_new", dt, dev, 3)
    _need(v_new, "v_new", dt, dev, 3)
    Hkv = k_new.shape[1]
    _need(k_cache, "k_cache", dt, dev, 5)
    _need(v_cache, "v_cache", dt, dev, 4)
    P, ps = k_cache.shape[0], k_cache.shape[3]
    if k_cache.shape != (P, Hkv, D // 32, ps, 32) or v_cache.shape != (P, Hkv, D, ps):
        raise ValueError("k_cache must be [P,Hkv,D/32,ps,32] and v_cache [P,Hkv,D,ps]")
    if k_new.shape != (T, Hkv, D) or v_new.shape != (T, Hkv, D):
        raise ValueError("k_new / v_new must be [T,Hkv,D]")
    _need(page_table, "page_table", torch.int32, dev, 2)
    _need(ctx_lens, "ctx_lens", torch.int32, dev, 1)
    _need(cu_q, "cu_q", torch.int32, dev, 1)
    B = ctx_lens.shape[0]
    if cu_q.shape[0] != B + 1 or page_table.shape[0] != B:
        raise ValueError("cu_q must be [B+1] and page_table [B, maxp]")
    if seq_ids is not None:
        _need(seq_ids, "seq_ids", torch.int32, dev, 1)
        n_seq = seq_ids.shape[0] if n_seq is None else n_seq
    elif n_seq is None:
        n_seq = B
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", dt, dev, 3)
    maxp = page_table.shape[1]
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, ps, P, seq_ids=seq_ids, n_seq=n_seq)
    if workspace is None:
        need = attn_workspace_size(n_seq, Hq, Hkv, D, max_q, maxp, ps)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().verify_attn_paged(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
        maxp, _ptr(ctx_lens), _ptr(cu_q), _ptr(seq_ids), n_seq, max_q, _ptr(out),
        Hq, Hkv, D, ps, P, float(scale), _dtype_code(dt), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(dev))
    _check("verify_attn_paged", st)
    return out


NOALLOC_SCRATCH_BYTES = 128 << 20


def verify_attn_paged_noalloc(q, k_new, v_new, k_cache, v_cache, page_table, ctx_lens, cu_q,
                              max_q: int, seq_ids=None, n_seq: Optional[int] = None,
                              scale: Optional[float] = None, out=None):
    """verify_attn_paged_noalloc (see include/ipdv.h): verify_attn_paged with
    its split-KV partials in the library's per-device scratch.  Allocates
    nothing when `out` is given."""
    dev = q.device
    dt = q.dtype
    _need(q, "q", dt, dev, 3)
    T, Hq, D = q.shape
    _need(k_new, "k_new", dt, dev, 3)
    _need(v_new, "v_new", dt, dev, 3)
    Hkv = k_new.shape[1]
    _need(k_cache, "k_cache", dt, dev, 5)
    _need(v_cache, "v_cache", dt, dev, 4)
    P, ps = k_cache.shape[0], k_cache.shape[3]
    if k_cache.shape != (P, Hkv, D // 32, ps, 32) or v_cache.shape != (P, Hkv, D, ps):
        raise ValueError("k_cache must be [P,Hkv,D/32,ps,32] and v_cache [P,Hkv,D,ps]")
    if k_new.shape != (T, Hkv, D) or v_new.shape != (T, Hkv, D):
        raise ValueError("k_new / v_new must be [T,Hkv,D]")
    _need(page_table, "page_table", torch.int32, dev, 2)
    _need(ctx_lens, "ctx_lens", torch.int32, dev, 1)
    _need(cu_q, "cu_q", torch.int32, dev, 1)
    B = ctx_lens.shape[0]
    if cu_q.shape[0] != B + 1 or page_table.shape[0] != B:
        raise ValueError("cu_q must be [B+1] and page_table [B, maxp]")
    if seq_ids is not None:
        _need(seq_ids, "seq_ids", torch.int32, dev, 1)
        n_seq = seq_ids.shape[0] if n_seq is None else n_seq
    elif n_seq is None:
        n_seq = B
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", dt, dev, 3)
    st = lib().verify_attn_paged_noalloc(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
        page_table.shape[1], _ptr(ctx_lens), _ptr(cu_q), _ptr(seq_ids), n_seq, max_q, _ptr(out),
        Hq, Hkv, D, ps, P, float(scale), _dtype_code(dt), _stream(dev))
    _check("verify_attn_paged_noalloc", st)
    return out


def lmhead_workspace_size(M, Hd, V, K) -> int:
    return int(lib().ipdv_lmhead_workspace_size(M, Hd, V, K))


W_TILED = 0x10


class PackedW:
    """The LM-head weight in the tiled layout written by lmhead_pack_w (see
    include/ipdv.h): ``data`` is the flat bf16 buffer; ``V`` and ``Hd`` the
    logical shape.  Accepted wherever a row-major W is."""

    def __init__(self, data, V: int, Hd: int):
        self.data, self.V, self.Hd = data, int(V), int(Hd)

    @property
    def device(self):
        return self.data.device

    @property
    def dtype(self):
        return self.data.dtype


def lmhead_pack_w(W) -> PackedW:
    """Repack a row-major bf16 W [V, Hd] into the tiled layout (one launch)."""
    dev = W.device
    _need(W, "W", torch.bfloat16, dev, 2)
    V, Hd = W.shape
    n = int(lib().ipdv_lmhead_packed_w_size(V, Hd))
    if n == 0:
        raise ValueError(f"unsupported LM-head shape V={V} Hd={Hd}")
    data = torch.empty(n // 2, dtype=torch.bfloat16, device=dev)
    st = lib().lmhead_pack_w(_ptr(W), V, Hd, _ptr(data), _dtype_code(torch.bfloat16), _stream(dev))
    _check("lmhead_pack_w", st)
    return PackedW(data, V, Hd)


def _w_arg(W, dt, dev, Hd):
    """(pointer, V, dtype code) for a row-major W [V, Hd] or a PackedW."""
    if isinstance(W, PackedW):
        if W.dtype != torch.bfloat16 or dt != torch.bfloat16:
            raise ValueError("a packed W needs bf16 hidden rows and weights")
        if W.device != dev:
            raise ValueError(f"W must be on {dev}")
        if W.Hd != Hd:
            raise ValueError("packed W has another hidden size")
        return _ptr(W.data), W.V, _dtype_code(dt) | W_TILED
    _need(W, "W", dt, dev, 2)
    if W.shape[1] != Hd:
        raise ValueError("W must be [V, Hd]")
    return _ptr(W), W.shape[0], _dtype_code(dt)


def lmhead_logsoftmax_verify(hidden, W, prop_tok, K: int, out_rows=None, n_out_rows=None,
                             with_entropy: bool = True, outs=None, workspace=None):
    """Verifier log-softmax outputs for each row (see include/ipdv.h).

    hidden [M,Hd], W [V,Hd] (bf16 or fp32), prop_tok [M] int32, out_rows [M]
    int32 or None.  Returns dict lse, logp_prop, argmax, topk_idx, topk_logp,
    entropy (rows = n_out_rows if out_rows is given, else M).
    """
    dev = hidden.device
    dt = hidden.dtype
    _need(hidden, "hidden", dt, dev, 2)
    M, Hd = hidden.shape
    w_ptr, V, code = _w_arg(W, dt, dev, Hd)
    _need(prop_tok, "prop_tok", torch.int32, dev, 1)
    if prop_tok.shape[0] != M:
        raise ValueError("prop_tok must be [M]")
    if out_rows is not None:
        _need(out_rows, "out_rows", torch.int32, dev, 1)
        R = int(n_out_rows)
    else:
        R = M
    if outs is None:
        outs = {
            "lse": torch.empty(R, dtype=torch.float32, device=dev),
            "logp_prop": torch.empty(R, dtype=torch.float32, device=dev),
            "argmax": torch.empty(R, dtype=torch.int32, device=dev),
            "topk_idx": torch.empty(R, K, dtype=torch.int32, device=dev),
            "topk_logp": torch.empty(R, K, dtype=torch.float32, device=dev),
            "entropy": torch.empty(R, dtype=torch.float32, device=dev) if with_entropy else None,
        }
    if workspace is None:
        need = lmhead_workspace_size(M, Hd, V, K)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().lmhead_logsoftmax_verify(
        _ptr(hidden), w_ptr, _ptr(prop_tok), _ptr(out_rows), M, Hd, V, K,
        _ptr(outs["lse"]), _ptr(outs["logp_prop"]), _ptr(outs["argmax"]), _ptr(outs["topk_idx"]),
        _ptr(outs["topk_logp"]), _ptr(outs["entropy"]), code, _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(dev))
    _check("lmhead_logsoftmax_verify", st)
    return outs


TAKE_COVERAGE, TAKE_ENTROPY = 0, 1
HAND_COVERAGE, HAND_FIXED_ONE, HAND_ENTROPY = 0, 1, 2


def _scan_args(cu_q, prop_tok, topk_idx, K, driver, ctx_lens, seq_lens, ent, uses_ent, outs):
    """Checks the verdict inputs and allocates the outputs when none are given."""
    dev = cu_q.device
    _need(cu_q, "cu_q", torch.int32, dev, 1)
    B = cu_q.shape[0] - 1
    _need(prop_tok, "prop_tok", torch.int32, dev, 1)
    T = prop_tok.shape[0]
    if uses_ent:
        _need(ent, "ent", torch.float32, dev, 1)
        if ent.shape[0] != T:
            raise ValueError("ent must be [T]")
    if K > 0 and topk_idx is not None:
        _need(topk_idx, "topk_idx", torch.int32, dev, 2)
        if topk_idx.shape[0] != T or topk_idx.shape[1] != K:
            raise ValueError("topk_idx must be [T, K]")
    _need(driver, "driver", torch.uint8, dev, 1)
    _need(ctx_lens, "ctx_lens", torch.int32, dev, 1)
    _need(seq_lens, "seq_lens", torch.int32, dev, 1)
    if outs is None:
        outs = {
            "n_acc": torch.empty(B, dtype=torch.int32, device=dev),
            "event_row": torch.empty(B, dtype=torch.int32, device=dev),
            "next_driver": torch.empty(B, dtype=torch.uint8, device=dev),
            "finished": torch.empty(B, dtype=torch.uint8, device=dev),
            "new_cache_len": torch.empty(B, dtype=torch.int32, device=dev),
            "src": torch.empty(T, dtype=torch.uint8, device=dev),
        }
    tk = _ptr(topk_idx) if (K > 0 and topk_idx is not None) else None
    return dev, B, tk, outs


def _scan_outs(outs):
    return (_ptr(outs["n_acc"]), _ptr(outs["event_row"]), _ptr(outs["next_driver"]),
            _ptr(outs["finished"]), _ptr(outs["new_cache_len"]), _ptr(outs["src"]))


def accept_scan(cu_q, prop_tok, topk_idx, K: int, driver, ctx_lens, seq_lens, eos_id: int,
                max_len: int, outs=None):
    """Verdict for each sequence's window (see include/ipdv.h).  Returns dict
    n_acc, event_row, next_driver, finished, new_cache_len, src."""
    dev, B, tk, outs = _scan_args(cu_q, prop_tok, topk_idx, K, driver, ctx_lens, seq_lens, None,
                                  False, outs)
    st = lib().accept_scan(_ptr(cu_q), _ptr(prop_tok), tk, K, _ptr(driver), _ptr(ctx_lens),
                           _ptr(seq_lens), int(eos_id), int(max_len), B, *_scan_outs(outs),
                           _stream(dev))
    _check("accept_scan", st)
    return outs


def accept_scan_rule(cu_q, prop_tok, topk_idx, K: int, driver, ctx_lens, seq_lens, eos_id: int,
                     max_len: int, take_rule: int = TAKE_COVERAGE, hand_rule: int = HAND_COVERAGE,
                     ent=None, tau_take: float = 0.0, tau_hand: float = 0.0, outs=None):
    """Verdict with the takeover / handback rule variants (see
    include/ipdv.h, accept_scan_rule).  ``ent`` is a [T] float32 entropy per
    row, needed by the entropy rules."""
    uses_ent = take_rule == TAKE_ENTROPY or hand_rule == HAND_ENTROPY
    dev, B, tk, outs = _scan_args(cu_q, prop_tok, topk_idx, K, driver, ctx_lens, seq_lens, ent,
                                  uses_ent, outs)
    st = lib().accept_scan_rule(
        _ptr(cu_q), _ptr(prop_tok), tk, K, _ptr(driver), _ptr(ctx_lens), _ptr(seq_lens),
        int(eos_id), int(max_len), B, int(take_rule), int(hand_rule),
        _ptr(ent) if uses_ent else None, float(tau_take), float(tau_hand), *_scan_outs(outs),
        _stream(dev))
    _check("accept_scan_rule", st)
    return outs


def sample_takeover(hidden, W, K: int, workspace, cu_q, driver, event_row, u, eos_id: int,
                    finished, row_local=None, seq_ids=None, token=None):
    """Teacher replacement tokens at the takeovers (see include/ipdv.h).

    hidden, W, K and workspace as passed to the preceding
    lmhead_logsoftmax_verify call (its records are read); cu_q [B+1] int32,
    driver [B] uint8, event_row [B] int32 (accept_scan's), u [B] float32
    uniforms in [0, 1), row_local [T] int32 or None, seq_ids [n] int32 or None
    (the sequences handled; None: all B), finished [B] uint8 (updated in
    place).  Returns token [B] int32 (-1: no draw; entries of sequences not
    handled are left as they were in `token`)."""
    dev = hidden.device
    dt = hidden.dtype
    _need(hidden, "hidden", dt, dev, 2)
    M, Hd = hidden.shape
    w_ptr, V, code = _w_arg(W, dt, dev, Hd)
    _need(cu_q, "cu_q", torch.int32, dev, 1)
    B = cu_q.shape[0] - 1
    _need(driver, "driver", torch.uint8, dev, 1)
    _need(event_row, "event_row", torch.int32, dev, 1)
    _need(u, "u", torch.float32, dev, 1)
    _need(finished, "finished", torch.uint8, dev, 1)
    if row_local is not None:
        _need(row_local, "row_local", torch.int32, dev, 1)
    n_seq = B
    if seq_ids is not None:
        _need(seq_ids, "seq_ids", torch.int32, dev, 1)
        n_seq = seq_ids.shape[0]
    if token is None:
        # every entry is written unless only some sequences are handled
        token = (torch.empty(B, dtype=torch.int32, device=dev) if seq_ids is None
                 else torch.full((B,), -1, dtype=torch.int32, device=dev))
    st = lib().sample_takeover(
        _ptr(hidden), w_ptr, M, Hd, V, K, _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(seq_ids), n_seq, _ptr(cu_q),
        _ptr(driver), _ptr(event_row), _ptr(row_local), _ptr(u), int(eos_id), _ptr(token),
        _ptr(finished), code, _stream(dev))
    _check("sample_takeover", st)
    return token


def lmhead_logp_gather(hidden, W, lse, idx, out=None):
    """log-softmax of hidden . W^T at idx [M, n] (see include/ipdv.h);
    lse [M] float32 from the same model's lmhead_logsoftmax_verify.  Returns
    logp [M, n] float32 (-inf for indices outside [0, V))."""
    dev = hidden.device
    dt = hidden.dtype
    _need(hidden, "hidden", dt, dev, 2)
    M, Hd = hidden.shape
    w_ptr, V, code = _w_arg(W, dt, dev, Hd)
    _need(lse, "lse", torch.float32, dev, 1)
    _need(idx, "idx", torch.int32, dev, 2)
    if lse.shape[0] != M or idx.shape[0] != M:
        raise ValueError("lse and idx must have M rows")
    n = idx.shape[1]
    if out is None:
        out = torch.empty(M, n, dtype=torch.float32, device=dev)
    st = lib().lmhead_logp_gather(_ptr(hidden), w_ptr, M, Hd, V, _ptr(lse), _ptr(idx), n,
                                  _ptr(out), code, _stream(dev))
    _check("lmhead_logp_gather", st)
    return out


SUPPORT_UNION, SUPPORT_STUDENT, SUPPORT_TEACHER, SUPPORT_INTERSECTION = 0, 1, 2, 3
LOSS_IPD_SPLIT, LOSS_PURE_REVERSE, LOSS_PURE_FORWARD, LOSS_INVERSE_SPLIT = 0, 1, 2, 3


def source_split_kl(s_idx, s_logp, s_at_t, t_idx, t_logp, t_at_s, src, support=SUPPORT_UNION,
                    loss_mode=LOSS_IPD_SPLIT, cu=None):
    """Per-position source-split KL values (see include/ipdv.h).  Inputs
    [M, K] (int32 indices, float32 log-probs) and src [M] uint8; cu [B+1]
    int32 segment offsets or None.  Returns dict kl_rev, kl_fwd, loss,
    overlap [M] and, with cu, seq_loss, t_ratio [B] (float32)."""
    dev = s_idx.device
    for t, name, dt in ((s_idx, "s_idx", torch.int32), (t_idx, "t_idx", torch.int32),
                        (s_logp, "s_logp", torch.float32), (s_at_t, "s_at_t", torch.float32),
                        (t_logp, "t_logp", torch.float32), (t_at_s, "t_at_s", torch.float32)):
        _need(t, name, dt, dev, 2)
    M, K = s_idx.shape
    for t in (s_logp, s_at_t, t_idx, t_logp, t_at_s):
        if t.shape != (M, K):
            raise ValueError("every list input must be [M, K]")
    _need(src, "src", torch.uint8, dev, 1)
    if src.shape[0] != M:
        raise ValueError("src must be [M]")
    out = {k: torch.empty(M, dtype=torch.float32, device=dev)
           for k in ("kl_rev", "kl_fwd", "loss", "overlap")}
    B = 0
    if cu is not None:
        _need(cu, "cu", torch.int32, dev, 1)
        B = cu.shape[0] - 1
        out["seq_loss"] = torch.empty(B, dtype=torch.float32, device=dev)
        out["t_ratio"] = torch.empty(B, dtype=torch.float32, device=dev)
    st = lib().source_split_kl(
        M, K, _ptr(s_idx), _ptr(s_logp), _ptr(s_at_t), _ptr(t_idx), _ptr(t_logp), _ptr(t_at_s),
        _ptr(src), int(support), int(loss_mode), _ptr(out["kl_rev"]), _ptr(out["kl_fwd"]),
        _ptr(out["loss"]), _ptr(out["overlap"]), _ptr(cu), B, _ptr(out.get("seq_loss")),
        _ptr(out.get("t_ratio")), _stream(dev))
    _check("source_split_kl", st)
    return out


def lmhead_sample(hidden, W, K: int, workspace, u, token=None):
    """One temperature-1 draw per row (see include/ipdv.h): hidden, W, K and
    workspace as passed to the preceding lmhead_logsoftmax_verify call; u [M]
    float32 uniforms in [0, 1).  Returns token [M] int32."""
    dev = hidden.device
    dt = hidden.dtype
    _need(hidden, "hidden", dt, dev, 2)
    M, Hd = hidden.shape
    w_ptr, V, code = _w_arg(W, dt, dev, Hd)
    _need(u, "u", torch.float32, dev, 1)
    if u.shape[0] != M:
        raise ValueError("u must be [M]")
    if token is None:
        token = torch.empty(M, dtype=torch.int32, device=dev)
    st = lib().lmhead_sample(_ptr(hidden), w_ptr, M, Hd, V, K, _ptr(workspace),
                             workspace.numel() * workspace.element_size(), _ptr(u), _ptr(token),
                             code, _stream(dev))
    _check("lmhead_sample", st)
    return token


# ---------------------------------------------------------------------------
# The 8-bit cache and what stands around it: rotary positions, the quantised
# append and its read-back, attention over it, filtered draws from logits.

ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_YARN = 0, 1, 2, 3


# The calls from here on check a tensor and give its address in one go: two of
# them make up a step of 8 us on the device, so each check that is made twice, or
# through an object that is built for it, shows.
def _at(t: torch.Tensor, name: str, dtype, dev, ndim: int) -> int:
    """_need, and the address."""
    try:
        if (t.dtype is dtype and t.get_device() == dev.index and t.dim() == ndim
                and t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass                          # not a tensor: named below
    _need(t, name, dtype, dev, ndim)
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, dtype, dev, ndim: int):
    """Like _at, but rows (dim 0) may lie further apart than they are long, as in
    a slice of a wider projection.  Returns the address, the row stride in
    elements and the shape."""
    try:
        if t.dtype is dtype and t.get_device() == dev.index:
            size, step = t.shape, t.stride()
            if len(size) == ndim and size[0] > 1 and step[-1] == 1 and (ndim == 2 or step[1] == size[2]):
                return t.data_ptr(), step[0], size    # a stride shorter than the row is refused by the library
    except AttributeError:
        pass                          # not a tensor: named below
    if isinstance(t, torch.Tensor) and t.dim() == ndim and t.shape[0] > 0 and not t.is_contiguous():
        _need(t[0], name, dtype, dev, ndim - 1)
        if t.shape[0] > 1:
            return t.data_ptr(), t.stride(0), t.shape
    else:
        _need(t, name, dtype, dev, ndim)
    n = 1
    for s in t.shape[1:]:
        n *= s
    return t.data_ptr(), n, t.shape


def _given_workspace(t, dev):
    if not (isinstance(t, torch.Tensor) and t.device == dev and t.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    return t.data_ptr(), t.numel() * t.element_size()


def _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev):
    """Addresses of ctx_lens, cu_q and seq_ids, the sequences to handle, and the batch."""
    ctx = _at(ctx_lens, "ctx_lens", torch.int32, dev, 1)
    cu = _at(cu_q, "cu_q", torch.int32, dev, 1)
    B = ctx_lens.size(0)
    if cu_q.size(0) != B + 1:
        raise ValueError("cu_q must be [B+1]")
    if seq_ids is None:
        if n_seq is None:
            n_seq = B
        elif n_seq > B:
            raise ValueError("n_seq exceeds the batch")
        return ctx, cu, None, n_seq, B
    ids = _at(seq_ids, "seq_ids", torch.int32, dev, 1)
    if n_seq is None:
        n_seq = seq_ids.size(0)
    elif n_seq > seq_ids.size(0):
        raise ValueError("n_seq exceeds seq_ids")
    return ctx, cu, ids, n_seq, B


def rope_inv_freq(rot: int, base: float = 10000.0, kind: int = ROPE_PLAIN, factor: float = 1.0,
                  original_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """Inverse frequencies [rot/2] (float32, on the CPU) and the factor on the
    rotation (see ipdv_rope_inv_freq)."""
    out = torch.empty(max(int(rot), 2) // 2, dtype=torch.float32)
    f = ctypes.c_float(1.0)
    st = lib().ipdv_rope_inv_freq(int(rot), float(base), int(kind), float(factor), int(original_len),
                                  float(beta_fast), float(beta_slow), out.data_ptr(), ctypes.byref(f))
    _check("ipdv_rope_inv_freq", st)
    return out, float(f.value)


def rope_window(q, k, inv_freq, ctx_lens, cu_q, max_q: int, seq_ids=None,
                n_seq: Optional[int] = None, layout: int = ROPE_HALF, factor: float = 1.0,
                inverse: bool = False, q_out=None, k_out=None):
    """Rotary positions of a window's queries and keys (see include/ipdv.h).

    q [T,Hq,D], k [T,Hkv,D] (bf16 or fp32; rows may be strided), inv_freq
    [rot/2] float32, ctx_lens [B], cu_q [B+1], seq_ids [n] int32 or None.
    inverse=True turns back: the gradient of q and k from that of the outputs
    (autograd does not record the call).  q_out / k_out may be q / k (in place).
    Returns (q_out, k_out)."""
    dev, dt = q.device, q.dtype
    code = _dtype_code(dt)
    qp, qs, q_shape = _rows(q, "q", dt, dev, 3)
    kp, ks, k_shape = _rows(k, "k", dt, dev, 3)
    T, Hq, D = q_shape
    Hkv = k_shape[1]
    if k_shape[0] != T or k_shape[2] != D:
        raise ValueError("k must be [T,Hkv,D]")
    freq = _at(inv_freq, "inv_freq", torch.float32, dev, 1)
    ctx, cu, ids, n_seq, _ = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    qos, kos = Hq * D, Hkv * D
    if q_out is None:
        q_out = torch.empty_like(q)       # dense rows; torch.empty of a torch.Size takes 0.8 us more
        qop = q_out.data_ptr()
    else:
        qop, qos, shape = _rows(q_out, "q_out", dt, dev, 3)
        if shape != q_shape:
            raise ValueError("q_out must have q's shape")
    if k_out is None:
        k_out = torch.empty_like(k)
        kop = k_out.data_ptr()
    else:
        kop, kos, shape = _rows(k_out, "k_out", dt, dev, 3)
        if shape != k_shape:
            raise ValueError("k_out must have k's shape")
    if T == 0:
        n_seq = 0
    st = lib().rope_window(qp, qs, kp, ks, qop, qos, kop, kos, freq, ctx, cu, ids, n_seq, max_q,
                           Hq, Hkv, D, 2 * inv_freq.size(0), int(layout), float(factor),
                           1 if inverse else 0, code, _stream(dev))
    _check("rope_window", st)
    return q_out, k_out


class Q8Cache:
    """A paged 8-bit cache (see kv_append_q8 in include/ipdv.h): ``k``
    [P,Hkv,D/16,ps,16] and ``v`` [P,Hkv,D,ps] in float8_e4m3fn, ``scale``
    [P,Hkv,2,ps] uint8.  The three tensors are the caller's."""

    def __init__(self, k, v, scale):
        dev = k.device
        _need(k, "k", torch.float8_e4m3fn, dev, 5)
        _need(v, "v", torch.float8_e4m3fn, dev, 4)
        _need(scale, "scale", torch.uint8, dev, 4)
        P, Hkv, D, ps = v.shape
        if k.shape != (P, Hkv, D // 16, ps, 16) or scale.shape != (P, Hkv, 2, ps) or D % 16:
            raise ValueError("k must be [P,Hkv,D/16,ps,16], v [P,Hkv,D,ps] and scale [P,Hkv,2,ps]")
        self.k, self.v, self.scale = k, v, scale
        self.num_pages, self.Hkv, self.D, self.page_size = P, Hkv, D, ps

    @classmethod
    def empty(cls, num_pages: int, Hkv: int, D: int, page_size: int = 16, device="cuda"):
        """An unwritten cache of `num_pages` pages."""
        f8 = torch.float8_e4m3fn
        return cls(torch.empty(num_pages, Hkv, D // 16, page_size, 16, dtype=f8, device=device),
                   torch.empty(num_pages, Hkv, D, page_size, dtype=f8, device=device),
                   torch.empty(num_pages, Hkv, 2, page_size, dtype=torch.uint8, device=device))

    @property
    def device(self):
        return self.k.device


def _q8_table(cache: Q8Cache, page_table, B, dev):
    """Address and width of the page table, once the cache is known to be on dev."""
    if not isinstance(cache, Q8Cache):
        raise TypeError("cache must be a Q8Cache")
    if cache.k.get_device() != dev.index:
        raise ValueError(f"cache must be on {dev} (is on {cache.device})")
    at = _at(page_table, "page_table", torch.int32, dev, 2)
    n, max_pages = page_table.shape
    if n != B:
        raise ValueError("page_table must be [B, maxp]")
    return at, max_pages


def kv_append_q8(k_new, v_new, cache: Q8Cache, page_table, ctx_lens, cu_q, max_q: int,
                 seq_ids=None, n_seq: Optional[int] = None, validate: bool = False):
    """Quantise the window's keys and values [T,Hkv,D] (bf16 or fp32; rows may
    be strided) into the cache at positions ctx_lens[b] + i (see
    include/ipdv.h).  validate=True first runs check_page_table on host copies."""
    dev, dt = k_new.device, k_new.dtype
    code = _dtype_code(dt)
    kp, ks, shape = _rows(k_new, "k_new", dt, dev, 3)
    vp, vs, v_shape = _rows(v_new, "v_new", dt, dev, 3)
    ctx, cu, ids, n_seq, B = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    table, max_pages = _q8_table(cache, page_table, B, dev)
    T, Hkv, D = shape
    if Hkv != cache.Hkv or D != cache.D or v_shape != shape:
        raise ValueError("k_new and v_new must be [T,Hkv,D] of the cache's heads")
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, cache.page_size, cache.num_pages,
                         seq_ids=seq_ids, n_seq=n_seq, rows=T)
    if T == 0:
        n_seq = 0
    st = lib().kv_append_q8(kp, ks, vp, vs, cache.k.data_ptr(), cache.v.data_ptr(),
                            cache.scale.data_ptr(), table, max_pages, ctx, cu, ids, n_seq, max_q,
                            Hkv, D, cache.page_size, cache.num_pages, code, _stream(dev))
    _check("kv_append_q8", st)


def kv_read_q8(cache: Q8Cache, page_table, ctx_lens, cu_q, max_q: int, rows: int, seq_ids=None,
               n_seq: Optional[int] = None, dtype=torch.bfloat16, k_out=None, v_out=None,
               validate: bool = False):
    """The values that positions ctx_lens[b] + i stand for, as rows cu_q[b] + i
    of two [rows,Hkv,D] tensors (see include/ipdv.h); with ctx_lens zero and
    the cached lengths in cu_q, whole sequences.  rows is cu_q's last entry, or
    at least where the last handled window ends: cu_q is read on the device
    alone, and rows beyond would be written behind the outputs.  validate=True
    checks that and the page table on host copies first.  Returns (k, v)."""
    dev = cache.device
    code = _dtype_code(dtype)
    ctx, cu, ids, n_seq, B = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    table, max_pages = _q8_table(cache, page_table, B, dev)
    Hkv, D = cache.Hkv, cache.D
    shape = (int(rows), Hkv, D)
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        if t is not None:
            _need(t, name, dtype, dev, 3)
            if t.shape != shape:
                raise ValueError(f"{name} must be [rows,Hkv,D]")
    if k_out is None:
        k_out = torch.empty(*shape, dtype=dtype, device=dev)
    if v_out is None:
        v_out = torch.empty_like(k_out)
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, cache.page_size, cache.num_pages,
                         seq_ids=seq_ids, n_seq=n_seq, rows=shape[0], writes=False)
    if shape[0] == 0:
        n_seq = 0
    st = lib().kv_read_q8(cache.k.data_ptr(), cache.v.data_ptr(), cache.scale.data_ptr(), table,
                          max_pages, ctx, cu, ids, n_seq, max_q, k_out.data_ptr(), v_out.data_ptr(),
                          Hkv, D, cache.page_size, cache.num_pages, code, _stream(dev))
    _check("kv_read_q8", st)
    return k_out, v_out


def attn_q8_workspace_size(n_seq, Hq, Hkv, D, max_q) -> int:
    return int(lib().ipdv_attn_q8_workspace_size(n_seq, Hq, Hkv, D, max_q))


def verify_attn_q8(q, cache: Q8Cache, page_table, ctx_lens, cu_q, max_q: int, seq_ids=None,
                   n_seq: Optional[int] = None, scale: Optional[float] = None, out=None,
                   workspace=None, validate: bool = False):
    """Causal GQA attention of the window rows q [T,Hq,D] (bf16 or fp32; rows
    may be strided) over the 8-bit cache, which already holds the window (see
    include/ipdv.h).  validate=True first runs check_page_table on host copies.
    Returns out [T,Hq,D]."""
    dev, dt = q.device, q.dtype
    code = _dtype_code(dt)
    qp, qs, shape = _rows(q, "q", dt, dev, 3)
    ctx, cu, ids, n_seq, B = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    table, max_pages = _q8_table(cache, page_table, B, dev)
    T, Hq, D = shape
    Hkv = cache.Hkv
    if D != cache.D:
        raise ValueError("q and the cache have different head dims")
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", dt, dev, 3)
        if out.shape != shape:
            raise ValueError("out must have q's shape")
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, cache.page_size, cache.num_pages,
                         seq_ids=seq_ids, n_seq=n_seq, rows=T, writes=False)
    if T == 0:
        n_seq = 0
    if workspace is None:
        size = max(attn_q8_workspace_size(n_seq, Hq, Hkv, D, max_q), 1)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    else:
        ws, size = _given_workspace(workspace, dev)
    st = lib().verify_attn_q8(qp, qs, cache.k.data_ptr(), cache.v.data_ptr(), cache.scale.data_ptr(),
                              table, max_pages, ctx, cu, ids, n_seq, max_q, out.data_ptr(), Hq, Hkv,
                              D, cache.page_size, cache.num_pages, float(scale), code, ws, size,
                              _stream(dev))
    _check("verify_attn_q8", st)
    return out


def sample_logits_workspace_size(M, V) -> int:
    return int(lib().ipdv_sample_logits_workspace_size(M, V))


def sample_logits(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, token=None,
                  logp=None, workspace=None):
    """One draw per row of logits [M,V] (bf16 or fp32; rows may be strided),
    each row with its own temperature, top_p, min_p [M] float32 and top_k [M]
    int32 (each None for off), from uniforms u [M] float32 in [0, 1) (see
    include/ipdv.h).  Returns (token [M] int32, logp [M] float32): the draws and
    their log-probs among what the filters kept."""
    dev, dt = logits.device, logits.dtype
    code = _dtype_code(dt)
    lp, ls, (M, V) = _rows(logits, "logits", dt, dev, 2)

    def of_rows(t, name, dtype):
        if t is None:
            return None
        at = _at(t, name, dtype, dev, 1)
        if t.size(0) != M:
            raise ValueError(f"{name} must be [M]")
        return at

    f32, i32 = torch.float32, torch.int32
    up = _at(u, "u", f32, dev, 1)
    if u.size(0) != M:
        raise ValueError("u must be [M]")
    tp = of_rows(temperature, "temperature", f32)
    kp = of_rows(top_k, "top_k", i32)
    pp = of_rows(top_p, "top_p", f32)
    mp = of_rows(min_p, "min_p", f32)
    of_rows(token, "token", i32)
    of_rows(logp, "logp", f32)
    token = torch.empty(M, dtype=i32, device=dev) if token is None else token
    logp = torch.empty(M, dtype=f32, device=dev) if logp is None else logp
    if workspace is None:
        size = max(sample_logits_workspace_size(M, V), 1)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    else:
        ws, size = _given_workspace(workspace, dev)
    st = lib().sample_logits(lp, ls, M, V, up, tp, kp, pp, mp, token.data_ptr(), logp.data_ptr(),
                             code, ws, size, _stream(dev))
    _check("sample_logits", st)
    return token, logp


# ---------------------------------------------------------------------------
# Attention with modified scores, the weights it gives and eviction by them, and
# the verdict on drafts by probabilities.

def _sized(t, name: str, dtype, dev, n: int):
    """Address of an optional [n] tensor."""
    if t is None:
        return None
    at = _at(t, name, dtype, dev, 1)
    if t.size(0) != n:
        raise ValueError(f"{name} must be [{n}]")
    return at


def _score_mod(slopes, first_key, end_key, T, Hq, dev):
    """Addresses of the scores' arrays."""
    if slopes is None and first_key is None and end_key is None:
        return None, None, None
    return (_sized(slopes, "slopes", torch.float32, dev, Hq),
            _sized(first_key, "first_key", torch.int32, dev, T),
            _sized(end_key, "end_key", torch.int32, dev, T))


def _paged(k_cache, page_table, dt, dev, D: int, B: int):
    """Addresses of the key pages and the page table, Hkv, page size, pages and table width."""
    kc = _at(k_cache, "k_cache", dt, dev, 5)
    P, Hkv, slices, ps, run = k_cache.shape
    if run != 32 or slices * 32 != D:
        raise ValueError("k_cache must be [P,Hkv,D/32,ps,32]")
    table = _at(page_table, "page_table", torch.int32, dev, 2)
    n, max_pages = page_table.shape
    if n != B:
        raise ValueError("page_table must be [B, maxp]")
    return kc, table, Hkv, ps, P, max_pages


@functools.lru_cache(maxsize=1024)      # a step asks for the same ones: 1.5 us each
def attn_masked_workspace_size(n_seq, Hq, Hkv, D, max_q, max_pages, page_size, window=0,
                               has_end_key=False) -> int:
    return int(lib().ipdv_attn_masked_workspace_size(n_seq, Hq, Hkv, D, max_q, max_pages, page_size,
                                                     window, 1 if has_end_key else 0))


def verify_attn_masked(q, k_new, v_new, k_cache, v_cache, page_table, ctx_lens, cu_q, max_q: int,
                       softcap: float = 0.0, window: int = 0, slopes=None, first_key=None,
                       end_key=None, seq_ids=None, n_seq: Optional[int] = None,
                       scale: Optional[float] = None, out=None, lse=None, workspace=None,
                       validate: bool = False):
    """verify_attn_paged with modified scores (see include/ipdv.h): a tanh cap, a
    sliding window, distance slopes [Hq] float32, and each row's first and end
    key [T] int32.

    q [T,Hq,D] (bf16 or fp32; rows may be strided), k_new/v_new [T,Hkv,D] or both
    None (the window is in the cache), k_cache [P,Hkv,D/32,ps,32], v_cache
    [P,Hkv,D,ps].  lse: a [T,Hq] float32 tensor to write, or True for a new one.
    validate=True first runs check_page_table on host copies.  Returns out
    [T,Hq,D], or (out, lse)."""
    dev, dt = q.device, q.dtype
    code = _dtype_code(dt)
    qp, qs, shape = _rows(q, "q", dt, dev, 3)
    T, Hq, D = shape
    ctx, cu, ids, n_seq, B = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    kc, table, Hkv, ps, P, max_pages = _paged(k_cache, page_table, dt, dev, D, B)
    vc = _at(v_cache, "v_cache", dt, dev, 4)
    if v_cache.shape != (P, Hkv, D, ps):
        raise ValueError("v_cache must be [P,Hkv,D,ps]")
    kn = vn = None
    if k_new is not None or v_new is not None:
        kn, vn = _at(k_new, "k_new", dt, dev, 3), _at(v_new, "v_new", dt, dev, 3)
        if k_new.shape != (T, Hkv, D) or v_new.shape != (T, Hkv, D):
            raise ValueError("k_new / v_new must be [T,Hkv,D]")
    slopes_p, first_p, end_p = _score_mod(slopes, first_key, end_key, T, Hq, dev)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", dt, dev, 3)
        if out.shape != shape:
            raise ValueError("out must have q's shape")
    if lse is True:
        lse = torch.empty(T, Hq, dtype=torch.float32, device=dev)
    elif lse is False:
        lse = None
    lp = None
    if lse is not None:
        lp = _at(lse, "lse", torch.float32, dev, 2)
        if lse.shape != (T, Hq):
            raise ValueError("lse must be [T,Hq]")
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, ps, P, seq_ids=seq_ids, n_seq=n_seq,
                         rows=T, writes=k_new is not None)
    if T == 0:
        n_seq = 0
    if workspace is None:
        size = max(attn_masked_workspace_size(n_seq, Hq, Hkv, D, max_q, max_pages, ps, int(window),
                                              end_key is not None), 1)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    else:
        ws, size = _given_workspace(workspace, dev)
    st = lib().verify_attn_masked(qp, qs, kn, vn, kc, vc, table, max_pages, ctx, cu, ids, n_seq,
                                  max_q, softcap, window, slopes_p, first_p, end_p, out.data_ptr(), lp,
                                  Hq, Hkv, D, ps, P, scale, code, ws, size, _stream(dev))
    _check("verify_attn_masked", st)
    return out if lse is None else (out, lse)


def attn_mass(q, k_cache, lse, page_table, ctx_lens, cu_q, max_q: int, mass=None,
              decay: float = 1.0, out=None, softcap: float = 0.0, window: int = 0, slopes=None,
              first_key=None, end_key=None, seq_ids=None, n_seq: Optional[int] = None,
              scale: Optional[float] = None, validate: bool = False):
    """The attention weight that every cached key gathers from a window (see
    include/ipdv.h), added to decay * mass.

    q, k_cache, the batch and the modifiers as in the verify_attn_masked call that
    gave lse [T,Hq]; mass [P,Hkv,ps] float32 is updated in place, or written to
    `out` (mass None: there is none yet).  Returns the updated tensor."""
    dev, dt = q.device, q.dtype
    code = _dtype_code(dt)
    qp, qs, (T, Hq, D) = _rows(q, "q", dt, dev, 3)
    ctx, cu, ids, n_seq, B = _window_args(ctx_lens, cu_q, seq_ids, n_seq, dev)
    kc, table, Hkv, ps, P, max_pages = _paged(k_cache, page_table, dt, dev, D, B)
    lp = _at(lse, "lse", torch.float32, dev, 2)
    if lse.shape != (T, Hq):
        raise ValueError("lse must be [T,Hq]")
    slopes_p, first_p, end_p = _score_mod(slopes, first_key, end_key, T, Hq, dev)
    if out is None:
        if mass is None:
            raise ValueError("mass or out must be given")
        out = mass
    mp = None
    for t, name in ((mass, "mass"), (out, "out")):
        if t is not None:
            mp = _at(t, name, torch.float32, dev, 3)
            if t.shape != (P, Hkv, ps):
                raise ValueError(f"{name} must be [P,Hkv,ps]")
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if validate:
        check_page_table(page_table, ctx_lens, cu_q, max_q, ps, P, seq_ids=seq_ids, n_seq=n_seq,
                         rows=T)
    if T == 0:                        # no rows: the masses decay
        qp = lp = None
    st = lib().attn_mass(qp, qs, kc, lp, table, max_pages, ctx, cu, ids, n_seq, max_q,
                         softcap, window, slopes_p, first_p, end_p,
                         None if mass is None else mass.data_ptr(), decay, mp, Hq, Hkv, D, ps, P,
                         scale, code, _stream(dev))
    _check("attn_mass", st)
    return out


def kv_evict(k_cache, v_cache, mass, page_table, dst_table, ctx_lens, keep, n_sink: int = 0,
             n_recent: int = 0, seq_ids=None, n_seq: Optional[int] = None, new_lens=None, kept=None,
             validate: bool = False):
    """Sequences cut to their heaviest keys, moved to dst_table's pages (see
    include/ipdv.h).

    k_cache [P,Hkv,D/32,ps,32], v_cache [P,Hkv,D,ps] (bf16 or fp32), mass
    [P,Hkv,ps] float32, page_table [B,maxp], dst_table [B,maxd], ctx_lens and keep
    [B] int32; new_lens may be ctx_lens or keep.  validate=True first checks both
    tables on host copies.  Returns (new_lens [B], kept [B,Hkv,maxd*ps]) int32."""
    dev, dt = k_cache.device, k_cache.dtype
    code = _dtype_code(dt)
    ctx = _at(ctx_lens, "ctx_lens", torch.int32, dev, 1)
    B = ctx_lens.size(0)
    if k_cache.dim() != 5:
        raise ValueError("k_cache must be [P,Hkv,D/32,ps,32]")
    D = 32 * k_cache.shape[2]
    kc, table, Hkv, ps, P, max_pages = _paged(k_cache, page_table, dt, dev, D, B)
    vc = _at(v_cache, "v_cache", dt, dev, 4)
    mp = _at(mass, "mass", torch.float32, dev, 3)
    if v_cache.shape != (P, Hkv, D, ps) or mass.shape != (P, Hkv, ps):
        raise ValueError("v_cache must be [P,Hkv,D,ps] and mass [P,Hkv,ps]")
    dst = _at(dst_table, "dst_table", torch.int32, dev, 2)
    if dst_table.shape[0] != B:
        raise ValueError("dst_table must be [B, maxd]")
    max_dst = dst_table.shape[1]
    kp = _at(keep, "keep", torch.int32, dev, 1)
    if keep.size(0) != B:
        raise ValueError("keep must be [B]")
    ids = None
    if seq_ids is not None:
        ids = _at(seq_ids, "seq_ids", torch.int32, dev, 1)
    most = B if seq_ids is None else seq_ids.size(0)
    if n_seq is None:
        n_seq = most
    elif n_seq > most:
        raise ValueError("n_seq exceeds the batch")
    slots = (B, Hkv, max_dst * ps)
    if new_lens is None:
        new_lens = torch.empty(B, dtype=torch.int32, device=dev)
    else:
        _sized(new_lens, "new_lens", torch.int32, dev, B)
    if kept is None:
        kept = torch.empty(*slots, dtype=torch.int32, device=dev)
    else:
        _need(kept, "kept", torch.int32, dev, 3)
        if kept.shape != slots:
            raise ValueError("kept must be [B,Hkv,maxd*ps]")
    if validate:
        _check_evict(page_table, dst_table, ctx_lens, keep, ps, P, seq_ids, n_seq)
    st = lib().kv_evict(kc, vc, mp, table, max_pages, dst, max_dst, ctx, kp, ids, n_seq, int(n_sink),
                        int(n_recent), new_lens.data_ptr(), kept.data_ptr(), Hkv, D, ps, P, code,
                        _stream(dev))
    _check("kv_evict", st)
    return new_lens, kept


def _check_evict(page_table, dst_table, ctx_lens, keep, ps, P, seq_ids, n_seq):
    """check_page_table of both tables, and that no page is both read and written."""
    import numpy as np

    host = lambda t: t.detach().cpu().numpy().astype(np.int64)  # noqa: E731
    ctx, want = host(ctx_lens), host(keep)
    B = ctx.shape[0]
    zero = np.zeros(B + 1, np.int32)
    check_page_table(page_table, ctx.astype(np.int32), zero, 1, ps, P, seq_ids=seq_ids, n_seq=n_seq)
    n = np.clip(want, 0, np.minimum(ctx, dst_table.shape[1] * ps))
    # the kept rows as windows of empty sequences: pages that they write are their own
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    check_page_table(dst_table, zero[:B], cu, max(1, int(n.max(initial=0))), ps, P, seq_ids=seq_ids,
                     n_seq=n_seq)
    ids = np.arange(n_seq) if seq_ids is None else host(seq_ids)[:n_seq]
    src, dst = host(page_table), host(dst_table)
    read = {int(p) for b in ids for p in src[b, : -(-int(ctx[b]) // ps)]}
    for b in ids:
        for p in dst[b, : -(-int(n[b]) // ps)]:
            if int(p) in read:
                raise IpdvError("kv_evict", -1, f"sequence {b}: page {int(p)} is read and written")


@functools.lru_cache(maxsize=1024)
def verify_drafts_workspace_size(T, V, B, target_filtered=False, draft_filtered=False) -> int:
    return int(lib().ipdv_verify_drafts_workspace_size(T, V, B, 1 if target_filtered else 0,
                                                       1 if draft_filtered else 0))


_NO_FILTERS = (None,) * 8


def verify_drafts(target_logits, draft_logits, prop_tok, cu_q, u_accept, u_draw, temperature=None,
                  top_k=None, top_p=None, min_p=None, draft_temperature=None, draft_top_k=None,
                  draft_top_p=None, draft_min_p=None, eos_id: int = -1, outs=None, workspace=None):
    """The verdict on drafted tokens by the two models' probabilities (see
    include/ipdv.h).

    target_logits, draft_logits [T,V] (bf16 or fp32; rows may be strided;
    draft_logits None: the drafts are certain), prop_tok [T] int32 (-1: no draft),
    cu_q [B+1] int32, u_accept [T] and u_draw [B] float32 in [0, 1); the target's
    and the draft's filters per row, as in sample_logits.  Returns dict n_acc,
    token [B] int32, finished [B] uint8, p_accept [T] float32, logp [B] float32
    (`outs` may hold these to be written).  p_accept of rows outside every window is
    not written: in a new tensor it may be anything."""
    dev, dt = target_logits.device, target_logits.dtype
    code = _dtype_code(dt)
    tp, ts, (T, V) = _rows(target_logits, "target_logits", dt, dev, 2)
    dp, ds = None, V
    if draft_logits is not None:
        dp, ds, shape = _rows(draft_logits, "draft_logits", dt, dev, 2)
        if shape != (T, V):
            raise ValueError("draft_logits must have target_logits' shape")
    elif any(t is not None for t in (draft_temperature, draft_top_k, draft_top_p, draft_min_p)):
        raise ValueError("the draft's filters need draft_logits")
    f32, i32 = torch.float32, torch.int32
    cu = _at(cu_q, "cu_q", i32, dev, 1)
    B = cu_q.size(0) - 1
    if B < 0:
        raise ValueError("cu_q must be [B+1]")
    if prop_tok is None or u_accept is None or u_draw is None:
        raise TypeError("prop_tok, u_accept and u_draw must be torch.Tensors")
    need = lambda t, name, dtype, n: _sized(t, name, dtype, dev, n)  # noqa: E731
    xp, ua, ud = need(prop_tok, "prop_tok", i32, T), need(u_accept, "u_accept", f32, T), need(u_draw, "u_draw", f32, B)
    target_cut = not (top_k is None and top_p is None and min_p is None)
    draft_cut = not (draft_top_k is None and draft_top_p is None and draft_min_p is None)
    filters = _NO_FILTERS
    if target_cut or draft_cut or temperature is not None or draft_temperature is not None:
        filters = (need(temperature, "temperature", f32, T), need(top_k, "top_k", i32, T),
                   need(top_p, "top_p", f32, T), need(min_p, "min_p", f32, T),
                   need(draft_temperature, "draft_temperature", f32, T),
                   need(draft_top_k, "draft_top_k", i32, T), need(draft_top_p, "draft_top_p", f32, T),
                   need(draft_min_p, "draft_min_p", f32, T))
    made = {}
    for name, dtype, n in (("n_acc", i32, B), ("token", i32, B), ("finished", torch.uint8, B),
                           ("p_accept", f32, T), ("logp", f32, B)):
        t = None if outs is None else outs.get(name)
        if t is None:
            t = torch.empty(n, dtype=dtype, device=dev)
        else:
            need(t, name, dtype, n)
        made[name] = t
    n_acc, token, finished, p_accept, logp = made.values()
    if workspace is None:
        size = max(verify_drafts_workspace_size(T, V, B, target_cut, draft_cut), 1)
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    else:
        ws, size = _given_workspace(workspace, dev)
    st = lib().verify_drafts(tp, ts, dp, ds, T, V, xp, cu, B, ua, ud, *filters, int(eos_id), n_acc.data_ptr(),
                             token.data_ptr(), finished.data_ptr(), p_accept.data_ptr(),
                             logp.data_ptr(), code, ws, size, _stream(dev))
    _check("verify_drafts", st)
    return made
