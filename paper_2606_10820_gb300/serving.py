"""Serving operators of libkforcing.so on torch tensors (include/kforcing_serving.h).

Argument checks and marshalling only: every operator runs in the CUDA library, on the
current torch stream of its tensors' device, without synchronising.  What a call
refuses raises ``KfError`` (the library's own checks) or ``ValueError`` (shapes,
types, devices); what only the device can see is reported by ``status()``.
Outputs and scratch come from torch's allocator, so they belong to the current
stream; tensors that are made on another stream need that stream's work
to be waited for, as with any torch operator.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import kforcing as kf

DEV_BAD_TOKEN, DEV_BAD_PAGE, DEV_TIMEOUT, DEV_BAD_ROW, DEV_NO_PAGES = 1, 2, 4, 8, 32
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_I32, _I64, _F32, _VP = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
_SIGNATURES = {
    "kf_op_token_scores": (ctypes.c_int, [_I32, _I64, _I32, _VP, _I64, _VP, _F32, _I32] + [_VP] * 6),
    "kf_op_token_scores_grad": (ctypes.c_int, [_I32, _I64, _I32, _VP, _I64, _VP, _F32] + [_VP] * 6 + [_I64, _VP]),
    "kf_op_prompt_attention_work": (_I64, [_I32, _I64]),
    "kf_op_prompt_attention": (ctypes.c_int, [_I32, _I32, _I64] + [_I32] * 4 + [_VP, _I64, _I64] * 4 + [_VP, _F32, _VP, _VP]),
    "kf_op_paged_attention_work": (_I64, [_I32]),
    "kf_op_paged_attention": (ctypes.c_int, [_I32] * 6 + [_VP] + [_I64] * 3 + [_VP, _I64, _I32, _VP, _I32, _VP, _F32] + [_VP] * 3),
    "kf_op_pages_work": (_I64, [_I32] * 3),
    "kf_op_pages_grow": (ctypes.c_int, [_I32, _VP, _VP, _VP, _I32, _VP, _I32, _I32, _VP, _I32, _VP, _VP]),
    "kf_op_pages_free": (ctypes.c_int, [_I32, _VP, _VP, _I32, _VP, _I32, _I32, _VP, _I32, _VP, _VP]),
    "kf_op_pages_fork": (ctypes.c_int, [_I32, _VP, _VP, _VP, _I32, _VP, _I32, _I32, _VP, _I32, _VP, _I32, _I64, _VP, _VP]),
    "kf_op_pages_compact": (ctypes.c_int, [_VP, _I32, _VP, _I32, _I32, _VP, _I32, _I64, _VP, _VP, _VP]),
    "kf_op_pages_copy": (ctypes.c_int, [_I32, _VP, _VP, _VP, _I32, _I32, _I64, _VP]),
    "kf_op_pages_append": (ctypes.c_int, [_I32, _VP, _VP, _I64, _I32, _I32, _VP, _I64, _I64, _VP, _I64, _I64, _VP, _I32, _I32, _VP,
                                          _I32, _I32, _VP, _VP]),
    "kf_op_status": (ctypes.c_int, [_VP]),
}
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = kf.load_library()
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
        _lib = lib
    return _lib


_stream = torch._C._cuda_getCurrentRawStream     # the current stream of a device, by its index
_empty, _F, _I = torch.empty, torch.float32, torch.int32


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _run(name, device, *args):
    """One call of the library with `device` current (argument checks come first)."""
    f = getattr(_lib or _library(), name)
    if torch.cuda.current_device() == device.index:
        rc = f(*args)
    else:
        with torch.cuda.device(device):
            rc = f(*args)
    if rc:
        kf._check(rc)


def _on(t, device, dtype, shape, what):
    if t.dtype != dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor {tuple(shape)} on {device} is wanted, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def status(device=None):
    """Waits for the current stream; raises KfError (KF_E_DEVICE) if an operator has flagged
    an error on this device since the last call."""
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        kf._check(_library().kf_op_status(torch.cuda.current_stream().cuda_stream))


# --------------------------------------------------------------- attention

_HALF = {torch.bfloat16: 1, torch.float16: 2}
_work_bytes = {}


def _scratch(name, device, *args):
    """Scratch of a call, from torch's allocator (one tensor per call: calls on several streams may overlap)."""
    key = (name, device.index, args)
    n = _work_bytes.get(key)
    if n is None:
        with torch.cuda.device(device):
            n = _work_bytes[key] = max(16, getattr(_lib or _library(), name)(*args))
    return _empty(n, dtype=torch.uint8, device=device)


def prompt_attention(q, k, v, starts, longest, scale=None, out=None):
    """Causal attention over packed prompts: q [T, Hq, hd], k and v [T, Hkv, hd] (bf16 or fp16; any strides but the
    last, so they may be parts of one projection's output), starts [n + 1] int32 on the GPU, the first tokens of the
    sequences and T; longest: at least the longest one's tokens.  scale: 1 / sqrt(hd)."""
    _need(q.is_cuda and q.dim() == k.dim() == v.dim() == 3 and q.dtype in _HALF, "q: [T, Hq, hd], k and v: [T, Hkv, hd], bf16 or fp16 on a GPU")
    T, Hq, hd = q.shape
    Hkv, dev, n = k.shape[1], q.device, starts.shape[0] - 1
    _need(k.shape == v.shape == (T, Hkv, hd) and k.dtype == v.dtype == q.dtype and k.device == v.device == dev
          and q.stride(2) == k.stride(2) == v.stride(2) == 1, "k and v: like q, heads of contiguous elements")
    if out is None:
        out = _empty((T, Hq, hd), dtype=q.dtype, device=dev)
    else:
        _need(out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.stride(2) == 1, "out: a tensor like q")
    work = _scratch("kf_op_prompt_attention_work", dev, n, T)
    _run("kf_op_prompt_attention", dev, _HALF[q.dtype], n, T, longest, Hq, Hkv, hd, q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(),
         k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
         _on(starts, dev, _I, (n + 1,), "starts"), 1.0 / math.sqrt(hd) if scale is None else scale, work.data_ptr(), _stream(dev.index))
    return out


def paged_attention(q, pool, table, lens, scale=None, out=None):
    """Attention of the newest rows of each sequence over a paged cache that holds their K and V.

    q [B, rows, Hq, hd] (bf16 or fp16; any strides but the last); pool [pages, 2, Hkv, page, hd],
    one layer's K and V; table [B, width] int32; lens [B] int32, the tokens of each sequence with the
    new rows.  Row i sees keys 0 .. lens - rows + i; a row that sees none is zeros.  scale: 1 / sqrt(hd)."""
    _need(q.is_cuda and q.dim() == 4 and pool.dim() == 5 and table.dim() == 2 and q.dtype in _HALF,
          "q: [B, rows, Hq, hd], pool: [pages, 2, Hkv, page, hd], table: [B, width], bf16 or fp16 on a GPU")
    B, rows, Hq, hd = q.shape
    n_pages, two, Hkv, page, _ = pool.shape
    dev = q.device
    _need(two == 2 and q.stride(3) == 1, "pool: K and V of each page; q: heads of contiguous elements")
    if out is None:
        out = _empty((B, rows, Hq, hd), dtype=q.dtype, device=dev)
    work = _scratch("kf_op_paged_attention_work", dev, hd)
    width = table.shape[1]
    _run("kf_op_paged_attention", dev, _HALF[q.dtype], B, rows, Hq, Hkv, hd, q.data_ptr(), q.stride(0), q.stride(1), q.stride(2),
         _on(pool, dev, q.dtype, (n_pages, 2, Hkv, page, hd), "pool"), n_pages, page,
         _on(table, dev, _I, (B, width), "table"), width, _on(lens, dev, _I, (B,), "lens"),
         1.0 / math.sqrt(hd) if scale is None else scale, _on(out, dev, q.dtype, q.shape, "out"), work.data_ptr(), _stream(dev.index))
    return out


# ------------------------------------------------------------------- pages
#
# The book of a cache: ``ref`` [pages] int32, ``table`` [slots, width] int32 (-1: no page) and ``lens``
# [slots] int32, changed in place.  The pool is [layers, pages, 2, Hkv, page, hd].

def new_book(n_pages, slots, width, device="cuda"):
    """An empty book: (ref, table, lens)."""
    return (torch.zeros(n_pages, dtype=_I, device=device), torch.full((slots, width), -1, dtype=_I, device=device),
            torch.zeros(slots, dtype=_I, device=device))


def _book(ref, table, lens=None):
    _need(ref.is_cuda and ref.dim() == 1 and table.dim() == 2, "ref: [pages], table: [slots, width], int32 on a GPU")
    dev, (slots, width) = ref.device, table.shape
    return (dev, ref.shape[0], slots, width, _on(ref, dev, _I, ref.shape, "ref"), _on(table, dev, _I, table.shape, "table"),
            None if lens is None else _on(lens, dev, _I, (slots,), "lens"))


def _list(x, dev, n, what):
    _need(x.dim() == 1, what + ": a list of int32 on the GPU")
    return _on(x, dev, _I, (n,), what)


def _pool(pool, dev, n_pages):
    """Address, layers and bytes of a page of one layer; pool [layers, pages, ...]."""
    _need(pool.dim() >= 3 and pool.device == dev and pool.is_contiguous() and pool.shape[1] == n_pages,
          "pool: a contiguous [layers, pages, ...] tensor on the book's device")
    return pool.data_ptr(), pool.shape[0], pool.stride(1) * pool.element_size()


def pages_grow(ref, table, lens, slots, new_lens, page=16):
    """Slot slots[i] gets pages for new_lens[i] (>= its length) tokens, lowest free page first."""
    dev, n_pages, n_slots, width, pr, pt, pl = _book(ref, table, lens)
    n = slots.shape[0]
    work = _scratch("kf_op_pages_work", dev, n_pages, n_slots, n)
    _run("kf_op_pages_grow", dev, n, _list(slots, dev, n, "slots"), _list(new_lens, dev, n, "new_lens"), pr, n_pages, pt, n_slots, width,
         pl, page, work.data_ptr(), _stream(dev.index))


def pages_free(ref, table, lens, slots, page=16):
    """The listed slots give up their pages and become empty."""
    dev, n_pages, n_slots, width, pr, pt, pl = _book(ref, table, lens)
    n = slots.shape[0]
    work = _scratch("kf_op_pages_work", dev, n_pages, n_slots, n)
    _run("kf_op_pages_free", dev, n, _list(slots, dev, n, "slots"), pr, n_pages, pt, n_slots, width, pl, page, work.data_ptr(), _stream(dev.index))


def pages_fork(pool, ref, table, lens, src, dst):
    """The sequence of slot src[i] continues in the empty slot dst[i] too: full pages are shared, a last page
    that is not full is copied, in every layer of pool [layers, pages, 2, Hkv, page, hd]."""
    dev, n_pages, n_slots, width, pr, pt, pl = _book(ref, table, lens)
    _need(pool.dim() == 6, "pool: [layers, pages, 2, Hkv, page, hd]")
    pp, layers, page_bytes = _pool(pool, dev, n_pages)
    n = src.shape[0]
    work = _scratch("kf_op_pages_work", dev, n_pages, n_slots, n)
    _run("kf_op_pages_fork", dev, n, _list(src, dev, n, "src"), _list(dst, dev, n, "dst"), pr, n_pages, pt, n_slots, width, pl,
         pool.shape[4], pp, layers, page_bytes, work.data_ptr(), _stream(dev.index))


def pages_compact(pool, ref, table, live=None):
    """The live pages move below their count (``live``, an int32 tensor of one, receives it); tables and references follow."""
    dev, n_pages, n_slots, width, pr, pt, _ = _book(ref, table)
    pp, layers, page_bytes = _pool(pool, dev, n_pages)
    work = _scratch("kf_op_pages_work", dev, n_pages, n_slots, 0)
    _run("kf_op_pages_compact", dev, pr, n_pages, pt, n_slots, width, pp, layers, page_bytes,
         None if live is None else _on(live, dev, _I, (1,), "live"), work.data_ptr(), _stream(dev.index))


def pages_copy(pool, src, dst):
    """Page src[i] to page dst[i] in every layer of pool [layers, pages, ...]."""
    _need(pool.is_cuda, "pool: on a GPU")
    dev, n = pool.device, src.shape[0]
    pp, layers, page_bytes = _pool(pool, dev, pool.shape[1])
    _run("kf_op_pages_copy", dev, n, _list(src, dev, n, "src"), _list(dst, dev, n, "dst"), pp, layers, pool.shape[1], page_bytes, _stream(dev.index))


def pages_append(pool, k, v, starts, table, lens, slots):
    """K and V rows of new tokens into their pages of one layer, pool [pages, 2, Hkv, page, hd]: rows
    starts[i] .. starts[i + 1] - 1 of k and v [T, Hkv, hd] are the last tokens of slot slots[i]."""
    _need(pool.is_cuda and pool.dim() == 5 and k.dim() == 3 and table.dim() == 2 and pool.element_size() == 2,
          "pool: [pages, 2, Hkv, page, hd], k and v: [T, Hkv, hd], 16-bit elements on a GPU")
    dev, (n_pages, two, Hkv, page, hd), (n_slots, width) = pool.device, pool.shape, table.shape
    T, n = k.shape[0], slots.shape[0]
    _need(two == 2 and pool.is_contiguous() and k.shape == v.shape == (T, Hkv, hd) and k.dtype == v.dtype == pool.dtype
          and k.device == v.device == dev and k.stride(2) == v.stride(2) == 1, "k and v: rows of the pool's heads and type")
    _run("kf_op_pages_append", dev, n, _list(slots, dev, n, "slots"), _list(starts, dev, n + 1, "starts"), T, Hkv, hd, k.data_ptr(),
         k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), pool.data_ptr(), n_pages, page,
         _on(table, dev, _I, table.shape, "table"), n_slots, width, _on(lens, dev, _I, (n_slots,), "lens"), _stream(dev.index))


# ------------------------------------------------------------------ scores

def _score_args(logits, tokens, tau):
    _need(logits.is_cuda and logits.dim() == 2 and logits.dtype in _TYPES, "logits: a 2-D fp32, bf16 or fp16 CUDA tensor")
    R, V = logits.shape
    _need(V > 0 and (logits.stride(1) == 1 or V == 1), "logits: rows of contiguous elements")
    stride = logits.stride(0) if R > 1 else V
    _need(stride >= V, "logits: rows that do not overlap")
    return R, V, stride, _on(tokens, logits.device, torch.int64, (R,), "tokens")


def token_scores(logits, tokens, top=0, tau=1.0):
    """Scores of ``tokens`` [R] (int64; negative: padding) under ``logits`` [R, V] / tau: a dict of
    ``logp``, ``entropy`` and ``lse`` [R] fp32 and, with top > 0, ``top_ids`` [R, top] int32 and
    ``top_logp`` [R, top] fp32 of the likeliest tokens (ties: the lowest id first)."""
    R, V, stride, tok = _score_args(logits, tokens, tau)
    _need(0 <= top <= min(64, V), "top: 0 to 64, and at most the vocabulary")
    dev = logits.device
    # (an allocation each: parts of one tensor whose whole is dropped cost more)
    logp, entropy, lse = _empty((R,), dtype=_F, device=dev), _empty((R,), dtype=_F, device=dev), _empty((R,), dtype=_F, device=dev)
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    ids = lps = None
    if top:
        out["top_ids"] = ids = _empty((R, top), dtype=_I, device=dev)
        out["top_logp"] = lps = _empty((R, top), dtype=_F, device=dev)
        ids, lps = ids.data_ptr(), lps.data_ptr()
    _run("kf_op_token_scores", dev, _TYPES[logits.dtype], R, V, logits.data_ptr(), stride, tok, tau, top, logp.data_ptr(),
         entropy.data_ptr(), lse.data_ptr(), ids, lps, _stream(dev.index))
    return out


def token_scores_grad(logits, tokens, g_logp=None, g_entropy=None, tau=1.0, out=None):
    """The scores and the gradient of ``sum(g_logp * logp + g_entropy * entropy)``: a dict of
    ``logp``, ``entropy``, ``lse`` [R] fp32 and ``grad`` [R, V] in the logits' type (``out``, which may be
    the logits themselves, where it is given)."""
    R, V, stride, tok = _score_args(logits, tokens, tau)
    dev = logits.device
    gl, gh = (None if g is None else _on(g, dev, torch.float32, (R,), n) for g, n in ((g_logp, "g_logp"), (g_entropy, "g_entropy")))
    grad = _empty((R, V), dtype=logits.dtype, device=dev) if out is None else out
    if out is not None:
        _need(out.dtype == logits.dtype and out.device == dev and out.shape == logits.shape and (out.stride(1) == 1 or V == 1),
              "out: a tensor like the logits")
    logp, entropy, lse = _empty((R,), dtype=_F, device=dev), _empty((R,), dtype=_F, device=dev), _empty((R,), dtype=_F, device=dev)
    _run("kf_op_token_scores_grad", dev, _TYPES[logits.dtype], R, V, logits.data_ptr(), stride, tok, tau, gl, gh, logp.data_ptr(),
         entropy.data_ptr(), lse.data_ptr(), grad.data_ptr(), grad.stride(0) if R > 1 else V, _stream(dev.index))
    return {"logp": logp, "entropy": entropy, "lse": lse, "grad": grad}
