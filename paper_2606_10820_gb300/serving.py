"""Serving operators of libkforcing.so on torch tensors (include/kforcing_serving.h).

Argument checks and marshalling only (csrc/py_serving.cpp): every operator runs in the CUDA
library, on the current torch stream of its tensors' device, without synchronising.  What a call
refuses raises ``KfError`` (the library's own checks) or ``ValueError`` (shapes,
types, devices); what only the device can see is reported by ``status()``.
Outputs and scratch come from torch's allocator, so they belong to the current
stream; tensors that are made on another stream need that stream's work
to be waited for, as with any torch operator.

The operators have no backward pass of their own: a tensor that requires a gradient raises ``ValueError``
while torch records gradients, instead of losing it.  ``token_scores_grad`` gives the logits' gradient
explicitly, so its logits may require one (``logits.backward(out["grad"])``).  What a call changes in
place counts up its version, so autograd notices a saved tensor that was written.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import kforcing as kf

DEV_BAD_TOKEN, DEV_BAD_PAGE, DEV_TIMEOUT, DEV_BAD_ROW, DEV_NO_PAGES = 1, 2, 4, 8, 32
_m = None


def _load():
    """The compiled binding (raises if it has not been built)."""
    global _m
    lib = kf.load_library()
    lib.kf_op_status.argtypes, lib.kf_op_status.restype = [ctypes.c_void_p], ctypes.c_int
    if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_serving.so")):
        raise RuntimeError("_serving.so is missing: build it with __graft_entry__.build() (with torch for CUDA, g++ and Python's headers)")
    from . import _serving
    _serving.set_check(kf._check)
    _m = _serving
    return _m


def status(device=None):
    """Waits for the current stream; raises KfError (KF_E_DEVICE) if an operator has flagged
    an error on this device since the last call."""
    _m or _load()
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        kf._check(kf.load_library().kf_op_status(torch.cuda.current_stream().cuda_stream))


# --------------------------------------------------------------- attention

def prompt_attention(q, k, v, starts, longest, scale=None, out=None):
    """Causal attention over packed prompts: q [T, Hq, hd], k and v [T, Hkv, hd] (bf16 or fp16; any strides but the
    last, so they may be parts of one projection's output), starts [n + 1] int32 on the GPU, the first tokens of the
    sequences and T; longest: at least the longest one's tokens.  scale: 1 / sqrt(hd)."""
    return (_m or _load()).prompt_attention(q, k, v, starts, longest, scale, out)


def paged_attention(q, pool, table, lens, scale=None, out=None):
    """Attention of the newest rows of each sequence over a paged cache that holds their K and V.

    q [B, rows, Hq, hd] (bf16 or fp16; any strides but the last); pool [pages, 2, Hkv, page, hd],
    one layer's K and V; table [B, width] int32; lens [B] int32, the tokens of each sequence with the
    new rows.  Row i sees keys 0 .. lens - rows + i; a row that sees none is zeros.  scale: 1 / sqrt(hd)."""
    return (_m or _load()).paged_attention(q, pool, table, lens, scale, out)


# ------------------------------------------------------------------- pages
#
# The book of a cache: ``ref`` [pages] int32, ``table`` [slots, width] int32 (-1: no page) and ``lens``
# [slots] int32, changed in place.  The pool is [layers, pages, 2, Hkv, page, hd].

def new_book(n_pages, slots, width, device="cuda"):
    """An empty book: (ref, table, lens)."""
    return (torch.zeros(n_pages, dtype=torch.int32, device=device), torch.full((slots, width), -1, dtype=torch.int32, device=device),
            torch.zeros(slots, dtype=torch.int32, device=device))


def pages_grow(ref, table, lens, slots, new_lens, page=16):
    """Slot slots[i] gets pages for new_lens[i] (>= its length) tokens, lowest free page first."""
    (_m or _load()).pages_grow(ref, table, lens, slots, new_lens, page)


def pages_free(ref, table, lens, slots, page=16):
    """The listed slots give up their pages and become empty."""
    (_m or _load()).pages_free(ref, table, lens, slots, page)


def pages_fork(pool, ref, table, lens, src, dst):
    """The sequence of slot src[i] continues in the empty slot dst[i] too: full pages are shared, a last page
    that is not full is copied, in every layer of pool [layers, pages, 2, Hkv, page, hd]."""
    (_m or _load()).pages_fork(pool, ref, table, lens, src, dst)


def pages_compact(pool, ref, table, live=None):
    """The live pages move below their count (``live``, an int32 tensor of one, receives it); tables and references follow."""
    (_m or _load()).pages_compact(pool, ref, table, live)


def pages_copy(pool, src, dst):
    """Page src[i] to page dst[i] in every layer of pool [layers, pages, ...]."""
    (_m or _load()).pages_copy(pool, src, dst)


def pages_append(pool, k, v, starts, table, lens, slots):
    """K and V rows of new tokens into their pages of one layer, pool [pages, 2, Hkv, page, hd]: rows
    starts[i] .. starts[i + 1] - 1 of k and v [T, Hkv, hd] are the last tokens of slot slots[i]."""
    (_m or _load()).pages_append(pool, k, v, starts, table, lens, slots)


# ------------------------------------------------------------------ scores

def token_scores(logits, tokens, top=0, tau=1.0):
    """Scores of ``tokens`` [R] (int64; negative: padding) under ``logits`` [R, V] / tau: a dict of
    ``logp``, ``entropy`` and ``lse`` [R] fp32 and, with top > 0, ``top_ids`` [R, top] int32 and
    ``top_logp`` [R, top] fp32 of the likeliest tokens (ties: the lowest id first)."""
    return (_m or _load()).token_scores(logits, tokens, top, tau)


def token_scores_grad(logits, tokens, g_logp=None, g_entropy=None, tau=1.0, out=None):
    """The scores and the gradient of ``sum(g_logp * logp + g_entropy * entropy)``: a dict of
    ``logp``, ``entropy``, ``lse`` [R] fp32 and ``grad`` [R, V] in the logits' type (``out``, which may be
    the logits themselves, where it is given)."""
    return (_m or _load()).token_scores_grad(logits, tokens, g_logp, g_entropy, tau, out)
