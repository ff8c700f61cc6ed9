"""Python binding of the COVER kernel library: same names as the C ABI.

Each function checks tensor dtypes / devices / contiguity, reads the sizes off
the tensors, and calls the C entry point on the current CUDA stream. All
arithmetic runs in the CUDA kernels; torch only provides device memory and
streams. A call of plain tensors is marshalled in native code (_binding); the
Python path behind it takes every other form and raises the errors.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import _lib


_nat = None


def _native():
    global _nat
    _nat = _lib.native()
    return _nat


def _done(fn_name, r):
    """What the native marshalling returned for a call it took: its results, or a status code to raise."""
    if type(r) is int:
        _lib.check(fn_name, r)
    return r


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _int32(name, x):
    """A number for an int of the C ABI, which ctypes would cut to its lower 32 bits."""
    x = int(x)
    if not -0x80000000 <= x <= 0x7fffffff:
        raise ValueError(f"{name} must fit 32 bits, got {x}")
    return x


def _sizes_fit(t, name):
    if t.numel() > 0x7fffffff and max(t.shape) > 0x7fffffff:
        raise ValueError(f"{name} must not be longer than 2^31 - 1 in a dimension, got {tuple(t.shape)}")


def _maker(stream, device):
    """make(shape, dtype, zero=False): a tensor that a call makes for itself, a result or a workspace. Of a given stream
    that is not the current one it comes from that stream's memory: a block of the current stream's may still be read
    or written by work that is pending there. The block is kept until the current stream, on which the caller goes on with it,
    is done with it too."""
    def make(shape, dtype, zero=False):
        return (torch.zeros if zero else torch.empty)(shape, dtype=dtype, device=device)

    if stream is None:
        return make
    current, s = torch.cuda.current_stream(device), _stream(stream)
    if s == current.cuda_stream:
        return make
    if isinstance(stream, torch.cuda.Stream):
        on = stream
    else:   # (ExternalStream(0) would be a stream of its own)
        on = torch.cuda.ExternalStream(s, device=current.device) if s else torch.cuda.default_stream(current.device)

    def make_there(shape, dtype, zero=False):
        with torch.cuda.stream(on):
            t = make(shape, dtype, zero)
        t.record_stream(current)
        return t
    return make_there


def _need(t: torch.Tensor, name: str, dtype, ndim: int):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    _sizes_fit(t, name)


def _attn(fn_name, dtype, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, out, lse, want_lse, stream):
    _need(q, "q", dtype, 4)
    _need(k_cached, "k_cached", dtype, 4)
    _need(v_cached, "v_cached", dtype, 4)
    B, Hq, L, D = q.shape
    Hkv = k_cached.shape[1]
    if tuple(k_cached.shape) != (B, Hkv, L, D) or tuple(v_cached.shape) != (B, Hkv, L, D):
        raise ValueError("k_cached / v_cached must be [B, Hkv, L, D] matching q")
    n_seeds = 0 if seed_idx is None else int(seed_idx.shape[1])
    if n_seeds > 0:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        _need(k_seedmask, "k_seedmask", dtype, 4)
        _need(v_seedmask, "v_seedmask", dtype, 4)
        if tuple(seed_idx.shape) != (B, n_seeds):
            raise ValueError("seed_idx must be [B, S]")
        if tuple(k_seedmask.shape) != (B, Hkv, n_seeds, D) or tuple(v_seedmask.shape) != (B, Hkv, n_seeds, D):
            raise ValueError("k_seedmask / v_seedmask must be [B, Hkv, S, D]")
    make = _maker(stream, q.device)
    if out is None:
        out = make(q.shape, q.dtype)
    else:
        _need(out, "out", dtype, 4)
        if out.shape != q.shape:
            raise ValueError("out must match q")
    if lse is None and want_lse:
        lse = make((B, Hq, L), torch.float32)
    elif lse is not None:
        _need(lse, "lse", torch.float32, 3)
        if tuple(lse.shape) != (B, Hq, L):
            raise ValueError("lse must be [B, Hq, L]")
    lib = _lib.load()
    code = getattr(lib, fn_name)(
        _ptr(q), _ptr(k_cached), _ptr(v_cached),
        _ptr(k_seedmask) if n_seeds else None, _ptr(v_seedmask) if n_seeds else None,
        _ptr(seed_idx) if n_seeds else None, n_seeds, B, Hq, Hkv, L, D,
        _ptr(out), _ptr(lse), _stream(stream))
    _lib.check(fn_name, code)
    return out, lse


def cover_attn_fwd(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *,
                   out=None, lse=None, want_lse=True, stream=None):
    """Two-view override attention (bf16). Returns (out [B,Hq,L,D] bf16, lse [B,Hq,L] f32 or None)."""
    if stream is None:
        r = (_nat or _native()).attn(0, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, 0, out, lse,
                                     want_lse, None)
        if r is not None:
            return _done("cover_attn_fwd", r)
    return _attn("cover_attn_fwd", torch.bfloat16, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx,
                 out, lse, want_lse, stream)


def cover_attn_fwd_f32(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *,
                       out=None, lse=None, want_lse=True, stream=None):
    """Two-view override attention in fp32 (CUDA cores)."""
    if stream is None:
        r = (_nat or _native()).attn(1, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, 0, out, lse,
                                     want_lse, None)
        if r is not None:
            return _done("cover_attn_fwd_f32", r)
    return _attn("cover_attn_fwd_f32", torch.float32, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx,
                 out, lse, want_lse, stream)


def _attn_prefix(fn_name, dtype, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, q0, out, lse, want_lse,
                 stream, extra=()):
    _need(q, "q", dtype, 4)
    _need(k_cached, "k_cached", dtype, 4)
    _need(v_cached, "v_cached", dtype, 4)
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k_cached.shape[1], k_cached.shape[2]
    if tuple(k_cached.shape) != (B, Hkv, Lk, D) or tuple(v_cached.shape) != (B, Hkv, Lk, D):
        raise ValueError("k_cached / v_cached must be [B, Hkv, Lk, D] matching q")
    n_seeds = 0 if seed_idx is None else int(seed_idx.shape[1])
    if n_seeds > 0:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        _need(k_seedmask, "k_seedmask", dtype, 4)
        _need(v_seedmask, "v_seedmask", dtype, 4)
        if tuple(seed_idx.shape) != (B, n_seeds):
            raise ValueError("seed_idx must be [B, S]")
        if tuple(k_seedmask.shape) != (B, Hkv, n_seeds, D) or tuple(v_seedmask.shape) != (B, Hkv, n_seeds, D):
            raise ValueError("k_seedmask / v_seedmask must be [B, Hkv, S, D]")
    make = _maker(stream, q.device)
    if out is None:
        out = make(q.shape, q.dtype)
    else:
        _need(out, "out", dtype, 4)
        if out.shape != q.shape:
            raise ValueError("out must match q")
    if lse is None and want_lse:
        lse = make((B, Hq, Lq), torch.float32)
    elif lse is not None:
        _need(lse, "lse", torch.float32, 3)
        if tuple(lse.shape) != (B, Hq, Lq):
            raise ValueError("lse must be [B, Hq, Lq]")
    code = getattr(_lib.load(), fn_name)(
        _ptr(q), _ptr(k_cached), _ptr(v_cached),
        _ptr(k_seedmask) if n_seeds else None, _ptr(v_seedmask) if n_seeds else None,
        _ptr(seed_idx) if n_seeds else None, n_seeds, B, Hq, Hkv, Lq, Lk, _int32("q0", q0), D,
        _ptr(out), _ptr(lse), *extra, _stream(stream))
    _lib.check(fn_name, code)
    return out, lse


def cover_attn_fwd_prefix(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *, q0: int,
                          out=None, lse=None, want_lse=True, stream=None):
    """Two-view attention for a window of Lq query rows at memory positions q0 .. q0+Lq-1 (bf16)."""
    if stream is None:
        r = (_nat or _native()).attn(2, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, q0, out, lse,
                                     want_lse, None)
        if r is not None:
            return _done("cover_attn_fwd_prefix", r)
    return _attn_prefix("cover_attn_fwd_prefix", torch.bfloat16, q, k_cached, v_cached, k_seedmask, v_seedmask,
                        seed_idx, q0, out, lse, want_lse, stream)


def cover_attn_fwd_prefix_f32(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *, q0: int,
                              out=None, lse=None, want_lse=True, stream=None):
    """The prefix-window attention in fp32 (CUDA cores)."""
    if stream is None:
        r = (_nat or _native()).attn(3, q, k_cached, v_cached, k_seedmask, v_seedmask, seed_idx, q0, out, lse,
                                     want_lse, None)
        if r is not None:
            return _done("cover_attn_fwd_prefix_f32", r)
    return _attn_prefix("cover_attn_fwd_prefix_f32", torch.float32, q, k_cached, v_cached, k_seedmask, v_seedmask,
                        seed_idx, q0, out, lse, want_lse, stream)


def _seed_route(fn_name, seed_idx, B, L, device, stream):
    n_seeds = 0 if seed_idx is None else int(seed_idx.shape[1])
    if n_seeds:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        device = seed_idx.device
    device = device or torch.device("cuda")
    make = _maker(stream, device)
    slot = make((B, L), torch.int32)
    bitmap = make((B, (L + 127) // 128, 4), torch.int32)
    n_invalid = make((1,), torch.int32)
    code = getattr(_lib.load(), fn_name)(_ptr(seed_idx) if n_seeds else None, n_seeds, B, L, _ptr(slot),
                                         _ptr(bitmap), _ptr(n_invalid), _stream(stream))
    _lib.check(fn_name, code)
    return slot, bitmap, n_invalid


def cover_seed_route(seed_idx: Optional[torch.Tensor], B: int, L: int, *, device=None, stream=None):
    """Seed routing as the kernels see it: (slot [B,L] int32, bitmap [B,ceil(L/128),4] int32 bits, n_invalid)."""
    return _seed_route("cover_seed_route", seed_idx, B, L, device, stream)


def cover_seed_route_debug(seed_idx: Optional[torch.Tensor], B: int, L: int, *, device=None, stream=None):
    """cover_seed_route under its boundary-table name (same C function behind it)."""
    return _seed_route("cover_seed_route_debug", seed_idx, B, L, device, stream)


def cover_score_workspace_bytes(n_seq: int) -> int:
    return int(_lib.load().cover_score_workspace_bytes(int(n_seq)))


def _score_workspace(n_seq):
    """Its shape and type."""
    return (max(cover_score_workspace_bytes(n_seq), 4) + 3) // 4, torch.int32


def score_workspace(n_seq: int, device=None) -> torch.Tensor:
    """A zero-filled workspace for cover_score_fwd (reusable across calls on one stream)."""
    return _maker(None, device or "cuda")(*_score_workspace(n_seq), zero=True)


def cover_score_fwd(logits, n_seq: int, topk: int, *, cur_tok=None, d_in=None, d_out=None, eligible=None,
                    workspace=None, out=None, stream=None):
    """Fused vocabulary scoring + per-segment top-k.

    Returns a dict of CUDA tensors: maxprob, entropy, argmax, score [N];
    topk_idx [n_seq, topk] int32 and topk_score [n_seq, topk] f32.
    """
    if stream is None and out is None and (workspace is not None or topk == 0):
        r = (_nat or _native()).score(logits, n_seq, topk, cur_tok, d_in, d_out, eligible, workspace, None, None)
        if r is not None:
            return _done("cover_score_fwd", r)
    _need(logits, "logits", torch.bfloat16, 2)
    N, V = logits.shape
    dev = logits.device
    if cur_tok is not None:
        _need(cur_tok, "cur_tok", torch.int32, 1)
    if d_in is not None:
        _need(d_in, "d_in", torch.float32, 1)
    if d_out is not None:
        _need(d_out, "d_out", torch.float32, 1)
    if eligible is not None:
        _need(eligible, "eligible", torch.uint8, 1)
    make = _maker(stream, dev)
    if out is None:
        out = dict(
            maxprob=make(N, torch.float32), entropy=make(N, torch.float32), argmax=make(N, torch.int32),
            score=make(N, torch.float32), topk_idx=make((n_seq, max(topk, 0)), torch.int32),
            topk_score=make((n_seq, max(topk, 0)), torch.float32),
        )
    if workspace is None and topk > 0:
        workspace = make(*_score_workspace(n_seq), zero=True)
    code = _lib.load().cover_score_fwd(
        _ptr(logits), N, V, n_seq, _ptr(cur_tok), _ptr(d_in), _ptr(d_out), _ptr(eligible), topk,
        _ptr(out["maxprob"]), _ptr(out["entropy"]), _ptr(out["argmax"]), _ptr(out["score"]),
        _ptr(out["topk_idx"]) if topk > 0 else None, _ptr(out["topk_score"]) if topk > 0 else None,
        _ptr(workspace), _stream(stream))
    _lib.check("cover_score_fwd", code)
    return out


def cover_score_fwd_noalloc(logits, n_seq: int, topk: int, *, cur_tok=None, d_in=None, d_out=None, eligible=None,
                            out=None, stream=None):
    """cover_score_fwd without a workspace: for callers that cannot allocate device memory.

    The per-sequence counters live in a fixed device array of the library
    (at most 4096 sequences). Calls that overlap on the GPU race on that array.
    The first call on a device looks up the array's address; make it before
    any stream capture. Returns the same dict as cover_score_fwd.
    """
    _need(logits, "logits", torch.bfloat16, 2)
    N, V = logits.shape
    dev = logits.device
    for name, t, dt in (("cur_tok", cur_tok, torch.int32), ("d_in", d_in, torch.float32),
                        ("d_out", d_out, torch.float32), ("eligible", eligible, torch.uint8)):
        if t is not None:
            _need(t, name, dt, 1)
    make = _maker(stream, dev)
    if out is None:
        out = dict(
            maxprob=make(N, torch.float32), entropy=make(N, torch.float32), argmax=make(N, torch.int32),
            score=make(N, torch.float32), topk_idx=make((n_seq, max(topk, 0)), torch.int32),
            topk_score=make((n_seq, max(topk, 0)), torch.float32),
        )
    code = _lib.load().cover_score_fwd_noalloc(
        _ptr(logits), N, V, n_seq, _ptr(cur_tok), _ptr(d_in), _ptr(d_out), _ptr(eligible), topk,
        _ptr(out["maxprob"]), _ptr(out["entropy"]), _ptr(out["argmax"]), _ptr(out["score"]),
        _ptr(out["topk_idx"]) if topk > 0 else None, _ptr(out["topk_score"]) if topk > 0 else None,
        _stream(stream))
    _lib.check("cover_score_fwd_noalloc", code)
    return out


def _seed_kv(fn_name, k, v, seed_idx, k_cache, v_cache, stream):
    if stream is None and seed_idx is not None:
        r = (_nat or _native()).kv(int(fn_name == "cover_seed_kv_override"), k, v, seed_idx, k_cache, v_cache, None)
        if r is not None:
            return _done(fn_name, r)
    if k.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("k must be bfloat16 or float32")
    _need(k, "k", k.dtype, 4)
    _need(v, "v", k.dtype, 4)
    B, Hkv, L, D = k.shape
    if tuple(v.shape) != (B, Hkv, L, D):
        raise ValueError("v must match k")
    S = 0 if seed_idx is None else int(seed_idx.shape[1])
    if S > 0:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        if tuple(seed_idx.shape) != (B, S):
            raise ValueError("seed_idx must be [B, S]")
        if k_cache is None:
            make = _maker(stream, k.device)
            k_cache, v_cache = (make((B, Hkv, S, D), k.dtype) for _ in range(2))
        _need(k_cache, "k_cache", k.dtype, 4)
        _need(v_cache, "v_cache", k.dtype, 4)
        if tuple(k_cache.shape) != (B, Hkv, S, D) or tuple(v_cache.shape) != (B, Hkv, S, D):
            raise ValueError("k_cache / v_cache must be [B, Hkv, S, D]")
    code = getattr(_lib.load(), fn_name)(
        _ptr(k), _ptr(v), _ptr(seed_idx) if S else None, S, B, Hkv, L, D, k.element_size(),
        _ptr(k_cache) if S else None, _ptr(v_cache) if S else None, _stream(stream))
    _lib.check(fn_name, code)
    return k_cache, v_cache


def cover_seed_kv_gather(k, v, seed_idx, *, k_cache=None, v_cache=None, stream=None):
    """Cache the seeds' states at selection: returns (k_cache, v_cache) [B, Hkv, S, D]."""
    return _seed_kv("cover_seed_kv_gather", k, v, seed_idx, k_cache, v_cache, stream)


def cover_seed_kv_override(k, v, seed_idx, k_cache, v_cache, *, stream=None):
    """Swap the cached seed states into k, v (in place); the caches then hold the masked-input pairs."""
    if seed_idx is not None and seed_idx.shape[1] > 0 and (k_cache is None or v_cache is None):
        raise ValueError("k_cache and v_cache are required")
    return _seed_kv("cover_seed_kv_override", k, v, seed_idx, k_cache, v_cache, stream)


def _rows_need(t, name: str, dtypes, device=None):
    """A [B, H, L, D] tensor of rows whose last dimension is dense."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 4:
        raise ValueError(f"{name} must have 4 dims, got {tuple(t.shape)}")
    if t.shape[3] > 1 and t.stride(3) != 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    _sizes_fit(t, name)
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} must be on {device}, got {t.device}")


def _strides(*tensors):
    """Their strides of the first three dimensions, in elements, 0 where a dimension has one entry."""
    vals = [t.stride(i) if t.shape[i] > 1 else 0 for t in tensors for i in range(3)]
    return (ctypes.c_int64 * len(vals))(*vals)


def _launch(fn_name, device, stream, args):
    """Calls the entry point on the tensors' device."""
    with torch.cuda.device(device):
        code = getattr(_lib.load(), fn_name)(*args, _stream(stream))
    _lib.check(fn_name, code)


_ROWS = (torch.bfloat16, torch.float32)


def _overlap(a, b):
    """Whether two tensors share a byte. Rows of one that lie between rows of the other do not (a projection's q and k).
    Exact but for layouts of many strides that no view of a projection has, which count as sharing one."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    pa, pb, ea, eb = a.data_ptr(), b.data_ptr(), a.element_size(), b.element_size()
    end = lambda t, p, e: p + e * (1 + sum((n - 1) * st for n, st in zip(t.shape, t.stride())))  # noqa: E731
    if pa >= end(b, pb, eb) or pb >= end(a, pa, ea):
        return False
    # the bytes between an element of a and one of b: base + sum_i c_i x_i with x_i in [lo_i, hi_i], a dimension each, those of
    # equal strides c as one; the elements share a byte if that is in (-size of a's element, size of b's)
    span = {}
    for t, e, sign in ((a, ea, 1), (b, eb, -1)):
        for n, st in zip(t.shape, t.stride()):
            if n > 1 and st:
                c = st * e
                lo, hi = span.get(c, (0, 0))
                span[c] = (lo, hi + n - 1) if sign > 0 else (lo - n + 1, hi)
    dims = sorted(span.items(), reverse=True)
    below, above = [0], [0]   # what the dimensions from the last one up add at least, at most
    for c, (lo, hi) in reversed(dims):
        below.append(below[-1] + c * lo)
        above.append(above[-1] + c * hi)
    left = 4096               # values to be looked at

    def meets(at, i):
        nonlocal left
        lowest, highest = 1 - ea - at, eb - 1 - at   # what the dimensions from i on have to add
        if i == len(dims):
            return lowest <= 0 <= highest
        c, (lo, hi) = dims[i]
        rest = len(dims) - i - 1
        # x_i with lowest <= c x_i + rest <= highest for some value of the rest
        for x in range(max(lo, -((above[rest] - lowest) // c)), min(hi, (highest - below[rest]) // c) + 1):
            left -= 1
            if left < 0 or meets(at + c * x, i + 1):
                return True
        return False
    return meets(pa - pb, 0)


def _rope_out(x, out, name, make):
    """The output for x: a new dense tensor, x itself (in place) or another one."""
    if out is None:
        return make(x.shape, x.dtype)
    _rows_need(out, name, (x.dtype,), x.device)
    if out.shape != x.shape:
        raise ValueError(f"{name} must have the shape {tuple(x.shape)}")
    if any(n > 1 and st == 0 for n, st in zip(out.shape, out.stride())):
        raise ValueError(f"{name} must not be expanded")
    return out


def _rope_aliases(pairs, rest):
    """Refuses given outputs that overlap anything but their own inputs, as which they lie in memory. pairs: (name, input, given output);
    rest: the other inputs."""
    seen = set()
    for i, (name, x, out) in enumerate(pairs):
        if out is None:
            continue
        in_place = out.data_ptr() == x.data_ptr() and all(n <= 1 or s == t for n, s, t in zip(x.shape, out.stride(), x.stride()))
        others = [t for j, p in enumerate(pairs) if j != i for t in p[1:]] + rest + ([] if in_place else [x])
        for t in others:
            if t is None or frozenset((id(out), id(t))) in seen:
                continue
            seen.add(frozenset((id(out), id(t))))
            if _overlap(out, t):
                raise ValueError(f"{name} must be its input or not overlap it, and overlap none of the other tensors")


def cover_rope_fwd(q, k, inv_freq, *, pos=None, pos0: int = 0, interleaved: bool = False, mscale: float = 1.0,
                   inverse: bool = False, out_q=None, out_k=None, stream=None):
    """Rotary positions of queries and keys. Returns (q, k) turned, dense unless out_q / out_k are given, which may be
    q / k themselves (in place) and share no byte with any other of the tensors (which is looked at in Python: such a
    call takes 37 us of host time, one that makes its results 5).

    q [B, Hq, L, D], k [B, Hkv, L, D] (or None): bf16 or fp32, dense in the last dimension only (a projection's
    [B, L, H, D] transposed will do). inv_freq: fp64 [R / 2], radians per position (rope_frequencies); the first
    R columns turn, in pairs (2i, 2i + 1) if ``interleaved``, else (i, i + R / 2). pos: int32 [B, L], or row l is
    at pos0 + l. ``inverse`` turns back, which is the gradient with respect to q and k too.
    """
    if stream is None and out_q is None and out_k is None and type(mscale) is float:
        r = (_nat or _native()).rope(q, k, inv_freq, pos, pos0, interleaved, mscale, inverse)
        if r is not None:
            return _done("cover_rope_fwd", r)
    _rows_need(q, "q", _ROWS)
    B, Hq, L, D = q.shape
    dev = q.device
    if k is not None:
        _rows_need(k, "k", (q.dtype,), dev)
        if k.shape[0] != B or tuple(k.shape[2:]) != (L, D):
            raise ValueError("k must be [B, Hkv, L, D] matching q")
    _need(inv_freq, "inv_freq", torch.float64, 1)
    if pos is not None:
        _need(pos, "pos", torch.int32, 2)
        if tuple(pos.shape) != (B, L):
            raise ValueError("pos must be [B, L]")
    _same_device(dev, inv_freq=inv_freq, pos=pos)
    if 2 * inv_freq.shape[0] > D:
        raise ValueError("inv_freq must have at most D / 2 entries")
    make = _maker(stream, dev)
    oq = _rope_out(q, out_q, "out_q", make)
    ok = None if k is None else _rope_out(k, out_k, "out_k", make)
    if out_q is not None or out_k is not None:
        _rope_aliases([("out_q", q, out_q)] + ([] if k is None else [("out_k", k, out_k)]), [inv_freq, pos])
    has_k = k is not None and k.shape[1] > 0
    st = _strides(q, k if has_k else q, oq, ok if has_k else oq)
    _launch("cover_rope_fwd", dev, stream,
            (_ptr(q), _ptr(k) if has_k else None, _ptr(oq), _ptr(ok) if has_k else None, ctypes.addressof(st), B, Hq,
             k.shape[1] if has_k else 0, L, D, 2 * inv_freq.shape[0], _ptr(inv_freq) or None, _ptr(pos), _int32("pos0", pos0),
             1 if interleaved else 0, float(mscale), 1 if inverse else 0, q.element_size()))
    return oq, ok


def rope_frequencies(R: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0,
                     trained: int = 4096, slow: float = 1.0, fast: float = 32.0, device=None):
    """(inv_freq, mscale) for cover_rope_fwd: R / 2 frequencies base^(-2i / R) in fp64, stretched by ``factor`` for
    contexts longer than the ``trained`` one.

    scaling: "none"; "linear": every frequency divided by the factor; "ntk": the base raised so that the slowest
    frequency is divided by it and the fastest kept; "yarn": pairs that turn at most ``slow`` times in the trained
    context are divided, those that turn ``fast`` times or more are kept, with a ramp between that is linear in the number of
    turns (code that ramps by the pair's index gives other frequencies: pass its own), and mscale = 0.1 ln(factor) + 1.
    """
    if R < 2 or R % 2:
        raise ValueError("R must be even and at least 2")
    if not factor >= 1.0:
        raise ValueError("factor must be at least 1")
    i = torch.arange(R // 2, dtype=torch.float64)
    mscale = 1.0
    if scaling == "ntk" and R > 2:
        base = base * factor ** (R / (R - 2))
    f = base ** (-2.0 * i / R)
    if scaling == "linear":
        f = f / factor
    elif scaling == "yarn":
        if not fast > slow:
            raise ValueError("fast must be above slow")
        keep = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
        mscale = 0.1 * math.log(factor) + 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return f.to(device or "cuda"), mscale


def kv8_memory(B: int, Hkv: int, L: int, D: int = 128, device=None):
    """An 8-bit key/value memory of zeros: (k8, v8, k_exp, v_exp), e4m3 codes [B, Hkv, L, D] and e8m0 bytes
    [B, Hkv, L]."""
    codes = [torch.zeros((B, Hkv, L, D), dtype=torch.uint8, device=device or "cuda").view(torch.float8_e4m3fn)
             for _ in range(2)]
    exps = [torch.full((B, Hkv, L), 127, dtype=torch.uint8, device=device or "cuda") for _ in range(2)]
    return codes[0], codes[1], exps[0], exps[1]


def _kv8_need(k8, v8, k_exp, v_exp):
    _need(k8, "k8", torch.float8_e4m3fn, 4)
    _need(v8, "v8", torch.float8_e4m3fn, 4)
    _need(k_exp, "k_exp", torch.uint8, 3)
    _need(v_exp, "v_exp", torch.uint8, 3)
    if v8.shape != k8.shape or k_exp.shape != k8.shape[:3] or v_exp.shape != k8.shape[:3]:
        raise ValueError("v8 must match k8 [B, Hkv, L, D], and k_exp, v_exp be [B, Hkv, L]")
    _same_device(k8.device, v8=v8, k_exp=k_exp, v_exp=v_exp)


def _kv8_pos(pos, B, n, device):
    if pos is None:
        return
    _need(pos, "pos", torch.int32, 2)
    if tuple(pos.shape) != (B, n):
        raise ValueError("pos must be [B, n]")
    _same_device(device, pos=pos)


def cover_kv8_write(k, v, k8, v8, k_exp, v_exp, *, pos=None, pos0: int = 0, stream=None) -> None:
    """Quantise rows k, v [B, Hkv, n, D] (bf16 or fp32, rows 16-byte aligned, in any layout that is dense in the last
    dimension) into the memory, in place: slot s at position pos0 + s, or at pos[b, s] (int32 [B, n]; entries
    outside the memory are left out, of those that name one position the lowest slot is taken)."""
    if stream is None:
        r = (_nat or _native()).kv8_write(k, v, k8, v8, k_exp, v_exp, pos, pos0)
        if r is not None:
            return None if r is True else _done("cover_kv8_write", r)
    _kv8_need(k8, v8, k_exp, v_exp)
    B, Hkv, L, D = k8.shape
    _rows_need(k, "k", _ROWS, k8.device)
    _rows_need(v, "v", (k.dtype,), k8.device)
    n = k.shape[2]
    if tuple(k.shape) != (B, Hkv, n, D) or v.shape != k.shape:
        raise ValueError("k and v must be [B, Hkv, n, D] matching the memory")
    _kv8_pos(pos, B, n, k8.device)
    st = _strides(k, v)
    _launch("cover_kv8_write", k8.device, stream,
            (_ptr(k), _ptr(v), ctypes.addressof(st), _ptr(pos) if n else None, _int32("pos0", pos0), n, B, Hkv, L, D, k.element_size(),
             _ptr(k8), _ptr(v8), _ptr(k_exp), _ptr(v_exp)))


def cover_kv8_read(k8, v8, k_exp, v_exp, *, pos=None, pos0: int = 0, n: Optional[int] = None, dtype=torch.bfloat16,
                   stream=None):
    """Read rows of the memory back: (k, v) [B, Hkv, n, D] in bf16 or fp32, exactly. Row s comes from position pos0 + s
    (n rows; to the end of the memory if None) or pos[b, s] (int32 [B, n]; zeros for entries outside it)."""
    if stream is None and dtype in _ROWS:
        r = (_nat or _native()).kv8_read(k8, v8, k_exp, v_exp, pos, pos0, n, dtype is torch.float32)
        if r is not None:
            return _done("cover_kv8_read", r)
    _kv8_need(k8, v8, k_exp, v_exp)
    if dtype not in _ROWS:
        raise TypeError(f"dtype must be torch.bfloat16 or torch.float32, got {dtype}")
    B, Hkv, L, D = k8.shape
    if n is None:
        n = int(pos.shape[1]) if pos is not None else max(0, L - _int32("pos0", pos0))
    if _int32("n", n) < 0:
        raise ValueError("n must not be negative")
    _kv8_pos(pos, B, n, k8.device)
    make = _maker(stream, k8.device)
    k, v = (make((B, Hkv, n, D), dtype) for _ in range(2))
    _launch("cover_kv8_read", k8.device, stream,
            (_ptr(k8), _ptr(v8), _ptr(k_exp), _ptr(v_exp), _ptr(pos) if n else None, _int32("pos0", pos0), n, B, Hkv, L, D,
             k.element_size(), _ptr(k) if n else None, _ptr(v) if n else None))
    return k, v


def cover_attn_prefix8_workspace_bytes(B: int, Hq: int, Hkv: int, Lq: int, Lk: int) -> int:
    sizes = [_int32(name, x) for name, x in (("B", B), ("Hq", Hq), ("Hkv", Hkv), ("Lq", Lq), ("Lk", Lk))]
    return int(_lib.load().cover_attn_prefix8_workspace_bytes(*sizes))


def _attn8_need(q, k8, v8, k_exp, v_exp, k_seedmask, v_seedmask, seed_idx, key_lo, key_hi):
    """Checks the inputs; returns the number of seeds."""
    _need(q, "q", torch.bfloat16, 4)
    _kv8_need(k8, v8, k_exp, v_exp)
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k8.shape[1], k8.shape[2]
    dev = q.device
    if tuple(k8.shape) != (B, Hkv, Lk, D):
        raise ValueError("the memory must be [B, Hkv, Lk, D] matching q")
    S = 0 if seed_idx is None else int(seed_idx.shape[1])
    if S > 0:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        _need(k_seedmask, "k_seedmask", torch.bfloat16, 4)
        _need(v_seedmask, "v_seedmask", torch.bfloat16, 4)
        if tuple(seed_idx.shape) != (B, S):
            raise ValueError("seed_idx must be [B, S]")
        if tuple(k_seedmask.shape) != (B, Hkv, S, D) or tuple(v_seedmask.shape) != (B, Hkv, S, D):
            raise ValueError("k_seedmask / v_seedmask must be [B, Hkv, S, D]")
        _same_device(dev, seed_idx=seed_idx, k_seedmask=k_seedmask, v_seedmask=v_seedmask)
    for name, t in (("key_lo", key_lo), ("key_hi", key_hi)):
        if t is not None:
            _need(t, name, torch.int32, 2)
            if tuple(t.shape) != (B, Lq):
                raise ValueError(f"{name} must be [B, Lq]")
    _same_device(dev, k8=k8, key_lo=key_lo, key_hi=key_hi)
    return S


def cover_attn_fwd_prefix8(q, k8, v8, k_exp, v_exp, k_seedmask=None, v_seedmask=None, seed_idx=None, *, q0: int,
                           key_lo=None, key_hi=None, softcap: float = 0.0, out=None, lse=None, want_lse=True,
                           workspace=None, stream=None):
    """cover_attn_fwd_prefix over an 8-bit memory. Returns (out [B,Hq,Lq,D] bf16, lse [B,Hq,Lq] f32 or None).

    key_lo, key_hi: int32 [B, Lq], the keys [lo, hi) that each row sees (all where None; none: out 0, lse -inf).
    softcap c > 0: scores become c tanh(score / c). workspace: uint8, at least cover_attn_prefix8_workspace_bytes,
    scratch of the call; allocated where None.
    """
    if stream is None and type(softcap) is float:
        r = (_nat or _native()).attn8(q, k8, v8, k_exp, v_exp, k_seedmask, v_seedmask, seed_idx, q0, key_lo, key_hi,
                                      softcap, out, lse, want_lse, workspace)
        if r is not None:
            return _done("cover_attn_fwd_prefix8", r)
    S = _attn8_need(q, k8, v8, k_exp, v_exp, k_seedmask, v_seedmask, seed_idx, key_lo, key_hi)
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k8.shape[1], k8.shape[2]
    dev = q.device
    make = _maker(stream, dev)
    if out is None:
        out = make(q.shape, q.dtype)
    else:
        _need(out, "out", torch.bfloat16, 4)
        if out.shape != q.shape:
            raise ValueError("out must match q")
    if lse is None and want_lse:
        lse = make((B, Hq, Lq), torch.float32)
    elif lse is not None:
        _need(lse, "lse", torch.float32, 3)
        if tuple(lse.shape) != (B, Hq, Lq):
            raise ValueError("lse must be [B, Hq, Lq]")
    nbytes = cover_attn_prefix8_workspace_bytes(B, Hq, Hkv, Lq, Lk)
    if workspace is not None:
        _need(workspace, "workspace", torch.uint8, 1)
        if workspace.numel() < nbytes:
            raise ValueError(f"workspace must have at least {nbytes} bytes")
    elif nbytes:
        workspace = make(nbytes, torch.uint8)
    _same_device(dev, out=out, lse=lse, workspace=workspace)
    _launch("cover_attn_fwd_prefix8", dev, stream,
            (_ptr(q), _ptr(k8), _ptr(v8), _ptr(k_exp), _ptr(v_exp), _ptr(k_seedmask) if S else None,
             _ptr(v_seedmask) if S else None, _ptr(seed_idx) if S else None, S, B, Hq, Hkv, Lq, Lk, _int32("q0", q0), D,
             _ptr(key_lo), _ptr(key_hi), float(softcap), _ptr(out), _ptr(lse), _ptr(workspace) if nbytes else None))
    return out, lse


def cover_decide_workspace_bytes(N: int, n_seq: int) -> int:
    return int(_lib.load().cover_decide_workspace_bytes(int(N), int(n_seq)))


def _decide_workspace(N, n_seq):
    """Its shape and type."""
    return ((max(cover_decide_workspace_bytes(N, n_seq), 16) + 15) // 16, 4), torch.int32


def decide_workspace(N: int, n_seq: int, device=None) -> torch.Tensor:
    """A zero-filled workspace for cover_score_decide_fwd (reusable across calls on one stream)."""
    return _maker(None, device or "cuda")(*_decide_workspace(N, n_seq), zero=True)


COVER_DECIDE_ALL = 0
COVER_DECIDE_UPDATE = 1


def cover_score_decide_fwd(logits, n_seq: int, tok, flags, remask_cnt, *, tau_draft: float, draft_budget: int,
                           remask_budget: int, mask_id: int, min_one: bool = True, pos0: int = 0,
                           max_seeds: int = 0, phase: int = COVER_DECIDE_ALL, d_in=None, d_out=None, draft_ok=None,
                           workspace=None, out=None, stream=None):
    """Scoring fused with one decoding step's decisions (drafting, revision, seed selection).

    tok (int32 [N]), flags and remask_cnt (uint8 [N]) are updated in place.
    Returns a dict of CUDA tensors: maxprob, entropy, argmax, score [N];
    seed_idx [n_seq, max_seeds] (positions, -1 padded), n_seeds [n_seq] and
    stats [n_seq, 6] (drafted, kept, replaced, remasked, n_t, n_above).
    With phase=COVER_DECIDE_UPDATE only drafting, revision and the state update
    run (score, seed_idx and n_seeds are left as they are); cover_attn_mass_fwd
    and cover_seed_select_fwd on the same workspace complete the step.
    """
    if stream is None and out is None and workspace is not None and type(tau_draft) is float:
        r = (_nat or _native()).decide(logits, n_seq, tok, flags, remask_cnt, tau_draft, draft_budget, remask_budget,
                                       mask_id, min_one, pos0, max_seeds, phase, d_in, d_out, draft_ok, workspace, None,
                                       None)
        if r is not None:
            return _done("cover_score_decide_fwd", r)
    _need(logits, "logits", torch.bfloat16, 2)
    N, V = logits.shape
    dev = logits.device
    _need(tok, "tok", torch.int32, 1)
    _need(flags, "flags", torch.uint8, 1)
    _need(remask_cnt, "remask_cnt", torch.uint8, 1)
    for name, t, dt in (("d_in", d_in, torch.float32), ("d_out", d_out, torch.float32),
                        ("draft_ok", draft_ok, torch.uint8)):
        if t is not None:
            _need(t, name, dt, 1)
    make = _maker(stream, dev)
    if out is None:
        out = dict(
            maxprob=make(N, torch.float32), entropy=make(N, torch.float32), argmax=make(N, torch.int32),
            score=make(N, torch.float32), seed_idx=make((n_seq, max(max_seeds, 0)), torch.int32),
            n_seeds=make(n_seq, torch.int32), stats=make((n_seq, 6), torch.int32),
        )
    if workspace is None:
        workspace = make(*_decide_workspace(N, n_seq), zero=True)
    code = _lib.load().cover_score_decide_fwd(
        _ptr(logits), N, V, n_seq, _ptr(d_in), _ptr(d_out), _ptr(draft_ok), float(tau_draft), int(draft_budget),
        int(remask_budget), int(mask_id), 1 if min_one else 0, _int32("pos0", pos0), int(max_seeds), int(phase),
        _ptr(tok), _ptr(flags), _ptr(remask_cnt), _ptr(out["maxprob"]), _ptr(out["entropy"]), _ptr(out["argmax"]),
        _ptr(out["score"]), _ptr(out["seed_idx"]) if max_seeds > 0 else None, _ptr(out["n_seeds"]),
        _ptr(out["stats"]), _ptr(workspace), _stream(stream))
    _lib.check("cover_score_decide_fwd", code)
    return out


def cover_seed_select_fwd(n_seq: int, tok, flags, remask_cnt, workspace, *, remask_budget: int, mask_id: int,
                          pos0: int = 0, max_seeds: int = 0, d_in=None, d_out=None, out=None, stream=None):
    """Seed score, adaptive revision rate and selection after a COVER_DECIDE_UPDATE call.

    `workspace` and the state tensors must be those of that call. Returns a
    dict of CUDA tensors: score [N], seed_idx [n_seq, max_seeds], n_seeds
    [n_seq], stats [n_seq, 6] (columns 4-5 written here).
    """
    _need(tok, "tok", torch.int32, 1)
    _need(flags, "flags", torch.uint8, 1)
    _need(remask_cnt, "remask_cnt", torch.uint8, 1)
    N = tok.shape[0]
    dev = tok.device
    for name, t in (("d_in", d_in), ("d_out", d_out)):
        if t is not None:
            _need(t, name, torch.float32, 1)
    if out is None:
        make = _maker(stream, dev)
        out = dict(score=make(N, torch.float32), seed_idx=make((n_seq, max(max_seeds, 0)), torch.int32),
                   n_seeds=make(n_seq, torch.int32), stats=make((n_seq, 6), torch.int32, zero=True))
    code = _lib.load().cover_seed_select_fwd(
        N, n_seq, _ptr(d_in), _ptr(d_out), int(remask_budget), int(mask_id), _int32("pos0", pos0), int(max_seeds),
        _ptr(tok), _ptr(flags), _ptr(remask_cnt), _ptr(out["score"]),
        _ptr(out["seed_idx"]) if max_seeds > 0 else None, _ptr(out["n_seeds"]), _ptr(out["stats"]),
        _ptr(workspace), _stream(stream))
    _lib.check("cover_seed_select_fwd", code)
    return out


def cover_attn_mass_workspace_bytes(B: int, Hq: int, per: int) -> int:
    return int(_lib.load().cover_attn_mass_workspace_bytes(int(B), int(Hq), int(per)))


def cover_attn_mass_fwd(q, k_cached, lse, tok, flags, *, mask_id: int, pos0: int, per: int, k_seedmask=None,
                        seed_idx=None, workspace=None, d_in=None, d_out=None, stream=None):
    """d_in / d_out (Section 5.3) of the response rows from the attention pass's q, K', lse.

    q [B, Hq, L, 128], k_cached [B, Hkv, L, 128] bf16, lse [B, Hq, L] f32 (as
    cover_attn_fwd wrote it), tok int32 / flags uint8 [B * per] (the state
    after a COVER_DECIDE_UPDATE call). Returns (d_in, d_out), float32 [B * per].
    """
    if stream is None and workspace is not None:
        r = (_nat or _native()).mass(q, k_cached, lse, tok, flags, mask_id, pos0, per, k_seedmask, seed_idx, workspace,
                                     d_in, d_out, None)
        if r is not None:
            return _done("cover_attn_mass_fwd", r)
    _need(q, "q", torch.bfloat16, 4)
    _need(k_cached, "k_cached", torch.bfloat16, 4)
    _need(lse, "lse", torch.float32, 3)
    _need(tok, "tok", torch.int32, 1)
    _need(flags, "flags", torch.uint8, 1)
    B, Hq, L, D = q.shape
    Hkv = k_cached.shape[1]
    n_seeds = 0 if seed_idx is None else int(seed_idx.shape[1])
    if n_seeds > 0:
        _need(seed_idx, "seed_idx", torch.int32, 2)
        _need(k_seedmask, "k_seedmask", torch.bfloat16, 4)
    if tok.shape[0] != B * per or flags.shape[0] != B * per:
        raise ValueError("tok / flags must have B * per entries")
    make = _maker(stream, q.device)
    if workspace is None:
        nbytes = cover_attn_mass_workspace_bytes(B, Hq, per)
        workspace = make(((nbytes + 15) // 16, 4), torch.int32)
    if d_in is None:
        d_in = make(B * per, torch.float32)
    if d_out is None:
        d_out = make(B * per, torch.float32)
    code = _lib.load().cover_attn_mass_fwd(
        _ptr(q), _ptr(k_cached), _ptr(k_seedmask) if n_seeds else None, _ptr(seed_idx) if n_seeds else None,
        n_seeds, _ptr(lse), B, Hq, Hkv, L, D, _ptr(tok), _ptr(flags), int(mask_id), _int32("pos0", pos0), int(per),
        _ptr(workspace), _ptr(d_in), _ptr(d_out), _stream(stream))
    _lib.check("cover_attn_mass_fwd", code)
    return d_in, d_out


def cover_device_status(stream=None) -> int:
    """Synchronise the stream; return and clear the device status word (0 = OK)."""
    return int(_lib.load().cover_device_status(_stream(stream)))


def cover_status_str(code: int) -> str:
    return _lib.status_str(code)


def cover_debug_umma_tile(a, b, p, v, *, stream=None):
    for name, t in (("a", a), ("b", b), ("p", p), ("v", v)):
        _need(t, name, torch.bfloat16, 2)
        if tuple(t.shape) != (128, 128):
            raise ValueError(f"{name} must be [128, 128]")
    make = _maker(stream, a.device)
    c1, c2 = (make((128, 128), torch.float32) for _ in range(2))
    code = _lib.load().cover_debug_umma_tile(_ptr(a), _ptr(b), _ptr(p), _ptr(v), _ptr(c1), _ptr(c2),
                                             _stream(stream))
    _lib.check("cover_debug_umma_tile", code)
    return c1, c2


def cover_debug_wait_timeout(limit_us: int, *, stream=None) -> None:
    _lib.check("cover_debug_wait_timeout", _lib.load().cover_debug_wait_timeout(int(limit_us), _stream(stream)))


def cover_debug_attn_prefix_packed(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *,
                                   q0: int, fault_cta: int = -1, limit_us: int = 0, out=None, lse=None,
                                   want_lse=True, stream=None):
    """The prefix-window attention (bf16) on the packed grouped-query window kernel, whichever kernel
    cover_attn_fwd_prefix would pick for the shape; fault_cta >= 0 or limit_us > 0 run its self-test
    instance (CTA fault_cta leaves out its first K load, waits give up after limit_us)."""
    return _attn_prefix("cover_debug_attn_prefix_packed", torch.bfloat16, q, k_cached, v_cached, k_seedmask,
                        v_seedmask, seed_idx, q0, out, lse, want_lse, stream,
                        extra=(int(fault_cta), int(limit_us)))


def cover_debug_attn_fault(q, k_cached, v_cached, k_seedmask=None, v_seedmask=None, seed_idx=None, *, q0: int = 0,
                           fault_cta: int, fault_entry: int, limit_us: int, out=None, lse=None, stream=None):
    """Self-test: the bf16 attention (window form) with CTA fault_cta leaving out one K tile load and every
    bounded wait limited to limit_us; read the outcome with cover_debug_status_detail()."""
    return _attn_prefix("cover_debug_attn_fault", torch.bfloat16, q, k_cached, v_cached, k_seedmask, v_seedmask,
                        seed_idx, q0, out, lse, True, stream,
                        extra=(int(fault_cta), int(fault_entry), int(limit_us)))


def cover_debug_attn_prefix8(q, k8, v8, k_exp, v_exp, k_seedmask=None, v_seedmask=None, seed_idx=None, *, q0: int, mode: int,
                             nsplit: int = 1, key_lo=None, key_hi=None, softcap: float = 0.0):
    """cover_attn_fwd_prefix8 on the kernel ``mode`` with the keys in ``nsplit`` parts (negative: -nsplit parts, joined
    in a cluster; above 100: nsplit - 100 parts of a KV head, shared out to the sequences). Returns (out, lse)."""
    S = _attn8_need(q, k8, v8, k_exp, v_exp, k_seedmask, v_seedmask, seed_idx, key_lo, key_hi)
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k8.shape[1], k8.shape[2]
    out = torch.empty_like(q)
    lse = torch.empty((B, Hq, Lq), dtype=torch.float32, device=q.device)
    nbytes = (4 * B * Hkv * Lk * D if mode >= 3 else 0) + (
        (nsplit - 100 + B) * Hq * Lq * 520 + 256 if nsplit > 100 else B * Hq * Lq * nsplit * 520 + 16 if nsplit > 1 else 0)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=q.device)
    _launch("cover_debug_attn_prefix8", q.device, None,
            (_ptr(q), _ptr(k8), _ptr(v8), _ptr(k_exp), _ptr(v_exp), _ptr(k_seedmask) if S else None,
             _ptr(v_seedmask) if S else None, _ptr(seed_idx) if S else None, S, B, Hq, Hkv, Lq, Lk, _int32("q0", q0), D,
             _ptr(key_lo), _ptr(key_hi), float(softcap), _ptr(out), _ptr(lse), _ptr(ws), ws.numel(), _int32("mode", mode), _int32("nsplit", nsplit)))
    return out, lse


def cover_debug_attn_prefix8_plan(B: int, Hq: int, Hkv: int, Lq: int, Lk: int, plain: bool, ranges: bool = False):
    """(mode, groups of rows a KV head, parts of the keys (as nsplit of cover_debug_attn_prefix8), predicted us)
    that cover_attn_fwd_prefix8 takes (no device needed)."""
    choice, us = (ctypes.c_int32 * 3)(), ctypes.c_double()
    code = _lib.load().cover_debug_attn_prefix8_plan(B, Hq, Hkv, Lq, Lk, 1 if plain else 0, 1 if ranges else 0, ctypes.addressof(choice),
                                                     ctypes.addressof(us))
    _lib.check("cover_debug_attn_prefix8_plan", code)
    return choice[0], choice[1], choice[2], us.value


def cover_debug_window_model(B: int, Hq: int, Hkv: int, Lq: int, Lk: int, q0: int, n_sm: int, max_clusters):
    """The prefix-window call's choice between the packed grouped-query kernel and the square kernel
    on a GPU with n_sm SMs and max_clusters[c - 1] resident clusters of c packed CTAs (c = 1 .. 8).
    Host arithmetic only (no device needed)."""
    mc = (ctypes.c_int32 * 8)(*[int(x) for x in max_clusters])
    choice = (ctypes.c_int32 * 6)()
    times = (ctypes.c_double * 2)()
    _lib.check("cover_debug_window_model",
               _lib.load().cover_debug_window_model(B, Hq, Hkv, Lq, Lk, q0, n_sm, mc, choice, times))
    return {"supported": bool(choice[0]), "resident": bool(choice[1]), "packed": bool(choice[2]),
            "T": int(choice[3]), "nsplit": int(choice[4]), "n_qt": int(choice[5]),
            "packed_us": float(times[0]), "square_us": float(times[1])}


def cover_debug_status_detail(stream=None):
    """(status code, site id, block id) of the current device's status block, which is then cleared."""
    detail = (ctypes.c_int32 * 3)()
    _lib.check("cover_debug_status_detail", _lib.load().cover_debug_status_detail(detail, _stream(stream)))
    return int(detail[0]), int(detail[1]), int(detail[2])
