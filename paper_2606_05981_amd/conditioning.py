"""Torch-facing wrappers of include/mte_cond.h, and of mte_proj.h's attention: the operators with which a
denoiser's layers read the encoder's conditioning (cross attention, also over a prefix that all
sequences share, an 8-bit key/value cache, group norm).

Tensors in, tensors out, as in ``encoder``: PyTorch provides memory and streams, every step
runs in libmte's HIP kernels, nothing falls back. Forward only: results carry no gradient, also where
inputs require one. Workspaces are taken from torch's
allocator call by call, on the stream the call runs on, so calls on several streams and
captured graphs share none. A call given a `stream` other than the current one orders
nothing by itself: the caller makes that stream wait for the inputs, and the current
one for the results.
"""
from __future__ import annotations

import math
from array import array
from typing import NamedTuple, Optional, Sequence

import torch

from . import binding as B

_DTYPE = {torch.float32: B.MTE_F32, torch.bfloat16: B.MTE_BF16}
_ACT = {None: B.MTE_ACT_NONE, "none": B.MTE_ACT_NONE, "silu": B.MTE_ACT_SILU}


# the current stream's handle without a Stream object around it (4 us of a call of 15)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _on(device: torch.device, stream: Optional[torch.cuda.Stream], used, fn):
    """fn(stream handle) with `device` and the stream current; `used` tensors (None allowed) and
    the results stay allocated until a stream other than their own is done with them."""
    if stream is None:
        if device.index == torch._C._cuda_getDevice():
            return fn(_raw_stream(device.index))
        with torch.cuda.device(device):
            return fn(_raw_stream(device.index))
    if stream.device != device:
        raise ValueError(f"stream: expected one of {device}, got one of {stream.device}")
    with torch.cuda.device(device):
        cur = torch.cuda.current_stream()
        if cur == stream:
            return fn(stream.cuda_stream)
        with torch.cuda.stream(stream):
            res = fn(stream.cuda_stream)
        for t in used:
            if t is not None:
                t.record_stream(stream)
        for t in res if isinstance(res, tuple) else (res,):
            if t is not None:
                t.record_stream(cur)
        return res


def _rows(name: str, t, dtype: torch.dtype, heads: int, d: int, device: torch.device):
    """Checks a [rows, heads, d] tensor and returns its (row, head) strides."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name}: expected a [tokens, heads, head_dim] tensor")
    if t.device != device:
        raise ValueError(f"{name}: expected a tensor on {device}, got one on {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    n, h, c = t.shape
    if h != heads or c != d:
        raise ValueError(f"{name}: expected shape (*, {heads}, {d}), got {tuple(t.shape)}")
    row, head, one = t.stride()
    if n <= 1:
        row = 0
    if heads == 1:
        head = 0
    if one != 1 or row % 8 or head % 8 or t.data_ptr() % 16:
        raise ValueError(f"{name}: expected contiguous heads at 16-byte aligned addresses, strides multiples of 8 "
                         f"elements; got strides {t.stride()}")
    return row, head


def _out_rows(out, q, row_head_of):
    """Checks a caller's out like q, and that its rows and heads do not overlap."""
    row, head = row_head_of
    d, n, heads = q.shape[2], q.shape[0], q.shape[1]
    if out.shape[0] != n:
        raise ValueError(f"out: expected {n} rows, got {out.shape[0]}")
    row, head = (row if n > 1 else None), (head if heads > 1 else None)
    small, big, count = (row, head, n) if row is not None and head is not None and row < head else (head, row, heads)
    if (small is not None and small < d) or (big is not None and big < (d if small is None else small * (count - 1) + d)):
        raise ValueError("out: rows or heads overlap")


def _query(q):
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not q.is_cuda or q.dtype not in _DTYPE:
        raise ValueError("q: expected a [tokens, heads, head_dim] bf16 or fp32 tensor on the GPU")
    return q.shape[1], q.shape[2], q.dtype, q.device


def _lens(name: str, lens: Sequence[int], rows: Optional[int]):
    """Host int32 lengths that sum to `rows` -> (the array, to be kept until the call is made, its address, count)."""
    a = array("i", lens)
    if rows is not None and sum(a) != rows:
        raise ValueError(f"{name}: expected lengths that sum to {rows}, got {sum(a)}")
    return a, a.buffer_info()[0], len(a)


def _spaced(device: torch.device, where: str, likely: bool, need, call) -> None:
    """call(workspace address or None, its bytes) with a workspace of need() bytes where it asks for
    one (likely: it will). A call that lacks it has enqueued nothing."""
    st = B.MTE_E_CAPACITY if likely else call(None, 0)
    if st == B.MTE_E_CAPACITY:
        n = need()
        ws = torch.empty(n, dtype=torch.uint8, device=device) if n else None
        st = call(ws.data_ptr() if n else None, n)
    B._check(st, where)


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_lens: Sequence[int], kv_lens: Sequence[int],
                    kv_index: Optional[Sequence[int]] = None, key_mask: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """mte_cross_attention: packed queries q [Tq, Hq, d] attend to packed conditioning tokens k, v
    [Tk, Hkv, d] of another length -> [Tq, Hq, d].

    q_lens / kv_lens: rows of each query / key sequence (0 allowed); kv_index: the key sequence
    of each query sequence (default: its own), so that one frame's conditioning can serve all
    ([0] * len(q_lens), as with TECache's batch_one); key_mask: uint8 or bool [Tk], 0 hides a
    token from every query; scale: default 1 / sqrt(d). A query that sees no token gets
    zeros. q, k, v (bf16 or fp32) may be strided over tokens and heads; out may be q."""
    hq, d, dtype, dev = _query(q)
    hkv = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0
    sq = _rows("q", q, dtype, hq, d, dev)
    sk, sv = _rows("k", k, dtype, hkv, d, dev), _rows("v", v, dtype, hkv, d, dev)
    if v.shape[0] != k.shape[0]:
        raise ValueError(f"v: expected {k.shape[0]} rows, got {v.shape[0]}")
    q_keep, ql, n_q = _lens("q_lens", q_lens, q.shape[0])
    kv_keep, kl, n_kv = _lens("kv_lens", kv_lens, k.shape[0])
    idx_keep, idx, n_idx = (None, None, n_q) if kv_index is None else _lens("kv_index", kv_index, None)
    if n_idx != n_q:
        raise ValueError(f"kv_index: expected {n_q} entries, got {n_idx}")
    if key_mask is not None:
        if not isinstance(key_mask, torch.Tensor) or key_mask.dtype not in (torch.uint8, torch.bool) or \
                key_mask.device != dev or tuple(key_mask.shape) != (k.shape[0],) or not key_mask.is_contiguous():
            raise ValueError(f"key_mask: expected a contiguous uint8 or bool tensor of {k.shape[0]} values on {dev}")
    so = None
    if out is not None:
        so = _rows("out", out, dtype, hq, d, dev)
        _out_rows(out, q, so)
    sc = 1.0 / math.sqrt(d) if scale is None else float(scale)

    def call(st):
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        shape = B.ATTN_SHAPE.pack(hq, hkv, d, _DTYPE[dtype], sc, *sq, *sk, *sv, *((hq * d, d) if so is None else so))
        _spaced(dev, "mte_cross_attention", n_kv > 0 and max(kv_keep) >= 384,
                lambda: B.mte_cross_attention_workspace(shape, ql, n_q, kl, n_kv, idx),
                lambda ws, n: B.lib.mte_cross_attention(
                    shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), None if key_mask is None else key_mask.data_ptr(),
                    ql, n_q, kl, n_kv, idx, o.data_ptr(), ws, n, st))
        return o
    return _on(dev, stream, (q, k, v, key_mask, out), call)


def prefix_attention(q: torch.Tensor, prefix_k: torch.Tensor, prefix_v: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                     q_lens: Sequence[int], kv_lens: Sequence[int], causal: bool = True, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """mte_prefix_attention: packed queries q [Tq, Hq, d] attend to the tokens that all sequences share,
    prefix_k, prefix_v [P, Hkv, d], and to their own, k, v [Tk, Hkv, d] -> [Tq, Hq, d].

    q_lens / kv_lens: query rows and own tokens of each sequence (0 allowed); causal: query u of q_lens[i] sees
    own tokens up to kv_lens[i] - q_lens[i] + u (all of the prefix in any case); scale: default
    1 / sqrt(d). A query that sees no token gets zeros. All may be strided over tokens and heads; out may be q, and
    otherwise shares no memory with what the call reads. Streams of single queries over a long prefix read it once
    between them."""
    hq, d, dtype, dev = _query(q)
    hkv = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0
    sq = _rows("q", q, dtype, hq, d, dev)
    sk, sv = _rows("k", k, dtype, hkv, d, dev), _rows("v", v, dtype, hkv, d, dev)
    spk, spv = _rows("prefix_k", prefix_k, dtype, hkv, d, dev), _rows("prefix_v", prefix_v, dtype, hkv, d, dev)
    p_len = prefix_k.shape[0]
    if v.shape[0] != k.shape[0]:
        raise ValueError(f"v: expected {k.shape[0]} rows, got {v.shape[0]}")
    if prefix_v.shape[0] != p_len:
        raise ValueError(f"prefix_v: expected {p_len} rows, got {prefix_v.shape[0]}")
    q_keep, ql, n = _lens("q_lens", q_lens, q.shape[0])
    kv_keep, kl, n_kv = _lens("kv_lens", kv_lens, k.shape[0])
    if n_kv != n:
        raise ValueError(f"kv_lens: expected {n} lengths, got {n_kv}")
    if p_len >= 1 << 31:
        raise ValueError(f"prefix_k: expected fewer than 2^31 rows, got {p_len}")
    so = None
    if out is not None:
        so = _rows("out", out, dtype, hq, d, dev)
        _out_rows(out, q, so)
    sc = 1.0 / math.sqrt(d) if scale is None else float(scale)

    def call(st):
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        shape = B.ATTN_SHAPE.pack(hq, hkv, d, _DTYPE[dtype], sc, *sq, *sk, *sv, *((hq * d, d) if so is None else so))
        _spaced(dev, "mte_prefix_attention", p_len >= 1024,
                lambda: B.mte_prefix_attention_workspace(shape, p_len, ql, kl, n),
                lambda ws, nb: B.lib.mte_prefix_attention(
                    shape, q.data_ptr(), prefix_k.data_ptr(), prefix_v.data_ptr(), *spk, *spv, p_len, k.data_ptr(),
                    v.data_ptr(), ql, kl, n, 1 if causal else 0, o.data_ptr(), ws, nb, st))
        return o
    return _on(dev, stream, (q, prefix_k, prefix_v, k, v, out), call)


class KV8Cache(NamedTuple):
    """A key/value cache in 8 bits (mte_kv8): blocks of 32 tokens of all kv heads, e4m3 codes with one
    power of two for each block, head and tensor. A sequence is a row of block numbers in a
    table and a length, both on the device and the caller's; any triple of such tensors
    serves as a cache."""
    k_codes: torch.Tensor    # uint8 [blocks, Hkv, d / 16, 32, 16]
    v_codes: torch.Tensor    # uint8 [blocks, Hkv, d, 32]
    scales: torch.Tensor     # float32 [blocks, Hkv, 2]


def kv8_cache(n_blocks: int, n_kv_heads: int, head_dim: int, device="cuda") -> KV8Cache:
    """An empty cache of n_blocks * 32 tokens (head_dim 64 or 128)."""
    if n_blocks <= 0 or n_kv_heads <= 0 or head_dim not in (64, 128):
        raise ValueError("expected n_blocks > 0, n_kv_heads > 0 and head_dim 64 or 128")
    return KV8Cache(torch.zeros((n_blocks, n_kv_heads, head_dim // 16, 32, 16), dtype=torch.uint8, device=device),
                    torch.zeros((n_blocks, n_kv_heads, head_dim, 32), dtype=torch.uint8, device=device),
                    torch.full((n_blocks, n_kv_heads, 2), 2.0 ** -126, dtype=torch.float32, device=device))


def _refuse_cache(cache, table, kv_lens, n: int, dev: torch.device):
    """Raises for what does not fit of a cache with the table and lengths of n sequences."""
    kc, vc, sc = cache
    for name, t, dt in (("k_codes", kc, torch.uint8), ("v_codes", vc, torch.uint8), ("scales", sc, torch.float32)):
        if not isinstance(t, torch.Tensor) or t.dtype != dt or t.device != dev or not t.is_contiguous():
            raise ValueError(f"cache {name}: expected a contiguous {dt} tensor on {dev}")
    if vc.dim() != 4:
        raise ValueError("cache v_codes: expected [blocks, heads, head_dim, 32]")
    nb, h, d, _ = vc.shape
    if vc.shape != (nb, h, d, 32) or kc.shape != (nb, h, d // 16, 32, 16) or sc.shape != (nb, h, 2):
        raise ValueError(f"cache: shapes {tuple(kc.shape)}, {tuple(vc.shape)}, {tuple(sc.shape)} do not fit together")
    if not isinstance(table, torch.Tensor) or table.dtype != torch.int32 or table.device != dev or \
            table.dim() != 2 or table.shape[0] != n or not 0 < table.shape[1] < 1 << 26 or \
            (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError(f"table: expected an int32 [{n}, blocks] tensor on {dev} with contiguous rows")
    raise ValueError(f"kv_lens: expected a contiguous int32 tensor of {n} lengths on {dev}")


def _cache(cache, table, kv_lens, n: int, dev: torch.device):
    """Checks a cache with the table and lengths of n sequences -> (mte_kv8 as bytes, heads, head_dim, width, table row)."""
    kc, vc, sc = cache
    try:
        nb, h, d, _ = vc.shape
        width, i = table.shape[1], dev.index
        fits = (kc.dtype is vc.dtype is torch.uint8 and sc.dtype is torch.float32 and
                table.dtype is kv_lens.dtype is torch.int32 and
                kc.get_device() == vc.get_device() == sc.get_device() == table.get_device() == kv_lens.get_device() == i and
                vc.shape == (nb, h, d, 32) and kc.shape == (nb, h, d // 16, 32, 16) and sc.shape == (nb, h, 2) and
                table.shape == (n, width) and 0 < width < 1 << 26 and (width == 1 or table.stride(1) == 1) and
                kv_lens.shape == (n,) and kc.is_contiguous() and vc.is_contiguous() and sc.is_contiguous() and
                kv_lens.is_contiguous())
    except (AttributeError, ValueError, IndexError):
        fits = False
    if not fits:
        _refuse_cache(cache, table, kv_lens, n, dev)
    return B.KV8.pack(kc.data_ptr(), vc.data_ptr(), sc.data_ptr(), nb, h, d), h, d, width, table.stride(0)


def kv8_append(cache, table: torch.Tensor, kv_lens: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               new_lens: Sequence[int], stream: Optional[torch.cuda.Stream] = None) -> None:
    """mte_kv8_append: rows k, v [sum(new_lens), Hkv, d] become the newest new_lens[i] tokens of each
    sequence, whose lengths afterwards are kv_lens (int32, device); table int32 [n, blocks], device."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3 or not k.is_cuda or k.dtype not in _DTYPE:
        raise ValueError("k: expected a [tokens, heads, head_dim] bf16 or fp32 tensor on the GPU")
    dev = k.device
    keep, lens, n = _lens("new_lens", new_lens, k.shape[0])
    c, h, d, width, row = _cache(cache, table, kv_lens, n, dev)
    sk, sv = _rows("k", k, k.dtype, h, d, dev), _rows("v", v, k.dtype, h, d, dev)
    if v.shape[0] != k.shape[0]:
        raise ValueError(f"v: expected {k.shape[0]} rows, got {v.shape[0]}")
    _on(dev, stream, (*cache, table, kv_lens, k, v),
        lambda st: B.mte_kv8_append(c, table.data_ptr(), width, row, kv_lens.data_ptr(), k.data_ptr(), *sk,
                                    v.data_ptr(), *sv, _DTYPE[k.dtype], lens, n, st) and None)


def kv8_read(cache, table: torch.Tensor, kv_lens: torch.Tensor, counts: Sequence[int],
             dtype: torch.dtype = torch.bfloat16, stream: Optional[torch.cuda.Stream] = None):
    """mte_kv8_read: the newest counts[i] tokens of each sequence -> (k, v), each
    [sum(counts), Hkv, d] of `dtype` (bf16 or fp32, both exact, but for bf16 magnitudes below 2^-126: rounded to
    multiples of 2^-133)."""
    if dtype not in _DTYPE:
        raise ValueError("dtype: expected torch.bfloat16 or torch.float32")
    dev = cache[0].device
    if dev.type != "cuda":
        raise ValueError("cache: expected tensors on the GPU")
    keep, lens, n = _lens("counts", counts, None)
    c, h, d, width, row = _cache(cache, table, kv_lens, n, dev)
    total = sum(keep)
    if n and min(keep) < 0:
        raise ValueError("counts: expected lengths of 0 or more")

    def call(st):
        k = torch.empty((total, h, d), dtype=dtype, device=dev)
        v = torch.empty((total, h, d), dtype=dtype, device=dev)
        B.mte_kv8_read(c, table.data_ptr(), width, row, kv_lens.data_ptr(), lens, n, k.data_ptr(), v.data_ptr(),
                       _DTYPE[dtype], st)
        return k, v
    return _on(dev, stream, (*cache, table, kv_lens), call)


def kv8_attention(q: torch.Tensor, cache, table: torch.Tensor, kv_lens: torch.Tensor, q_lens: Sequence[int],
                  causal: bool = False, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """mte_kv8_attention: packed queries q [Tq, Hq, d] attend to their sequence's cached tokens ->
    [Tq, Hq, d]. causal: query u of q_lens[i] sees the tokens up to kv_lens[i] - q_lens[i] + u
    (append its own token first). out may be q. The work is split for sequences as long as the table is wide:
    a narrower view table[:, :m] serves shorter ones better."""
    hq, d, dtype, dev = _query(q)
    keep, lens, n = _lens("q_lens", q_lens, q.shape[0])
    c, hkv, dc, width, row = _cache(cache, table, kv_lens, n, dev)
    sq = _rows("q", q, dtype, hq, dc, dev)
    so = None
    if out is not None:
        so = _rows("out", out, dtype, hq, d, dev)
        _out_rows(out, q, so)
    sc = 1.0 / math.sqrt(d) if scale is None else float(scale)

    def call(st):
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        shape = B.ATTN_SHAPE.pack(hq, hkv, d, _DTYPE[dtype], sc, *sq, 0, 0, 0, 0,
                                  *((hq * d, d) if so is None else so))
        _spaced(dev, "mte_kv8_attention", width > 16, lambda: B.mte_kv8_attention_workspace(shape, lens, n, width),
                lambda ws, nb: B.lib.mte_kv8_attention(shape, c, table.data_ptr(), width, row, kv_lens.data_ptr(),
                                                       q.data_ptr(), lens, n, 1 if causal else 0, o.data_ptr(), ws, nb,
                                                       st))
        return o
    return _on(dev, stream, (q, *cache, table, kv_lens, out), call)


def _pixels(name: str, t: torch.Tensor):
    """(image stride, row stride, pixels) of a channels-last [N, P, C] or [N, H, W, C] tensor."""
    shape, st = t.shape, t.stride()
    if shape[-1] > 1 and st[-1] != 1:
        raise ValueError(f"{name}: expected contiguous channels (the last dimension), got strides {st}")
    if len(shape) == 3:
        row, px = st[1], shape[1]
    else:
        h, w = shape[1], shape[2]
        if h > 1 and w > 1 and st[1] != w * st[2]:
            raise ValueError(f"{name}: expected pixels at one stride, got strides {st}")
        row, px = st[2] if w > 1 else st[1], h * w
    return st[0] if shape[0] > 1 else 0, row if px > 1 else 0, px


def group_norm(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None,
               beta: Optional[torch.Tensor] = None, eps: float = 1e-5, act: Optional[str] = None,
               out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """mte_group_norm: act(group norm of x), x channels last [N, P, C] or [N, H, W, C] (bf16 or fp32; a
    channels_last NCHW tensor is x.permute(0, 2, 3, 1)), channels contiguous, pixels at one stride
    (a slice of a wider buffer's channels is fine). gamma, beta: [C] of x's dtype; act: None or
    "silu". out: like x, or x itself."""
    if not isinstance(x, torch.Tensor) or x.dim() not in (3, 4) or not x.is_cuda or x.dtype not in _DTYPE:
        raise ValueError("x: expected a [N, P, C] or [N, H, W, C] bf16 or fp32 tensor on the GPU")
    if act not in _ACT:
        raise ValueError(f"act: expected None or 'silu', got {act!r}")
    dev, dtype, C = x.device, x.dtype, x.shape[-1]
    for name, t in (("gamma", gamma), ("beta", beta)):
        if t is not None and (t.dtype != dtype or t.device != dev or tuple(t.shape) != (C,) or not t.is_contiguous()):
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of {C} values on {dev}")
    xi, xr, px = _pixels("x", x)
    n = x.shape[0]
    if not 0 < groups < 1 << 31 or max(n, px, C) >= 1 << 31:      # (counted in 31 bits)
        raise ValueError(f"x, groups: expected fewer than 2^31 images, pixels, channels and groups, got {n} of {px} of "
                         f"{C} in {groups}")
    oi = orow = 0
    if out is not None:
        if not isinstance(out, torch.Tensor) or out.shape != x.shape or out.dtype != dtype or out.device != dev:
            raise ValueError(f"out: expected a {dtype} tensor of shape {tuple(x.shape)} on {dev}")
        oi, orow, _ = _pixels("out", out)
        if (px > 1 and orow < C) or (n > 1 and oi < (px - 1) * orow + C):
            raise ValueError("out: pixels or images overlap")

    def call(st):
        if out is None:
            y, yi, yr = torch.empty_like(x, memory_format=torch.contiguous_format), px * C, C
        else:
            y, yi, yr = out, oi, orow
        _spaced(dev, "mte_group_norm", False, lambda: B.mte_group_norm_workspace(n, px, C, groups, _DTYPE[dtype]),
                lambda ws, nb: B.lib.mte_group_norm(
                    x.data_ptr(), xr, xi, n, px, C, groups, None if gamma is None else gamma.data_ptr(),
                    None if beta is None else beta.data_ptr(), eps, _ACT[act], _DTYPE[dtype], y.data_ptr(), yr, yi, ws,
                    nb, st))
        return y
    return _on(dev, stream, (x, gamma, beta, out), call)
