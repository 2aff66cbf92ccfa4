"""Torch-facing wrappers of include/mte_proj.h: what stands between the encoder's hidden states and
the attention that reads them (``conditioning``): linear layers in 8-bit integers, rotary positions.

Conventions as in ``conditioning``: tensors in, tensors out, every step in libmte's HIP kernels,
nothing falls back, no gradients (a rotation's is its inverse), workspaces from torch's
allocator on the stream of the call.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import binding as B
from .conditioning import _ACT, _DTYPE, _on, _out_rows, _rows, _spaced


class I8Rows(NamedTuple):
    """Rows in 8 bits (mte_i8_quantize_rows): row r is codes[r, :cols] * scales[r]."""
    codes: torch.Tensor      # int8 [rows, cols rounded up to a multiple of 128], zeros past cols
    scales: torch.Tensor     # float32 [rows]
    cols: int


def _matrix(name: str, x, most: int = B.MTE_I8_COLS):
    """A [..., K] bf16 or fp32 GPU tensor, K up to `most`, as rows -> (the 2-d view, its row stride)."""
    if not isinstance(x, torch.Tensor) or x.dim() < 1 or not x.is_cuda or x.dtype not in _DTYPE:
        raise ValueError(f"{name}: expected a [..., channels] bf16 or fp32 tensor on the GPU")
    k = x.shape[-1]
    if not 0 < k <= most:
        raise ValueError(f"{name}: expected 1 to {most} channels, got {k}")
    if x.dim() != 2:
        try:
            x = x.view(-1, k) if x.numel() else x.reshape(0, k)
        except RuntimeError:
            raise ValueError(f"{name}: expected rows at one stride, got shape {tuple(x.shape)}, strides {x.stride()}") from None
    row, one = x.stride()
    if k > 1 and one != 1:
        raise ValueError(f"{name}: expected contiguous channels, got strides {x.stride()}")
    if x.shape[0] >= 1 << 31:                        # (counted in 31 bits)
        raise ValueError(f"{name}: expected fewer than 2^31 rows, got {x.shape[0]}")
    return x, row if x.shape[0] > 1 else 0


def _meet(a, b) -> bool:
    """Whether two pieces of memory, rows at one stride as (address, rows, bytes from row to row, bytes of a row),
    share a byte. Rows that lie between the other's are apart; at two strides that do not tell, they are taken to meet."""
    (p, m, s, w), (q, n, t, u) = ((x[0], 1, 0, (x[1] - 1) * x[2] + x[3]) if x[2] <= x[3] else x for x in (a, b))
    if p + (m - 1) * s + w <= q or q + (n - 1) * t + u <= p:
        return False
    every = math.gcd(s if m > 1 else 0, t if n > 1 else 0)
    at = (q - p) % every if every else 0
    return at < w or at + u > every


def _whole(t: torch.Tensor):
    return t.data_ptr(), 1, 0, t.numel() * t.element_size()


def _i8_rows(name: str, t, dev: torch.device):
    """Checks 8-bit rows -> (codes, scales, rows, cols)."""
    codes, scales, cols = t
    try:                                             # one expression: a call is bound by the host
        n, pitch = codes.shape
        fits = (codes.dtype is torch.int8 and scales.dtype is torch.float32 and
                codes.get_device() == scales.get_device() == dev.index and 0 < cols <= B.MTE_I8_COLS and
                pitch == (cols + 127) & -128 and scales.shape == (n,) and n < 1 << 31 and codes.is_contiguous() and
                scales.is_contiguous() and codes.data_ptr() % 16 == 0)
    except (AttributeError, ValueError, TypeError):
        fits = False
    if fits:
        return codes, scales, n, cols
    if not isinstance(cols, int) or not 0 < cols <= B.MTE_I8_COLS:
        raise ValueError(f"{name}: expected 1 to {B.MTE_I8_COLS} channels, got {cols}")
    raise ValueError(f"{name}: expected fewer than 2^31 rows as contiguous int8 codes [rows, {(cols + 127) // 128 * 128}], "
                     f"aligned to 16 bytes, and float32 scales [rows], both on {dev}")


def quantize_rows(x: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> I8Rows:
    """mte_i8_quantize_rows: the rows of x [..., K] (bf16 or fp32) in 8 bits, a scale each: the weight
    [N, K] of a linear layer once, or tokens that several layers read."""
    x, row = _matrix("x", x)
    m, k = x.shape
    dev = x.device

    def call(st):
        codes = torch.empty((m, (k + 127) // 128 * 128), dtype=torch.int8, device=dev)
        scales = torch.empty((m,), dtype=torch.float32, device=dev)
        B.mte_i8_quantize_rows(x.data_ptr(), row, m, k, _DTYPE[x.dtype], codes.data_ptr(), scales.data_ptr(), st)
        return codes, scales
    return I8Rows(*_on(dev, stream, (x,), call), k)


def i8_linear(x, weight: I8Rows, bias: Optional[torch.Tensor] = None, act: Optional[str] = None,
              dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """mte_i8_linear: act(x weight^T + bias) with tokens and weight in 8 bits -> [..., N].

    x: [..., K] bf16 or fp32, quantised within the call, or the I8Rows of M tokens; weight: I8Rows of
    N rows of K; bias: [N] of the result's dtype; act: None or "silu"; dtype of the result: bf16 or fp32, by
    default x's (I8Rows: bf16). out: [M, N] or x's leading shape, rows at one stride; it shares no memory with what
    the call reads (workgroups store rows while others read x)."""
    if act not in _ACT:
        raise ValueError(f"act: expected None or 'silu', got {act!r}")
    if isinstance(x, torch.Tensor):
        lead = x.shape[:-1]
        src, row = _matrix("x", x)
        m, k = src.shape
        dev, x_type, x_scales = src.device, _DTYPE[src.dtype], None
        dtype = src.dtype if dtype is None else dtype
    else:
        dev = x[0].device
        if dev.type != "cuda":
            raise ValueError("x: expected tensors on the GPU")
        src, x_scales, m, k = _i8_rows("x", x, dev)
        lead, row, x_type = (m,), 0, B.MTE_I8_CODES
        dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in _DTYPE:
        raise ValueError("dtype: expected torch.bfloat16 or torch.float32")
    w, w_scales, n, kw = _i8_rows("weight", weight, dev)
    if kw != k:
        raise ValueError(f"weight: expected rows of {k} channels, got {kw}")
    if n == 0:
        raise ValueError("weight: expected at least one row")
    if bias is not None and (not isinstance(bias, torch.Tensor) or bias.dtype != dtype or bias.device != dev or
                             tuple(bias.shape) != (n,) or not bias.is_contiguous()):
        raise ValueError(f"bias: expected a contiguous {dtype} tensor of {n} values on {dev}")
    orow = n
    if out is not None:
        if not isinstance(out, torch.Tensor) or out.dtype != dtype or out.device != dev or tuple(out.shape) != (*lead, n):
            raise ValueError(f"out: expected a {dtype} tensor of shape {(*lead, n)} on {dev}")
        flat, orow = _matrix("out", out, n)
        if flat.shape[0] > 1 and orow < n:
            raise ValueError("out: rows overlap")
        to, es = (out.data_ptr(), m, orow * out.element_size(), n * out.element_size()), src.element_size()
        reads = [(src.data_ptr(), m, row * es, k * es)] if x_scales is None else [_whole(src), _whole(x_scales)]
        reads += [_whole(t) for t in (w, w_scales, bias) if t is not None]
        if m and any(_meet(to, r) for r in reads):
            raise ValueError("out: expected memory that the call does not read")

    def call(st):
        y = w.new_empty((*lead, n), dtype=dtype) if out is None else out
        args = (src.data_ptr(), row, None if x_scales is None else x_scales.data_ptr(), x_type, m, k, w.data_ptr(),
                w_scales.data_ptr(), n, None if bias is None else bias.data_ptr(), _ACT[act], y.data_ptr(), orow, _DTYPE[dtype])
        _spaced(dev, "mte_i8_linear", x_scales is None and 32 < m < 32768, lambda: B.mte_i8_linear_workspace(x_type, m, k, n),
                lambda ws, nb: B.lib.mte_i8_linear(*args, ws, nb, st))
        return y
    return _on(dev, stream, (src, x_scales, w, w_scales, bias, out), call)


def rotary_frequencies(rot_dim: int, theta: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       original_length: Optional[int] = None, fast: float = 32.0, slow: float = 1.0,
                       device="cuda") -> Tuple[torch.Tensor, float]:
    """Angular frequencies of rot_dim / 2 pairs, w_i = theta^(-2 i / rot_dim), as the float64 tensor that
    ``rotary`` takes, and its factor. scaling, for contexts `factor` = s times as long as the
    model was trained for:
      "linear": w_i / s (positions are interpolated);
      "ntk":    theta s^(r / (r - 2)) in place of theta (r = rot_dim > 2; the slowest pair by s, the fastest not);
      "yarn":   g w_i + (1 - g) w_i / s, g = (L w_i / 2 pi - slow) / (fast - slow) within [0, 1]: pairs that turn at
                least `fast` times over the original_length L are kept, those under `slow` turns interpolated;
                the returned factor is 0.1 ln(s) + 1 for s > 1, which multiplies queries and keys alike."""
    if not isinstance(rot_dim, int) or rot_dim <= 0 or rot_dim % 2:
        raise ValueError(f"rot_dim: expected an even number above 0, got {rot_dim}")
    if not (theta > 0 and math.isfinite(theta)) or not (factor > 0 and math.isfinite(factor)):
        raise ValueError("theta, factor: expected finite numbers above 0")
    if scaling not in (None, "linear", "ntk", "yarn"):
        raise ValueError(f"scaling: expected None, 'linear', 'ntk' or 'yarn', got {scaling!r}")
    gain = 1.0
    if scaling == "ntk":
        if rot_dim == 2:
            raise ValueError("rot_dim: expected more than one pair with 'ntk'")
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    w = [theta ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling == "linear":
        w = [x / factor for x in w]
    elif scaling == "yarn":
        if original_length is None or original_length <= 0 or not fast > slow:
            raise ValueError("original_length, fast, slow: expected a length above 0 and fast > slow with 'yarn'")
        keep = [min(max((original_length * x / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0) for x in w]
        w = [g * x + (1 - g) * x / factor for g, x in zip(keep, w)]
        gain = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return torch.tensor(w, dtype=torch.float64, device=device), gain


def rotary(q: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, k: Optional[torch.Tensor] = None,
           interleaved: bool = False, sections: Optional[Sequence[int]] = None, factor: float = 1.0,
           inverse: bool = False, out=None, stream: Optional[torch.cuda.Stream] = None):
    """mte_rotary: rotates the first 2 len(freq) channels of every head of q [T, Hq, d] and, in the same
    launch, of k [T, Hk, d], by positions * freq -> (q, k), k None where none was given.

    positions: int32 [T], or [axes, T] (2 to 4 axes, such as the encoder's t, h, w) with sections, the pairs of
    each axis; freq: float64, device (``rotary_frequencies``); interleaved: pairs are neighbouring
    channels instead of the two halves; inverse: turns back (with the same factor, the gradient).
    out: (q_out, k_out or None), which may be q and k themselves, and otherwise share no memory with what the call
    reads, nor with each other. q and k may be strided over tokens and heads."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not q.is_cuda or q.dtype not in _DTYPE:
        raise ValueError("q: expected a [tokens, heads, head_dim] bf16 or fp32 tensor on the GPU")
    t, hq, d = q.shape
    dev, dtype = q.device, q.dtype
    if max(t, hq, d) >= 1 << 31:                     # (counted in 31 bits)
        raise ValueError(f"q: expected fewer than 2^31 tokens and heads, got shape {tuple(q.shape)}")
    sq, hk, sk = _rows("q", q, dtype, hq, d, dev), 0, (0, 0)
    if k is not None:
        hk = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0
        sk = _rows("k", k, dtype, hk, d, dev)
        if k.shape[0] != t:
            raise ValueError(f"k: expected {t} rows, got {k.shape[0]}")
        if not 0 < hk < 1 << 31:
            raise ValueError(f"k: expected 1 to 2^31 - 1 heads, got {hk}")
    if not isinstance(freq, torch.Tensor) or freq.dtype != torch.float64 or freq.device != dev or freq.dim() != 1 or \
            not 0 < freq.shape[0] <= d // 2 or not freq.is_contiguous():
        raise ValueError(f"freq: expected a contiguous float64 tensor of 1 to {d // 2} values on {dev}")
    pairs = freq.shape[0]
    axes = 1 if sections is None else len(sections)
    shape = (t,) if sections is None else (axes, t)
    if sections is not None and (not 2 <= axes <= 4 or min(sections) < 0 or sum(sections) != pairs):
        raise ValueError(f"sections: expected 2 to 4 counts that sum to {pairs}, got {tuple(sections)}")
    if not isinstance(positions, torch.Tensor) or positions.dtype != torch.int32 or positions.device != dev or \
            tuple(positions.shape) != shape or (t > 1 and positions.stride(-1) != 1):
        raise ValueError(f"positions: expected an int32 tensor of shape {shape} on {dev}, tokens contiguous")
    if sections is not None and positions.stride(0) < 0:
        raise ValueError("positions: expected strides of 0 or more")
    if not math.isfinite(factor):
        raise ValueError("factor: expected a finite number")
    if out is None:
        oq = ok = None
    else:
        oq, ok = out
        if (ok is None) != (k is None):
            raise ValueError("out: expected a pair (q, k), k None where there is none")
        for name, o, x, h in (("out q", oq, q, hq), ("out k", ok, k, hk)):
            if x is not None:
                _out_rows(o, x, _rows(name, o, dtype, h, d, dev))
    sec = (0, 0, 0, 0) if sections is None else (*sections, 0, 0, 0)[:4]

    def call(st):
        yq = torch.empty_like(q, memory_format=torch.contiguous_format) if oq is None else oq
        yk = (None if k is None else torch.empty_like(k, memory_format=torch.contiguous_format)) if ok is None else ok
        so = (hq * d, d) if oq is None else _rows("out q", oq, dtype, hq, d, dev)
        ko = (hk * d, d) if ok is None else _rows("out k", ok, dtype, hk, d, dev)
        s = B.ROTARY_SHAPE.pack(hq, hk, d, 2 * pairs, _DTYPE[dtype], 1 if interleaved else 0, 1 if inverse else 0, axes,
                                *sec, factor, *sq, *sk, *so, *ko)
        B.mte_rotary(s, q.data_ptr(), None if k is None else k.data_ptr(), positions.data_ptr(),
                     0 if sections is None else positions.stride(0), freq.data_ptr(), t, yq.data_ptr(),
                     None if yk is None else yk.data_ptr(), st)
        return yq, yk
    return _on(dev, stream, (q, k, positions, freq, oq, ok), call)
