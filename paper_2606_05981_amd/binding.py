"""ctypes binding of libmte (include/mte.h, mte_vision.h, mte_cond.h, mte_proj.h): argument marshalling only.

Every function keeps the C name and returns what the C call returns, except
that a negative status raises MteError. Device buffers are passed as integer
addresses (``tensor.data_ptr()``) and streams as ``hipStream_t`` handles
(``torch.cuda.current_stream().cuda_stream``). There is no fallback: if the
library is not built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmte.so")

MTE_F32, MTE_BF16 = 0, 1
MTE_MROPE_SECTIONS, MTE_MROPE_INTERLEAVED = 0, 1
MTE_WEIGHTS_DTYPE, MTE_WEIGHTS_E4M3 = 0, 1
MTE_E_CAPACITY = -2
STATUS = {0: "MTE_OK", -1: "MTE_E_INVALID", -2: "MTE_E_CAPACITY", -3: "MTE_E_HIP",
          -4: "MTE_E_OOM", -5: "MTE_E_UNSUPPORTED"}
MTE_ACT_NONE, MTE_ACT_SILU = 0, 1
MTE_KV8_BLOCK = 32
MTE_I8_CODES, MTE_I8_COLS = 2, 131071
KERNEL_CLASSES = {"qkv_gemm": 0, "attention": 1, "o_gemm": 2, "gate_up_gemm": 3, "down_gemm": 4}


class MteError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({mte_status_string(status)})")


class mte_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("mrope_section", C.c_int32 * 3), ("mrope_layout", C.c_int32),
                ("qk_norm", C.c_int32), ("dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("max_tokens", C.c_int32), ("max_batch", C.c_int32), ("max_seq", C.c_int32),
                ("weight_format", C.c_int32)]


class mte_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "w_q", "w_k", "w_v", "q_norm", "k_norm",
                                          "w_o", "mlp_norm", "w_gate", "w_up", "w_down")]


class mte_weights(C.Structure):
    _fields_ = [("layers", C.POINTER(mte_layer_weights)), ("final_norm", C.c_void_p)]


class mte_seq_layout(C.Structure):
    _fields_ = [("n_text_before", C.c_int32), ("grid_t", C.c_int32), ("grid_h", C.c_int32),
                ("grid_w", C.c_int32), ("n_text_after", C.c_int32)]


class mte_vision_config(C.Structure):
    _fields_ = [("depth", C.c_int32), ("hidden", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("ffn", C.c_int32), ("patch", C.c_int32), ("merge", C.c_int32), ("in_channels", C.c_int32),
                ("out_hidden", C.c_int32), ("ln_eps", C.c_float), ("rope_theta", C.c_float),
                ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("max_images", C.c_int32),
                ("max_side", C.c_int32)]


VISION_LAYER_FIELDS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b", "w_fc1", "b_fc1",
                       "w_fc2", "b_fc2")
VISION_OUTER_FIELDS = ("patch_w", "patch_b", "merge_ln_g", "merge_ln_b", "merge_w1", "merge_b1", "merge_w2",
                       "merge_b2")


class mte_vision_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in VISION_LAYER_FIELDS]


class mte_vision_weights(C.Structure):
    _fields_ = [("patch_w", C.c_void_p), ("patch_b", C.c_void_p),
                ("layers", C.POINTER(mte_vision_layer_weights)),
                ("merge_ln_g", C.c_void_p), ("merge_ln_b", C.c_void_p), ("merge_w1", C.c_void_p),
                ("merge_b1", C.c_void_p), ("merge_w2", C.c_void_p), ("merge_b2", C.c_void_p)]


class mte_attn_shape(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("scale", C.c_float),
                ("q_row", C.c_int64), ("q_head", C.c_int64), ("k_row", C.c_int64), ("k_head", C.c_int64),
                ("v_row", C.c_int64), ("v_head", C.c_int64), ("o_row", C.c_int64), ("o_head", C.c_int64)]


class mte_kv8(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("scales", C.c_void_p),
                ("n_blocks", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class mte_rotary_shape(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_k_heads", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32),
                ("dtype", C.c_int32), ("interleaved", C.c_int32), ("inverse", C.c_int32), ("n_axes", C.c_int32),
                ("section", C.c_int32 * 4), ("factor", C.c_float),
                ("q_row", C.c_int64), ("q_head", C.c_int64), ("k_row", C.c_int64), ("k_head", C.c_int64),
                ("qo_row", C.c_int64), ("qo_head", C.c_int64), ("ko_row", C.c_int64), ("ko_head", C.c_int64)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_05981_amd.build`")
lib = C.CDLL(LIB_PATH)

_P = C.c_void_p
_sig = {
    "mte_config_validate": (C.c_int, [C.POINTER(mte_config)]),
    "mte_check_batch": (C.c_int, [C.POINTER(mte_config), C.POINTER(C.c_int32), C.c_int32,
                                  C.POINTER(C.c_int32)]),
    "mte_encoder_create": (C.c_int, [C.POINTER(mte_config), C.POINTER(mte_weights), _P,
                                     C.POINTER(_P)]),
    "mte_encode": (C.c_int, [_P, _P, _P, C.POINTER(C.c_int32), C.c_int32, _P, _P]),
    "mte_encode_static": (C.c_int, [_P, _P, _P, C.POINTER(C.c_int32), C.c_int32, _P, _P]),
    "mte_encode_layers": (C.c_int, [_P, _P, _P, C.POINTER(C.c_int32), C.c_int32, C.c_int32,
                                    C.c_int32, _P, _P]),
    "mte_build_positions": (C.c_int, [C.POINTER(mte_seq_layout), C.c_int32, _P, _P]),
    "mte_encoder_reserve_prefix": (C.c_int, [_P, C.c_int32]),
    "mte_encode_prefixed": (C.c_int, [_P, _P, _P, C.c_int32, _P, _P, C.POINTER(C.c_int32), C.c_int32, _P,
                                      _P, _P]),
    "mte_encoder_destroy": (None, [_P]),
    "mte_status_string": (C.c_char_p, [C.c_int]),
    "mte_timing_enable": (C.c_int, [_P, C.c_int32, C.c_int32]),
    "mte_timing_read": (C.c_int, [_P, C.POINTER(C.c_int32), C.POINTER(C.c_double)]),
    "mte_timing_disable": (C.c_int, [_P]),
    "mte_quantize_e4m3_rows": (C.c_int, [_P, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P]),
    "mte_vision_config_validate": (C.c_int, [C.POINTER(mte_vision_config)]),
    "mte_vision_create": (C.c_int, [C.POINTER(mte_vision_config), C.POINTER(mte_vision_weights), _P,
                                    C.POINTER(_P)]),
    "mte_vision_encode": (C.c_int, [_P, _P, C.c_int32, C.c_int32, C.c_int32, _P, _P]),
    "mte_vision_encode_strided": (C.c_int, [_P, _P, C.c_int32, C.c_int32, C.c_int32, _P, C.c_int32, _P]),
    "mte_vision_destroy": (None, [_P]),
    # descriptors and host arrays as plain addresses: a ctypes object, bytes of the struct or an int
    "mte_cross_attention": (C.c_int, [_P, _P, _P, _P, _P, _P, C.c_int32, _P, C.c_int32, _P, _P, _P, C.c_int64, _P]),
    "mte_cross_attention_workspace": (C.c_int64, [_P, _P, C.c_int32, _P, C.c_int32, _P]),
    "mte_kv8_append": (C.c_int, [_P, _P, C.c_int32, C.c_int64, _P, _P, C.c_int64, C.c_int64, _P, C.c_int64,
                                 C.c_int64, C.c_int32, _P, C.c_int32, _P]),
    "mte_kv8_read": (C.c_int, [_P, _P, C.c_int32, C.c_int64, _P, _P, C.c_int32, _P, _P, C.c_int32, _P]),
    "mte_kv8_attention": (C.c_int, [_P, _P, _P, C.c_int32, C.c_int64, _P, _P, _P, C.c_int32, C.c_int32, _P, _P,
                                    C.c_int64, _P]),
    "mte_kv8_attention_workspace": (C.c_int64, [_P, _P, C.c_int32, C.c_int32]),
    "mte_group_norm": (C.c_int, [_P, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, _P,
                                 C.c_float, C.c_int32, C.c_int32, _P, C.c_int64, C.c_int64, _P, C.c_int64, _P]),
    "mte_group_norm_workspace": (C.c_int64, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "mte_i8_pitch": (C.c_int64, [C.c_int32]),
    "mte_i8_quantize_rows": (C.c_int, [_P, C.c_int64, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P]),
    "mte_i8_linear": (C.c_int, [_P, C.c_int64, _P, C.c_int32, C.c_int32, C.c_int32, _P, _P, C.c_int32, _P, C.c_int32, _P,
                                C.c_int64, C.c_int32, _P, C.c_int64, _P]),
    "mte_i8_linear_workspace": (C.c_int64, [C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "mte_prefix_attention": (C.c_int, [_P, _P, _P, _P, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_int32, _P, _P, _P, _P,
                                       C.c_int32, C.c_int32, _P, _P, C.c_int64, _P]),
    "mte_prefix_attention_workspace": (C.c_int64, [_P, C.c_int32, _P, _P, C.c_int32]),
    "mte_rotary": (C.c_int, [_P, _P, _P, _P, C.c_int64, _P, C.c_int32, _P, _P, _P]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(lib, _name)
    _f.restype, _f.argtypes = _res, _args


def _check(st: int, where: str) -> int:
    if st < 0:
        raise MteError(st, where)
    return st


def _i32(values: Sequence[int]):
    return (C.c_int32 * len(values))(*[int(v) for v in values])


def make_config(n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, rms_eps=1e-6,
                rope_theta=5e6, mrope_section=(24, 20, 20), mrope_layout=0, qk_norm=1,
                dtype=MTE_BF16, out_dtype=None, max_tokens=4096, max_batch=64,
                max_seq=4096, weight_format=MTE_WEIGHTS_DTYPE) -> mte_config:
    c = mte_config()
    c.n_layers, c.hidden, c.n_q_heads, c.n_kv_heads = n_layers, hidden, n_q_heads, n_kv_heads
    c.head_dim, c.ffn, c.rms_eps, c.rope_theta = head_dim, ffn, rms_eps, rope_theta
    c.mrope_section[:] = list(mrope_section)
    c.mrope_layout, c.qk_norm, c.dtype = mrope_layout, qk_norm, dtype
    c.out_dtype = dtype if out_dtype is None else out_dtype
    c.max_tokens, c.max_batch, c.max_seq = max_tokens, max_batch, max_seq
    c.weight_format = weight_format
    return c


def mte_status_string(status: int) -> str:
    return lib.mte_status_string(int(status)).decode()


def mte_config_validate(cfg: mte_config) -> int:
    return lib.mte_config_validate(C.byref(cfg))


def mte_check_batch(cfg: Optional[mte_config], seq_lens: Optional[Sequence[int]],
                    batch: Optional[int] = None):
    """Returns (status, total_tokens)."""
    tot = C.c_int32(-1)
    arr = _i32(seq_lens) if seq_lens is not None else None
    n = len(seq_lens) if batch is None else batch
    st = lib.mte_check_batch(C.byref(cfg) if cfg is not None else None, arr, n, C.byref(tot))
    return st, tot.value


def mte_encoder_create(cfg: mte_config, layers: Sequence[dict], final_norm: int, stream: int) -> int:
    """layers: per layer a dict of device addresses keyed like mte_layer_weights."""
    arr = (mte_layer_weights * max(1, len(layers)))()
    for i, L in enumerate(layers):
        for k, v in L.items():
            setattr(arr[i], k, v)
    w = mte_weights(arr if layers else None, final_norm)
    h = _P()
    _check(lib.mte_encoder_create(C.byref(cfg), C.byref(w), stream, C.byref(h)), "mte_encoder_create")
    return h.value


def mte_encode(enc: int, embeds: int, pos_thw: int, seq_lens: Sequence[int], batch: int,
               out_hidden: int, stream: int) -> int:
    return _check(lib.mte_encode(enc, embeds, pos_thw, _i32(seq_lens), batch, out_hidden, stream),
                  "mte_encode")


def mte_encode_static(enc: int, embeds: int, pos_thw: int, seq_lens: Sequence[int], batch: int,
                      out_hidden: int, stream: int) -> int:
    return _check(lib.mte_encode_static(enc, embeds, pos_thw, _i32(seq_lens), batch, out_hidden, stream),
                  "mte_encode_static")


def mte_encode_layers(enc: int, h_in: int, pos_thw: int, seq_lens: Sequence[int], batch: int,
                      layer_begin: int, layer_end: int, h_out: int, stream: int) -> int:
    return _check(lib.mte_encode_layers(enc, h_in, pos_thw, _i32(seq_lens), batch, layer_begin,
                                        layer_end, h_out, stream), "mte_encode_layers")


def mte_build_positions(layouts: Sequence[Sequence[int]], pos_thw: int, stream: int) -> int:
    arr = (mte_seq_layout * max(1, len(layouts)))()
    for i, s in enumerate(layouts):
        arr[i] = mte_seq_layout(*[int(v) for v in s])
    return _check(lib.mte_build_positions(arr, len(layouts), pos_thw, stream), "mte_build_positions")


def mte_encoder_reserve_prefix(enc: int, max_prefix: int) -> int:
    return _check(lib.mte_encoder_reserve_prefix(enc, max_prefix), "mte_encoder_reserve_prefix")


def mte_encode_prefixed(enc: int, prefix_embeds: int, prefix_pos: int, prefix_len: int, embeds: int,
                        pos_thw: int, seq_lens: Sequence[int], batch: int, out_prefix: int,
                        out_hidden: int, stream: int) -> int:
    return _check(lib.mte_encode_prefixed(enc, prefix_embeds, prefix_pos, prefix_len, embeds, pos_thw,
                                          _i32(seq_lens), batch, out_prefix, out_hidden, stream),
                  "mte_encode_prefixed")


def mte_encoder_destroy(enc: int) -> None:
    lib.mte_encoder_destroy(enc)


def mte_timing_enable(enc: int, kernel_class: int, capacity: int) -> int:
    return _check(lib.mte_timing_enable(enc, kernel_class, capacity), "mte_timing_enable")


def mte_timing_read(enc: int):
    n, ms = C.c_int32(0), C.c_double(0.0)
    _check(lib.mte_timing_read(enc, C.byref(n), C.byref(ms)), "mte_timing_read")
    return n.value, ms.value


def mte_timing_disable(enc: int) -> int:
    return _check(lib.mte_timing_disable(enc), "mte_timing_disable")


def mte_quantize_e4m3_rows(src: int, src_dtype: int, rows: int, cols: int, codes: int, scales: int,
                           stream: int) -> int:
    return _check(lib.mte_quantize_e4m3_rows(src, src_dtype, rows, cols, codes, scales, stream),
                  "mte_quantize_e4m3_rows")


def make_vision_config(depth, hidden, n_heads, head_dim, ffn, patch=16, merge=2, in_channels=3, out_hidden=2048,
                       ln_eps=1e-6, rope_theta=10000.0, dtype=MTE_BF16, out_dtype=None, max_images=16,
                       max_side=256) -> mte_vision_config:
    c = mte_vision_config()
    c.depth, c.hidden, c.n_heads, c.head_dim, c.ffn = depth, hidden, n_heads, head_dim, ffn
    c.patch, c.merge, c.in_channels, c.out_hidden = patch, merge, in_channels, out_hidden
    c.ln_eps, c.rope_theta, c.dtype = ln_eps, rope_theta, dtype
    c.out_dtype = dtype if out_dtype is None else out_dtype
    c.max_images, c.max_side = max_images, max_side
    return c


def mte_vision_config_validate(cfg: mte_vision_config) -> int:
    return lib.mte_vision_config_validate(C.byref(cfg))


def mte_vision_create(cfg: mte_vision_config, outer: dict, layers: Sequence[dict], stream: int) -> int:
    """outer: device addresses keyed like VISION_OUTER_FIELDS; layers: per block keyed like
    VISION_LAYER_FIELDS."""
    arr = (mte_vision_layer_weights * max(1, len(layers)))()
    for i, L in enumerate(layers):
        for k, v in L.items():
            setattr(arr[i], k, v)
    w = mte_vision_weights()
    for k in VISION_OUTER_FIELDS:
        setattr(w, k, outer[k])
    w.layers = arr if layers else None
    h = _P()
    _check(lib.mte_vision_create(C.byref(cfg), C.byref(w), stream, C.byref(h)), "mte_vision_create")
    return h.value


def mte_vision_encode(enc: int, pixels: int, n_images: int, height: int, width: int, out: int,
                      stream: int) -> int:
    return _check(lib.mte_vision_encode(enc, pixels, n_images, height, width, out, stream), "mte_vision_encode")


def mte_vision_destroy(enc: int) -> None:
    lib.mte_vision_destroy(enc)


def mte_vision_encode_strided(enc: int, pixels: int, n_images: int, height: int, width: int, out: int,
                              image_stride: int, stream: int) -> int:
    return _check(lib.mte_vision_encode_strided(enc, pixels, n_images, height, width, out, image_stride, stream),
                  "mte_vision_encode_strided")


# The descriptors of mte_cond.h as bytes (what a call passes): the same layout as the structures above.
ATTN_SHAPE = struct.Struct("@iiiif4x8q")
KV8 = struct.Struct("@PPPiii4x")
assert ATTN_SHAPE.size == C.sizeof(mte_attn_shape) and KV8.size == C.sizeof(mte_kv8)


def make_attn_shape(n_q_heads, n_kv_heads, head_dim, dtype, scale, q=(0, 0), k=(0, 0), v=(0, 0),
                    out=(0, 0)) -> mte_attn_shape:
    """q, k, v, out: (row, head) strides in elements."""
    return mte_attn_shape(n_q_heads, n_kv_heads, head_dim, dtype, scale, *q, *k, *v, *out)


# shape, cache: bytes (ATTN_SHAPE / KV8) or the structures by reference; q_lens, kv_lens (host), kv_index,
# new_lens, counts: int32 arrays as _i32 makes them, or their address.

def mte_cross_attention_workspace(shape, q_lens, n_q: int, kv_lens, n_kv: int, kv_index) -> int:
    return _check(lib.mte_cross_attention_workspace(shape, q_lens, n_q, kv_lens, n_kv, kv_index),
                  "mte_cross_attention_workspace")


def mte_cross_attention(shape, q: int, k: int, v: int, key_mask: Optional[int], q_lens, n_q: int, kv_lens, n_kv: int,
                        kv_index, out: int, workspace: Optional[int], workspace_bytes: int, stream: int) -> int:
    return _check(lib.mte_cross_attention(shape, q, k, v, key_mask, q_lens, n_q, kv_lens, n_kv, kv_index, out,
                                          workspace, workspace_bytes, stream), "mte_cross_attention")


def mte_kv8_append(cache, table: int, table_width: int, table_row: int, kv_lens: int, k: int, k_row: int, k_head: int,
                   v: int, v_row: int, v_head: int, dtype: int, new_lens, n: int, stream: int) -> int:
    return _check(lib.mte_kv8_append(cache, table, table_width, table_row, kv_lens, k, k_row, k_head, v, v_row, v_head,
                                     dtype, new_lens, n, stream), "mte_kv8_append")


def mte_kv8_read(cache, table: int, table_width: int, table_row: int, kv_lens: int, counts, n: int, k: int, v: int,
                 dtype: int, stream: int) -> int:
    return _check(lib.mte_kv8_read(cache, table, table_width, table_row, kv_lens, counts, n, k, v, dtype, stream),
                  "mte_kv8_read")


def mte_kv8_attention_workspace(shape, q_lens, n: int, table_width: int) -> int:
    return _check(lib.mte_kv8_attention_workspace(shape, q_lens, n, table_width), "mte_kv8_attention_workspace")


def mte_kv8_attention(shape, cache, table: int, table_width: int, table_row: int, kv_lens: int, q: int, q_lens, n: int,
                      causal: int, out: int, workspace: Optional[int], workspace_bytes: int, stream: int) -> int:
    return _check(lib.mte_kv8_attention(shape, cache, table, table_width, table_row, kv_lens, q, q_lens, n, causal, out,
                                        workspace, workspace_bytes, stream), "mte_kv8_attention")


def mte_group_norm_workspace(n: int, pixels: int, channels: int, groups: int, dtype: int) -> int:
    return _check(lib.mte_group_norm_workspace(n, pixels, channels, groups, dtype), "mte_group_norm_workspace")


def mte_group_norm(x: int, x_row: int, x_image: int, n: int, pixels: int, channels: int, groups: int,
                   gamma: Optional[int], beta: Optional[int], eps: float, act: int, dtype: int, y: int, y_row: int,
                   y_image: int, workspace: Optional[int], workspace_bytes: int, stream: int) -> int:
    return _check(lib.mte_group_norm(x, x_row, x_image, n, pixels, channels, groups, gamma, beta, eps, act, dtype, y,
                                     y_row, y_image, workspace, workspace_bytes, stream), "mte_group_norm")


# mte_proj.h; ROTARY_SHAPE: mte_rotary_shape as bytes.
ROTARY_SHAPE = struct.Struct("@8i4if4x8q")
assert ROTARY_SHAPE.size == C.sizeof(mte_rotary_shape)


def mte_i8_pitch(cols: int) -> int:
    return _check(lib.mte_i8_pitch(cols), "mte_i8_pitch")


def mte_i8_quantize_rows(x: int, x_row: int, rows: int, cols: int, dtype: int, codes: int, scales: int,
                         stream: int) -> int:
    return _check(lib.mte_i8_quantize_rows(x, x_row, rows, cols, dtype, codes, scales, stream), "mte_i8_quantize_rows")


def mte_i8_linear_workspace(x_type: int, m: int, k: int, n: int) -> int:
    return _check(lib.mte_i8_linear_workspace(x_type, m, k, n), "mte_i8_linear_workspace")


def mte_i8_linear(x: int, x_row: int, x_scales: Optional[int], x_type: int, m: int, k: int, w: int, w_scales: int, n: int,
                  bias: Optional[int], act: int, out: int, out_row: int, dtype: int, workspace: Optional[int],
                  workspace_bytes: int, stream: int) -> int:
    return _check(lib.mte_i8_linear(x, x_row, x_scales, x_type, m, k, w, w_scales, n, bias, act, out, out_row, dtype,
                                    workspace, workspace_bytes, stream), "mte_i8_linear")


def mte_rotary(shape, q: int, k: Optional[int], positions: int, axis_stride: int, freq: int, tokens: int, q_out: int,
               k_out: Optional[int], stream: int) -> int:
    return _check(lib.mte_rotary(shape, q, k, positions, axis_stride, freq, tokens, q_out, k_out, stream), "mte_rotary")


def mte_prefix_attention_workspace(shape, prefix_len: int, q_lens, kv_lens, n: int) -> int:
    return _check(lib.mte_prefix_attention_workspace(shape, prefix_len, q_lens, kv_lens, n),
                  "mte_prefix_attention_workspace")


def mte_prefix_attention(shape, q: int, prefix_k: Optional[int], prefix_v: Optional[int], pk_row: int, pk_head: int,
                         pv_row: int, pv_head: int, prefix_len: int, k: Optional[int], v: Optional[int], q_lens, kv_lens,
                         n: int, causal: int, out: int, workspace: Optional[int], workspace_bytes: int,
                         stream: int) -> int:
    return _check(lib.mte_prefix_attention(shape, q, prefix_k, prefix_v, pk_row, pk_head, pv_row, pv_head, prefix_len, k, v,
                                           q_lens, kv_lens, n, causal, out, workspace, workspace_bytes, stream),
                  "mte_prefix_attention")
