"""Limits of include/mte_cond.h's arguments at which a call is still taken, and past which it is turned down (runs
without a GPU; the addresses are never touched)."""
import ctypes

import pytest

INVALID = -1
P = 4096                    # an aligned address that no call may reach


@pytest.fixture(scope="module")
def B():
    from paper_2606_05981_amd import binding
    return binding


@pytest.mark.parametrize("scale,status", [(2.35e38, 0), (2.37e38, INVALID), (3.4e38, INVALID), (1e-45, 0)])
def test_attention_scale(B, scale, status):
    """Scores are taken in units of log 2: scale * log2(e) has to be within fp32, too."""
    s = B.make_attn_shape(4, 2, 64, B.MTE_BF16, scale, q=(256, 64), k=(128, 64), v=(128, 64), out=(256, 64))
    none, one, kv = B._i32([0]), B._i32([1]), B._i32([96])
    ref = ctypes.byref(s)
    assert B.lib.mte_cross_attention(ref, P, P, P, None, none, 1, kv, 1, None, P, P, 1 << 40, None) == status
    assert B.lib.mte_cross_attention_workspace(ref, one, 1, kv, 1, None) == status
    c = B.mte_kv8(P, P, P, 64, 2, 64)
    assert B.lib.mte_kv8_attention(ref, ctypes.byref(c), P, 4, 4, P, P, none, 1, 0, P, P, 1 << 40, None) == status
    assert B.lib.mte_kv8_attention_workspace(ref, one, 1, 4) == status


def test_attention_sizes(B):
    """Rows of queries (token and head) and key tokens are counted in 31 bits, with room for the last tile's end."""
    top = 2**31 - 4097
    shape = lambda hq, hkv, d=64: ctypes.byref(B.make_attn_shape(hq, hkv, d, B.MTE_BF16, 0.1, q=(hq * d, d), k=(0, 0), v=(0, 0),
                                                                 out=(hq * d, d)))
    one = B._i32([1])
    cross = lambda s, ql, kl: B.lib.mte_cross_attention_workspace(s, B._i32(ql), len(ql), B._i32(kl), len(kl), None)
    assert cross(shape(1, 1), [1], [top]) > 0 and cross(shape(1, 1), [top], [1]) == 0
    assert cross(shape(1, 1), [1], [top + 1]) == INVALID and cross(shape(1, 1), [top + 1], [1]) == INVALID
    assert cross(shape(1, 1), [1, 1], [top, 1]) == INVALID
    assert cross(shape(4, 2), [top // 4 + 1], [1]) == INVALID
    kv8 = lambda s, ql: B.lib.mte_kv8_attention_workspace(s, B._i32(ql), len(ql), 4)
    assert kv8(shape(1, 1), [top]) >= 0
    assert kv8(shape(1, 1), [top + 1]) == INVALID and kv8(shape(2, 1), [top // 2 + 1]) == INVALID
    c = ctypes.byref(B.mte_kv8(P, P, P, 64, 2, 64))
    assert B.lib.mte_kv8_read(c, P, 4, 4, P, B._i32([top + 1]), 1, P, P, 1, None) == INVALID
    assert B.lib.mte_kv8_append(c, P, 4, 4, P, P, 0, 0, P, 0, 0, 1, B._i32([top + 1]), 1, None) == INVALID
