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
