"""include/mte_cond.h through the binding, as a program without torch would call it: buffers and a workspace of its own of
just the stated size; what lies behind them stays as it was, and results equal the wrappers'."""
import ctypes
import sys

import pytest

from tests.test_gpu_cond import _fill, _randn

pytestmark = pytest.mark.gpu
GUARD, MARK = 4096, 0xA5


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "no GPU"
    return torch


@pytest.fixture(scope="module")
def C():
    from paper_2606_05981_amd import conditioning
    return conditioning


@pytest.fixture(scope="module")
def B():
    from paper_2606_05981_amd import binding
    return binding


class Guarded:
    """`nbytes` of device memory with marked bytes behind them."""

    def __init__(self, torch, nbytes):
        self.n = nbytes
        self.mem = torch.full((nbytes + GUARD,), MARK, dtype=torch.uint8, device="cuda")

    def address(self):
        return self.mem.data_ptr() if self.n else None

    def kept(self):
        return bool((self.mem[self.n:] == MARK).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,hkv,d", [([5, 0, 40], [96, 7, 70], 4, 2, 64), ([2], [2500], 8, 2, 64),
                                            ([1, 0, 30, 1], [1500, 9, 2000, 12], 16, 8, 128), ([600], [2500], 16, 16, 64),
                                            ([1100, 33], [96, 70], 16, 8, 72)])
def test_cross_attention(torch, C, B, ql, kl, hq, hkv, d, dtype):
    _say(f"binding, cross {ql} x {kl} {dtype}")
    q = _randn(torch, 120, sum(ql), hq, d, dtype=dtype)
    k, v = _randn(torch, 121, sum(kl), hkv, d, dtype=dtype), _randn(torch, 122, sum(kl), hkv, d, dtype=dtype)
    shape = ctypes.byref(B.make_attn_shape(hq, hkv, d, C._DTYPE[q.dtype], d ** -0.5, q=(hq * d, d), k=(hkv * d, d), v=(hkv * d, d),
                                           out=(hq * d, d)))
    a, b = B._i32(ql), B._i32(kl)
    need = B.mte_cross_attention_workspace(shape, a, len(ql), b, len(kl), None)
    ws, out = Guarded(torch, need), Guarded(torch, q.numel() * q.element_size())
    args = (shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), None, a, len(ql), b, len(kl), None, out.address())
    stream = torch.cuda.current_stream().cuda_stream
    if need:
        with pytest.raises(B.MteError) as e:
            B.mte_cross_attention(*args, ws.address(), need - 1, stream)
        assert e.value.status == B.MTE_E_CAPACITY
    B.mte_cross_attention(*args, ws.address(), need, stream)
    assert torch.equal(out.mem[:out.n].view(q.dtype).view(q.shape), C.cross_attention(q, k, v, ql, kl))
    assert ws.kept() and out.kept()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,hkv,d,width", [([1, 0, 2], [100, 5, 700], 16, 8, 128, None), ([1] * 130, [40] * 130, 4, 2, 64, 50),
                                                  ([300], [310], 32, 4, 64, None), ([300, 3], [310, 900], 32, 4, 64, 40),
                                                  ([20], [3000], 4, 2, 128, None)])
def test_kv8_attention(torch, C, B, ql, kl, hq, hkv, d, width, dtype):
    _say(f"binding, cached {ql[:4]} x {kl[:4]} {dtype}")
    cache, table, kv, k, v = _fill(torch, C, kl, hkv, d, width=width)
    width = table.shape[1]
    q = _randn(torch, 123, sum(ql), hq, d, dtype=dtype)
    shape = ctypes.byref(B.make_attn_shape(hq, hkv, d, C._DTYPE[q.dtype], d ** -0.5, q=(hq * d, d), out=(hq * d, d)))
    kv8 = ctypes.byref(B.mte_kv8(*(t.data_ptr() for t in cache), cache.k_codes.shape[0], hkv, d))
    a, stream = B._i32(ql), torch.cuda.current_stream().cuda_stream
    need = B.mte_kv8_attention_workspace(shape, a, len(ql), width)
    for causal in (0, 1):
        ws, out = Guarded(torch, need), Guarded(torch, q.numel() * q.element_size())
        args = (shape, kv8, table.data_ptr(), width, table.stride(0), kv.data_ptr(), q.data_ptr(), a, len(ql), causal, out.address())
        if need:
            with pytest.raises(B.MteError) as e:
                B.mte_kv8_attention(*args, ws.address(), need - 1, stream)
            assert e.value.status == B.MTE_E_CAPACITY
        B.mte_kv8_attention(*args, ws.address(), need, stream)
        assert torch.equal(out.mem[:out.n].view(q.dtype).view(q.shape),
                           C.kv8_attention(q, cache, table, kv, ql, causal=bool(causal)))
        assert ws.kept() and out.kept()
    # the rows of a read, and what lies behind them
    counts = [min(n, 33) for n in kl]
    rk, rv = (Guarded(torch, sum(counts) * hkv * d * q.element_size()) for _ in range(2))
    B.mte_kv8_read(kv8, table.data_ptr(), width, table.stride(0), kv.data_ptr(), B._i32(counts), len(kl), rk.address(), rv.address(),
                   C._DTYPE[q.dtype], stream)
    for got, want in zip((rk, rv), C.kv8_read(cache, table, kv, counts, dtype=q.dtype)):
        assert torch.equal(got.mem[:got.n].view(q.dtype).view(want.shape), want) and got.kept()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,px,c,groups", [(2, 64, 1280, 32), (1, 4096, 320, 32), (3, 1023, 33, 11), (1, 10000, 64, 1)])
def test_group_norm(torch, C, B, n, px, c, groups, dtype):
    _say(f"binding, group norm {n} x {px} x {c} {dtype}")
    x = _randn(torch, 124, n, px, c, dtype=dtype)
    code = C._DTYPE[x.dtype]
    need = B.mte_group_norm_workspace(n, px, c, groups, code)
    ws, y = Guarded(torch, need), Guarded(torch, x.numel() * x.element_size())
    B.mte_group_norm(x.data_ptr(), c, px * c, n, px, c, groups, None, None, 1e-5, B.MTE_ACT_SILU, code, y.address(), c, px * c,
                     ws.address(), need, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y.mem[:y.n].view(x.dtype).view(x.shape), C.group_norm(x, groups, act="silu"))
    assert ws.kept() and y.kept()
