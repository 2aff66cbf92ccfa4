"""Host-side checks of include/mte_cond.h: every entry point is exported and turns bad arguments
down before any HIP call (runs without a GPU; the addresses are never touched)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, CAPACITY, UNSUPPORTED = -1, -2, -5
P = 4096                    # an aligned address that no call may reach


@pytest.fixture(scope="module")
def B():
    from paper_2606_05981_amd import binding
    return binding


def test_header_and_library_agree(B):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mte_cond.h")).read(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|int64_t)\s+(mte_[a-z0-9_]+)\s*\(", src, flags=re.M))
    assert names == {"mte_cross_attention", "mte_cross_attention_workspace", "mte_kv8_append", "mte_kv8_read",
                     "mte_kv8_attention", "mte_kv8_attention_workspace", "mte_group_norm",
                     "mte_group_norm_workspace"}
    lib = ctypes.CDLL(B.LIB_PATH)
    assert not [n for n in names if not hasattr(lib, n)]
    assert ctypes.sizeof(B.mte_attn_shape) == 88 and ctypes.sizeof(B.mte_kv8) == 40


def _shape(B, hq=16, hkv=8, d=128, dtype=1, scale=0.1, **kw):
    s = B.make_attn_shape(hq, hkv, d, dtype, scale, q=(hq * d, d), k=(hkv * d, d), v=(hkv * d, d), out=(hq * d, d))
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _cross(B, shape=None, q=P, k=P, v=P, mask=None, ql=(4, 5), kl=(96, 33), index=None, out=P, ws=P, nbytes=1 << 40,
           n_q=None, n_kv=None, **kw):
    shape = _shape(B, **kw) if shape is None else shape
    return B.lib.mte_cross_attention(
        ctypes.byref(shape) if shape else None, q, k, v, mask, None if ql is None else B._i32(ql),
        len(ql or ()) if n_q is None else n_q, None if kl is None else B._i32(kl), len(kl or ()) if n_kv is None else n_kv,
        None if index is None else B._i32(index), out, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(out=None), INVALID), (dict(ql=None), INVALID), (dict(kl=None), INVALID),
    (dict(n_q=0), INVALID), (dict(n_kv=0), INVALID), (dict(n_q=-3), INVALID),
    (dict(ql=(4, -1)), INVALID), (dict(kl=(-96, 33)), INVALID),
    (dict(ql=(4,)), INVALID),                                   # 1 query sequence, 2 key sequences, no index
    (dict(index=(0, 2)), INVALID), (dict(index=(-1, 0)), INVALID),
    (dict(hq=10, hkv=4), INVALID), (dict(hq=0), INVALID), (dict(hkv=-1), INVALID), (dict(d=0), INVALID),
    (dict(hq=65536, hkv=65536), INVALID),
    (dict(dtype=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(q_row=2044), INVALID), (dict(k_head=-128), INVALID), (dict(v_row=1 << 41), INVALID), (dict(o_head=4), INVALID),
    (dict(q=P + 8), INVALID), (dict(k=P + 2), INVALID), (dict(v=P + 4), INVALID), (dict(out=P + 1), INVALID),
    (dict(ql=(2**31 - 1, 0)), INVALID),                         # tokens x heads beyond 31 bits
    (dict(ql=(2**30, 2**30)), INVALID), (dict(kl=(2**31 - 1, 1)), INVALID),
    (dict(d=136), UNSUPPORTED), (dict(d=20), UNSUPPORTED), (dict(d=256), UNSUPPORTED),
    (dict(ql=(1, 1), kl=(8192, 8192), nbytes=16), CAPACITY),    # a long key range is split: needs a workspace
    (dict(ql=(1, 1), kl=(8192, 8192), ws=None), INVALID),
    (dict(ql=(1, 1), kl=(8192, 8192), ws=P + 4), INVALID),
])
def test_cross_attention(B, kw, status):
    assert _cross(B, **kw) == status


def test_cross_attention_without_queries(B):
    assert _cross(B, ql=(0, 0), q=None, out=None, ws=None, nbytes=0) == 0
    assert _cross(B, ql=(0, 0), q=None, out=None, index=(1, 2)) == INVALID       # still checked


def test_cross_workspace(B):
    w = lambda ql, kl, idx=None, **kw: B.lib.mte_cross_attention_workspace(
        ctypes.byref(_shape(B, **kw)), B._i32(ql), len(ql), B._i32(kl), len(kl), None if idx is None else B._i32(idx))
    assert w((4096,) * 16, (96,) * 16) == 0
    assert w((1,), (8192,)) > 0
    assert w((0,), (8192,)) == 0
    assert w((1,), (8192,), (1,)) == INVALID
    assert w((1,), (96,), d=136) == UNSUPPORTED


def _kv8(B, nb=64, h=8, d=128, k=P, v=P, s=P):
    return B.mte_kv8(k, v, s, nb, h, d)


CACHE = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(s=None), INVALID), (dict(nb=0), INVALID),
         (dict(h=0), INVALID), (dict(h=70000), INVALID), (dict(d=0), INVALID), (dict(k=P + 8), INVALID),
         (dict(v=P + 1), INVALID), (dict(s=P + 4), INVALID), (dict(d=80), UNSUPPORTED), (dict(d=32), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache(B, kw, status):
    c = _kv8(B, **kw)
    one = B._i32([1])
    d = kw.get("d", 128)
    assert B.lib.mte_kv8_append(ctypes.byref(c), P, 4, 4, P, P, 1024, 128, P, 1024, 128, 1, one, 1, None) == status
    assert B.lib.mte_kv8_read(ctypes.byref(c), P, 4, 4, P, one, 1, P, P, 1, None) == status
    if d > 0 and kw.get("h", 8) == 8:
        s = _shape(B, d=d)
        assert B.lib.mte_kv8_attention(ctypes.byref(s), ctypes.byref(c), P, 4, 4, P, P, one, 1, 0, P, P, 1 << 40,
                                       None) == status


@pytest.mark.parametrize("table,width,row,lens", [(None, 4, 4, P), (P, 0, 4, P), (P, -1, 4, P), (P, 1 << 26, 4, P),
                                                  (P, 4, -1, P), (P, 4, 4, None)])
def test_table(B, table, width, row, lens):
    c, one, s = ctypes.byref(_kv8(B)), B._i32([1]), _shape(B)
    assert B.lib.mte_kv8_append(c, table, width, row, lens, P, 1024, 128, P, 1024, 128, 1, one, 1, None) == INVALID
    assert B.lib.mte_kv8_read(c, table, width, row, lens, one, 1, P, P, 1, None) == INVALID
    assert B.lib.mte_kv8_attention(ctypes.byref(s), c, table, width, row, lens, P, one, 1, 0, P, P, 1 << 40,
                                   None) == INVALID


def test_append_and_read(B):
    c = ctypes.byref(_kv8(B))
    app = lambda k=P, kr=1024, kh=128, v=P, vr=1024, vh=128, dt=1, new=(1,), n=None: B.lib.mte_kv8_append(
        c, P, 4, 4, P, k, kr, kh, v, vr, vh, dt, None if new is None else B._i32(new), len(new or ()) if n is None else n,
        None)
    for kw in (dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(kr=1023), dict(kh=-8), dict(vr=4),
               dict(vh=1 << 41), dict(dt=2), dict(new=None), dict(n=0), dict(new=(1, -1)), dict(new=(2**31 - 1, 1))):
        assert app(**kw) == INVALID, kw
    assert app(new=(0, 0), k=None, v=None) == 0
    rd = lambda cnt=(1,), n=None, k=P, v=P, dt=1: B.lib.mte_kv8_read(
        c, P, 4, 4, P, None if cnt is None else B._i32(cnt), len(cnt or ()) if n is None else n, k, v, dt, None)
    for kw in (dict(cnt=None), dict(n=0), dict(cnt=(-1,)), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 4),
               dict(dt=-1)):
        assert rd(**kw) == INVALID, kw
    assert rd(cnt=(0,), k=None, v=None) == 0


def test_kv8_attention(B):
    def att(c=None, s=None, ql=(1,), n=None, q=P, out=P, causal=0, width=4, ws=P, nbytes=1 << 40, **kw):
        s = _shape(B, **kw) if s is None else s
        return B.lib.mte_kv8_attention(ctypes.byref(s), ctypes.byref(c or _kv8(B)), P, width, width, P, q,
                                       None if ql is None else B._i32(ql), len(ql or ()) if n is None else n, causal, out,
                                       ws, nbytes, None)
    for kw in (dict(ql=None), dict(n=0), dict(ql=(-1,)), dict(q=None), dict(out=None), dict(q=P + 4), dict(out=P + 8),
               dict(causal=2), dict(causal=-1), dict(hkv=16), dict(d=64), dict(dtype=9), dict(scale=0.0),
               dict(q_row=4), dict(o_row=-8), dict(ql=(2**31 - 1,))):
        assert att(**kw) == INVALID, kw
    assert att(width=4096, nbytes=0) == CAPACITY
    assert att(width=4096, ws=None) == INVALID
    assert att(ql=(0,), q=None, out=None, ws=None, nbytes=0) == 0
    w = lambda ql, width, **kw: B.lib.mte_kv8_attention_workspace(ctypes.byref(_shape(B, **kw)), B._i32(ql), len(ql),
                                                                  width)
    assert w((1,), 4096) > 0 and w((1,), 4) == 0 and w((0,), 4096) == 0
    assert w((1,), 0) == INVALID and w((1,), 1 << 26) == INVALID and w((1,), 4, d=80) == UNSUPPORTED


def test_group_norm(B):
    def gn(x=P, xr=320, xi=320 * 64, n=2, px=64, c=320, g=32, gamma=P, beta=P, eps=1e-5, act=1, dt=1, y=P, yr=320,
           yi=320 * 64, ws=P, nbytes=1 << 40):
        return B.lib.mte_group_norm(x, xr, xi, n, px, c, g, gamma, beta, eps, act, dt, y, yr, yi, ws, nbytes, None)
    for kw in (dict(x=None), dict(y=None), dict(n=-1), dict(n=65536), dict(px=-1), dict(c=0), dict(g=0), dict(g=33),
               dict(c=70000, g=70000), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(act=2),
               dict(act=-1), dict(dt=3), dict(xr=-1), dict(xi=-1), dict(yr=-8), dict(yi=1 << 41), dict(x=P + 1),
               dict(y=P + 1), dict(gamma=P + 1), dict(beta=P + 1), dict(dt=0, x=P + 2)):
        assert gn(**kw) == INVALID, kw
    assert gn(n=0) == 0 and gn(px=0, x=None, y=None) == 0
    assert gn(px=1 << 16, nbytes=0) == CAPACITY
    assert gn(px=1 << 16, ws=None) == INVALID
    assert gn(px=1 << 16, ws=P + 8) == INVALID
    w = B.lib.mte_group_norm_workspace
    assert w(1, 1 << 16, 320, 32, 1) > 0 and w(0, 64, 320, 32, 1) == 0
    assert w(1, 64, 320, 33, 1) == INVALID


def test_wrappers_take_gpu_tensors_only(B):
    import torch
    from paper_2606_05981_amd import conditioning as C
    q = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        C.cross_attention(q, q, q, [4], [4])
    with pytest.raises(ValueError):
        C.group_norm(torch.zeros(1, 4, 32), 8)
    with pytest.raises(ValueError):
        C.kv8_cache(4, 2, 80, device="cpu")
    cache = C.kv8_cache(4, 2, 64, device="cpu")
    with pytest.raises(ValueError):
        C.kv8_attention(q, cache, torch.zeros((1, 4), dtype=torch.int32), torch.ones(1, dtype=torch.int32), [4])
    with pytest.raises(ValueError):
        C.kv8_append(cache, torch.zeros((1, 4), dtype=torch.int32), torch.ones(1, dtype=torch.int32), q, q, [4])


def test_binding_raises(B):
    with pytest.raises(B.MteError) as e:
        B.mte_group_norm(P, 320, 0, 1, 64, 320, 33, None, None, 1e-5, 0, 1, P, 320, 0, None, 0, None)
    assert e.value.status == INVALID
    with pytest.raises(B.MteError):
        B.mte_kv8_attention_workspace(ctypes.byref(_shape(B, d=80)), B._i32([1]), 1, 4)
