"""Host-side checks of include/mte_proj.h: every entry point is exported and turns bad arguments
down before any HIP call (runs without a GPU; the addresses are never touched)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, CAPACITY, UNSUPPORTED = -1, -2, -5
P = 4096                    # an aligned address that no call may reach
TOP = 2**31 - 4097
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2606_05981_amd import binding
    return binding


def test_header_and_library_agree(B):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mte_proj.h")).read(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|int64_t)\s+(mte_[a-z0-9_]+)\s*\(", src, flags=re.M))
    assert names == set(n for n in B._sig if n.startswith(("mte_i8_", "mte_rotary", "mte_prefix_")))
    assert names == {"mte_i8_pitch", "mte_i8_quantize_rows", "mte_i8_linear", "mte_i8_linear_workspace", "mte_rotary",
                     "mte_prefix_attention", "mte_prefix_attention_workspace"}
    lib = ctypes.CDLL(B.LIB_PATH)
    assert not [n for n in names if not hasattr(lib, n)]
    assert ctypes.sizeof(B.mte_rotary_shape) == 120


def test_i8_pitch(B):
    assert [B.lib.mte_i8_pitch(c) for c in (1, 127, 128, 129, 2048, 131071)] == [128, 128, 128, 256, 2048, 131072]
    assert [B.lib.mte_i8_pitch(c) for c in (0, -5, 131072)] == [INVALID] * 3


def test_i8_quantize(B):
    def q(x=P, row=320, rows=4, cols=320, dt=1, codes=P, scales=P):
        return B.lib.mte_i8_quantize_rows(x, row, rows, cols, dt, codes, scales, None)
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(row=-1), dict(row=1 << 41), dict(rows=-1),
               dict(rows=TOP + 1), dict(cols=0), dict(cols=131072), dict(dt=2), dict(dt=-1), dict(x=P + 1),
               dict(dt=0, x=P + 2), dict(codes=P + 8), dict(scales=P + 2)):
        assert q(**kw) == INVALID, kw
    assert q(rows=0, x=None, codes=None, scales=None) == 0


def _lin(B, x=P, row=320, xs=None, xt=1, m=4, k=320, w=P, ws=P, n=640, bias=None, act=0, out=P, orow=640, dt=1, work=P,
         nbytes=1 << 50):
    return B.lib.mte_i8_linear(x, row, xs, xt, m, k, w, ws, n, bias, act, out, orow, dt, work, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(ws=None), INVALID), (dict(out=None), INVALID),
    (dict(xt=3), INVALID), (dict(xt=-1), INVALID), (dict(dt=2), INVALID), (dict(dt=-1), INVALID),
    (dict(act=2), INVALID), (dict(act=-1), INVALID), (dict(m=-1), INVALID), (dict(m=TOP + 1), INVALID),
    (dict(n=0), INVALID), (dict(n=TOP + 1, orow=1 << 31), INVALID), (dict(k=0), INVALID), (dict(k=131072), INVALID),
    (dict(row=-1), INVALID), (dict(row=1 << 41), INVALID), (dict(orow=639), INVALID), (dict(orow=1 << 41), INVALID),
    (dict(x=P + 1), INVALID), (dict(xt=0, x=P + 2), INVALID), (dict(w=P + 8), INVALID), (dict(ws=P + 2), INVALID),
    (dict(out=P + 1), INVALID), (dict(dt=0, out=P + 2), INVALID), (dict(bias=P + 1), INVALID),
    (dict(dt=0, bias=P + 2), INVALID), (dict(xt=2), INVALID), (dict(xt=2, xs=P + 1), INVALID),
    (dict(xt=2, xs=P, x=P + 8), INVALID), (dict(m=300, nbytes=300), CAPACITY), (dict(m=300, work=None), INVALID),
    (dict(m=300, work=P + 8), INVALID), (dict(m=0, x=None, w=None, ws=None, out=None, work=None, nbytes=0), 0),
    (dict(m=0, n=-1), INVALID), (dict(m=0, act=7), INVALID),
])
def test_i8_linear(B, kw, status):
    assert _lin(B, **kw) == status


def test_i8_linear_workspace(B):
    w = B.lib.mte_i8_linear_workspace
    assert w(1, 300, 320, 640) >= 300 * (384 + 4) and w(0, 300, 321, 640) >= 300 * (384 + 4)
    assert w(2, 300, 320, 640) >= 0 and w(1, 0, 320, 640) == 0
    assert w(1, TOP, 131071, 1) > 1 << 47                            # sizes past 32 bits
    for a in ((3, 4, 320, 640), (1, -1, 320, 640), (1, 4, 0, 640), (1, 4, 131072, 640), (1, 4, 320, 0), (1, TOP + 1, 1, 1)):
        assert w(*a) == INVALID


def _rot(B, q=P, k=P, pos=P, axis=64, freq=P, tokens=64, qo=P, ko=P, shape=None, **kw):
    s = dict(n_q_heads=16, n_k_heads=8, head_dim=128, rot_dim=128, dtype=1, interleaved=0, inverse=0, n_axes=1,
             factor=1.0, q_row=2048, q_head=128, k_row=1024, k_head=128, qo_row=2048, qo_head=128, ko_row=1024, ko_head=128)
    section = kw.pop("section", (0, 0, 0, 0))
    s.update(kw)
    c = B.mte_rotary_shape(**s)
    c.section[:] = list(section)
    return B.lib.mte_rotary(None if shape is False else ctypes.byref(c), q, k, pos, axis, freq, tokens, qo, ko, None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(pos=None), INVALID),
    (dict(freq=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID),
    (dict(n_q_heads=0), INVALID), (dict(n_q_heads=65536), INVALID), (dict(n_k_heads=-1), INVALID),
    (dict(n_k_heads=65536), INVALID), (dict(head_dim=0), INVALID),
    (dict(rot_dim=0), INVALID), (dict(rot_dim=127), INVALID), (dict(rot_dim=130), INVALID), (dict(rot_dim=-2), INVALID),
    (dict(dtype=2), INVALID), (dict(interleaved=2), INVALID), (dict(interleaved=-1), INVALID), (dict(inverse=2), INVALID),
    (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID), (dict(factor=NAN), INVALID), (dict(factor=INF), INVALID),
    (dict(n_axes=3, section=(24, 20, 19, 0)), INVALID), (dict(n_axes=2, section=(65, -1, 0, 0)), INVALID),
    (dict(n_axes=2, section=(2**31 - 1, 2**31 - 1, 0, 0)), INVALID), (dict(n_axes=2, section=(32, 32, 0, 0), axis=-1), INVALID),
    (dict(tokens=-1), INVALID), (dict(tokens=TOP // 24 + 1), INVALID),
    (dict(qo_row=4096), INVALID), (dict(qo_head=256), INVALID), (dict(ko_row=2048), INVALID),   # in place, other rows
    (dict(q_row=2044), INVALID), (dict(q_head=-8), INVALID), (dict(k_row=4), INVALID), (dict(ko_head=1 << 41), INVALID),
    (dict(q=P + 8), INVALID), (dict(k=P + 2), INVALID), (dict(qo=P + 4), INVALID), (dict(ko=P + 8), INVALID),
    (dict(pos=P + 2), INVALID), (dict(freq=P + 4), INVALID),
    (dict(head_dim=132, rot_dim=128), UNSUPPORTED), (dict(head_dim=520), UNSUPPORTED), (dict(head_dim=20, rot_dim=20), UNSUPPORTED),
    (dict(tokens=0, q=None, k=None, pos=None, freq=None, qo=None, ko=None), 0), (dict(tokens=0, rot_dim=3), INVALID),
    (dict(tokens=0, n_k_heads=0, k_row=3), 0),
])
def test_rotary(B, kw, status):
    assert _rot(B, **kw) == status


def _pre(B, shape=None, q=P, pk=P, pv=P, ps=(1024, 128, 1024, 128), p_len=96, k=P, v=P, ql=(4, 5), kl=(7, 9), n=None,
         causal=1, out=P, ws=P, nbytes=1 << 40, hq=16, hkv=8, d=128, dtype=1, scale=0.1, **kw):
    s = B.make_attn_shape(hq, hkv, d, dtype, scale, q=(hq * d, d), k=(hkv * d, d), v=(hkv * d, d), out=(hq * d, d))
    for name, value in kw.items():
        setattr(s, name, value)
    return B.lib.mte_prefix_attention(
        None if shape is False else ctypes.byref(s), q, pk, pv, *ps, p_len, k, v, None if ql is None else B._i32(ql),
        None if kl is None else B._i32(kl), len(ql or ()) if n is None else n, causal, out, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(shape=False), INVALID), (dict(q=None), INVALID), (dict(pk=None), INVALID), (dict(pv=None), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(ql=None), INVALID),
    (dict(kl=None), INVALID), (dict(n=0), INVALID), (dict(n=-1), INVALID), (dict(ql=(4, -1)), INVALID),
    (dict(kl=(-7, 9)), INVALID), (dict(p_len=-1), INVALID), (dict(causal=2), INVALID), (dict(causal=-1), INVALID),
    (dict(hq=10, hkv=4), INVALID), (dict(hq=0), INVALID), (dict(hkv=-1), INVALID), (dict(d=0), INVALID),
    (dict(dtype=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=2.4e38), INVALID),
    (dict(q_row=2044), INVALID), (dict(k_head=-128), INVALID), (dict(v_row=1 << 41), INVALID), (dict(o_head=4), INVALID),
    (dict(ps=(1020, 128, 1024, 128)), INVALID), (dict(ps=(1024, -8, 1024, 128)), INVALID),
    (dict(ps=(1024, 128, 1 << 41, 128)), INVALID), (dict(ps=(1024, 128, 1024, 4)), INVALID),
    (dict(q=P + 8), INVALID), (dict(pk=P + 2), INVALID), (dict(pv=P + 8), INVALID), (dict(k=P + 2), INVALID),
    (dict(v=P + 4), INVALID), (dict(out=P + 1), INVALID), (dict(ql=(2**31 - 1, 0)), INVALID),
    (dict(kl=(2**31 - 1, 1)), INVALID), (dict(kl=(TOP - 90, 0)), INVALID),            # with the prefix past 31 bits
    (dict(d=136), UNSUPPORTED), (dict(d=20), UNSUPPORTED),
    (dict(ql=(1, 1), kl=(1, 1), p_len=16384, nbytes=16), CAPACITY),
    (dict(ql=(1, 1), kl=(1, 1), p_len=16384, ws=None), INVALID), (dict(ql=(1, 1), kl=(1, 1), p_len=16384, ws=P + 4), INVALID),
    (dict(ql=(0, 0), q=None, out=None, ws=None, nbytes=0), 0), (dict(ql=(0, 0), causal=3), INVALID),
])
def test_prefix_attention(B, kw, status):
    assert _pre(B, **kw) == status


def test_prefix_workspace(B):
    s = B.make_attn_shape(16, 8, 128, 1, 0.1, q=(2048, 128), k=(1024, 128), v=(1024, 128), out=(2048, 128))
    w = lambda p, ql, kl, sh=s: B.lib.mte_prefix_attention_workspace(ctypes.byref(sh), p, B._i32(ql), B._i32(kl), len(ql))
    assert w(96, (4096,) * 16, (96,) * 16) == 0 and w(96, (0, 0), (4, 5)) == 0
    assert w(16384, (1,) * 64, (96,) * 64) > 0 and w(0, (1,), (9000,)) > 0
    assert w(-1, (1,), (1,)) == INVALID and w(96, (-1,), (1,)) == INVALID and w(96, (1,), (-1,)) == INVALID
    s.head_dim = 136
    assert w(96, (1,), (1,)) == UNSUPPORTED


def test_binding_raises(B):
    with pytest.raises(B.MteError) as e:
        B.mte_i8_linear(P, 320, None, 1, 4, 320, P, P, 640, None, 9, P, 640, 1, P, 1 << 40, 0)
    assert e.value.status == INVALID
    with pytest.raises(B.MteError):
        B.mte_i8_pitch(0)
    with pytest.raises(B.MteError):
        B.mte_i8_linear_workspace(1, 4, 0, 640)
    with pytest.raises(B.MteError):
        B.mte_i8_quantize_rows(None, 320, 4, 320, 1, P, P, 0)


def test_wrappers_take_gpu_tensors_only(B):
    import torch
    from paper_2606_05981_amd import conditioning as C
    from paper_2606_05981_amd import projections as J
    x = torch.zeros(4, 64)
    w = J.I8Rows(torch.zeros((8, 128), dtype=torch.int8), torch.ones(8), 64)
    for call in (lambda: J.quantize_rows(x), lambda: J.i8_linear(x, w), lambda: J.i8_linear(w, w),
                 lambda: J.rotary(torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.ones(32, dtype=torch.float64)),
                 lambda: J.i8_linear(x, w, act="gelu"),
                 lambda: C.prefix_attention(*[torch.zeros(4, 2, 64)] * 5, [4], [4])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=8, theta=0.0), dict(rot_dim=8, theta=INF),
                                dict(rot_dim=8, factor=0.0), dict(rot_dim=8, factor=NAN), dict(rot_dim=8, scaling="dynamic"),
                                dict(rot_dim=2, scaling="ntk", factor=2.0), dict(rot_dim=8, scaling="yarn", factor=2.0),
                                dict(rot_dim=8, scaling="yarn", factor=2.0, original_length=4096, fast=1.0, slow=1.0)])
def test_rotary_frequencies_refuses(B, kw):
    from paper_2606_05981_amd import projections as J
    with pytest.raises(ValueError):
        J.rotary_frequencies(device="cpu", **kw)


def test_rows_that_meet():
    """Rows at strides against rows at strides, byte by byte: what shares one is found; what does not is told apart where
    one of the two is a single run, or both have one stride."""
    import itertools
    from paper_2606_05981_amd import projections as J
    cells = lambda x: {x[0] + r * x[2] + b for r in range(x[1]) for b in range(x[3])}
    pieces = [(0, rows, step, width) for rows, step, width in ((1, 0, 5), (3, 4, 4), (3, 2, 5), (4, 0, 3), (3, 7, 3), (4, 12, 5), (2, 6, 1))]
    told = 0
    for a, b in itertools.product(pieces, pieces):
        for at in range(60):
            x, y = (20, *a[1:]), (at, *b[1:])
            share = bool(cells(x) & cells(y))
            runs = [p[1] == 1 or p[2] <= p[3] for p in (x, y)]
            if share or any(runs) or x[2] == y[2]:
                assert J._meet(x, y) == share, (x, y)
                assert J._meet(y, x) == share, (x, y)
                told += not share
    assert told > 500
