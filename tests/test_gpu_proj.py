"""Linear layers in 8-bit integers and rotary positions (include/mte_proj.h) against their float64
oracle, through the Python wrappers.

Tolerances are the operators' own rounding, element by element (U16 = 2^-8 for bf16, U = 2^-24 for
fp32, half a step relative to the value each):
 - codes and scales are defined to the last bit: equal;
 - a product p is an exact sum, rounded to fp32 and multiplied by two scales (3 U |p|), the bias is added
   (U |z|): e = 3 U |p| + U |z|. SiLU has a slope of at most 1.1; its own steps are the exponent -z log2 e, rounded
   (|z| U, and as much again for the constant, relative), exp2, 1 + e, reciprocal and product (2 U each at
   most): 1.1 e + (2 |z| + 8) U |y|, and 2^-126 |z| where exp2 or the reciprocal leave fp32's range;
 - a rotation: the reduced angle in fp32 (pi U), sine and cosine (4 U: two units in the last place each), two products, their
   sum and the factor (4 U): (pi + 8) U f (|x1| + |x2|);
 - the result, U16 or U of itself.
"""
import math
import sys

import numpy as np
import pytest

from oracle import proj_oracle as O

pytestmark = pytest.mark.gpu

U, U16 = 2.0 ** -24, 2.0 ** -8


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "no GPU"
    return torch


@pytest.fixture(scope="module")
def P():
    from paper_2606_05981_amd import projections
    return projections


def _dt(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _f64(t):
    return t.detach().double().cpu().numpy()


def _randn(torch, seed, *shape, std=1.0, dtype="bf16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(_dt(torch, dtype)).cuda()


def _within(got, ref, tol, dtype):
    g = _f64(got)
    assert g.shape == ref.shape and np.isfinite(g).all()
    tol = tol + (U16 if dtype == "bf16" else U) * (np.abs(ref) + tol) + 1e-40
    worst = float((np.abs(g - ref) / tol).max()) if g.size else 0.0
    _say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0


# ---- rows in 8 bits -----------------------------------------------------------------------------


def _check_rows(rows, x):
    codes, scales = O.i8_rows(_f64(x))
    c = rows.codes.cpu().numpy()
    k = x.shape[1]
    assert c.shape[1] % 128 == 0 and c.shape[1] - k < 128
    assert np.array_equal(rows.scales.cpu().numpy(), scales, equal_nan=True)
    assert np.array_equal(c[:, :k], codes.astype(np.int8))
    assert (c[:, k:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k", [(1, 1), (300, 1), (1, 2048), (3, 7), (700, 7), (3, 8), (3, 9), (3, 15), (5, 127), (4, 128), (2, 129), (9, 511), (65, 513), (7, 1001),
                                 (33, 2047), (6, 4096), (5, 4097), (3, 6144), (2, 20011), (1, 131071), (1030, 320)])
def test_quantize(torch, P, m, k, dtype):
    _say(f"quantize {m} x {k}, {dtype}")
    x = _randn(torch, m + k, m, k, std=3.0, dtype=dtype)
    rows = P.quantize_rows(x)
    assert rows.cols == k
    _check_rows(rows, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_borders(torch, P, dtype):
    """Quotients on and next to halves: rows whose largest value is a power of two, 127 or 254 steps, and their
    neighbours in the type; rows of zeros, of tiny and of the largest values; infinities and NaN."""
    dt = _dt(torch, dtype)
    rows = []
    for top in (1.0, 127.0, 254.0, 63.5, 0.75, 3.0, 2.0 ** -119, 2.0 ** -126, 2.0 ** -130, 1e-38, 3e38, 0.0):
        steps = torch.arange(128, dtype=torch.float64) + 0.5
        x = torch.cat([steps / 127 * top, -steps / 127 * top, torch.tensor([top, -top / 2, top / 254, 0.0])]).clamp(-top, top)
        x = x.to(dt)
        rows += [x, torch.nextafter(x.float(), torch.zeros(1)).to(dt), -x]
    x = torch.stack(rows).cuda()
    _check_rows(P.quantize_rows(x), x)
    y = x[:5].clone()
    y[0, 3], y[1, 0], y[2, 259], y[3, 100] = math.inf, math.nan, -math.inf, -math.nan
    got = P.quantize_rows(y)
    _check_rows(got, y)
    assert torch.isnan(got.scales[:4]).all() and not torch.isnan(got.scales[4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_are_those_that_torch_computes_here(torch, P, dtype):
    """max |x| / 127 as torch has it on this device, bit for bit: rows of every bf16 mantissa, and of others in fp32. It is
    not the rounded quotient of 64 bits, which differs for some of them."""
    x = torch.cat([1 + torch.arange(128) / 128] + [torch.rand(4000, generator=torch.Generator().manual_seed(9)) + 2.0 ** e for e in (-20, 0, 9)])
    x = x[:, None].mul(torch.tensor([0.25, -1.0, 0.5])).to(_dt(torch, dtype)).cuda()
    rows, top = P.quantize_rows(x), x.float().abs().amax(1)
    assert torch.equal(rows.scales, top / 127)
    assert (rows.scales != (top.double() / 127).float()).any()
    _check_rows(rows, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,wide,skip", [(5, 320, 3, 0), (5, 320, 8, 0), (4, 77, 0, 1), (6, 640, 1, 5), (3, 5000, 11, 3)])
def test_quantize_strided(torch, P, m, k, wide, skip, dtype):
    """Rows of a wider buffer, at odd strides and addresses."""
    full = _randn(torch, 5, m, k + wide + skip, dtype=dtype)
    x = full[:, skip:skip + k]
    _check_rows(P.quantize_rows(x), x)
    x = full[:1, skip:skip + k].expand(m, k)         # one row for all
    _check_rows(P.quantize_rows(x), x)


@pytest.mark.parametrize("k", [8, 5, 4100])
def test_quantize_more_rows_than_a_grid(torch, P, k):
    """More rows than a launch has workgroups for: the first, some in between and the last."""
    m = {8: (1 << 24) + 9, 5: (1 << 24) + 9, 4100: (1 << 22) + 3}[k]
    x = _randn(torch, 1, 1, k).expand(m, k) if k == 4100 else \
        torch.randn((m, k), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    got = P.quantize_rows(x)
    at = torch.tensor([0, 1, 4095, m // 2, m - 6, m - 2, m - 1], device="cuda")
    _check_rows(P.I8Rows(got.codes[at], got.scales[at], k), x[at])


# ---- products -----------------------------------------------------------------------------------


def _check_linear(got, x, w, bias, silu, dtype):
    """x, w: (codes, scales) of the oracle."""
    y, z, p = O.i8_linear(*x, *w, bias, silu)
    e = 3 * U * np.abs(p) + U * np.abs(z)
    if silu:
        e = 1.1 * e + (2 * np.abs(z) + 8) * U * np.abs(y) + 2.0 ** -126 * np.abs(z)
    _within(got, y, e, dtype)


LINEAR = [
    # m, k, n
    (1, 1, 1), (5, 7, 20), (16, 8, 5), (3, 9, 70), (40, 3, 9), (8200, 5, 40), (33000, 8, 40), (33000, 7, 9), (1, 2048, 2048), (1, 30000, 37), (1, 100000, 20), (2, 9000, 70), (4, 640, 5000), (7, 3000, 4200), (16, 5000, 33), (16, 6144, 40), (16, 8192, 40), (9, 8192, 9000), (2, 130, 17), (3, 128, 16), (15, 127, 33), (16, 320, 640), (17, 320, 40), (16, 2048, 1283),
    (17, 2048, 4096), (17, 2048, 4097), (32, 2048, 40), (20, 2900, 70), (24, 3100, 40), (32, 2944, 33), (32, 8, 1), (31, 640, 64), (33, 1001, 129), (64, 2048, 512), (65, 2048, 257), (96, 2048, 1024), (127, 513, 255), (128, 512, 256),
    (129, 129, 257), (200, 6144, 300), (255, 320, 640), (256, 384, 1283), (257, 4096, 1000), (777, 1001, 1283),
    (1030, 320, 640), (1536, 640, 1100), (2049, 300, 77), (300, 20000, 70),
    # many short rows
    (8192, 320, 640), (32768, 320, 320), (32769, 100, 70), (33000, 257, 129), (32897, 384, 1), (40000, 128, 131), (32900, 130, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", LINEAR)
def test_linear(torch, P, m, k, n, dtype):
    """Rows that the call quantises, with and without bias and activation by turns."""
    bias, silu = (m + n) % 2 == 1, (m + k) % 3 == 0
    _say(f"linear {m} x {k} x {n}, {dtype}, bias {bias}, silu {silu}")
    x, w = _randn(torch, 1, m, k, std=2.0, dtype=dtype), _randn(torch, 2, n, k, std=1 / math.sqrt(k), dtype=dtype)
    b = _randn(torch, 3, n, dtype=dtype) if bias else None
    weight = P.quantize_rows(w)
    got = P.i8_linear(x, weight, b, act="silu" if silu else None)
    assert got.dtype == x.dtype
    _check_linear(got, O.i8_rows(_f64(x)), O.i8_rows(_f64(w)), None if b is None else _f64(b), silu, dtype)


@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(1, 2048, 640), (30, 1500, 90), (32, 2944, 33), (40, 640, 130), (300, 1000, 515)])
def test_linear_of_codes(torch, P, m, k, n, out_dtype):
    """Tokens quantised once for several layers, both result types; the largest sums (all codes -128 or 127)."""
    g = torch.Generator().manual_seed(7)
    pad = (k + 127) // 128 * 128
    a, b = torch.zeros((m, pad), dtype=torch.int8), torch.zeros((n, pad), dtype=torch.int8)
    a[:, :k], b[:, :k] = torch.randint(-128, 128, (m, k), generator=g), torch.randint(-128, 128, (n, k), generator=g)
    a[0, :k], b[0, :k], b[1, :k] = -128, -128, 127
    s, t = torch.rand(m, generator=g) + 0.01, torch.rand(n, generator=g) + 0.01
    x, w = P.I8Rows(a.cuda(), s.cuda(), k), P.I8Rows(b.cuda(), t.cuda(), k)
    got = P.i8_linear(x, w, dtype=_dt(torch, out_dtype))
    _check_linear(got, (a[:, :k].double().numpy(), s.numpy()), (b[:, :k].double().numpy(), t.numpy()), None, False, out_dtype)


@pytest.mark.parametrize("src,dst", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("m,k,n", [(3, 300, 70), (24, 500, 130), (30, 7, 9), (300, 1001, 130), (33000, 120, 70), (32900, 250, 130),
                                   (33000, 300, 64)])
def test_linear_of_two_types(torch, P, m, k, n, silu, src, dst):
    """Rows of one type, bias and result of the other."""
    x, w, b = _randn(torch, 1, m, k, std=2.0, dtype=src), _randn(torch, 2, n, k, std=1 / math.sqrt(k)), _randn(torch, 3, n, dtype=dst)
    got = P.i8_linear(x, P.quantize_rows(w), b, act="silu" if silu else None, dtype=_dt(torch, dst))
    assert got.dtype == _dt(torch, dst)
    _check_linear(got, O.i8_rows(_f64(x)), O.i8_rows(_f64(w)), _f64(b), silu, dst)
    bare = P.i8_linear(x, P.quantize_rows(w), act="silu" if silu else None, dtype=_dt(torch, dst))
    _check_linear(bare, O.i8_rows(_f64(x)), O.i8_rows(_f64(w)), None, silu, dst)


@pytest.mark.parametrize("dst", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(5, 640, 70), (30, 1500, 90), (40, 640, 130), (300, 1000, 515), (33000, 100, 70)])
def test_linear_of_codes_with_bias(torch, P, m, k, n, dst):
    """Ready codes, with bias and with SiLU: what the rows themselves give."""
    x, w, b = _randn(torch, 1, m, k, std=2.0), _randn(torch, 2, n, k, std=1 / math.sqrt(k)), _randn(torch, 3, n, dtype=dst)
    codes, weight = P.quantize_rows(x), P.quantize_rows(w)
    for bias in (None, b):
        for act in (None, "silu"):
            got = P.i8_linear(codes, weight, bias, act=act, dtype=_dt(torch, dst))
            _check_linear(got, O.i8_rows(_f64(x)), O.i8_rows(_f64(w)), None if bias is None else _f64(bias), act is not None, dst)
            assert torch.equal(got, P.i8_linear(x, weight, bias, act=act, dtype=_dt(torch, dst)))


@pytest.mark.parametrize("m", [1, 16, 17, 32])
@pytest.mark.parametrize("k,n", [(2048, 12288), (6144, 2048)])
def test_linear_feed_forward_steps(torch, P, m, k, n):
    """The two widths of a feed-forward layer for a step's rows, of rows and of codes."""
    x, w = _randn(torch, 1, m, k, std=2.0), _randn(torch, 2, n, k, std=1 / math.sqrt(k))
    weight = P.quantize_rows(w)
    got = P.i8_linear(x, weight)
    _check_linear(got, O.i8_rows(_f64(x)), O.i8_rows(_f64(w)), None, False, "bf16")
    assert torch.equal(P.i8_linear(P.quantize_rows(x), weight), got)


def test_linear_longest_rows(torch, P):
    """131071 products of -128 and -128 still fit the sum."""
    k = 131071
    a, b = torch.zeros((2, 131072), dtype=torch.int8), torch.zeros((3, 131072), dtype=torch.int8)
    a[:, :k], b[:, :k] = -128, -128
    b[1, :k] = 127
    s, t = torch.tensor([1.0, 0.5]), torch.tensor([1.0, 2.0, 0.25])
    got = P.i8_linear(P.I8Rows(a.cuda(), s.cuda(), k), P.I8Rows(b.cuda(), t.cuda(), k), dtype=torch.float32)
    _check_linear(got, (a[:, :k].double().numpy(), s.numpy()), (b[:, :k].double().numpy(), t.numpy()), None, False, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [5, 300, 32768])
def test_linear_strides(torch, P, m, dtype):
    """x a slice of wider rows at an odd address, out a slice whose other channels stay, leading dimensions, a
    second call's results, and rows behind the last one."""
    k, n = 333, 217
    full = _randn(torch, 1, m, k + 5, std=2.0, dtype=dtype)
    x = full[:, 3:3 + k]
    w = _randn(torch, 2, n, k, std=0.05, dtype=dtype)
    weight = P.quantize_rows(w)
    ref = (O.i8_rows(_f64(x)), O.i8_rows(_f64(w)))
    for off, wide in ((0, 7), (1, 0), (8, 23), (3, 4)):
        buf = torch.full((m + 2, off + n + wide), 7.0, dtype=x.dtype, device="cuda")
        out = buf[:m, off:off + n]
        assert P.i8_linear(x, weight, out=out) is out
        _check_linear(out, *ref, None, False, dtype)
        assert (buf[:, :off] == 7).all() and (buf[:, off + n:] == 7).all() and (buf[m:] == 7).all()
    if m == 300:
        y = P.i8_linear(x.contiguous().view(3, 4, 25, k), weight)
        assert y.shape == (3, 4, 25, n)
        assert torch.equal(y.view(m, n), P.i8_linear(x, weight))


@pytest.mark.parametrize("off,wide", [(0, 0), (8, 24), (3, 2)])
def test_linear_result_wider_than_the_longest_rows(torch, P, off, wide):
    """What bounds a row's channels (the sum) does not bound the weight's rows: a vocabulary's worth of them, into
    a result of the caller's, whole and as a slice."""
    m, k, n = 2, 64, 140000
    x, weight = _randn(torch, 1, m, k), P.quantize_rows(_randn(torch, 2, n, k))
    ref = P.i8_linear(x, weight)
    buf = torch.full((m, off + n + wide), 7.0, dtype=x.dtype, device="cuda")
    out = buf[:, off:off + n]
    assert P.i8_linear(x, weight, out=out) is out
    assert torch.equal(out, ref)
    assert (buf[:, :off] == 7).all() and (buf[:, off + n:] == 7).all()


def test_linear_more_tiles_than_a_grid(torch, P):
    """More tiles of 64 rows than a launch takes workgroups for, 2^24; rows that overlap in memory, so that what is large
    are the codes that the call makes."""
    m, k = (1 << 30) + 70, 5
    if torch.cuda.mem_get_info()[0] < m * 134 + (8 << 30):
        pytest.skip("needs the memory of a whole MI355X")
    x = _randn(torch, 1, m + k).as_strided((m, k), (1, 1))
    weight, bias = P.quantize_rows(_randn(torch, 2, 1, k)), _randn(torch, 3, 1)
    got = P.i8_linear(x, weight, bias)
    for at in (0, (1 << 28) - 150, (1 << 29) - 150, m // 2, m - 300):
        assert torch.equal(got[at:at + 300], P.i8_linear(x[at:at + 300], weight, bias)), at
    del x, got
    torch.cuda.empty_cache()


def test_linear_more_tiles_across_than_a_launch(torch, P):
    """The same of the weight's rows: 2^22 tiles of 64 columns a launch."""
    m, k, n = 17, 5, (1 << 28) + 70
    if torch.cuda.mem_get_info()[0] < n * (134 + 2 * m) + (8 << 30):
        pytest.skip("needs the memory of a whole MI355X")
    x, bias = _randn(torch, 1, m, k), _randn(torch, 3, 70).repeat(n // 70 + 1)[:n]
    w = P.quantize_rows(_randn(torch, 2, n + k).as_strided((n, k), (1, 1)))
    got = P.i8_linear(x, w, bias)
    for at in (0, (1 << 27) - 150, (1 << 28) - 150, n - 300):
        part = P.I8Rows(w.codes[at:at + 300], w.scales[at:at + 300], k)
        assert torch.equal(got[:, at:at + 300], P.i8_linear(x, part, bias[at:at + 300].contiguous())), at
    del w, bias, got, part
    torch.cuda.empty_cache()


def test_linear_batch_invariant(torch, P):
    """A row's result does not depend on the rows beside it, nor on the kernel that takes them: the sums are exact."""
    x, w = _randn(torch, 1, 33000, 320, std=2.0), _randn(torch, 2, 330, 320, std=0.05)
    weight, b = P.quantize_rows(w), _randn(torch, 3, 330)
    whole = P.i8_linear(x, weight, b, act="silu")
    for a, e in ((0, 1), (3, 17), (6, 30), (5, 69), (100, 400), (7, 32900)):
        assert torch.equal(P.i8_linear(x[a:e], weight, b, act="silu"), whole[a:e])
    assert torch.equal(P.i8_linear(P.quantize_rows(x), weight, b, act="silu"), whole)


@pytest.mark.parametrize("m", [3, 150, 33000])
def test_linear_nan_rows(torch, P, m):
    """A token with an infinity or NaN gives a row of NaN, a weight row with one a column; the others are
    what they are without."""
    x, w = _randn(torch, 1, m, 200), _randn(torch, 2, 70, 200)
    ref = P.i8_linear(x, P.quantize_rows(w))
    x2, w2 = x.clone(), w.clone()
    x2[1, 5], w2[66, 199] = math.inf, math.nan
    got = P.i8_linear(x2, P.quantize_rows(w2))
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[1], bad[:, 66] = True, True
    assert torch.isnan(got[bad]).all()
    assert torch.equal(got[~bad], ref[~bad])


def test_linear_magnitudes(torch, P):
    """Scales far apart whose product is in range: rows near fp32's largest times small weights, and the reverse."""
    k, n = 256, 48
    x = torch.cat([_randn(torch, 1, 2, k, std=3e37, dtype="f32"), _randn(torch, 2, 2, k, std=1e-24, dtype="f32")]).clamp(-3e38, 3e38)
    for std in (1e-12, 1.0, 1e20):
        w = _randn(torch, 3, n, k, std=std, dtype="f32")
        rows = x if std < 1 else x[2:]
        got = P.i8_linear(rows, P.quantize_rows(w))
        _check_linear(got, O.i8_rows(_f64(rows)), O.i8_rows(_f64(w)), None, False, "f32")


def test_linear_empty(torch, P):
    weight = P.quantize_rows(_randn(torch, 2, 20, 64))
    assert P.i8_linear(_randn(torch, 1, 0, 64), weight).shape == (0, 20)
    assert P.i8_linear(torch.zeros((2, 0, 64), dtype=torch.bfloat16, device="cuda"), weight).shape == (2, 0, 20)
    assert P.quantize_rows(_randn(torch, 1, 0, 64)).codes.shape == (0, 128)


def test_linear_approximates_the_product(torch, P):
    """Against the unquantised product: a code is off by half a step, 1/254 of its row's largest value."""
    x, w = _randn(torch, 1, 40, 640, dtype="f32"), _randn(torch, 2, 100, 640, dtype="f32")
    got, xs, ws = _f64(P.i8_linear(x, P.quantize_rows(w))), _f64(x), _f64(w)
    ex, ew = np.abs(xs).max(1, keepdims=True) / 253, np.abs(ws).max(1, keepdims=True) / 253
    bound = np.abs(xs).sum(1, keepdims=True) * ew.T + ex * np.abs(ws).sum(1)[None] + 640 * ex * ew.T
    assert (np.abs(got - xs @ ws.T) <= bound).all()


# ---- rotary positions ---------------------------------------------------------------------------


def _freq(P, pairs, theta=5e6, **kw):
    return P.rotary_frequencies(2 * pairs, theta, **kw)[0]


def _check_rotary(got, x, pos, freq, dtype, **kw):
    x, pos, freq = _f64(x), pos.cpu().numpy(), freq.cpu().numpy()
    ref = O.rotary(x, pos, freq, **kw)
    n, mag = len(freq), np.zeros_like(ref)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if kw.get("interleaved") else (slice(0, n), slice(n, 2 * n))
    both = abs(kw.get("factor", 1.0)) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    mag[..., a], mag[..., b] = both, both
    _within(got, ref, (math.pi + 8) * U * mag, dtype)
    assert np.array_equal(_f64(got)[..., 2 * n:], x[..., 2 * n:])


ROTARY = [
    # tokens, q heads, k heads, d, pairs, far, axes
    (1, 1, 0, 8, 4, 100, 1), (1, 16, 8, 128, 64, 131072, 1), (5, 4, 2, 64, 32, 1 << 30, 1), (64, 16, 8, 128, 64, 131072, 1),
    (33, 3, 1, 40, 20, 5000, 2), (17, 5, 5, 80, 21, 300, 1), (7, 2, 2, 64, 1, 1 << 20, 1), (130, 8, 1, 128, 31, 2000, 3),
    (1000, 10, 10, 64, 16, 64, 2), (9, 2, 1, 512, 256, 4096, 4), (2049, 4, 2, 64, 30, 4096, 3), (3, 300, 7, 16, 6, 99, 1),
    (4099, 1, 1, 8, 3, 1 << 16, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("t,hq,hk,d,pairs,far,axes", ROTARY)
def test_rotary(torch, P, t, hq, hk, d, pairs, far, axes, inter, dtype):
    _say(f"rotary {t} tokens, heads {hq}/{hk} of {d}, {pairs} pairs, below {far}, {axes} axes, inter {inter}, {dtype}")
    q = _randn(torch, 1, t, hq, d, std=2.0, dtype=dtype)
    k = _randn(torch, 2, t, hk, d, std=2.0, dtype=dtype) if hk else None
    g = torch.Generator().manual_seed(4)
    pos = torch.randint(-far, far, (axes, t) if axes > 1 else (t,), generator=g, dtype=torch.int32).cuda()
    sections = None if axes == 1 else [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1)
    freq = _freq(P, pairs)
    kw = dict(interleaved=inter, sections=sections, factor=1.25)
    gq, gk = P.rotary(q, pos, freq, k=k, **kw)
    _check_rotary(gq, q, pos, freq, dtype, **kw)
    if hk:
        _check_rotary(gk, k, pos, freq, dtype, **kw)
    else:
        assert gk is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_rotary_in_place_and_strided(torch, P, inter, dtype):
    """q and k in one fused projection's rows, rotated where they lie and into head-major results; v stays."""
    t, hq, hk, d, pairs = 70, 4, 2, 64, 24
    both = _randn(torch, 1, t, hq + 2 * hk, d, dtype=dtype)
    before = both.clone()
    pos, freq = torch.arange(1000, 1000 + t, dtype=torch.int32, device="cuda"), _freq(P, pairs)
    q, k = both[:, :hq], both[:, hq:hq + hk]
    hq_major, hk_major = (torch.zeros((h, t, d), dtype=both.dtype, device="cuda") for h in (hq, hk))
    P.rotary(q, pos, freq, k=k, interleaved=inter, out=(hq_major.transpose(0, 1), hk_major.transpose(0, 1)))
    assert torch.equal(both, before)
    rq, rk = P.rotary(q, pos, freq, k=k, interleaved=inter, out=(q, k))
    assert rq is q and rk is k
    assert torch.equal(both[:, hq + hk:], before[:, hq + hk:])
    _check_rotary(q, before[:, :hq], pos, freq, dtype, interleaved=inter)
    _check_rotary(k, before[:, hq:hq + hk], pos, freq, dtype, interleaved=inter)
    assert torch.equal(hq_major.transpose(0, 1), q) and torch.equal(hk_major.transpose(0, 1), k)


@pytest.mark.parametrize("inter,heads", [(False, 3), (True, 6)])
def test_rotary_more_workgroups_than_a_grid(torch, P, inter, heads):
    """A token a workgroup, 2^24 of them and a few more: one token's queries and keys for all, turned by positions of
    its own (the second axis's)."""
    t, d = (1 << 24) + 5, 344
    if torch.cuda.mem_get_info()[0] < t * heads * d * 2 + (4 << 30):
        pytest.skip("needs the memory of a whole MI355X")
    q, k = (_randn(torch, h, 1, h, d).expand(t, h, d) for h in (heads - 1, 1))
    pos = torch.stack([torch.zeros(t, dtype=torch.int32, device="cuda"), torch.arange(t, dtype=torch.int32, device="cuda")])
    freq, kw = _freq(P, 1), dict(interleaved=inter, sections=(0, 1))
    got = P.rotary(q, pos, freq, k=k, **kw)
    at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, (1 << 23) + 3, t - 6, t - 5, t - 1], device="cuda")
    for x, y in zip((q, k), got):
        _check_rotary(y[at], x[:len(at)], pos[:, at], freq, "bf16", **kw)
    del got, y
    torch.cuda.empty_cache()


def test_rotary_inverse_is_the_gradient(torch, P):
    """Turning back undoes a turn, and is the gradient: <R x, g> = <x, R^-1 g>, also against differences."""
    t, h, d, pairs = 12, 3, 40, 15
    x, g = _randn(torch, 1, t, h, d, dtype="f32"), _randn(torch, 2, t, h, d, dtype="f32")
    pos = torch.arange(t, dtype=torch.int32, device="cuda") * 37
    freq = _freq(P, pairs)
    f = 1.5
    y, _ = P.rotary(x, pos, freq, factor=f)
    back, _ = P.rotary(g, pos, freq, factor=f, inverse=True)
    unit = lambda z: f if z < 2 * pairs else 1.0
    gain = torch.tensor([unit(c) ** 2 for c in range(d)], device="cuda")
    again, _ = P.rotary(y, pos, freq, factor=f, inverse=True)
    assert torch.allclose(again, x * gain, rtol=0, atol=40 * U * f * f * float(x.abs().max()))
    lhs, rhs = (_f64(y) * _f64(g)).sum((1, 2)), (_f64(x) * _f64(back)).sum((1, 2))
    # 2 (pi + 9) U f (|x1| + |x2|) |g| a channel, from the bound above
    assert np.abs(lhs - rhs).max() <= 4 * (math.pi + 9) * U * f * (np.abs(_f64(x)).sum((1, 2)).max() * np.abs(_f64(g)).max() * 2)
    for c in (0, pairs - 1, pairs, 2 * pairs, d - 1):
        # the map is linear: a difference over a step of 1 is the derivative, up to the roundings of two results
        e = x.clone()
        e[..., c] += 1
        step = (_f64(P.rotary(e, pos, freq, factor=f)[0]) - _f64(y)) * _f64(g)
        tol = 4 * (math.pi + 9) * U * f * (2 * np.abs(_f64(x)).max() + 1) * 2 * np.abs(_f64(g)).max()
        assert np.abs(step.sum(2) - _f64(back)[..., c]).max() <= tol


def test_rotary_frequencies(P):
    w, f = P.rotary_frequencies(8, 1e4, device="cpu")
    assert f == 1.0 and np.allclose(w.numpy(), [1, 0.1, 0.01, 0.001], rtol=1e-15)
    lin, f = P.rotary_frequencies(8, 1e4, "linear", 4.0, device="cpu")
    assert f == 1.0 and np.allclose(lin.numpy(), w.numpy() / 4, rtol=1e-15)
    ntk, f = P.rotary_frequencies(8, 1e4, "ntk", 4.0, device="cpu")
    assert f == 1.0 and ntk[0] == 1 and np.isclose(ntk[3], w[3] / 4, rtol=1e-14)
    yarn, f = P.rotary_frequencies(8, 1e4, "yarn", 4.0, original_length=4096, device="cpu")
    turns = 4096 * w.numpy() / (2 * math.pi)
    g = np.clip((turns - 1) / 31, 0, 1)
    assert np.isclose(f, 0.1 * math.log(4) + 1) and np.allclose(yarn.numpy(), g * w.numpy() + (1 - g) * w.numpy() / 4, rtol=1e-14)
    assert g[0] == 1 and g[3] == 0 and 0 < g[2] < 1


def test_rotary_empty(torch, P):
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    gq, gk = P.rotary(q, torch.zeros(0, dtype=torch.int32, device="cuda"), _freq(P, 32), k=q[:, :2])
    assert gq.shape == (0, 4, 64) and gk.shape == (0, 2, 64)


def test_rotary_matches_the_encoders_layout(torch, P):
    """The encoder's M-RoPE sections: three axes, frequencies over the whole head, angles in its oracle."""
    from oracle import te_oracle as T
    d, sec, t = 128, (24, 20, 20), 50
    pos = torch.randint(0, 500, (3, t), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    q = _randn(torch, 1, t, 2, d, dtype="f32")
    got, _ = P.rotary(q, pos.cuda(), _freq(P, 64), sections=sec)
    x = _f64(q)
    ref = T.mrope(x, pos.numpy(), d, 5e6, sec, 0)
    _within(got, ref, (math.pi + 8) * U * 2 * np.abs(x).max() * np.ones_like(ref), "f32")
