"""The operators over cached codes and conditioning rows (include/mte_cond.h) where magnitudes part: value
scales of one block far above another's, NaN that only some rows see, scores past fp32's whole
numbers, factors at the ends of the range; against the float64 oracle."""
import sys

import numpy as np
import pytest

from oracle import cond_oracle as O
from tests.test_gpu_cond import U, U16, _check_norm, _f64, _fill, _held, _i32, _randn

pytestmark = pytest.mark.gpu


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


# q_len, kv_len, table width, Hq, Hkv: one token, few rows of a long cache, chunks of them, rows over tables that
# fit LDS twice and once, and over one that does not (heads of 64)
CACHED = [(1, 200, None, 4, 2), (3, 2500, None, 4, 2), (40, 300, None, 4, 2), (130, 140, None, 32, 4),
          (300, 310, None, 32, 4), (300, 310, 40, 32, 4)]


def _sees(q_len, kv_len, causal):
    return np.arange(kv_len)[None] <= kv_len - q_len + np.arange(q_len)[:, None] if causal else np.ones((q_len, kv_len), bool)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread,away", [(20, 16), (25, 64), (40, 64), (40, 28), (60, 44), (100, 64), (-60, 0)])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_values_of_unlike_magnitude(torch, C, ql, kl, width, hq, h, spread, away, dtype):
    """The first or the last block's values are 2^spread times the others', its keys `away` (natural log)
    below: precision goes by what weight and scale come to together in the row, not by the largest scale.

    Bound: as in tests/test_gpu_cond.py, but what fp16 cannot hold of a term, at most half its smallest step, 2^-25 of
    operands whose largest in the row is 2^7 or more, is 2^-32 of the row's largest p_j scale_j, times codes of at
    most 448, for each of n keys."""
    d = 64
    for first in (True, False):
        _say(f"cached values 2^{spread} apart, away {away}, {ql} x {kl}, width {width}, {dtype}, first {first}")
        big = slice(0, 32) if first else slice((kl - 1) // 32 * 32, kl)
        cache, table, kv, k, v = _fill(torch, C, [kl], h, d, width=width, spread=False)
        k[..., 0] = 0
        k[big, :, 0] = -away
        v[big] *= 2.0 ** spread
        C.kv8_append(cache, table, kv, k, v, [kl])
        q = _randn(torch, 110, ql, hq, d, dtype=dtype)
        q[..., 0] = 8
        got = _f64(C.kv8_attention(q, cache, table, kv, [ql]))
        (kk, vv), = _held(torch, cache, table, [kl])
        ref, mag, reach = O.attend(_f64(q), kk, vv, _sees(ql, kl, False), 1 / 8)
        vs = cache.scales[table[0, :(kl + 31) // 32].long(), :, 1].double().cpu().numpy().repeat(32, 0)[:kl]
        s = np.einsum("ihd,jhd->hij", _f64(q), kk.repeat(hq // h, 1)) / 8
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        top = (p * vs.repeat(hq // h, 1).T[:, None]).max(-1).T[..., None]           # [ql, hq, 1]
        D = (d + 4) * U * reach[..., None] + 2 * U
        t = 4 * D * mag + 2 * (kl + 16) * U * mag + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * mag
        t = t + kl * 2.0 ** -32 * 448 * top
        t = t + (U16 if dtype == "bf16" else U) * (np.abs(ref) + t) + 1e-30
        worst = float((np.abs(got - ref) / t).max())
        _say(f"  worst error / bound {worst:.3f}")
        assert worst <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,width,hq,h", [(4, 100, None, 4, 2), (4, 2500, None, 4, 2), (40, 64, None, 4, 2), (130, 140, None, 32, 4),
                                              (300, 310, None, 32, 4), (300, 310, 40, 32, 4)])
def test_kv8_unseen_nan(torch, C, ql, kl, width, hq, h, d, dtype):
    """A causal row's result does not depend on NaN that it does not see: a cached NaN value reaches the rows that
    see its token, in its channel; a NaN key the rows that see it, whole."""
    _say(f"cached NaN, {ql} x {kl} of {d}, width {width}, {dtype}")
    cache, table, kv, k, v = _fill(torch, C, [kl], h, d, width=width)
    q = _randn(torch, 111, ql, hq, d, dtype=dtype)
    seen_by = lambda tok: torch.arange(ql, device="cuda") >= tok - (kl - ql)     # rows that see a token
    for tok, chan in ((kl - ql + 1, 5), (kl - 1, d - 1), (kl - (ql + 1) // 2, 0)):
        bad = v.clone()
        bad[tok, 0, chan] = 0                      # (no scale hangs on it)
        C.kv8_append(cache, table, kv, k, bad, [kl])
        clean = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
        every = C.kv8_attention(q, cache, table, kv, [ql])
        bad[tok, 0, chan] = float("nan")
        C.kv8_append(cache, table, kv, k, bad, [kl])
        want = clean.clone()
        rows = seen_by(tok)
        want[:, :hq // h, chan] = torch.where(rows[:, None], torch.full_like(want[:, :hq // h, chan], float("nan")),
                                              want[:, :hq // h, chan])
        got = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
        assert bool(rows.any()) and not bool(rows.all())
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
        got = C.kv8_attention(q, cache, table, kv, [ql])                        # seen by all
        assert bool(torch.isnan(got[:, :hq // h, chan]).all())
        got[:, :hq // h, chan] = every[:, :hq // h, chan]
        assert torch.equal(got, every)
    bad = k.clone()
    bad[kl - 2, 0, 3] = 0
    C.kv8_append(cache, table, kv, bad, v, [kl])
    clean = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
    bad[kl - 2, 0, 3] = float("nan")
    C.kv8_append(cache, table, kv, bad, v, [kl])
    got = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
    rows = seen_by(kl - 2)
    assert bool(torch.isnan(got[rows][:, :hq // h]).all())
    got[rows, :hq // h] = clean[rows, :hq // h]
    assert torch.equal(got, clean)


def _far(torch, q_len, kv_len, hq, h, d, sign, dtype):
    """One channel: queries of 165 * 2^10, keys of 9 * 2^14, the heaviest 9 * 2^15 (sign -1: -9 * 2^15 and -9 * 2^14): scores of
    1485 * 2^24 and twice that, exact, in units of which any scale takes fp32 past its whole numbers."""
    win = kv_len * 2 // 3
    q = torch.zeros(q_len, hq, d)
    k = torch.zeros(kv_len, h, d)
    q[..., 3] = 165 * 2.0 ** 10
    k[..., 3] = 9 * 2.0 ** 14 * (1 if sign > 0 else -2)
    k[win, :, 3] = 9 * 2.0 ** 14 * (2 if sign > 0 else -1)
    return q.to(dtype).cuda(), k.to(dtype).cuda(), win


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,h,d", [(1, 96, 4, 2, 64), (33, 130, 4, 2, 128), (2, 2500, 4, 2, 64), (2100, 96, 8, 8, 64),
                                          (2100, 96, 4, 2, 128), (600, 2500, 16, 16, 64)])
def test_cross_scores_far_out(torch, C, ql, kl, hq, h, d, dtype):
    """Scores past fp32's whole numbers: the heaviest key takes all, exactly."""
    _say(f"cross, scores of 2^34, {ql} x {kl}, {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    v = _randn(torch, 112, kl, h, d, dtype=dtype)
    for sign in (1, -1):
        q, k, win = _far(torch, ql, kl, hq, h, d, sign, dt)
        for scale in (1.0, 1.3, 0.9, 0.071):
            got = C.cross_attention(q, k, v, [ql], [kl], scale=scale)
            assert torch.equal(got, v[win].repeat_interleave(hq // h, 0)[None].expand(ql, -1, -1)), (sign, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_scores_far_out(torch, C, ql, kl, width, hq, h, d, dtype):
    _say(f"cached, scores of 2^34, {ql} x {kl} of {d}, width {width}, {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, table, kv, _, v = _fill(torch, C, [kl], h, d, width=width)
    for sign in (1, -1):
        q, k, win = _far(torch, ql, kl, hq, h, d, sign, dt)
        C.kv8_append(cache, table, kv, k.to(v.dtype), v, [kl])
        _, rv = C.kv8_read(cache, table, kv, [kl], dtype=dt)
        for scale in (1.0, 1.3, 0.9, 0.071):
            got = C.kv8_attention(q, cache, table, kv, [ql], scale=scale)
            assert torch.equal(got, rv[win].repeat_interleave(hq // h, 0)[None].expand(ql, -1, -1)), (sign, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_largest_keys_under_zero_queries(torch, C, ql, kl, width, hq, h, dtype):
    """Keys at the largest block scale and a large factor: their product is beyond fp32, a score of 0 is 0 all
    the same, and all tokens weigh alike."""
    _say(f"cached, zero queries over the largest keys, {ql} x {kl}, width {width}, {dtype}")
    d = 64
    cache, table, kv, k, v = _fill(torch, C, [kl], h, d, width=width, spread=False)
    k[:] = 3.2e38
    C.kv8_append(cache, table, kv, k, v, [kl])
    assert bool((cache.scales[table[0, :(kl + 31) // 32].long(), :, 0] == 2.0 ** 120).all())
    q = torch.zeros((ql, hq, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    got = _f64(C.kv8_attention(q, cache, table, kv, [ql], scale=512.0))
    (_, vv), = _held(torch, cache, table, [kl])
    ref, mag = vv.mean(0).repeat(hq // h, 0)[None], np.abs(vv).mean(0).repeat(hq // h, 0)[None]
    # p = 1 exactly: sums of kl terms, their quotient, the result
    t = 2 * (kl + 16) * U * mag + (U16 if dtype == "bf16" else U) * np.abs(ref)
    assert (np.abs(got - ref) <= t).all()


@pytest.mark.parametrize("d", [64, 128])
def test_kv8_append_beside_refused_sequences(torch, C, d):
    """A length that does not fit leaves its own sequence's blocks as they were; the sequences beside it are
    written, from their own rows."""
    _say(f"append beside refused sequences, d {d}")
    h, new = 2, [20, 0, 35, 20]
    k, v = _randn(torch, 113, sum(new), h, d), _randn(torch, 114, sum(new), h, d)
    start = [0, 20, 20, 55, 75]
    for lens in ([20, 0, 34, 20], [19, 5, 40, 20], [20, 0, 35, 65], [-5, 0, 64, 2**31 - 1], [64, -1, 36, -2**31]):
        cache = C.kv8_cache(8, h, d)
        table = _i32(torch, [[7, 2], [3, 5], [0, 6], [4, 1]])
        C.kv8_append(cache, table, _i32(torch, lens), k, v, new)
        for i, (n, m) in enumerate(zip(lens, new)):
            blocks = table[i].long()
            if m == 0 or n < m or n > 64:
                assert not bool(cache.k_codes[blocks].any()) and not bool(cache.v_codes[blocks].any())
                assert bool((cache.scales[blocks] == 2.0 ** -126).all())
                continue
            one = C.kv8_cache(8, h, d)               # the same rows alone
            C.kv8_append(one, table[i:i + 1], _i32(torch, [n]), k[start[i]:start[i + 1]], v[start[i]:start[i + 1]], [m])
            assert bool(one.k_codes[blocks].any())
            for a, b in zip(cache, one):
                assert torch.equal(a[blocks], b[blocks])
            (kk, vv), = _held(torch, cache, table[i:i + 1], [n])
            for rows, got in ((k, kk), (v, vv)):
                ref = O.Cache(h, d)
                if n > m:
                    ref.append(np.zeros((n - m, h, d)))
                ref.append(_f64(rows[start[i]:start[i + 1]]))
                np.testing.assert_array_equal(got, ref.values())


def test_kv8_read_smallest_values(torch, C):
    """Values at the smallest scale, 2^-126: fp32 holds them all, bf16 those that are multiples of 2^-133; the others
    are rounded to one, ties to even."""
    _say("read, smallest values")
    h, d = 1, 64
    codes = torch.tensor([c for c in range(256) if c & 0x7F != 0x7F], dtype=torch.int64)   # all but NaN
    rows = torch.cat([codes, codes[:2]]).reshape(4, 1, 64)
    cache = C.kv8_cache(1, h, d)
    lut = torch.from_numpy(O.Q.decode_table()).double()
    x = (lut[rows] * 2.0 ** -126).float()            # exact
    C.kv8_append(cache, _i32(torch, [[0]]), _i32(torch, [4]), x.cuda(), x.cuda(), [4])
    assert bool((cache.scales == 2.0 ** -126).all())
    for got in C.kv8_read(cache, _i32(torch, [[0]]), _i32(torch, [4]), [4], dtype=torch.float32):
        assert torch.equal(got.cpu(), x)
    steps = torch.round(x.double() * 2.0 ** 133) * 2.0 ** -133                  # ties to even
    want = torch.where(x.double().abs() < 2.0 ** -126, steps, x.double())
    for got in C.kv8_read(cache, _i32(torch, [[0]]), _i32(torch, [4]), [4]):
        assert torch.equal(got.double().cpu(), want)
    assert not torch.equal(want, x.double())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,h,d", [([40, 3], [96, 7], 4, 2, 64), ([3, 2], [2500, 40], 4, 2, 64), ([2100], [96], 16, 8, 128),
                                          ([1300, 9], [130, 70], 8, 8, 40), ([600], [2500], 16, 16, 64)])
def test_cross_in_place_of_the_queries(torch, C, ql, kl, hq, h, d, dtype):
    _say(f"cross, out = q, {ql} x {kl} {dtype}")
    q = _randn(torch, 116, sum(ql), hq, d, dtype=dtype)
    k, v = _randn(torch, 117, sum(kl), h, d, dtype=dtype), _randn(torch, 118, sum(kl), h, d, dtype=dtype)
    want = C.cross_attention(q, k, v, ql, kl)
    got = C.cross_attention(q, k, v, ql, kl, out=q)
    assert got is q and torch.equal(q, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_in_place_of_the_queries(torch, C, ql, kl, width, hq, h, d, dtype):
    _say(f"cached, out = q, {ql} x {kl} of {d}, width {width}, {dtype}")
    cache, table, kv, _, _ = _fill(torch, C, [kl], h, d, width=width)
    q = _randn(torch, 119, ql, hq, d, dtype=dtype)
    want = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
    got = C.kv8_attention(q, cache, table, kv, [ql], causal=True, out=q)
    assert got is q and torch.equal(q, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,px,c,groups", [(1, 4096, 5, 5), (1, 9, 64, 8), (2, 2048, 6, 3)])
def test_group_norm_mean_whose_square_overflows(torch, C, n, px, c, groups, dtype):
    """A mean of 1.5 * 2^64, beyond fp32 when squared, under a spread of 2^57.6: only differences are squared."""
    _say(f"group norm, mean of 2^64.6, {n} x {px} x {c} / {groups}, {dtype}")
    g = torch.Generator().manual_seed(125)
    x = 1.5 * (1 + 2.0 ** -7 * torch.randint(-1, 2, (n, px, c), generator=g)) * 2.0 ** 64   # (8 bits: exact in bf16)
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    _check_norm(torch, C.group_norm(x, groups), x, groups, None, None, 1e-5, None, dtype)


def test_cross_more_heads_than_fp32_counts(torch, C):
    """2^24 query heads on one kv head, rows of a wider buffer: rows are found by whole numbers, not in fp32."""
    _say("cross, 2^24 heads")
    hq, d = 1 << 24, 8
    wide = [torch.full((2, hq * d + 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, out = (w.as_strided((2, hq, d), (hq * d + 64, d, 1)) for w in wide)
    q.copy_(torch.randn(2, hq, d, generator=torch.Generator("cuda").manual_seed(126), device="cuda"))
    k, v = _randn(torch, 127, 3, 1, d), _randn(torch, 128, 3, 1, d)
    C.cross_attention(q, k, v, [2], [3], out=out)
    kf, vf = k[:, 0].float(), v[:, 0].float()
    for i in range(2):
        p = torch.softmax(torch.stack([(q[i].float() * x).sum(-1) for x in kf], -1) / d ** 0.5, -1)
        ref = sum(p[:, j:j + 1] * vf[j] for j in range(3))
        mag = sum(p[:, j:j + 1] * vf[j].abs() for j in range(3))
        # the probabilities' and the result's rounding; fp32 on both sides: (d + 16) u each of the scores, |s| < 40
        assert bool(((out[i].float() - ref).abs() <= U16 * (mag + ref.abs()) * 1.01 + 4 * 40 * (d + 16) * U * mag).all())
    assert all(bool((w[:, -64:] == 7.0).all()) for w in wide)


def _alike(torch, got, ref, mag, n, dtype):
    """Equal weights: sums of n terms, their quotient, and the result's rounding."""
    t = 2 * (n + 16) * U * mag + (U16 if dtype == "bf16" else U) * np.abs(ref)
    assert (np.abs(_f64(got) - ref) <= t + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,h,d", [(3, 96, 4, 2, 64), (2, 2500, 4, 2, 64), (2100, 96, 8, 8, 64), (2100, 130, 4, 2, 128)])
def test_cross_scores_far_out_masked(torch, C, ql, kl, hq, h, d, dtype):
    """The heaviest key masked: the others, of one score, weigh alike; and a sequence beside it that sees nothing."""
    _say(f"cross, far scores, heaviest masked, {ql} x {kl} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    v = _randn(torch, 129, kl, h, d, dtype=dtype)
    for sign in (1, -1):
        q, k, win = _far(torch, ql, kl, hq, h, d, sign, dt)
        mask = torch.ones(2 * kl, dtype=torch.bool)
        mask[win], mask[kl:] = False, False
        got = C.cross_attention(torch.cat([q, q]), torch.cat([k, k]), torch.cat([v, v]), [ql, ql], [kl, kl],
                                key_mask=mask.cuda(), scale=1.3)
        vv = np.delete(_f64(v), win, 0).repeat(hq // h, 1)
        _alike(torch, got[:ql], vv.mean(0)[None], np.abs(vv).mean(0)[None], kl, dtype)
        assert not bool(got[ql:].any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_scores_far_out_causal(torch, C, ql, kl, width, hq, h, dtype):
    """Rows from the heaviest key on are its value, those before it the mean of what they see."""
    _say(f"cached, far scores, causal, {ql} x {kl}, width {width}, {dtype}")
    d, dt = 64, torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, table, kv, _, v = _fill(torch, C, [kl], h, d, width=width)
    for sign in (1, -1):
        q, k, _ = _far(torch, ql, kl, hq, h, d, sign, dt)
        win, rest = kl - (ql + 1) // 2, k[:1].clone()
        k[:] = rest
        k[win] *= 2.0 if sign > 0 else 0.5
        C.kv8_append(cache, table, kv, k.to(v.dtype), v, [kl])
        got = C.kv8_attention(q, cache, table, kv, [ql], causal=True, scale=1.3)
        (_, vv), = _held(torch, cache, table, [kl])
        vv = vv.repeat(hq // h, 1)
        for u in range(ql):
            n = kl - ql + u + 1
            if n > win:
                assert np.array_equal(_f64(got[u]), _f64(torch.from_numpy(vv[win]).to(dt)))
            else:
                _alike(torch, got[u], vv[:n].mean(0), np.abs(vv[:n]).mean(0), n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,width,hq,h", CACHED)
def test_kv8_scales_that_are_no_powers_of_two(torch, C, ql, kl, width, hq, h, dtype):
    """A cache that another program filled, its scales between powers of two: attention takes them as they are. (The
    logarithm of a value scale is within 2^-21 here, |log2| < 8: its weights move by less.)"""
    _say(f"cached, scales of any value, {ql} x {kl}, width {width}, {dtype}")
    d = 64
    cache, table, kv, _, _ = _fill(torch, C, [kl], h, d, width=width, spread=False)
    cache.scales.mul_(1 + torch.rand(cache.scales.shape, generator=torch.Generator().manual_seed(130)).cuda() * 0.99)
    q = _randn(torch, 131, ql, hq, d, dtype=dtype)
    got = _f64(C.kv8_attention(q, cache, table, kv, [ql]))
    (kk, vv), = _held(torch, cache, table, [kl])
    ref, mag, reach = O.attend(_f64(q), kk, vv, _sees(ql, kl, False), 1 / 8)
    D = (d + 4) * U * reach[..., None] + 2 * U
    t = 4 * D * mag + 2 * (kl + 16) * U * mag + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * mag + 2.0 ** -21 * mag
    t = t + kl * 2.0 ** -32 * 448 * float(cache.scales[..., 1].max())
    t = t + (U16 if dtype == "bf16" else U) * (np.abs(ref) + t) + 1e-30
    worst = float((np.abs(got - ref) / t).max())
    _say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0
