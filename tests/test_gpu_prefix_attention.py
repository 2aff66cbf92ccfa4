"""Attention over a shared prefix and each sequence's own tokens (mte_prefix_attention) against its float64
oracle, through the Python wrapper.

Tolerances are the operator's own rounding, element by element (U16 = 2^-8 for bf16, U = 2^-24 for
fp32, half a step relative to the value each). With A = sum_j p_j |v_j| and S = the largest
scale * sum |q| |k| of the row, both from the oracle:
 - a score is a dot product of d terms and three further fp32 steps, so off by at most
   D = (d + 4) U S, plus 2 U for exp2 itself; a probability by 2 (D + 2 U) of itself, numerator and
   denominator: 2 (D + 2 U) A each;
 - sums over n keys, in fp32 and joined over parts: (n + 16) U A twice (O and l);
 - bf16: the probabilities' rounding U16 A and the result's U16 |o|; fp32: U |o|.
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
def C():
    from paper_2606_05981_amd import conditioning
    return conditioning


def _dt(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _f64(t):
    return t.detach().double().cpu().numpy()


def _randn(torch, seed, *shape, std=1.0, dtype="bf16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(_dt(torch, dtype)).cuda()


def _compare(got, ref, n, d, dtype):
    out, mag, reach = ref
    g = _f64(got)
    assert g.shape == out.shape and np.isfinite(g).all()
    D = (d + 4) * U * reach[..., None] + 2 * U
    t = 4 * D * mag + 2 * (n + 16) * U * mag + (U16 * mag if dtype == "bf16" else 0)
    t = t + (U16 if dtype == "bf16" else U) * (np.abs(out) + t) + 1e-30
    worst = float((np.abs(g - out) / t).max()) if g.size else 0.0
    _say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0


def _make(torch, ql, p, kl, hq, hkv, d, dtype, fused=False):
    q = _randn(torch, 1, sum(ql), hq, d, std=1.5, dtype=dtype)
    if fused:
        a, b = _randn(torch, 2, p, 2, hkv, d, dtype=dtype), _randn(torch, 3, sum(kl), 2, hkv, d, dtype=dtype)
        return q, a[:, 0], a[:, 1], b[:, 0], b[:, 1]
    return (q, *(_randn(torch, 2 + i, n, hkv, d, dtype=dtype) for i, n in enumerate((p, p, sum(kl), sum(kl)))))


CASES = [
    # q_lens, prefix, kv_lens, Hq, Hkv, d
    ([1], 1, [1], 1, 1, 64), ([1], 0, [1], 1, 1, 8), ([1], 96, [0], 16, 8, 128), ([3], 0, [0], 2, 2, 64),
    ([1, 1, 1], 33, [96, 0, 31], 16, 8, 128), ([5, 1, 0, 33], 65, [5, 7, 9, 33], 4, 2, 64),
    ([2, 9, 4], 31, [1, 4, 0], 4, 4, 72),                         # fewer own tokens than queries: rows that see the prefix alone
    ([4, 7], 0, [2, 7], 4, 2, 64),                                # ... or nothing
    ([32], 32, [32], 4, 4, 64), ([31], 33, [33], 4, 4, 64), ([33], 127, [65], 8, 1, 128), ([70], 129, [170], 12, 4, 40),
    # shared: many streams of few rows over a long prefix
    ([1] * 64, 1024, [96] * 40 + [33] * 24, 16, 8, 128), ([1] * 33, 2500, list(range(33)), 8, 8, 64),
    ([1, 2, 4, 0, 1, 24] * 8, 1500, [1, 320, 4, 7, 0, 24] * 8, 12, 4, 80), ([3] * 130, 700, [5] * 130, 5, 5, 40),
    ([1] * 300, 600, [2] * 300, 8, 2, 64),                        # more sequences than a launch takes
    ([2], 5000, [3], 16, 8, 128), ([1], 9000, [1], 8, 1, 64),     # one stream: the list is cut
    ([1] * 8, 40, [3000, 5, 0, 1, 700, 64, 65, 1], 8, 2, 128),    # long own ranges
    # many rows: tiles of 128 in one pass
    ([2100, 33], 96, [70, 33], 8, 8, 64), ([1030], 320, [1030], 16, 8, 128), ([700, 1, 0, 900], 33, [10, 5, 5, 901], 12, 4, 40),
    ([1500, 129], 65, [31, 129], 6, 6, 72), ([520, 3], 1200, [9, 3], 16, 16, 128),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,p,kl,hq,hkv,d", CASES)
def test_prefix_attention(torch, C, ql, p, kl, hq, hkv, d, causal, dtype):
    _say(f"prefix {p} + {kl[:8]} x {ql[:8]}, heads {hq}/{hkv} of {d}, causal {causal}, {dtype}")
    q, pk, pv, k, v = _make(torch, ql, p, kl, hq, hkv, d, dtype, fused=d == 64)
    got = C.prefix_attention(q, pk, pv, k, v, ql, kl, causal=causal)
    _compare(got, O.prefix(*map(_f64, (q, pk, pv, k, v)), ql, kl, causal), p + max(kl), d, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,p,kl,hq,hkv,d", [([1] * 40, 1100, [64] * 40, 8, 4, 64), ([300, 40], 70, [300, 41], 4, 4, 128),
                                              ([9, 1], 50, [9, 4], 4, 2, 72)])
def test_unseen_tokens_reach_nothing(torch, C, ql, p, kl, hq, hkv, d, dtype):
    """Infinities and NaN in own tokens that causal queries do not see: those rows are what they are without; the
    rows that see a NaN have it."""
    q, pk, pv, k, v = _make(torch, ql, p, kl, hq, hkv, d, dtype)
    k2, v2 = k.clone(), v.clone()
    at, row, bad = 0, 0, torch.zeros(q.shape[0], dtype=torch.bool)
    for i, (n, m) in enumerate(zip(ql, kl)):
        if n > 1:
            # the last token is seen by the last query only, one in the middle by those from its own on
            for j, (kv, vv) in ((m - 1, (math.nan, math.inf)), (m - 1 - n // 2, (1.0, math.nan))):
                k2[at + j, :, 3], v2[at + j, :, 5] = kv, vv
                bad[row + max(j - (m - n), 0):row + n] = True
        at, row = at + m, row + n
    got = C.prefix_attention(q, pk, pv, k2, v2, ql, kl)
    good = ~bad.cuda()
    assert torch.isfinite(got[good].float()).all()
    full = O.prefix(*map(_f64, (q, pk, pv, k, v)), ql, kl, True)
    keep = good.cpu().numpy()
    _compare(got[good], tuple(x[keep] for x in full), p + max(kl), d, dtype)
    if bad.any():
        assert torch.isnan(got[bad.cuda()].float()).any(-1).all()


def test_wild_values_are_seen(torch, C):
    """A value of infinity is the result of the rows that see it, in its channel alone."""
    ql, p, kl, h, d = [40], 20, [40], 2, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, h, h, d, "bf16")
    v[10, :, 7] = math.inf
    got = C.prefix_attention(q, pk, pv, k, v, ql, kl)
    assert torch.isfinite(got[:10].float()).all()
    assert (got[10:, :, 7] == math.inf).all()
    other = [c for c in range(d) if c != 7]
    assert torch.isfinite(got[10:][..., other].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wild_values_beside_far_scores(torch, C, dtype):
    """An infinite value of a heavy key, with scores of the other keys 300 below: 32 own keys and the prefix, which
    another wave of the workgroup takes."""
    ql, p, kl, h, d = [40], 20, [40], 2, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, h, h, d, dtype)
    one = torch.zeros_like(q)
    one[..., 0] = 8.0                                                # a score is k[.., 0] (of 64: 8 / sqrt(64))
    pk[..., 0], k[:32, :, 0], k[32:, :, 0] = -300.0, -300.0, 0.0
    v[35, :, 7] = -math.inf
    got = C.prefix_attention(one, pk, pv, k, v, ql, kl)
    assert torch.isfinite(got[:35].float()).all()
    assert (got[35:, :, 7] == -math.inf).all()
    other = [c for c in range(d) if c != 7]
    assert torch.isfinite(got[35:][..., other].float()).all()


# Every way through the keys whose own tokens hold infinities and NaN: q_lens, prefix, kv_lens, Hq, Hkv, d, far (rows of
# the prefix too far apart for the copies of the streamed tiles)
WAYS = [
    ([2, 3] * 20, 1100, [64, 70] * 20, 8, 4, 64, False), ([2, 3] * 20, 1100, [64, 70] * 20, 4, 4, 120, False),   # shared
    ([2, 5] * 20, 1500, [400, 1500] * 20, 8, 4, 128, False),          # shared, own ranges cut
    ([1030], 320, [1030], 16, 8, 128, False),                         # tiles of 128 rows in one pass, cut
    ([700, 900], 33, [700, 901], 12, 4, 40, False), ([1500, 129], 65, [1400, 129], 6, 6, 104, False),
    ([1030, 64], 70, [40, 64], 8, 4, 64, False), ([1030, 64], 70, [40, 64], 8, 4, 64, True),                     # whole
    ([2, 3] * 20, 1100, [64, 70] * 20, 8, 4, 64, True),
    ([3], 5000, [600], 16, 8, 128, False), ([9, 4], 50, [9, 4], 4, 2, 72, False),                                # tiles of 32
]


def _wild(torch, C, case, dtype, key, value):
    """Attention with `key` in channel 3 and `value` in channel 5 of two own tokens of each sequence, the last and one in
    the middle -> result, oracle without them, the rows that see one."""
    ql, p, kl, hq, hkv, d, far = case
    q, pk, pv, k, v = _make(torch, ql, p, kl, hq, hkv, d, dtype)
    full = O.prefix(*map(_f64, (q, pk, pv, k, v)), ql, kl, True)
    at, row, bad = 0, 0, torch.zeros(q.shape[0], dtype=torch.bool)
    for n, m in zip(ql, kl):
        for j in (m - 1, max(m - 1 - n // 2, 0)):
            if key is not None:
                k[at + j, :, 3] = key
            v[at + j, :, 5] = value
            bad[row + max(j - (m - n), 0):row + n] = True
        at, row = at + m, row + n
    if far:
        step = 1 << 24
        box = torch.zeros(((p - 1) * step + hkv * d,), dtype=q.dtype, device="cuda").as_strided((p, hkv, d), (step, d, 1))
        box.copy_(pk)
        pk = box
    got = C.prefix_attention(q, pk, pv, k, v, ql, kl)
    assert bad.any() and not bad.all()
    return got, full, bad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", WAYS)
def test_unseen_tokens_in_every_way(torch, C, case, dtype):
    _say(f"unseen {case}, {dtype}")
    for key, value in ((math.nan, math.inf), (math.inf, math.nan), (None, math.nan)):
        got, full, bad = _wild(torch, C, case, dtype, key, value)
        keep = ~bad
        _compare(got[keep.cuda()], tuple(x[keep.numpy()] for x in full), case[1] + max(case[2]), case[5], dtype)
        assert torch.isnan(got[bad.cuda()].float()).any(-1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", WAYS)
def test_infinite_values_in_every_way(torch, C, case, dtype):
    """An infinity of the rows that see it, in its channel alone; all else is what it is without."""
    _say(f"infinite {case}, {dtype}")
    for value in (math.inf, -math.inf):
        got, full, bad = _wild(torch, C, case, dtype, None, value)
        seen = got[bad.cuda()]
        assert (seen[..., 5] == value).all()
        got[..., 5][bad.cuda()] = 0.0
        full[0][..., 5][bad.numpy()] = 0.0
        _compare(got, full, case[1] + max(case[2]), case[5], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,p,kl", [([1] * 50, 800, [7] * 50), ([400], 100, [64])])
def test_strides_out_and_in_place(torch, C, ql, p, kl, dtype):
    """Queries within fused rows, head-major keys, out in place of the queries; other channels and rows stay."""
    hq, hkv, d = 8, 4, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, hq, hkv, d, dtype)
    ref = C.prefix_attention(q, pk, pv, k, v, ql, kl)
    major = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(C.prefix_attention(q, major(pk), major(pv), major(k), major(v), ql, kl), ref)
    wide = torch.full((q.shape[0] + 2, hq + 3, d), 7.0, dtype=q.dtype, device="cuda")
    inner = wide[:q.shape[0], 1:hq + 1]
    inner.copy_(q)
    assert C.prefix_attention(inner, pk, pv, k, v, ql, kl, out=inner) is inner
    assert torch.equal(inner, ref)
    assert (wide[:, 0] == 7).all() and (wide[:, hq + 1:] == 7).all() and (wide[q.shape[0]:] == 7).all()


def test_far_rows(torch, C):
    """Key rows too far apart for 32-bit offsets within a tile."""
    ql, p, kl, h, d = [300, 40], 70, [50, 40], 4, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, h, h, d, "bf16")
    ref = C.prefix_attention(q, pk, pv, k, v, ql, kl)
    big = torch.zeros(((p - 1) * (1 << 24) + h * d,), dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((p, h, d), (1 << 24, d, 1))
    far.copy_(pk)
    got = C.prefix_attention(q, far, pv, k, v, ql, kl)
    full = O.prefix(*map(_f64, (q, pk, pv, k, v)), ql, kl, True)
    _compare(got, full, p + 50, d, "bf16")
    _compare(ref, full, p + 50, d, "bf16")


def test_same_as_one_sequence(torch, C):
    """Over a prefix alone, and over own tokens alone, it is cross attention."""
    q, pk, pv, k, v = _make(torch, [3, 200], 96, [50, 60], 8, 4, 64, "bf16")
    none = k[:0]
    full = O.prefix(*map(_f64, (q, pk, pv, none, none)), [3, 200], [0, 0], False)
    _compare(C.prefix_attention(q, pk, pv, none, none, [3, 200], [0, 0]), full, 96, 64, "bf16")
    _compare(C.cross_attention(q, pk, pv, [3, 200], [96], kv_index=[0, 0]), full, 96, 64, "bf16")
    own = C.prefix_attention(q, none, none, k, v, [3, 200], [50, 60], causal=False)
    _compare(own, O.prefix(*map(_f64, (q, none, none, k, v)), [3, 200], [50, 60], False), 60, 64, "bf16")


def test_large_scores(torch, C):
    """Scores of tens of thousands on either side, where the heaviest key alone counts."""
    ql, p, kl, h, d = [1] * 40, 900, [33] * 40, 4, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, h, h, d, "bf16")
    k = k * 64
    got = C.prefix_attention(q, pk, pv, k, v, ql, kl, scale=64.0)
    qd, pkd, kd = q.double(), pk.double(), k.double()
    for i in (0, 7, 39):
        for g in range(h):
            s = (kd[33 * i:33 * i + 33, g] @ qd[i, g]) * 64.0
            best, gap = int(s.argmax()), float(s.topk(2).values.diff().abs())
            if gap > 1000 and float(s.max()) > float((pkd[:, g] @ qd[i, g]).max()) * 64.0 + 1000:
                assert torch.equal(got[i, g], v[33 * i + best, g])


def test_large_scores_are_decided(torch, C):
    """As above with keys that make it so: the heaviest of every row and head leads by more than 1000, by turns an own
    token and one of the prefix."""
    ql, p, kl, h, d = [1] * 40, 900, [33] * 40, 4, 64
    q, pk, pv, k, v = _make(torch, ql, p, kl, h, h, d, "bf16")
    own = torch.arange(0, 40, 2)
    k[33 * own + 5] = 16 * q[own]
    pk[100 + own + 1] = 16 * q[own + 1]
    got = C.prefix_attention(q, pk, pv, k, v, ql, kl, scale=64.0)
    for i in range(40):
        keys, values = torch.cat([pk, k[33 * i:33 * i + 33]]), torch.cat([pv, v[33 * i:33 * i + 33]])
        for g in range(h):
            s = (keys[:, g].double() @ q[i, g].double()) * 64.0
            two = s.topk(2)
            assert float(two.values[0] - two.values[1]) > 1000
            assert torch.equal(got[i, g], values[two.indices[0], g])


def test_no_queries(torch, C):
    q, pk, pv, k, v = _make(torch, [0, 0], 5, [3, 0], 4, 2, 64, "bf16")
    assert C.prefix_attention(q, pk, pv, k, v, [0, 0], [3, 0]).shape == (0, 4, 64)


# 257 tiles of 128 rows for each of 65535 heads: more workgroups than a launch takes. One token's queries for all.
MANY, HEADS = [129] * 127 + [257], 65535


@pytest.mark.parametrize("form", ["own", "cross", "cache"])
def test_more_workgroups_than_a_grid(torch, C, form):
    """Every sequence has one token, whose value is its result; the same of cross attention and of the 8-bit cache (a
    token for all)."""
    n, d = len(MANY), 64 if form == "cache" else 8
    if torch.cuda.mem_get_info()[0] < sum(MANY) * HEADS * d * 2 + (4 << 30):
        pytest.skip("needs the memory of a whole MI355X")
    q = _randn(torch, 1, 1, HEADS, d).expand(sum(MANY), HEADS, d)
    if form == "cache":
        cache = C.kv8_cache(1, HEADS, d)
        table, lens = torch.zeros((n, 21), dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
        k = _randn(torch, 2, 1, HEADS, d)
        C.kv8_append(cache, table[:1], lens[:1], k, k, [1])
        v = C.kv8_read(cache, table[:1], lens[:1], [1])[1].expand(n, HEADS, d)
        got = C.kv8_attention(q, cache, table, lens, MANY)
    else:
        k, v = (_randn(torch, i, n, HEADS, d) for i in (2, 3))
        got = C.cross_attention(q, k, v, MANY, [1] * n) if form == "cross" else \
            C.prefix_attention(q, k[:0], k[:0], k, v, MANY, [1] * n, causal=False)
    at = 0
    for i, rows in enumerate(MANY):
        assert bool((got[at:at + rows] == v[i]).all()), i
        at += rows
    del got
    torch.cuda.empty_cache()
