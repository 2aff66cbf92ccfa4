"""The operators that read the conditioning (include/mte_cond.h) against their float64 oracle, through
the Python wrappers.

Tolerances are the operators' own rounding, element by element (u16 = 2^-8 for bf16, u = 2^-24 for
fp32, half a step relative to the value each). With A = sum_j p_j |v_j| and S = the largest
scale * sum |q| |k| of the row, both from the oracle:
 - a score is a dot product of d terms and three further fp32 steps, so off by at most
   D = (d + 4) u S, plus 2 u for exp2 itself; a probability by 2 (D + 2 u) of itself, numerator and
   denominator: 2 (D + 2 u) A each;
 - sums over n keys, in fp32 and joined over splits: (n + 16) u A twice (O and l);
 - bf16: the probabilities' rounding u16 A and the result's u16 |o|; fp32: u |o|;
 - cache: bf16 calls round probabilities to fp16, 2^-11 A, and small ones by half fp16's smallest
   step, 2^-25, where the row's largest is held as 2^7 at least (it lies in [2^7, 2^15], so that the
   reference may lag): 2^-25 / 2^7 = 2^-32 of it, on a value of at most vmax each: n 2^-32 vmax;
   fp32 calls carry two fp16 terms: 2^-22 A and the same absolute part.
"""
import sys

import numpy as np
import pytest

from oracle import cond_oracle as O

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


def _tol(ref, mag, reach, n, d, dtype, cached=0.0):
    """Element bounds of an attention result (module docstring); cached: the largest cached |v|."""
    D = (d + 4) * U * reach[..., None] + 2 * U
    t = 4 * D * mag + 2 * (n + 16) * U * mag
    if cached:
        t = t + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * mag + n * 2.0 ** -32 * cached
    elif dtype == "bf16":
        t = t + U16 * mag
    return t + (U16 if dtype == "bf16" else U) * (np.abs(ref) + t) + 1e-30


def _compare(got, ref, mag, reach, n, d, dtype, cached=0.0):
    g = _f64(got)
    assert np.isfinite(g).all()
    over = np.abs(g - ref) / _tol(ref, mag, reach, n, d, dtype, cached)
    worst = float(over.max()) if over.size else 0.0
    _say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0


def _randn(torch, seed, *shape, std=1.0, dtype="bf16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(_dt(torch, dtype)).cuda()


# ---- cross attention ----------------------------------------------------------------------------

CROSS = [
    # q_lens, kv_lens, Hq, Hkv, d
    ([1], [1], 1, 1, 64),
    ([1], [96], 16, 8, 128),
    ([1, 1, 1], [96, 31, 130], 16, 8, 128),
    ([5, 1, 0, 33], [0, 1, 7, 64], 4, 2, 64),
    ([32], [32], 4, 4, 64), ([31], [33], 4, 4, 64), ([33], [65], 4, 4, 64),
    ([127, 128, 129], [127, 128, 129], 2, 2, 128),
    ([64, 3], [63, 320], 8, 1, 128),             # all query heads on one kv head
    ([70], [40], 12, 4, 64),                     # groups of three
    ([40, 9], [100, 17], 5, 5, 40), ([40, 9], [100, 17], 3, 3, 80), ([9], [50], 2, 1, 8), ([17], [50], 2, 2, 72),
    ([300], [1], 4, 2, 64),
    ([2], [2500], 8, 2, 64),                     # a long range of keys, few rows: split and joined
    ([1], [5000], 16, 8, 128), ([130], [1500], 2, 2, 128),
    ([8, 8], [1000, 3], 2, 2, 64),               # a split plan of which one sequence uses one part
    # enough rows for the tiles of 128: ends inside tiles, no keys, one key, padded heads, groups
    ([2100, 33], [96, 70], 8, 8, 64), ([1030], [320], 16, 8, 128), ([700, 1, 0, 900], [33, 0, 5, 1], 12, 4, 40),
    ([1500, 129], [65, 31], 6, 6, 72), ([4099], [64], 4, 2, 128),
    ([600], [2500], 16, 16, 64), ([520, 3], [1200, 9], 16, 16, 128),   # and split
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,hkv,d", CROSS)
def test_cross_attention(torch, C, ql, kl, hq, hkv, d, dtype):
    _say(f"cross {ql} x {kl}, heads {hq}/{hkv} of {d}, {dtype}")
    q = _randn(torch, 1, sum(ql), hq, d, std=1.5, dtype=dtype)
    k, v = _randn(torch, 2, sum(kl), hkv, d, dtype=dtype), _randn(torch, 3, sum(kl), hkv, d, dtype=dtype)
    got = C.cross_attention(q, k, v, ql, kl)
    ref = O.cross(_f64(q), _f64(k), _f64(v), ql, kl)
    _compare(got, *ref, max(kl), d, dtype)
    again = C.cross_attention(q, k, v, ql, kl)
    assert torch.equal(got, again)                # no order of sums depends on the run


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,hq,hkv,d", [([3, 40, 1], [96, 70, 33], 4, 2, 64), ([1, 1], [200, 31], 16, 8, 128),
                                            ([200], [130], 2, 2, 128), ([1], [3000], 4, 4, 64),
                                            ([1100, 40], [96, 70], 16, 8, 128), ([600], [2500], 16, 16, 64)])
def test_cross_attention_mask(torch, C, ql, kl, hq, hkv, d, dtype):
    """Masked tokens hold infinities and NaN; one sequence is masked whole."""
    _say(f"masked cross {ql} x {kl} {dtype}")
    q = _randn(torch, 4, sum(ql), hq, d, std=1.5, dtype=dtype)
    k, v = _randn(torch, 5, sum(kl), hkv, d, dtype=dtype), _randn(torch, 6, sum(kl), hkv, d, dtype=dtype)
    mask = torch.rand(sum(kl), generator=torch.Generator().manual_seed(7)) < 0.6
    mask[-1] = False                              # the last token of all, next to what is not there
    if len(kl) > 1:
        mask[kl[0]:kl[0] + kl[1]] = False
    bad = torch.tensor([float("inf"), float("nan"), float("-inf"), torch.finfo(_dt(torch, dtype)).min])
    fill = bad[torch.arange(sum(kl)) % 4].to(_dt(torch, dtype)).cuda()[:, None, None]
    gm = mask.cuda()
    k, v = torch.where(gm[:, None, None], k, fill), torch.where(gm[:, None, None], v, fill)
    ref = O.cross(_f64(q), _f64(k), _f64(v), ql, kl, key_mask=mask.numpy())
    for m in (gm, gm.to(torch.uint8) * 3):
        got = C.cross_attention(q, k, v, ql, kl, key_mask=m)
        _compare(got, *ref, max(kl), d, dtype)
    if len(kl) > 1:
        assert not bool(got[ql[0]:ql[0] + ql[1]].any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,hq,hkv,d", [(9, 4, 2, 40), (2100, 8, 4, 40), (2100, 8, 4, 72), (2100, 4, 2, 128)])
def test_cross_attention_infinite_scores(torch, C, ql, hq, hkv, d, dtype):
    """A key whose score is -inf weighs nothing, also where head_dim is padded."""
    _say(f"cross with scores of -inf {ql} rows of {d} {dtype}")
    q = _randn(torch, 80, ql, hq, d, dtype=dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    k, v = _randn(torch, 81, 96, hkv, d, dtype=dtype), _randn(torch, 82, 96, hkv, d, dtype=dtype)
    gone = np.arange(96) % 5 == 1
    ref = O.cross(_f64(q), _f64(k), _f64(v), [ql], [96], key_mask=~gone)
    k[torch.from_numpy(gone).cuda(), :, 0] = float("-inf")
    _compare(C.cross_attention(q, k, v, [ql], [96]), *ref, 96, d, dtype)


def test_cross_attention_index(torch, C):
    """One frame's conditioning for all, the same one twice, an order that goes back, and one that
    nobody reads."""
    _say("cross with kv_index")
    ql, kl = [5, 40, 1, 33], [70, 9, 96]
    q = _randn(torch, 8, sum(ql), 4, 64)
    k, v = _randn(torch, 9, sum(kl), 2, 64), _randn(torch, 10, sum(kl), 2, 64)
    for idx in ([0, 0, 0, 0], [2, 1, 2, 0], [1, 1, 2, 2]):
        got = C.cross_attention(q, k, v, ql, kl, kv_index=idx)
        _compare(got, *O.cross(_f64(q), _f64(k), _f64(v), ql, kl, idx), max(kl), 64, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_attention_layouts(torch, C, dtype):
    """Fused key/value rows, head-major tensors, queries and results inside wider buffers; what lies
    around the result stays as it was."""
    _say("cross layouts", dtype)
    ql, kl, hq, hkv, d = [50, 3], [40, 77], 4, 2, 64
    q = _randn(torch, 11, sum(ql), hq, d, dtype=dtype)
    both = _randn(torch, 12, sum(kl), 2, hkv, d, dtype=dtype)
    plain = C.cross_attention(q, both[:, 0].contiguous(), both[:, 1].contiguous(), ql, kl)
    assert torch.equal(plain, C.cross_attention(q, both[:, 0], both[:, 1], ql, kl))
    qh = q.transpose(0, 1).contiguous().transpose(0, 1)                       # [H, T, d] in memory
    kh = both[:, 0].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(plain, C.cross_attention(qh, kh, both[:, 1], ql, kl))
    wide = torch.full((sum(ql) + 2, hq, d + 16), 7.0, dtype=q.dtype, device="cuda")
    qw = torch.zeros_like(wide)
    qw[:-2, :, 8:-8] = q
    out = wide[:-2, :, 8:-8]
    res = C.cross_attention(qw[:-2, :, 8:-8], both[:, 0], both[:, 1], ql, kl, out=out)
    assert res is out and torch.equal(out, plain)
    rest = wide.clone()
    rest[:-2, :, 8:-8] = 7.0
    assert bool((rest == 7.0).all())
    oh = torch.empty((hq, sum(ql), d), dtype=q.dtype, device="cuda").transpose(0, 1)
    assert torch.equal(plain, C.cross_attention(q, both[:, 0], both[:, 1], ql, kl, out=oh))


def test_cross_attention_many_sequences(torch, C):
    """More sequences than one launch takes, some of them empty."""
    _say("cross, 300 sequences")
    rng = np.random.default_rng(13)
    ql = [int(x) for x in rng.integers(0, 5, 300)]
    kl = [int(x) for x in rng.integers(0, 20, 300)]
    q = _randn(torch, 14, sum(ql), 2, 64)
    k, v = _randn(torch, 15, sum(kl), 2, 64), _randn(torch, 16, sum(kl), 2, 64)
    _compare(C.cross_attention(q, k, v, ql, kl), *O.cross(_f64(q), _f64(k), _f64(v), ql, kl), max(kl), 64, "bf16")


def test_cross_attention_scale_and_large_scores(torch, C):
    """Scores of hundreds: one key takes all, nothing overflows."""
    _say("cross, large scores")
    ql, kl, d = [64, 2], [90, 33], 64
    q, k = _randn(torch, 17, sum(ql), 2, d, std=8), _randn(torch, 18, sum(kl), 2, d, std=8)
    v = _randn(torch, 19, sum(kl), 2, d)
    for scale in (1.0, 0.01):
        got = C.cross_attention(q, k, v, ql, kl, scale=scale)
        _compare(got, *O.cross(_f64(q), _f64(k), _f64(v), ql, kl, scale=scale), max(kl), d, "bf16")


def test_cross_attention_strides_past_32_bits(torch, C):
    """Rows 2^30 elements apart (4 GiB and more from the first)."""
    _say("cross, rows 2 GiB apart")
    step = 1 << 30
    buf = torch.empty(3 * step + 128, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((4, 2, 64), (step, 64, 1))
    q = _randn(torch, 20, 4, 2, 64)
    k, v = _randn(torch, 21, 4, 2, 64), _randn(torch, 22, 4, 2, 64)
    plain = C.cross_attention(q, k, v, [4], [4])
    far.copy_(k)
    assert torch.equal(plain, C.cross_attention(q, far, v, [4], [4]))
    far.copy_(v)
    assert torch.equal(plain, C.cross_attention(q, k, far, [4], [4]))
    far.copy_(q)
    assert torch.equal(plain, C.cross_attention(far, k, v, [4], [4], out=far))


@pytest.mark.parametrize("ql,kl,d", [(8500, 70, 64), (8500, 70, 104), (20, 600, 64)])
def test_cross_attention_rows_far_apart(torch, C, ql, kl, d):
    """Keys too far apart for 32-bit offsets within a tile, under many rows and few."""
    _say(f"cross, {ql} rows over keys 2^24 elements apart")
    step = 1 << 24
    buf = torch.empty((kl - 1) * step + 2 * d, dtype=torch.bfloat16, device="cuda")
    k, v = (buf.as_strided((kl, 1, d), (step, d, 1), x) for x in (0, d))
    k.copy_(_randn(torch, 23, kl, 1, d)), v.copy_(_randn(torch, 24, kl, 1, d))
    q = _randn(torch, 25, ql, 2, d, std=1.5)
    mask = torch.rand(kl, generator=torch.Generator().manual_seed(26)) < 0.7
    for m in (None, mask):
        got = C.cross_attention(q, k, v, [ql], [kl], key_mask=None if m is None else m.cuda())
        _compare(got, *O.cross(_f64(q), _f64(k), _f64(v), [ql], [kl], key_mask=None if m is None else m.numpy()), kl, d,
                 "bf16")


@pytest.mark.parametrize("step", [1 << 29, 1 << 30])
def test_attention_heads_far_apart(torch, C, step):
    """Many rows of queries and results whose heads lie as far apart as 32-bit offsets reach, and farther."""
    _say(f"attention, heads {step} elements apart")
    n, hq, hkv, d = 2100, 4, 2, 64
    buf = torch.empty((hq - 1) * step + n * d, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((n, hq, d), (d, step, 1))
    q = _randn(torch, 86, n, hq, d)
    k, v = _randn(torch, 87, 96, hkv, d), _randn(torch, 88, 96, hkv, d)
    ref = O.cross(_f64(q), _f64(k), _f64(v), [n], [96])
    cache = C.kv8_cache(3, hkv, d)
    table, kv = _i32(torch, [[2, 0, 1]]), _i32(torch, [96])
    C.kv8_append(cache, table, kv, k, v, [96])
    plain = C.kv8_attention(q, cache, table, kv, [n])
    far.copy_(q)
    _compare(C.cross_attention(far, k, v, [n], [96], out=far), *ref, 96, d, "bf16")
    far.copy_(q)
    got = C.kv8_attention(far, cache, table, kv, [n], out=far)
    assert got is far and torch.equal(plain, far)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cross_attention_index_split(torch, C, dtype):
    """Several sequences, long and short, over one long one that is split; a masked half."""
    _say("cross with kv_index, split", dtype)
    ql, kl, idx = [3, 30, 0, 1], [5, 3300], [1, 1, 0, 0]
    q = _randn(torch, 27, sum(ql), 4, 64, dtype=dtype)
    k, v = _randn(torch, 28, sum(kl), 2, 64, dtype=dtype), _randn(torch, 29, sum(kl), 2, 64, dtype=dtype)
    mask = torch.ones(sum(kl), dtype=torch.bool)
    mask[400:2000] = False                        # whole parts see nothing
    for m in (None, mask):
        got = C.cross_attention(q, k, v, ql, kl, kv_index=idx, key_mask=None if m is None else m.cuda())
        ref = O.cross(_f64(q), _f64(k), _f64(v), ql, kl, idx, key_mask=None if m is None else m.numpy())
        _compare(got, *ref, max(kl), 64, dtype)


# ---- the cache ----------------------------------------------------------------------------------


def _tables(torch, lens, width, n_blocks, seed=0):
    """Disjoint rows of block numbers in a shuffled order."""
    nb = [(x + 31) // 32 for x in lens]
    order = np.random.default_rng(seed).permutation(n_blocks)
    t = np.zeros((len(lens), width), np.int32)
    at = 0
    for i, n in enumerate(nb):
        t[i, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(t).cuda()


def _i32(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _fill(torch, C, lens, h, d, dtype="bf16", seed=30, spread=True, width=None, spare=3):
    """A cache filled in one append per sequence set -> (cache, table, lens tensor, k, v rows)."""
    nb = sum((x + 31) // 32 for x in lens)
    width = max((max(lens) + 31) // 32, 1) if width is None else width
    cache = C.kv8_cache(nb + spare, h, d)
    table = _tables(torch, lens, width, nb + spare, seed)
    k = _randn(torch, seed + 1, sum(lens), h, d, dtype=dtype)
    v = _randn(torch, seed + 2, sum(lens), h, d, dtype=dtype)
    if spread:                                    # blocks and heads of unlike magnitude
        f = 2.0 ** torch.randint(-9, 9, (sum(lens), h, 1), generator=torch.Generator().manual_seed(seed + 3)).cuda()
        v = (v * f).to(v.dtype)
    kv = _i32(torch, lens)
    C.kv8_append(cache, table, kv, k, v, lens)
    return cache, table, kv, k, v


def _held(torch, cache, table, lens):
    """The cached values by the documented layout: per sequence (k, v) [len, H, d] float64."""
    k, v = O.block_values(*(t.cpu().numpy() for t in cache))
    t = table.cpu().numpy()
    out = []
    for i, n in enumerate(lens):
        b = t[i, :(n + 31) // 32]
        out.append((k[b].reshape(-1, *k.shape[2:])[:n], v[b].reshape(-1, *v.shape[2:])[:n]))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("steps", [
    [[1, 32, 33, 0, 100]],                                       # whole sequences at once
    [[5, 31, 32, 1, 0], [1, 1, 1, 1, 1], [40, 0, 31, 64, 3]],    # continued at every kind of place
    [[1, 1, 1, 1, 1]] * 40,                                      # token by token
])
def test_kv8_append_and_read(torch, C, steps, d, dtype):
    """Codes and scales exactly as defined, whatever the steps; values of a block grow and shrink by
    powers of two so that scales rise in the middle of blocks; blocks that no step touches and the
    spare ones keep their bytes."""
    _say(f"append {len(steps)} steps of {steps[0]}, d {d}, {dtype}")
    h, n = 3, len(steps[0])
    final = [sum(s[i] for s in steps) for i in range(n)]
    width = (max(final) + 31) // 32 + 1
    n_blocks = sum((x + 31) // 32 for x in final) + 4
    cache = C.KV8Cache(torch.full((n_blocks, h, d // 16, 32, 16), 0x55, dtype=torch.uint8, device="cuda"),
                       torch.full((n_blocks, h, d, 32), 0x55, dtype=torch.uint8, device="cuda"),
                       torch.full((n_blocks, h, 2), 3.0, device="cuda"))
    table = _tables(torch, final, width, n_blocks, 40)
    refs = [(O.Cache(h, d), O.Cache(h, d)) for _ in range(n)]
    lens = [0] * n
    g = torch.Generator().manual_seed(41)
    for step, new in enumerate(steps):
        lens = [a + b for a, b in zip(lens, new)]
        rows = []
        for t in range(2):
            x = torch.randn(sum(new), h, d, generator=g) * 2.0 ** torch.randint(-12, 12, (sum(new), h, 1), generator=g)
            x = x.to(_dt(torch, dtype))
            if t == 1 and step == 0:
                x[0] = 0                          # a block that opens with zeros
            rows.append(x)
        C.kv8_append(cache, table, _i32(torch, lens), rows[0].cuda(), rows[1].cuda(), new)
        at = 0
        for i, m in enumerate(new):
            for t in range(2):
                refs[i][t].append(_f64(rows[t][at:at + m]))
            at += m
    for i, (k, v) in enumerate(_held(torch, cache, table, lens)):
        np.testing.assert_array_equal(k, refs[i][0].values())
        np.testing.assert_array_equal(v, refs[i][1].values())
    kv = _i32(torch, lens)
    for out_dtype in ("bf16", "f32"):
        for counts in (lens, [min(x, 33) for x in lens], [min(x, 1) for x in lens]):
            k, v = C.kv8_read(cache, table, kv, counts, dtype=_dt(torch, out_dtype))
            for t, got in enumerate((k, v)):
                want = np.concatenate([r[t].values()[len_ - c:] for r, len_, c in zip(refs, lens, counts)])
                np.testing.assert_array_equal(_f64(got), want)
    # past the length a touched block holds zeros, all others what they held
    used = {int(b) for i, x in enumerate(lens) for b in table[i, :(x + 31) // 32]}
    spare = [b for b in range(n_blocks) if b not in used]
    assert spare and bool((cache.k_codes[spare] == 0x55).all()) and bool((cache.v_codes[spare] == 0x55).all())
    assert bool((cache.scales[spare] == 3.0).all())
    for i, x in enumerate(lens):
        if x % 32:
            b = int(table[i, x // 32])
            assert not bool(cache.k_codes[b, :, :, x % 32:].any())
            place = [p for p, tok in enumerate(O.V_ORDER) if tok >= x % 32]
            assert not bool(cache.v_codes[b][..., place].any())


def test_kv8_append_every_value(torch, C):
    """Codes over the whole range: every bf16 magnitude of a block's eleven binades and below, ties
    and the edges of the format among them; infinities saturate, NaN stays; zero blocks."""
    _say("append, every value")
    h, d = 1, 128
    bits = torch.arange(0, 1 << 16, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    x = x[torch.isfinite(x)]
    x = x[(x.abs() <= 448) & (x.abs() >= 2.0 ** -14)]
    n = (x.numel() // d) // 32 * 32
    x = x[:n * d].reshape(n, 1, d).clone()
    x[::32, :, 0] = 448.0                          # every block at scale 1
    cache = C.kv8_cache(n // 32, h, d)
    table = torch.arange(n // 32, dtype=torch.int32, device="cuda")[None]
    kv = _i32(torch, [n])
    C.kv8_append(cache, table, kv, x.to(torch.bfloat16).cuda(), x.to(torch.bfloat16).cuda(), [n])
    from oracle import e4m3 as Q
    want = Q.decode_table()[Q.encode(_f64(x)).astype(int)]
    k, v = C.kv8_read(cache, table, kv, [n], dtype=torch.float32)
    np.testing.assert_array_equal(_f64(k), want)
    np.testing.assert_array_equal(_f64(v), want)
    assert bool((cache.scales == 1.0).all())
    # infinities, NaN, the largest and the smallest values, zeros
    rows = torch.zeros(5 * 32, 1, d)
    rows[0, 0, 0], rows[1, 0, 1] = float("inf"), -1.0
    rows[32, 0, 3], rows[33, 0, 4] = float("nan"), 5.0
    rows[64, 0, 0] = 3.3e38
    rows[96, 0, 7] = 2.0 ** -133
    cache = C.kv8_cache(5, h, d)
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    C.kv8_append(cache, table, _i32(torch, [160]), rows.cuda(), rows.cuda(), [160])
    k, v = C.kv8_read(cache, table, _i32(torch, [160]), [160], dtype=torch.float32)
    for t, got in enumerate((k, v)):
        ref = O.Cache(h, d)
        ref.append(_f64(rows))
        np.testing.assert_array_equal(_f64(got), ref.values())
        assert cache.scales[:, 0, t].tolist() == [2.0 ** 120, 2.0 ** -6, 2.0 ** 120, 2.0 ** -126, 2.0 ** -126]


def test_kv8_append_refuses_on_the_device(torch, C):
    """Lengths that do not fit (below the new rows, past the table) and block numbers that are none
    write nothing; reads give zeros there."""
    _say("append, bad lengths and blocks")
    h, d = 2, 64
    cache = C.kv8_cache(4, h, d)
    k = _randn(torch, 50, 40, h, d)
    table = _i32(torch, [[0, 1], [2, 3]])
    for lens in ([-5, 10], [19, 65], [-2**31, 2**31 - 1]):
        C.kv8_append(cache, table, _i32(torch, lens), k, k, [20, 20])
        torch.cuda.synchronize()
        assert bool(cache.k_codes.any()) == (lens == [-9, 10])
        assert not bool(cache.k_codes[:2].any())
        cache.k_codes.zero_(), cache.v_codes.zero_()
    bad = _i32(torch, [[-1, 1], [4, 2**31 - 1]])
    C.kv8_append(cache, bad, _i32(torch, [40, 40]), torch.cat([k, k]), torch.cat([k, k]), [40, 40])
    rk, rv = C.kv8_read(cache, bad, _i32(torch, [40, 40]), [40, 40])
    assert not bool(rk[:32].any()) and not bool(rv[40:].any()) and bool(rk[32:40].any())
    assert not bool(cache.k_codes[[0, 2, 3]].any())
    rk, _ = C.kv8_read(cache, bad, _i32(torch, [-7, 2**31 - 1]), [5, 5])
    assert not bool(rk.any())


CACHED = [
    # q_lens, kv_lens, Hq, Hkv, d
    ([1], [1], 16, 8, 128), ([1], [31], 4, 2, 64), ([1, 1, 1], [32, 33, 700], 16, 8, 128),
    ([1, 0, 2, 4], [100, 5, 64, 257], 8, 1, 128),
    ([3], [5000], 2, 2, 64),                       # split and joined
    ([1, 1], [4000, 7], 16, 8, 128),
    ([40, 64], [40, 90], 4, 2, 64), ([65, 128, 129], [65, 300, 129], 2, 2, 128),
    ([100, 1, 33, 1], [320, 96, 33, 2000], 12, 4, 64),   # both kernels in one call
    ([20], [3000], 4, 2, 128),                     # rows past one tile, keys split
    ([16], [40], 8, 4, 64), ([17], [40], 8, 4, 64),
    # enough rows for the tiles of 128: over tables that fit LDS, of each width, and that do not
    ([600, 1, 90], [320, 96, 77], 16, 8, 128), ([1030, 70], [128, 500], 16, 8, 128), ([700, 33], [640, 31], 8, 8, 64),
    ([410, 40], [96, 40], 10, 10, 64), ([900, 65], [900, 700], 12, 4, 64), ([300, 170], [1500, 200], 16, 16, 128),
    ([40, 3], [50, 700], 66, 2, 64),               # 33 heads: one token is more than 32 rows
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,kl,hq,hkv,d", CACHED)
def test_kv8_attention(torch, C, ql, kl, hq, hkv, d, causal, dtype):
    _say(f"cached {ql} x {kl}, heads {hq}/{hkv} of {d}, causal {causal}, {dtype}")
    cache, table, kv, _, _ = _fill(torch, C, kl, hkv, d)
    q = _randn(torch, 60, sum(ql), hq, d, std=1.5, dtype=dtype)
    got = C.kv8_attention(q, cache, table, kv, ql, causal=causal)
    held = _held(torch, cache, table, kl)
    parts, at = [], 0
    for (k, v), n, m in zip(held, ql, kl):
        see = np.arange(m)[None] <= m - n + np.arange(n)[:, None] if causal else np.ones((n, m), bool)
        parts.append(O.attend(_f64(q[at:at + n]), k, v, see, 1 / np.sqrt(d)))
        at += n
    ref = [np.concatenate([p[x] for p in parts]) for x in range(3)]
    vmax = max(np.abs(v).max() for _, v in held)
    _compare(got, *ref, max(kl), d, dtype, vmax)
    assert torch.equal(got, C.kv8_attention(q, cache, table, kv, ql, causal=causal))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql", [[2, 3, 1], [60, 70, 50]])
def test_kv8_attention_on_the_device(torch, C, ql, dtype):
    """Lengths and block numbers that only the device sees: a length of zero, below zero and past the
    table, blocks that are none in the middle and at the end, causal rows before the first token.
    Blocks never written hold NaN codes."""
    _say("cached, device-side lengths and blocks", ql, dtype)
    h, d, kl = 2, 64, [100, 130, 40]
    cache, table, kv, _, _ = _fill(torch, C, kl, h, d, width=6)
    used = {int(b) for i, x in enumerate(kl) for b in table[i, :(x + 31) // 32]}
    free = [b for b in range(cache.k_codes.shape[0]) if b not in used]
    cache.k_codes[free], cache.v_codes[free] = 0x7F, 0xFF
    q = _randn(torch, 61, sum(ql), 4, d, dtype=dtype)
    table = table.clone()
    table[1, 1], table[1, 4] = -3, cache.k_codes.shape[0]
    held = _held(torch, cache, _i32(torch, table.clamp(0, cache.k_codes.shape[0] - 1).tolist()), kl)
    for causal in (False, True):
        for lens in ([100, 130, 0], [100, 130, -7], [1, 1000, 40]):
            eff = [min(max(x, 0), 6 * 32) for x in lens]
            if eff[1] == 192:                      # past the table: its last block is none either
                table[1, 5] = 2**31 - 1
            got = C.kv8_attention(q, cache, table, _i32(torch, lens), ql, causal=causal)
            parts, at = [], 0
            for i, (n, m) in enumerate(zip(ql, eff)):
                k, v = (np.zeros((m, h, d)) for _ in range(2))
                have = min(m, kl[i])
                k[:have], v[:have] = held[i][0][:have], held[i][1][:have]
                see = np.arange(m)[None] <= m - n + np.arange(n)[:, None] if causal else np.ones((n, m), bool)
                if i == 1:
                    see = see.copy()
                    see[:, 32:64] = False
                    see[:, 128:] = False
                parts.append(O.attend(_f64(q[at:at + n]), k, v, see, 1 / np.sqrt(d)))
                at += n
            ref = [np.concatenate([p[x] for p in parts]) for x in range(3)]
            _compare(got, *ref, 192, d, dtype, max(np.abs(v).max() for _, v in held))


def test_kv8_shared_blocks_and_narrow_table(torch, C):
    """Two sequences over the same blocks, a table that is a view of a wider one, queries inside a
    wider buffer, a caller's out."""
    _say("cached, shared blocks")
    cache, table, kv, _, _ = _fill(torch, C, [90], 2, 64)
    wide = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, :3] = table
    lens = _i32(torch, [90, 90, 33])
    q = _randn(torch, 62, 60, 4, 64)
    alone = [C.kv8_attention(q[i * 20:(i + 1) * 20], cache, wide[:1, :3], lens[i:i + 1], [20]) for i in range(3)]
    box = torch.zeros((60, 4, 80), dtype=q.dtype, device="cuda")
    box[..., :64] = q
    out = torch.full((60, 4, 72), 5.0, dtype=q.dtype, device="cuda")
    got = C.kv8_attention(box[..., :64], cache, wide[:, :3], lens, [20] * 3, out=out[..., :64])
    assert torch.equal(got, torch.cat(alone)) and bool((out[..., 64:] == 5.0).all())


def test_kv8_offsets_past_32_bits(torch, C):
    """Blocks behind the first 4 GiB of codes."""
    _say("cached, a cache of 2 x 4.3 GB")
    h, d, nb = 8, 128, 131072 + 64
    cache = C.KV8Cache(torch.empty((nb, h, d // 16, 32, 16), dtype=torch.uint8, device="cuda"),
                       torch.empty((nb, h, d, 32), dtype=torch.uint8, device="cuda"),
                       torch.empty((nb, h, 2), device="cuda"))
    small = C.kv8_cache(3, h, d)
    k, v = _randn(torch, 63, 80, h, d), _randn(torch, 64, 80, h, d)
    far, near = _i32(torch, [[nb - 1, 131072, nb - 2]]), _i32(torch, [[0, 1, 2]])
    kv = _i32(torch, [80])
    for q_len in (2, 70):
        q = _randn(torch, 65, q_len, 16, d)
        res = []
        for c, t in ((cache, far), (small, near)):
            C.kv8_append(c, t, kv, k, v, [80])
            res.append((*C.kv8_read(c, t, kv, [80]), C.kv8_attention(q, c, t, kv, [q_len], causal=True)))
        assert all(torch.equal(a, b) for a, b in zip(*res))


def test_kv8_many_sequences(torch, C):
    _say("cached, 200 sequences")
    rng = np.random.default_rng(66)
    kl = [int(x) for x in rng.integers(0, 60, 200)]
    ql = [int(x) for x in rng.integers(0, 4, 200)]
    cache, table, kv, _, _ = _fill(torch, C, kl, 2, 64, spread=False)
    q = _randn(torch, 67, sum(ql), 2, 64)
    got = C.kv8_attention(q, cache, table, kv, ql)
    parts, at = [], 0
    for (k, v), n in zip(_held(torch, cache, table, kl), ql):
        parts.append(O.attend(_f64(q[at:at + n]), k, v, np.ones((n, k.shape[0]), bool), 1 / 8))
        at += n
    _compare(got, *(np.concatenate([p[x] for p in parts]) for x in range(3)), 60, 64, "bf16", 8.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl,width,hq,h", [(16, 40, None, 4, 2), (64, 64, None, 4, 2), (64, 64, 30, 4, 2),
                                              (300, 310, None, 32, 4), (300, 310, 40, 32, 4)])
def test_kv8_values_of_unseen_blocks(torch, C, ql, kl, width, hq, h, dtype):
    """A causal row's result does not depend on how large the values are that it does not see."""
    _say("cached, values of unseen blocks", ql, kl, width, dtype)
    d = 64
    v = torch.randn(kl, h, d, generator=torch.Generator().manual_seed(93))
    v[32:] *= 2.0 ** 40
    cache, table, kv, _, _ = _fill(torch, C, [kl], h, d, width=width)
    k = _randn(torch, 94, kl, h, d)
    C.kv8_append(cache, table, kv, k, v.to(torch.bfloat16).cuda(), [kl])
    q = _randn(torch, 95, ql, hq, d, dtype=dtype)
    got = C.kv8_attention(q, cache, table, kv, [ql], causal=True)
    (kk, vv), = _held(torch, cache, table, [kl])
    see = np.arange(kl)[None] <= kl - ql + np.arange(ql)[:, None]
    ref = O.attend(_f64(q), kk, vv, see, 1 / 8)
    edge = 32 - (kl - ql)                         # rows before it see the first block only
    for part, m in ((slice(0, edge), 32), (slice(edge, ql), kl)):
        _compare(got[part], *(x[part] for x in ref), m, d, dtype, np.abs(vv[:m]).max())


@pytest.mark.parametrize("ql,kl", [([1], [4000]), ([40], [3000]), ([40], [64])])
def test_kv8_smallest_keys(torch, C, ql, kl):
    """Keys at the smallest scale under queries that make up for it."""
    _say("cached, smallest keys", ql, kl)
    h, d = 2, 64
    cache = C.kv8_cache((kl[0] + 31) // 32, h, d)
    table = torch.arange(cache.scales.shape[0], dtype=torch.int32, device="cuda")[None]
    k, v = _randn(torch, 96, kl[0], h, d, dtype="f32") * 2.0 ** -126, _randn(torch, 97, kl[0], h, d, dtype="f32")
    kv = _i32(torch, kl)
    C.kv8_append(cache, table, kv, k, v, kl)
    assert bool((cache.scales[..., 0] == 2.0 ** -126).all())
    q = _randn(torch, 98, sum(ql), 4, d, dtype="f32") * 2.0 ** 120
    got = C.kv8_attention(q, cache, table, kv, ql)
    (kk, vv), = _held(torch, cache, table, kl)
    ref = O.attend(_f64(q), kk, vv, np.ones((ql[0], kl[0]), bool), 1 / 8)
    # what scores are multiplied by, 1.44 * 2^-129, is subnormal: off by 2^-150 at most, 2^-21.5 of itself,
    # less than 6 u more
    _compare(got, *ref, kl[0], d + 6, "f32", np.abs(vv).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ql,kl", [([1], [4000]), ([40], [3000]), ([40], [64])])
def test_kv8_largest_values(torch, C, ql, kl, dtype):
    """Values next to fp32's largest: sums are kept in units of the scale, partial results as means."""
    _say("cached, largest values", ql, kl, dtype)
    h, d = 2, 64
    cache = C.kv8_cache((kl[0] + 31) // 32, h, d)
    table = torch.arange(cache.scales.shape[0], dtype=torch.int32, device="cuda")[None]
    g = torch.Generator().manual_seed(90)
    v = (torch.rand(kl[0], h, d, generator=g) * 2.9e38).cuda()
    k = _randn(torch, 91, kl[0], h, d, dtype="f32")
    kv = _i32(torch, kl)
    C.kv8_append(cache, table, kv, k, v, kl)
    q = _randn(torch, 92, sum(ql), 4, d, dtype=dtype)
    got = C.kv8_attention(q, cache, table, kv, ql)
    (kk, vv), = _held(torch, cache, table, kl)
    ref = O.attend(_f64(q), kk, vv, np.ones((ql[0], kl[0]), bool), 1 / 8)
    _compare(got, *ref, kl[0], d, dtype, np.abs(vv).max())


@pytest.mark.parametrize("causal", [False, True])
def test_kv8_many_sequences_cut(torch, C, causal):
    """More sequences than one launch takes, long ones among them, each cut into its own number of parts;
    lengths that change under the same call."""
    _say("cached, 150 sequences, long ones cut", causal)
    rng = np.random.default_rng(68)
    kl = [int(x) for x in rng.integers(0, 50, 150)]
    kl[3], kl[40], kl[127], kl[128], kl[149] = 2000, 700, 900, 1100, 33
    ql = [int(x) for x in rng.integers(0, 3, 150)]
    ql[3], ql[40], ql[127], ql[128] = 1, 2, 1, 2
    cache, table, _, _, _ = _fill(torch, C, kl, 2, 64, spread=False)
    q = _randn(torch, 69, sum(ql), 4, 64)
    held = _held(torch, cache, table, kl)
    for lens in (kl, [x // 2 for x in kl], [x if i == 128 else min(x, 1) for i, x in enumerate(kl)]):
        got = C.kv8_attention(q, cache, table, _i32(torch, lens), ql, causal=causal)
        parts, at = [], 0
        for (k, v), n, m in zip(held, ql, lens):
            see = np.arange(m)[None] <= m - n + np.arange(n)[:, None] if causal else np.ones((n, m), bool)
            parts.append(O.attend(_f64(q[at:at + n]), k[:m], v[:m], see, 1 / 8))
            at += n
        _compare(got, *(np.concatenate([p[x] for p in parts]) for x in range(3)), 2000, 64, "bf16",
                 max(np.abs(v).max() for _, v in held if v.size))


# ---- group norm ---------------------------------------------------------------------------------
#
# Sums: a thread adds up to 32 values, LDS runs and trees at most ~90 more, parts are joined once:
# K = 128 roundings bound every sum. mean: K u mean|x| =: e; variance: 2 (K + 4) u of itself and e^2;
# so (x - mean) rstd is off by rstd (e + u |x - mean|) + |z0| (K + 8) u, then two steps of the
# affine part, at most 1.1 times that through SiLU (its slope) and 2^-20 of its own (exp2, rcp).

NORMS = [
    # n, (h, w), channels, groups
    (1, (1, 1), 32, 32), (1, (1, 1), 64, 8), (2, (8, 8), 1280, 32), (1, (8, 8), 320, 32), (3, (5, 7), 30, 3),
    (2, (16, 16), 640, 32), (1, (64, 64), 320, 32), (2, (33, 31), 96, 32), (1, (64, 65), 33, 11),
    (1, (40, 40), 2560, 32), (1, (3, 3), 5120, 1), (2, (17, 1), 9000, 2), (1, (100, 100), 64, 1), (1, (64, 64), 5, 5),
    (4, (2, 3), 24, 4), (1, (128, 64), 32, 8),
    # a full slab and sums per channel: together more than a workgroup's LDS
    (8, (40, 40), 320, 32), (4, (40, 40), 96, 8),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hw,c,groups", NORMS)
def test_group_norm(torch, C, n, hw, c, groups, dtype):
    _say(f"group norm {n} x {hw} x {c} / {groups} {dtype}")
    g = torch.Generator().manual_seed(70)
    x = torch.randn(n, *hw, c, generator=g) * torch.exp(torch.randn(c, generator=g)) + 4 * torch.randn(c, generator=g)
    x = x.to(_dt(torch, dtype)).cuda()
    gamma, beta = 1 + _randn(torch, 71, c, std=0.2, dtype=dtype), _randn(torch, 72, c, std=0.3, dtype=dtype)
    for affine in (True, False):
        for act in (None, "silu"):
            a = (gamma, beta) if affine else (None, None)
            got = C.group_norm(x, groups, *a, eps=1e-5, act=act)
            _check_norm(torch, got, x.reshape(n, -1, c), groups, *a, 1e-5, act, dtype)
            assert torch.equal(got, C.group_norm(x, groups, *a, eps=1e-5, act=act))


def _check_norm(torch, got, x, groups, gamma, beta, eps, act, dtype):
    ga, be = (None, None) if gamma is None else (_f64(gamma), _f64(beta))
    ref, z, rstd, mabs = O.group_norm(_f64(x), groups, ga, be, eps, act == "silu")
    K = 128
    ga, be = (1.0, 0.0) if ga is None else (np.abs(ga), np.abs(be))
    z0 = (np.abs(z) + be)                         # |gamma (x - mean) rstd| at most
    t = ga * rstd * (K * U * mabs) + z0 * (K + 12) * U + 2 * U * (np.abs(z) + be)
    t = 1.1 * t + 2.0 ** -20 * np.abs(ref) + 2.0 ** -22 if act else t
    t = t + (U16 if dtype == "bf16" else U) * (np.abs(ref) + t) + 1e-30
    g = _f64(got).reshape(ref.shape)
    assert np.isfinite(g).all()
    worst = float((np.abs(g - ref) / t).max())
    _say(f"  worst error / bound {worst:.3f}")
    assert worst <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hw", [(4, 4), (64, 64)])
def test_group_norm_layouts(torch, C, hw, dtype):
    """Slices of wider buffers at any alignment, a channels_last NCHW tensor, in place, a caller's out
    whose surroundings stay as they were."""
    _say("group norm layouts", hw, dtype)
    n, c, groups = 2, 64, 8
    x = _randn(torch, 73, n, *hw, c, dtype=dtype)
    plain = C.group_norm(x, groups, act="silu")
    for off, extra in ((8, 16), (1, 3), (2, 6), (4, 4)):
        box = torch.zeros((n, *hw, c + extra), dtype=x.dtype, device="cuda")
        view = box[..., off:off + c] if off + c <= c + extra else box[..., :c]
        view.copy_(x)
        out = torch.full((n, *hw, c + extra), 9.0, dtype=x.dtype, device="cuda")
        got = C.group_norm(view, groups, act="silu", out=out[..., :c])
        _check_norm(torch, got.contiguous(), x.reshape(n, -1, c), groups, None, None, 1e-5, "silu", dtype)
        assert bool((out[..., c:] == 9.0).all())
    nchw = x.permute(0, 3, 1, 2)                  # channels_last in memory
    assert torch.equal(plain, C.group_norm(nchw.permute(0, 2, 3, 1), groups, act="silu"))
    y = x.clone()
    assert C.group_norm(y, groups, act="silu", out=y) is y and torch.equal(y, plain)


def test_group_norm_large_mean(torch, C):
    """A mean 10^4 times the spread, and one outlier in the first place: squares around the mean, not
    a difference of sums."""
    _say("group norm, large mean")
    x = _randn(torch, 74, 1, 4096, 32, dtype="f32")
    x[0, 0] = 100.0
    x = x + 10000.0
    got = C.group_norm(x, 4)
    _check_norm(torch, got, x, 4, None, None, 1e-5, None, "f32")


def test_group_norm_empty(torch, C):
    assert C.group_norm(torch.empty((0, 4, 32), device="cuda"), 4).shape == (0, 4, 32)
    assert C.group_norm(torch.empty((2, 0, 32), device="cuda"), 4).shape == (2, 0, 32)
