"""The operators that read the conditioning as a denoiser uses them: a group norm of latents and cross
attention to what the encoder returned, directly and over the 8-bit cache that keeps it across calls;
captured and replayed while the cache grows, on several streams, and what the wrappers turn down."""
import sys

import numpy as np
import pytest

from oracle import cond_oracle as O
from synth import workloads as W
from tests.gpu_common import layout_tuples, make_encoder
from tests.test_gpu_cond import _compare, _f64, _held, _i32, _randn, _tables

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


def test_denoiser_reads_the_encoder(torch, C):
    """Two frames through the tiny encoder; their states are projected to keys and values, read by
    normalised latents of 8x8 each, and again, from the cache, in a second call that does not encode
    (TECache with refresh_every = 2)."""
    from paper_2606_05981_amd.encoder import TECache, build_positions
    wl = W.workload("tiny_fp32")
    d = wl.dims
    enc = make_encoder(d, max_tokens=256, max_batch=8, max_seq=128)
    emb = torch.from_numpy(W.embeddings(d, wl.layouts)).cuda()
    lens = W.seq_lens(wl.layouts)
    n = len(lens)
    _say(f"denoiser path: {n} frames of {lens} tokens")
    pos = build_positions(layout_tuples(wl.layouts))
    te = TECache(enc, refresh_every=2)
    hq, hkv, hd, ch = 4, 2, 64, 256
    w_q = _randn(torch, 100, ch, hq * hd, std=ch ** -0.5, dtype="f32")
    w_kv = _randn(torch, 101, d.hidden, 2 * hkv * hd, std=d.hidden ** -0.5, dtype="f32")
    gamma, beta = 1 + _randn(torch, 102, ch, std=0.1, dtype="f32"), _randn(torch, 103, ch, std=0.1, dtype="f32")
    cache = C.kv8_cache(sum((x + 31) // 32 for x in lens) + 1, hkv, hd)
    table = _tables(torch, lens, max((x + 31) // 32 for x in lens), cache.k_codes.shape[0], 104)
    kv = _i32(torch, lens)
    ql = [64] * n
    held = None
    for call in range(2):
        latents = _randn(torch, 105 + call, n, 8, 8, ch, std=2.0, dtype="f32")
        hidden = te(emb, pos, lens)
        x = C.group_norm(latents, 32, gamma, beta, eps=1e-6)
        ref, _, _, _ = O.group_norm(_f64(latents).reshape(n, 64, ch), 32, _f64(gamma), _f64(beta), 1e-6)
        assert np.abs(_f64(x).reshape(ref.shape) - ref).max() <= 1e-5   # 128 roundings of 2^-24 at |z| < 6
        q = torch.matmul(x.reshape(-1, ch), w_q).reshape(-1, hq, hd)
        both = torch.matmul(hidden, w_kv).reshape(-1, 2, hkv, hd)
        if call == 0:
            C.kv8_append(cache, table, kv, both[:, 0], both[:, 1], lens)
            held = _held(torch, cache, table, lens)
        direct = C.cross_attention(q, both[:, 0], both[:, 1], ql, lens)
        _compare(direct, *O.cross(_f64(q), _f64(both[:, 0]), _f64(both[:, 1]), ql, lens), max(lens), hd, "f32")
        cached = C.kv8_attention(q, cache, table, kv, ql)
        parts = [O.attend(_f64(q[64 * i:64 * i + 64]), k, v, np.ones((64, k.shape[0]), bool), hd ** -0.5)
                 for i, (k, v) in enumerate(held)]
        _compare(cached, *(np.concatenate([p[j] for p in parts]) for j in range(3)), max(lens), hd, "f32",
                 max(np.abs(v).max() for _, v in held))
    assert te.encodes == 1
    # one frame's conditioning for all, as batch_one hands it on
    one = C.cross_attention(q, both[:lens[0], 0], both[:lens[0], 1], ql, lens[:1], kv_index=[0] * n)
    shared = C.kv8_attention(q, cache, table[:1].expand(n, -1), kv[:1].repeat(n), ql)
    assert torch.equal(one[:64], direct[:64]) and torch.equal(shared[:64], cached[:64])
    enc.close()


def test_cached_step_captured_while_the_cache_grows(torch, C):
    """A step (lengths up by one, append, attend) captured once and replayed: every replay equals the
    same step run eagerly on a second cache, through block ends and with other work in between."""
    _say("captured step")
    h, hq, d, n, steps = 4, 8, 128, 3, 40
    start = [1, 30, 300]
    width = (max(start) + steps + 31) // 32
    blocks = n * width
    a, b = C.kv8_cache(blocks, h, d), C.kv8_cache(blocks, h, d)
    table = _i32(torch, np.random.default_rng(110).permutation(blocks).reshape(n, width).tolist())
    k0, v0 = _randn(torch, 111, sum(start), h, d), _randn(torch, 112, sum(start), h, d)
    for c in (a, b):
        C.kv8_append(c, table, _i32(torch, start), k0, v0, start)
    lens_a, lens_b = _i32(torch, start), _i32(torch, start)
    k, v, q = (torch.zeros((n, x, d), dtype=torch.bfloat16, device="cuda") for x in (h, h, hq))

    def step(c, lens):
        lens.add_(1)
        C.kv8_append(c, table, lens, k, v, [1] * n)
        return C.kv8_attention(q, c, table, lens, [1] * n, causal=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                  # warm up on copies
        step(C.KV8Cache(*(t.clone() for t in a)), lens_a.clone())
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(a, lens_a)
    for s in range(steps):
        for t, seed in ((k, 200), (v, 300), (q, 400)):
            t.copy_(_randn(torch, seed + s, *t.shape, std=1.0 + (s % 5)))
        g.replay()
        ref = step(b, lens_b)
        assert torch.equal(out, ref), s
        assert torch.equal(lens_a, lens_b)
        torch.mm(torch.randn(64, 64, device="cuda"), torch.randn(64, 64, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_reads(torch, C):
    """Cross attention (split and whole), attention over the cache and group norm (one launch and two) in
    one graph, replayed over new inputs."""
    _say("captured reads")
    d = 64
    q = _randn(torch, 120, 300, 4, d)
    k, v = _randn(torch, 121, 2600, 2, d), _randn(torch, 122, 2600, 2, d)
    x, small = _randn(torch, 123, 2, 64, 64, 64), _randn(torch, 124, 2, 4, 4, 64)
    cache = C.kv8_cache(4, 2, d)
    table, kv = _i32(torch, [[3, 0, 2]]), _i32(torch, [90])
    C.kv8_append(cache, table, kv, k[:90], v[:90], [90])

    def run():
        return (C.cross_attention(q[:3], k, v, [3], [2600]), C.cross_attention(q, k[:100], v[:100], [300], [100]),
                C.kv8_attention(q, cache, table, kv, [300]), C.group_norm(x, 8, act="silu"), C.group_norm(small, 8))
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for s in range(3):
        q.copy_(_randn(torch, 130 + s, *q.shape))
        x.copy_(_randn(torch, 140 + s, *x.shape))
        small.copy_(_randn(torch, 150 + s, *small.shape))
        g.replay()
        for a, b in zip(got, run()):
            assert torch.equal(a, b), s


def test_two_graphs(torch, C):
    """Two captured graphs of split calls and a two-launch norm, replayed in turn and on two streams at
    once: their workspaces are their own."""
    _say("two graphs")
    xs = [_randn(torch, 200 + i, 3, 4, 64) for i in range(2)]
    k, v = _randn(torch, 202, 4000, 2, 64), _randn(torch, 203, 4000, 2, 64)
    im = [_randn(torch, 204 + i, 2, 64, 64, 64) for i in range(2)]
    cache = C.kv8_cache(125, 2, 64)
    table, kv = torch.arange(125, dtype=torch.int32, device="cuda")[None], _i32(torch, [4000])
    C.kv8_append(cache, table, kv, k, v, [4000])

    def run(i):
        return (C.cross_attention(xs[i], k, v, [3], [4000]), C.kv8_attention(xs[i], cache, table, kv, [3], causal=True),
                C.group_norm(im[i], 8, act="silu"))
    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, got = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(run(i))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for both in (False, True, True, False):
        for i in (0, 1):
            for t in got[i]:
                t.zero_()
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.stream(streams[i] if both else torch.cuda.current_stream()):
                for _ in range(3):
                    graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i])), (both, i)


def test_streams(torch, C):
    """Calls on two streams at once, inputs of one stream read on another (ordered by the caller and
    dropped right after), and a stream handed over by argument."""
    _say("streams")
    qs = [_randn(torch, 160 + i, 3, 16, 128) for i in range(2)]
    ks = [_randn(torch, 170 + i, 9000, 8, 128) for i in range(2)]
    want = [C.cross_attention(qs[i], ks[i], ks[1 - i], [3], [9000]) for i in range(2)]
    xs = _randn(torch, 180, 4, 64, 64, 64)
    wx = C.group_norm(xs, 8)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append((C.cross_attention(qs[i], ks[i], ks[1 - i], [3], [9000]), C.group_norm(xs, 8)))
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for i in range(2):
            assert torch.equal(got[i][0], want[i]) and torch.equal(got[i][1], wx)
    s = streams[0]
    for _ in range(5):
        y = xs.clone()
        s.wait_stream(torch.cuda.current_stream())
        out = C.group_norm(y, 8, stream=s)
        del y
        junk = torch.full_like(xs, float("nan"))    # would take y's memory if it were free
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(out, wx)
        del junk


def test_wrappers_refuse(torch, C):
    """What would reach the kernels wrong raises before anything is enqueued."""
    from paper_2606_05981_amd.binding import MteError
    q, k = _randn(torch, 190, 8, 4, 64), _randn(torch, 191, 10, 2, 64)
    ok = dict(q=q, k=k, v=k, q_lens=[8], kv_lens=[10])
    C.cross_attention(**ok)
    buf = torch.zeros(8 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q.float()), dict(k=k.float()), dict(v=k[:9]), dict(v=k[:, :1]), dict(q=q[:, :, :32]),
                dict(q_lens=[7]), dict(kv_lens=[11]), dict(kv_lens=[5, 5]), dict(kv_index=[1]), dict(kv_index=[0, 0]),
                dict(q_lens=[9, -1]), dict(q=q.cpu()), dict(k=k.cpu()), dict(scale=0.0), dict(scale=float("nan")),
                dict(key_mask=torch.ones(9, dtype=torch.bool, device="cuda")),
                dict(key_mask=torch.ones(10, device="cuda")), dict(key_mask=torch.ones(10, dtype=torch.bool)),
                dict(q=buf[1:1 + 2048].view(8, 4, 64)),                     # not 16-byte aligned
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)),     # head_dim strided
                dict(out=torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda").expand(8, 4, 64)),
                dict(out=torch.empty(8, 4, 64, device="cuda")), dict(out=q[:7]),
                dict(q=_randn(torch, 192, 8, 3, 64))):                      # 3 query heads on 2
        with pytest.raises((ValueError, MteError)):
            C.cross_attention(**{**ok, **bad})
    cache = C.kv8_cache(4, 2, 64)
    table, kv = _i32(torch, [[0, 1]]), _i32(torch, [10])
    app = dict(cache=cache, table=table, kv_lens=kv, k=k, v=k, new_lens=[10])
    C.kv8_append(**app)
    att = dict(q=q, cache=cache, table=table, kv_lens=kv, q_lens=[8])
    C.kv8_attention(**att)
    for bad in (dict(table=table.long()), dict(table=table[0]), dict(table=_i32(torch, [[0, 1], [2, 3]])),
                dict(table=table.cpu()), dict(kv_lens=kv.long()), dict(kv_lens=_i32(torch, [1, 2])),
                dict(kv_lens=kv.cpu()), dict(cache=C.kv8_cache(4, 2, 128)), dict(cache=C.kv8_cache(4, 3, 64)),
                dict(cache=(cache[0], cache[1], cache[2].double())), dict(cache=(cache[0], cache[1][:3], cache[2])),
                dict(cache=(cache[1], cache[0], cache[2]))):
        with pytest.raises((ValueError, MteError)):
            C.kv8_attention(**{**att, **bad})
        with pytest.raises((ValueError, MteError)):
            C.kv8_append(**{**app, **bad})
    with pytest.raises(ValueError):
        C.kv8_read(cache, table, kv, [10], dtype=torch.float16)
    with pytest.raises(ValueError):
        C.kv8_read(cache, table, kv, [-1])
    x = _randn(torch, 193, 2, 4, 4, 64)
    C.group_norm(x, 8)
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(groups=7), dict(groups=0), dict(act="gelu"), dict(gamma=g.float()), dict(gamma=g[:32]),
                dict(beta=g.cpu()), dict(eps=-1.0), dict(x=x.half()), dict(x=x[0, 0]),
                dict(x=x.permute(0, 3, 1, 2).contiguous().permute(0, 2, 3, 1)),   # channels strided
                dict(x=x[:, :, :2]),                                              # pixels at two strides
                dict(out=x[:1]), dict(out=x.float()), dict(out=x[:, :1].expand(2, 4, 4, 64)),
                dict(stream=object())):
        with pytest.raises((ValueError, MteError, AttributeError)):
            C.group_norm(**{**dict(x=x, groups=8), **bad})


def test_sizes_past_31_bits_are_refused(torch, C):
    """Sizes that the C interface counts in 31 bits raise instead of wrapping round."""
    x = torch.zeros(1, 1, 8, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(x=x.expand(1, (1 << 32) + 1, 8), groups=1), dict(x=x.expand((1 << 32) + 1, 1, 8), groups=1),
                dict(x=x, groups=(1 << 32) + 1)):
        with pytest.raises(ValueError):
            C.group_norm(**bad)
    cache = [t.cpu() for t in C.kv8_cache(1, 2, 64)]
    with pytest.raises(ValueError):
        C.kv8_read(cache, torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32), [1])
