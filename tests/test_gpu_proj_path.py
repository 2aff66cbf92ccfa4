"""Projections, rotary positions and attention over a shared prefix as a denoiser uses them together: from
what the encoder returned to the attention that reads it, directly and through the 8-bit cache; captured
and replayed over new inputs, in two graphs, on several streams, and what the wrappers turn down."""
import sys

import numpy as np
import pytest

from oracle import proj_oracle as O
from synth import workloads as W
from tests.gpu_common import layout_tuples, make_encoder

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


@pytest.fixture(scope="module")
def P():
    from paper_2606_05981_amd import projections
    return projections


def _f64(t):
    return t.detach().double().cpu().numpy()


def _randn(torch, seed, *shape, std=1.0, dtype="bf16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def test_from_hidden_states_to_attention(torch, C, P):
    """Frames through the tiny encoder; their states become rotated keys and values by an 8-bit projection, latents
    become rotated queries, which attend to a shared instruction's tokens and to their frame's. Every step
    against the oracle of the step, given the step's own inputs: the bounds are those of the single operators."""
    from paper_2606_05981_amd.encoder import build_positions
    wl = W.workload("tiny_fp32")
    d = wl.dims
    enc = make_encoder(d, max_tokens=256, max_batch=8, max_seq=128)
    emb = torch.from_numpy(W.embeddings(d, wl.layouts)).cuda()
    lens = W.seq_lens(wl.layouts)
    pos = build_positions(layout_tuples(wl.layouts))
    hidden = enc.encode(emb, pos, lens)
    hq, hkv, hd, ch, n = 4, 2, 64, 250, len(lens)
    w_kv = P.quantize_rows(_randn(torch, 1, 2 * hkv * hd, d.hidden, std=d.hidden ** -0.5, dtype="f32"))
    w_q = P.quantize_rows(_randn(torch, 2, hq * hd, ch, std=ch ** -0.5, dtype="f32"))
    latents = _randn(torch, 3, n, 64, ch, std=2.0, dtype="f32")

    kv = P.i8_linear(hidden, w_kv).view(-1, 2, hkv, hd)
    q = P.i8_linear(latents, w_q).view(-1, hq, hd)
    for got, x, w in ((kv, hidden, w_kv), (q, latents, w_q)):
        x = _f64(x).reshape(-1, x.shape[-1])
        cols = w.cols
        y, z, p = O.i8_linear(*O.i8_rows(x), _f64(w.codes)[:, :cols], w.scales.cpu().numpy())
        assert (np.abs(_f64(got).reshape(y.shape) - y) <= 5 * U * np.abs(p) + 1e-40).all()

    freq, gain = P.rotary_frequencies(hd, 1e4, "yarn", 4.0, original_length=64)
    sec = (12, 10, 10)
    at = torch.arange(64, dtype=torch.int32, device="cuda")
    grid = torch.stack([torch.zeros_like(at), at // 8, at % 8]).repeat(1, n)
    before = kv.clone()
    qr, _ = P.rotary(q, grid, freq, sections=sec, factor=gain)
    P.rotary(kv[:, 0], pos, freq, sections=sec, factor=gain, out=(kv[:, 0], None))     # where they lie
    assert torch.equal(kv[:, 1], before[:, 1])
    for got, x, p in ((qr, q, grid), (kv[:, 0], before[:, 0], pos)):
        ref = O.rotary(_f64(x), p.cpu().numpy(), freq.cpu().numpy(), sections=sec, factor=gain)
        assert np.abs(_f64(got) - ref).max() <= 13 * U * gain * 2 * np.abs(_f64(x)).max()

    shared = _randn(torch, 4, 40, 2, hkv, hd, dtype="f32")
    ql = [64] * n
    o = C.prefix_attention(qr, shared[:, 0], shared[:, 1], kv[:, 0], kv[:, 1], ql, lens, causal=False)
    ref, mag, reach = O.prefix(*map(_f64, (qr, shared[:, 0], shared[:, 1], kv[:, 0], kv[:, 1])), ql, lens, False)
    D = (hd + 4) * U * reach[..., None] + 2 * U
    assert (np.abs(_f64(o) - ref) <= 4 * D * mag + 2 * (40 + max(lens) + 16) * U * mag + U * np.abs(ref) + 1e-30).all()
    enc.close()


def test_step_with_a_cache(torch, C, P):
    """One token of several streams: project, rotate, append, attend over the 8-bit cache, captured once and replayed while
    the streams grow; every replay equals the same step run eagerly on a second cache."""
    n, hq, hkv, hd, ch, steps = 5, 8, 2, 128, 320, 12
    w = P.quantize_rows(_randn(torch, 1, (hq + 2 * hkv) * hd, ch, std=ch ** -0.5))
    freq, _ = P.rotary_frequencies(hd, 5e6)
    a, b = C.kv8_cache(n * 2, hkv, hd), C.kv8_cache(n * 2, hkv, hd)
    table = torch.arange(2 * n, dtype=torch.int32, device="cuda").view(n, 2)
    x = torch.zeros((n, ch), dtype=torch.bfloat16, device="cuda")
    lens_a, lens_b = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))

    def step(cache, lens):
        at = lens.clone()
        lens.add_(1)
        h = P.i8_linear(x, w).view(n, hq + 2 * hkv, hd)
        P.rotary(h[:, :hq], at, freq, k=h[:, hq:hq + hkv], out=(h[:, :hq], h[:, hq:hq + hkv]))
        C.kv8_append(cache, table, lens, h[:, hq:hq + hkv], h[:, hq + hkv:], [1] * n)
        return C.kv8_attention(h[:, :hq], cache, table, lens, [1] * n, causal=True)

    step(C.KV8Cache(*(t.clone() for t in a)), lens_a.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(a, lens_a)
    for s in range(steps):
        x.copy_(_randn(torch, 50 + s, n, ch, std=1.0 + s))
        g.replay()
        ref = step(b, lens_b)
        assert torch.equal(out, ref) and torch.equal(lens_a, lens_b), s
        torch.mm(torch.randn(64, 64, device="cuda"), torch.randn(64, 64, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def _many(torch, C, P, seed):
    """Inputs of every way through the operators, and a function that runs them all."""
    hq, hkv, d = 8, 4, 64
    x = {m: _randn(torch, seed + m, m, 200, std=2.0) for m in (3, 200, 33000)}
    w = P.quantize_rows(_randn(torch, seed + 1, 130, 200))
    q = _randn(torch, seed + 2, 40, hq, d)
    big = _randn(torch, seed + 3, 700, hq, d)
    pk, k = _randn(torch, seed + 4, 1500, hkv, d), _randn(torch, seed + 5, 800, hkv, d)
    freq, _ = P.rotary_frequencies(d)
    pos = torch.arange(40, dtype=torch.int32, device="cuda") * 1000

    def run():
        return (*(P.i8_linear(x[m], w, act="silu") for m in x), *P.quantize_rows(x[200])[:2],
                *P.rotary(q, pos, freq, k=q[:, :hkv]),
                C.prefix_attention(q, pk, pk, k[:400], k[:400], [1] * 40, [10] * 40),           # shared
                C.prefix_attention(q[:2], pk, pk, k[:3], k[:3], [2], [3]),                      # one stream, cut
                C.prefix_attention(big, pk[:50], pk[:50], k, k, [700], [800]))                  # one pass
    return [*x.values(), q, big, pk, k], run


def test_captured(torch, C, P):
    """Every way in one graph, replayed over new inputs with eager work and waits between the replays."""
    inputs, run = _many(torch, C, P, 1000)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for s in range(4):
        for i, t in enumerate(inputs):
            t.copy_(_randn(torch, 2000 + 10 * s + i, *t.shape))
        g.replay()
        for i, (a, b) in enumerate(zip(got, run())):
            assert torch.equal(a, b), (s, i)
        torch.cuda.synchronize()


def test_two_graphs(torch, C, P):
    """Two captured graphs, replayed in turn and on two streams at once: their workspaces are their own."""
    runs = [_many(torch, C, P, seed)[1] for seed in (3000, 4000)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    graphs, got = [], []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(r())
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


def test_streams(torch, C, P):
    """Calls on two streams at once, a stream handed over by argument, its inputs dropped right after."""
    runs = [_many(torch, C, P, seed)[1] for seed in (5000, 6000)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for r, s in zip(runs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(r())
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    s = streams[0]
    x, w = _randn(torch, 1, 300, 640), P.quantize_rows(_randn(torch, 2, 200, 640))
    pk = _randn(torch, 3, 2000, 4, 64)
    q, freq = _randn(torch, 4, 50, 4, 64), P.rotary_frequencies(64)[0]
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    calls = (lambda t, st: P.i8_linear(t, w, stream=st), lambda t, st: P.quantize_rows(t, stream=st).codes,
             lambda t, st: P.rotary(t, pos, freq, stream=st)[0],
             lambda t, st: C.prefix_attention(t, pk, pk, q, q, [1] * 50, [1] * 50, stream=st))
    for src, call in zip((x, x, q, q), calls):
        ref = call(src, None)
        for _ in range(3):
            y = src.clone()
            s.wait_stream(torch.cuda.current_stream())
            out = call(y, s)
            del y
            junk = torch.full_like(src, float("nan"))   # would take y's memory if it were free
            torch.cuda.current_stream().wait_stream(s)
            assert torch.equal(out, ref)
            del junk


def test_wrappers_refuse(torch, C, P):
    """What would reach the kernels wrong raises before anything is enqueued."""
    from paper_2606_05981_amd.binding import MteError
    x, w = _randn(torch, 1, 6, 96), P.quantize_rows(_randn(torch, 2, 40, 96))
    bias, out = _randn(torch, 3, 40), torch.zeros((6, 40), dtype=torch.bfloat16, device="cuda")
    ok = dict(x=x, weight=w, bias=bias, out=out)
    P.i8_linear(**ok)
    for bad in (dict(x=x.half()), dict(x=x.cpu()), dict(x=x[:, :95]), dict(x=x.t()), dict(x=x[:, ::2]),
                dict(x=torch.zeros((2, 3, 2, 96), dtype=torch.bfloat16, device="cuda").transpose(0, 1)),
                dict(bias=bias.float()), dict(bias=bias[:39]), dict(bias=bias.cpu()), dict(act="gelu"), dict(dtype=torch.float16),
                dict(out=out[:5]), dict(out=out.float()), dict(out=out.t().contiguous().t()), dict(out=out[:1].expand(6, 40)),
                dict(weight=(w.codes, w.scales, 200)), dict(weight=(w.codes[:, :64], w.scales, 96)),
                dict(weight=(w.codes, w.scales.double(), 96)), dict(weight=(w.codes, w.scales[:3], 96)),
                dict(weight=(w.codes.cpu(), w.scales, 96)), dict(weight=(w.codes.to(torch.uint8), w.scales, 96)),
                dict(weight=(w.codes[:0], w.scales[:0], 96)), dict(weight=(w.codes, w.scales, 95)),
                dict(weight=(w.codes.view(-1)[8:-120].view(-1, 128), w.scales[:39], 96)),          # not 16-byte aligned
                dict(x=P.quantize_rows(_randn(torch, 4, 6, 97))), dict(x=x, stream=object())):
        with pytest.raises((ValueError, MteError, AttributeError)):
            P.i8_linear(**{**ok, **bad})
    for bad in (x.half(), x.cpu(), x.t(), torch.zeros((4, 0), device="cuda"), torch.zeros((4, 131072), device="cuda"),
                x[:1].expand((1 << 31) + 1, 96), 3):
        with pytest.raises(ValueError):
            P.quantize_rows(bad)
    q, k = _randn(torch, 5, 7, 4, 64), _randn(torch, 6, 7, 2, 64)
    pos, freq = torch.arange(7, dtype=torch.int32, device="cuda"), P.rotary_frequencies(64)[0]
    ok = dict(q=q, positions=pos, freq=freq, k=k)
    P.rotary(**ok)
    three = pos.expand(3, 7)
    P.rotary(**{**ok, "positions": three, "sections": (12, 10, 10)})
    for bad in (dict(q=q.half()), dict(q=q.cpu()), dict(q=q[:, :, :63]), dict(k=k[:6]), dict(k=k.float()), dict(k=k[:, :0]),
                dict(q=q.transpose(1, 2)), dict(positions=pos.long()), dict(positions=pos[:6]), dict(positions=three),
                dict(positions=pos.cpu()), dict(positions=three, sections=(12, 10, 9)), dict(positions=three, sections=(12, 20)),
                dict(positions=three, sections=(43, -1, -10)), dict(sections=(32,)), dict(freq=freq.float()),
                dict(freq=freq[:0]), dict(freq=freq.cpu()), dict(freq=torch.cat([freq, freq])), dict(freq=freq[::2]),
                dict(factor=float("nan")), dict(out=(q, None)), dict(out=(q[:6], k)), dict(out=(q.float(), k)),
                dict(out=(q[:1].expand(7, 4, 64), k)), dict(q=q[:1].expand((1 << 31) + 1, 4, 64), k=None)):
        with pytest.raises((ValueError, MteError)):
            P.rotary(**{**ok, **bad})
    ok = dict(q=q, prefix_k=k, prefix_v=k, k=k, v=k, q_lens=[3, 4], kv_lens=[5, 2])
    C.prefix_attention(**ok)
    for bad in (dict(q=q.float()), dict(prefix_k=k.float()), dict(prefix_v=k[:6]), dict(prefix_k=k[:, :1]), dict(k=k[:6]),
                dict(v=k[:6]), dict(q_lens=[3, 3]), dict(kv_lens=[5, 3]), dict(kv_lens=[7]), dict(q_lens=[8, -1]),
                dict(q=q.cpu()), dict(prefix_k=k.cpu()), dict(scale=0.0), dict(scale=float("nan")), dict(out=q[:6]),
                dict(out=q[:1].expand(7, 4, 64)), dict(q=_randn(torch, 7, 7, 3, 64)), dict(prefix_v=k.transpose(1, 2))):
        with pytest.raises((ValueError, MteError)):
            C.prefix_attention(**{**ok, **bad})


def test_products_refuse_a_result_in_what_they_read(torch, P):
    """A result in the memory of the rows (a square layer in place), of codes, weight or bias raises: workgroups store
    while others read. Columns beside the rows, in one buffer, are taken."""
    k = 128
    for m in (5, 40):
        x, w, bias = _randn(torch, 1, m, k), P.quantize_rows(_randn(torch, 2, k, k)), _randn(torch, 3, k)
        ref = P.i8_linear(x, w, bias)
        box = torch.zeros((m + 1, 2 * k), dtype=x.dtype, device="cuda")
        rows, beside = box[:m, :k], box[:m, k:]
        rows.copy_(x)
        twice = torch.zeros((2 * m, k), dtype=torch.int8, device="cuda")        # codes in the first half
        codes = P.I8Rows(twice[:m], P.quantize_rows(x).scales, k)
        as_result = lambda t: t.view(-1).view(torch.bfloat16)[:m * k].view(m, k)
        held = box.clone()
        for src, out in ((x, x), (rows, rows), (rows, box[:m, 8:k + 8]), (rows, box[1:, :k]),
                         (rows, box.view(-1)[k:(m + 1) * k].view(m, k)), (codes, as_result(twice)), (x, as_result(w.codes)),
                         (x[:1], bias.view(1, k)), (x[:1], w.scales.view(torch.bfloat16)[:k].view(1, k))):
            with pytest.raises(ValueError, match="out"):
                P.i8_linear(src, w, bias, out=out)
        assert torch.equal(box, held)
        assert torch.equal(P.i8_linear(rows, w, bias, out=beside), ref) and torch.equal(rows, x)
