"""The operators with which a denoiser reads the encoder's conditioning, as cases to time and compare.

Three of them: cross attention from latent positions to the encoder's tokens
(`cross`), the 8-bit key/value cache that keeps such tokens across calls (`append`
stores rows and reads them back, `cached` attends to them) and group norm with an
activation on channels-last latents (`norm`). Head shapes are those of this
repository's encoder (16 query / 8 kv heads of 128, 4 / 2 of 64) and generic
denoiser ones; key lengths are the encoder's sequences (96 to 320 tokens, the mixed
batch of synth.workloads) and, for the cache, streams that grow.

listed() is the fixed set, draw() gives further cases of the same ranges, prepare()
what a program holds before the call, run() one call in plain torch or through the
framework (`own`), work() what it cannot do without, exact() the result in 64 bits.

The 8-bit cache, as prepare() lays it out: blocks of 32 tokens; keys [block, head,
d / 16, 32 tokens, 16], values [block, head, d, 32 tokens in the order of _ORDER],
e4m3 codes; scales [block, head, 2] (keys, values), powers of two.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
# value position 16 h + 8 t + 4 a + i of a block holds token 16 t + 8 a + 4 h + i
_ORDER = [16 * t + 8 * a + 4 * h + i for h in range(2) for t in range(2) for a in range(2) for i in range(4)]

# 32 key lengths of 102 .. 319 tokens: the mixed batch of synth.workloads
MIXED = ("126,124,275,208,228,231,256,102,205,129,186,304,219,111,218,125,"
         "265,309,316,235,291,179,128,211,195,245,319,157,288,127,174,273")


def _cross(name, q_lens, kv_lens, hq, hkv, d, dtype="bf16", mask=False, fused=False, shared=False):
    """Queries of q_lens positions attend to kv_lens tokens ("4096x16" or "33,1,96"). mask: some keys
    are masked out; fused: keys and values are the halves of one projection's rows; shared: one
    frame's keys for all (the encoder's batch_one caching), kv_lens then names one sequence."""
    c = {"kind": "cross", "q": q_lens, "kv": kv_lens, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "mask": mask,
         "fused": fused, "shared": shared}
    return dict(c, name=name) if name else c


def _append(name, kv_lens, new_lens, hkv, d, dtype="bf16"):
    """new_lens rows join sequences that kv_lens tokens long afterwards; what is read back are the
    rows of the blocks that the call touched."""
    c = {"kind": "append", "kv": kv_lens, "new": new_lens, "hkv": hkv, "d": d, "dtype": dtype}
    return dict(c, name=name) if name else c


def _cached(name, q_lens, kv_lens, hq, hkv, d, dtype="bf16", causal=False):
    c = {"kind": "cached", "q": q_lens, "kv": kv_lens, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "causal": causal}
    return dict(c, name=name) if name else c


def _norm(name, n, side_h, side_w, c, groups, act=True, dtype="bf16", wide=0):
    """wide: channels that the rows of x have beyond c (a slice of a concatenated buffer)."""
    c = {"kind": "norm", "n": n, "h": side_h, "w": side_w, "c": c, "groups": groups, "act": act, "dtype": dtype,
         "wide": wide}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One query for each of 16 streams to its frame's tokens: a pooled readout, all latency.
        _cross("cross_tokens_16x1", "1x16", "96x16", 16, 8, 128),
        # One frame's 32x32 latents to its 96 conditioning tokens: a stream that goes frame by frame.
        _cross("cross_frame_1024x96", "1024", "96", 10, 10, 64, fused=True),
        # The batched dispatch: 16 frames of 64x64 latents, the largest read and write.
        _cross("cross_batch_16x4096x96", "4096x16", "96x16", 10, 10, 64, fused=True),
        # 32 frames of mixed sizes, padded keys masked out, grouped heads: the matrix cores' case.
        _cross("cross_mixed32_masked", "1000x32", MIXED, 16, 8, 128, mask=True),
        # The fp32 configuration's heads, odd lengths.
        _cross("cross_f32_ragged", "256,77,1,1024,513", "96,33,320,1,200", 4, 2, 64, dtype="f32"),
        # Storing the keys and values of 16 frames of 512x512 sources (320 tokens), bytes in and out.
        _append("append_prompt_16x320", "320x16", "320x16", 8, 128),
        # One token joins each of 64 streams, inside blocks that hold others.
        _append("append_step_64", "77x20,1000x20,4097x24", "1x64", 8, 128),
        # A step of 32 streams of unequal history: one query each over the cached tokens.
        _cached("cached_step_32", "1x32", "8192x8,5000x8,777x8,96x8", 16, 8, 128, causal=True),
        # One stream with a long history: a single query over 131071 tokens.
        _cached("cached_long_131071", "1", "131071", 16, 8, 128, causal=True),
        # 16 frames' 32x32 latents over conditioning kept in 8 bits.
        _cached("cached_frames_16x1024x320", "1024x16", "320x16", 16, 8, 128),
        # The innermost level of one frame: 8x8 latents, many channels.
        _norm("norm_8x8x1280", 1, 8, 8, 1280, 32),
        # The outermost level of 16 frames.
        _norm("norm_16x64x64x320", 16, 64, 64, 320, 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_lens(rng, n, lo, hi, equal=0.3):
    if rng.random() < equal:
        return "%dx%d" % (_log_int(rng, lo, hi), n)
    return ",".join(str(_log_int(rng, lo, hi)) for _ in range(n))


def draw(rng):
    r = rng.random()
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    hq, hkv = rng.choice([(8, 8), (10, 10), (20, 20), (16, 8), (4, 2), (16, 2), (8, 1), (12, 4), (5, 5)])
    if r < 0.35:
        n = _log_int(rng, 1, 24)
        shared = rng.random() < 0.15
        top = 1024 if dtype == "bf16" else 320
        kv = _draw_lens(rng, 1 if shared else n, 1, top)
        if n > 1 and not shared and rng.random() < 0.2:  # a frame without tokens: its rows are zero
            kv = ",".join(["0"] + [str(x) for x in _lens(kv)][1:])
        return _cross("", _draw_lens(rng, n, 1, 4096 if n <= 12 else 900), kv,
                      hq, hkv, rng.choice([64, 64, 128, 128, 40, 80]), dtype, mask=rng.random() < 0.3,
                      fused=rng.random() < 0.4, shared=shared)
    if r < 0.50:
        n = _log_int(rng, 1, 64)
        kv = [_log_int(rng, 1, 2000) for _ in range(n)]
        step = rng.random() < 0.5
        new = [1 if step else rng.randint(1, x) for x in kv]
        return _append("", ",".join(map(str, kv)), ",".join(map(str, new)), hkv, rng.choice([64, 128]), dtype)
    if r < 0.80:
        d = rng.choice([64, 128])
        if rng.random() < 0.5:  # single tokens, a few at most
            n = _log_int(rng, 1, 32)
            kv = [_log_int(rng, 4, 131072 * 8 // max(hkv, 8) // n) for _ in range(n)]
            q = [rng.choice([1, 1, 1, 2, 4]) for _ in range(n)]
        else:
            n = _log_int(rng, 1, 16)
            kv = [_log_int(rng, 16, 1024) for _ in range(n)]
            q = [_log_int(rng, 1, x) for x in kv]
        return _cached("", ",".join(map(str, q)), ",".join(map(str, kv)), hq, hkv, d, dtype, causal=rng.random() < 0.6)
    groups = rng.choice([32, 32, 32, 16, 8, 5])
    c = groups * _log_int(rng, 1, 40)
    h, w = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    n = max(1, min(_log_int(rng, 1, 16), 20_000_000 // (h * w * c)))
    return _norm("", n, h, w, c, groups, rng.random() < 0.7, dtype, wide=rng.choice([0, 0, 0, 8, 3]))


def _lens(text):
    """"96x16" or "33,1,7x2" -> list of lengths."""
    parts = [p.split("x") for p in text.split(",")]
    return [int(p[0]) for p in parts for _ in range(int(p[1]) if len(p) > 1 else 1)]


def _start(lens):
    return [sum(lens[:i]) for i in range(len(lens))]


def _ramp(n):
    return torch.arange(n, device="cuda")


def _rows(lens, starts=None):
    """Padded gather of packed rows: (row of [sequence, position], whether it is one)."""
    L = torch.tensor(lens, device="cuda").view(-1, 1)
    s = torch.tensor(_start(lens) if starts is None else starts, device="cuda").view(-1, 1)
    at = _ramp(max(max(lens), 1)).view(1, -1)
    return torch.where(at < L, s + at, torch.zeros_like(s)), at < L


def _unpad(lens):
    """The inverse: flat padded index of every packed row."""
    top = max(max(lens), 1)
    n, s = torch.tensor(lens, device="cuda"), torch.tensor(_start(lens), device="cuda")
    seq = torch.repeat_interleave(_ramp(len(lens)), n)
    return seq * top + _ramp(sum(lens)) - s[seq]


# ---- inputs -------------------------------------------------------------------------------------


def _e4m3_scale(amax):
    """2^e, e the smallest integer >= -126 with amax <= 448 * 2^e (448 = 0.875 * 2^9)."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)   # the power itself, no pow()


def _codes(x, scale):
    """e4m3 codes of x / scale, as torch.float8_e4m3fn."""
    return (x / scale).to(torch.float8_e4m3fn)


def _lay_out(k8, v8):
    """Codes [blocks, head, 32, d] of keys and values in the cache's two layouts (uint8)."""
    n, h, t, d = k8.shape
    k8 = k8.view(torch.uint8).view(n, h, t, d // 16, 16).transpose(2, 3).contiguous()
    v8 = v8.view(torch.uint8)[:, :, torch.tensor(_ORDER, device="cuda")].transpose(2, 3).contiguous()
    return k8, v8


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    dt = DT[case["dtype"]]

    def pool(lens, hkv, d, spare=3):
        """A pool whose blocks hold `lens` tokens of each sequence, in a shuffled order, and its table."""
        nb = [(x + BLOCK - 1) // BLOCK for x in lens]
        total = sum(nb) + spare
        order = torch.randperm(total, generator=g, device="cuda")
        rows, valid = _rows(nb)
        table = torch.where(valid, order[rows], torch.zeros_like(rows)).to(torch.int32).contiguous()
        spread = torch.exp(torch.randn((1, hkv, 1, 1), generator=g, device="cuda"))
        parts, scales = [], []
        for i in range(2):
            x = torch.randn((total, hkv, BLOCK, d), generator=g, device="cuda") * (1.0 if i == 0 else spread)
            s = _e4m3_scale(x.abs().amax((2, 3)))
            parts.append(_codes(x, s[:, :, None, None]))
            scales.append(s)
            del x
        k8, v8 = _lay_out(*parts)
        return k8, v8, torch.stack(scales, -1).contiguous(), table

    def append_plan(kv, new, table):
        """Index tensors of a plain append: for every touched block its pool index, the packed row that
        lands in each of its 32 places (or -1), whether a place holds a token from before; and for every row read
        back its place."""
        at, block, row, kept, back = [], [], [], [], []
        s = 0
        for i, (a, b) in enumerate(zip(kv, new)):
            lo = (a - b) // BLOCK
            for j in range(lo, (a + BLOCK - 1) // BLOCK):
                pos = torch.arange(j * BLOCK, (j + 1) * BLOCK)
                at.append((i, j))
                is_new = (pos >= a - b) & (pos < a)
                row.append(torch.where(is_new, s + pos - (a - b), torch.full_like(pos, -1)))
                kept.append(pos < a - b)
            back.append(len(block) * BLOCK + torch.arange(a - lo * BLOCK))
            block += [None] * (len(at) - len(block))
            s += b
        at = torch.tensor(at, device="cuda")
        return {"block": table[at[:, 0], at[:, 1]].long(), "row": torch.stack(row).cuda(),
                "kept": torch.stack(kept).cuda(), "back": torch.cat(back).cuda()}

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dt)

    if kind == "norm":
        n, h, w, c = case["n"], case["h"], case["w"], case["c"]
        full = c + case["wide"]
        x = torch.randn((n, h, w, full), generator=g, device="cuda")
        x = (x * torch.exp(0.5 * torch.randn((full,), generator=g, device="cuda")) +
             torch.randn((full,), generator=g, device="cuda")).to(dt)
        gamma = (1 + 0.2 * torch.randn((c,), generator=g, device="cuda")).to(dt)
        return {"case": case, "x": x[..., :c], "gamma": gamma, "beta": normal(c, std=0.2)}
    kv = _lens(case["kv"])
    if kind == "append":
        new = _lens(case["new"])
        k8, v8, sc, table = pool(kv, case["hkv"], case["d"])
        # rows read back: those of the touched blocks
        first = [(a - b) // BLOCK * BLOCK for a, b in zip(kv, new)]
        return {"case": case, "k8": k8, "v8": v8, "scales": sc, "table": table, "new": new,
                "counts": [a - f for a, f in zip(kv, first)],
                "kv_lens": torch.tensor(kv, dtype=torch.int32, device="cuda"),
                "k": normal(sum(new), case["hkv"], case["d"], std=1.5), "v": normal(sum(new), case["hkv"], case["d"], std=3.0),
                "plan": append_plan(kv, new, table)}
    ql = _lens(case["q"])
    q = normal(sum(ql), case["hq"], case["d"], std=1.5)
    base = {"case": case, "q": q, "q_lens": ql, "q_rows": _rows(ql), "q_flat": _unpad(ql)}
    if kind == "cached":
        k8, v8, sc, table = pool(kv, case["hkv"], case["d"])
        return dict(base, k8=k8, v8=v8, scales=sc, table=table,
                    kv_lens=torch.tensor(kv, dtype=torch.int32, device="cuda"),
                    q_count=torch.tensor(ql, device="cuda"))
    n, T = len(ql), sum(kv)
    index = [0] * n if case["shared"] else list(range(n))
    if case["fused"]:
        both = normal(T, 2, case["hkv"], case["d"])
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = normal(T, case["hkv"], case["d"]), normal(T, case["hkv"], case["d"])
    mask = (torch.rand((T,), generator=g, device="cuda") < 0.8) if case["mask"] else None
    starts = _start(kv)
    return dict(base, k=k, v=v, mask=mask, kv_lens=kv, index=index,
                k_rows=_rows([kv[i] for i in index], [starts[i] for i in index]))


# ---- plain forms --------------------------------------------------------------------------------


def _softmax_read(q, k, v, see, scale):
    """Attention on padded float tensors: q [n, Hq, Lq, d], k, v [n, Hkv, Lk, d], see broadcast to
    [n, 1, Lq, Lk] -> [n, Lq, Hq, d]; rows that see nothing are zero."""
    n, hq, lq, d = q.shape
    rep = hq // k.shape[1]
    q = q.reshape(n, hq // rep, rep * lq, d)
    s = (q @ k.transpose(2, 3).contiguous()).reshape(n, hq, lq, -1) * scale
    s = torch.where(see, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = p.reshape(n, hq // rep, rep * lq, -1) @ v
    return o.reshape(n, hq, lq, d).transpose(1, 2)


def _plain_cross(st):
    q_rows, q_valid = st["q_rows"]
    k_rows, see = st["k_rows"]
    if st["mask"] is not None:
        see = see & st["mask"][k_rows]
    q = st["q"].float()[q_rows].transpose(1, 2)
    k = st["k"].float()[k_rows].transpose(1, 2).contiguous()
    v = st["v"].float()[k_rows].transpose(1, 2).contiguous()
    o = _softmax_read(q, k, v, see[:, None, None, :], 1 / math.sqrt(q.shape[-1]))
    return o.reshape(-1, *o.shape[2:])[st["q_flat"]].to(st["q"].dtype)


def _values(codes, scale):
    return codes.view(torch.float8_e4m3fn).float() * scale


def _plain_pages(k8, v8, scales, blocks):
    """Blocks of the pool as fp32 keys and values [..., head, 32, d] of any index shape."""
    sc = scales[blocks]
    k = k8[blocks]
    k = _values(k.transpose(-3, -2).reshape(*k.shape[:-3], BLOCK, -1), sc[..., 0, None, None])
    back = torch.argsort(torch.tensor(_ORDER, device="cuda"))
    v = _values(v8[blocks][..., back].transpose(-1, -2).contiguous(), sc[..., 1, None, None])
    return k, v


def _plain_cached(st):
    q_rows, q_valid = st["q_rows"]
    k, v = _plain_pages(st["k8"], st["v8"], st["scales"], st["table"].long())   # [n, nb, H, 32, d]
    n, nb, h, t, d = k.shape
    k = k.transpose(1, 2).reshape(n, h, nb * t, d)
    v = v.transpose(1, 2).reshape(n, h, nb * t, d)
    q = st["q"].float()[q_rows].transpose(1, 2)
    at = _ramp(nb * t).view(1, 1, -1)
    see = at < st["kv_lens"].view(-1, 1, 1)
    if st["case"]["causal"]:
        mine = (st["kv_lens"] - st["q_count"]).view(-1, 1, 1) + _ramp(q.shape[2]).view(1, -1, 1)
        see = see & (at <= mine)
    o = _softmax_read(q, k, v, see[:, None], 1 / math.sqrt(d))
    return o.reshape(-1, *o.shape[2:])[st["q_flat"]].to(st["q"].dtype)


def _plain_append(st):
    plan = st["plan"]
    block, row, kept = plan["block"], plan["row"], plan["kept"][:, None, :, None]
    old_scale = st["scales"][block]
    olds = _plain_pages(st["k8"], st["v8"], st["scales"], block)
    any_kept = plan["kept"].any(1)[:, None]
    fresh = (row >= 0)[:, None, :, None]

    def merge(x, old, s_old):
        x = torch.where(fresh, x.float()[row.clamp(min=0)].transpose(1, 2), torch.zeros_like(old))
        s = _e4m3_scale(x.abs().amax((2, 3)))
        s = torch.where(any_kept, torch.maximum(s, s_old), s)
        return _codes(torch.where(kept, old, x), s[:, :, None, None]), s

    k8, ks = merge(st["k"], olds[0], old_scale[..., 0])
    v8, vs = merge(st["v"], olds[1], old_scale[..., 1])
    lk, lv = _lay_out(k8, v8)
    st["k8"][block], st["v8"][block], st["scales"][block] = lk, lv, torch.stack([ks, vs], -1)
    k = _values(k8.transpose(1, 2).reshape(-1, *k8.shape[1:2], k8.shape[3])[plan["back"]], torch.repeat_interleave(ks, BLOCK, 0)[plan["back"]][..., None])
    v = _values(v8.transpose(1, 2).reshape(-1, *v8.shape[1:2], v8.shape[3])[plan["back"]], torch.repeat_interleave(vs, BLOCK, 0)[plan["back"]][..., None])
    return k.to(st["k"].dtype), v.to(st["v"].dtype)


def _plain_norm(st):
    c = st["case"]
    x = st["x"].float()
    z = x.reshape(c["n"], c["h"] * c["w"], c["groups"], -1)
    z = z - z.mean((1, 3), keepdim=True)
    z = z / torch.sqrt((z * z).mean((1, 3), keepdim=True) + 1e-5)
    z = z.reshape(x.shape) * st["gamma"].float() + st["beta"].float()
    if c["act"]:
        z = z / (1 + torch.exp(-z))
    return z.to(st["x"].dtype)


def run(st):
    kind = st["case"]["kind"]
    if own:
        from paper_2606_05981_amd import conditioning as C
        if kind == "cross":
            return C.cross_attention(st["q"], st["k"], st["v"], st["q_lens"], st["kv_lens"], kv_index=st["index"],
                                     key_mask=st["mask"])
        if kind == "norm":
            return C.group_norm(st["x"], st["case"]["groups"], st["gamma"], st["beta"], eps=1e-5,
                                act="silu" if st["case"]["act"] else None)
        cache = (st["k8"], st["v8"], st["scales"])
        if kind == "append":
            C.kv8_append(cache, st["table"], st["kv_lens"], st["k"], st["v"], st["new"])
            return C.kv8_read(cache, st["table"], st["kv_lens"], st["counts"], dtype=st["k"].dtype)
        return C.kv8_attention(st["q"], cache, st["table"], st["kv_lens"], st["q_lens"], causal=st["case"]["causal"])
    if kind == "cross":
        return _plain_cross(st)
    if kind == "cached":
        return _plain_cached(st)
    return _plain_append(st) if kind == "append" else _plain_norm(st)


# ---- what it cannot do without ------------------------------------------------------------------


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        n = case["n"] * case["h"] * case["w"] * case["c"]
        return {"bytes": 2 * n * es + 2 * case["c"] * es, "flops": 8 * n}
    kv, hkv, d = _lens(case["kv"]), case["hkv"], case["d"]
    if case["kind"] == "append":
        new = _lens(case["new"])
        back = sum(a - (a - b) // BLOCK * BLOCK for a, b in zip(kv, new))
        rows = 2 * hkv * d
        return {"bytes": rows * (sum(new) * (es + 1) + back * (es + 1)), "flops": 4 * rows * sum(new)}
    q = _lens(case["q"])
    io = 2 * sum(q) * case["hq"] * d * es
    if case["kind"] == "cross":
        pairs = sum(a * b for a, b in zip(q, kv * len(q) if case["shared"] else kv))
        b = io + 2 * sum(kv) * hkv * d * es + (sum(kv) if case["mask"] else 0)
    else:
        pairs = sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(q, kv))
        b = io + sum(kv) * 2 * hkv * d + sum((x + BLOCK - 1) // BLOCK for x in kv) * (8 * hkv + 4)
    return {"bytes": b, "flops": 4 * case["hq"] * d * pairs}


# ---- 64 bits ------------------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]

    def e4m3_table():
        """The value of every e4m3 code, from the format's definition."""
        t = []
        for c in range(256):
            e, m = (c >> 3) & 15, c & 7
            v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
            t.append(math.nan if e == 15 and m == 7 else -v if c & 128 else v)
        return torch.tensor(t, dtype=torch.float64, device="cuda")

    def nearest(x):
        """The e4m3 value nearest to x (|x| <= 448), ties to the even code, by search."""
        vals = e4m3_table()[:127].contiguous()
        a = x.abs().contiguous()
        hi = torch.searchsorted(vals, a).clamp(0, 126)
        lo = (hi - 1).clamp(min=0)
        dl, dh = a - vals[lo], vals[hi] - a
        up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
        return torch.where(up, vals[hi], vals[lo]) * torch.sign(x)

    def power(amax):
        """The smallest 2^e, e >= -126, with amax <= 448 * 2^e, by search."""
        steps = torch.tensor([2.0 ** e for e in range(-126, 121)], dtype=torch.float64, device="cuda")
        return steps[torch.searchsorted(448 * steps, amax).clamp(max=len(steps) - 1)]

    def decoded(st, i, blocks):
        """Keys and values [head, tokens, d] of one sequence in float64, token by token of the layout."""
        lut = e4m3_table()
        b = st["table"][i, :blocks].long()
        sc = st["scales"][b].double()
        k = lut[st["k8"][b].long()].permute(1, 0, 3, 2, 4).reshape(sc.shape[1], blocks * BLOCK, -1)
        v = lut[st["v8"][b].long()]
        place = [_ORDER.index(t) for t in range(BLOCK)]
        v = torch.stack([v[..., p] for p in place], 2).permute(1, 0, 2, 3).reshape(sc.shape[1], blocks * BLOCK, -1)
        wide = torch.repeat_interleave(sc, BLOCK, 0).permute(1, 0, 2)
        return k * wide[..., :1], v * wide[..., 1:]

    def exact_rows(q, k, v, see):
        """One sequence: q [Lq, Hq, d], k, v [Hkv, Lk, d] float64, see [Lq or 1, Lk]."""
        lq, hq, d = q.shape
        out = torch.zeros_like(q)
        for h in range(hq):
            g = h // (hq // k.shape[0])
            s = torch.matmul(q[:, h], k[g].T) / math.sqrt(d)
            s = s.masked_fill(~see.expand_as(s), -math.inf)
            p = torch.nan_to_num(torch.softmax(s, -1), nan=0.0)
            out[:, h] = torch.matmul(p, v[g])
        return out

    if kind == "norm":
        x = st["x"].double()
        y = torch.empty_like(x)
        per = case["c"] // case["groups"]
        for g in range(case["groups"]):
            a = slice(g * per, (g + 1) * per)
            z = x[..., a]
            var, mean = torch.var_mean(z, (1, 2, 3), keepdim=True, correction=0)
            y[..., a] = (z - mean) * torch.rsqrt(var + 1e-5) * st["gamma"][a].double() + st["beta"][a].double()
        return y * torch.sigmoid(y) if case["act"] else y
    kv = _lens(case["kv"])
    if kind == "append":
        got, s = ([], []), 0
        for i, (a, b) in enumerate(zip(kv, st["new"])):
            lo = (a - b) // BLOCK
            olds = decoded(st, i, (a + BLOCK - 1) // BLOCK)
            for t, x in enumerate((st["k"], st["v"])):
                rows = x[s:s + b].double().transpose(0, 1)
                whole = torch.cat([olds[t][:, :a - b], rows], 1)
                for j in range(lo, (a + BLOCK - 1) // BLOCK):
                    part = whole[:, j * BLOCK:min(a, (j + 1) * BLOCK)]
                    n_old = max(0, a - b - j * BLOCK)
                    scale = power(part[:, n_old:].abs().amax((1, 2)))
                    if n_old:
                        scale = torch.maximum(scale, st["scales"][st["table"][i, j].long(), :, t].double())
                    scale = scale[:, None, None]
                    got[t].append((nearest(part / scale) * scale).transpose(0, 1))
            s += b
        return torch.cat(got[0]), torch.cat(got[1])
    out, s = [], 0
    starts = _start(kv)
    for i, n in enumerate(st["q_lens"]):
        q = st["q"][s:s + n].double()
        if kind == "cross":
            j = st["index"][i]
            a, b = starts[j], starts[j] + kv[j]
            k, v = st["k"][a:b].double().transpose(0, 1), st["v"][a:b].double().transpose(0, 1)
            see = (torch.ones((1, b - a), dtype=torch.bool, device="cuda") if st["mask"] is None else st["mask"][None, a:b])
        else:
            k, v = (x[:, :kv[i]] for x in decoded(st, i, (kv[i] + BLOCK - 1) // BLOCK))
            at = torch.arange(kv[i], device="cuda")[None]
            see = at <= kv[i] - n + torch.arange(n, device="cuda")[:, None] if case["causal"] else at >= 0
        out.append(exact_rows(q, k, v, see))
        s += n
    return torch.cat(out)
