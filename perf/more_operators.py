"""The operators between the encoder's hidden states and the attention that reads them, as cases to
time and compare.

Three of them: a product in 8-bit integers with a scale for each token and each channel (`i8`: q,
kv and feed-forward projections), rotary positions (`rot`: half or interleaved pairs, part of
the head, several axes, far positions) and attention of a batch whose sequences share a long
prefix (`prefix`). Widths and heads are those of this repository's encoder (2048, 16 query / 8 kv
heads of 128, SwiGLU of 6144, 96 or 320 tokens a frame) and generic denoiser ones (320 channels, 10
heads of 64); context lengths are generic.

listed() is the fixed set, draw() gives further cases of the same ranges, prepare()
what a program holds before the call, run() one call in plain torch or through the
framework (`own`), work() what it cannot do without, exact() the result in 64 bits.

8-bit rows: scale s = max |x| / 127 of a row, rounded to fp32 (at least 2^-126), codes x / s rounded to
the nearest whole number, ties to the even one; stored with rows of a multiple of 128 bytes.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i8(name, m, k, n, dtype="bf16", bias=False, act=False, wide=0):
    """x [m, k] times an 8-bit weight [n, k]. act: SiLU; wide: elements that the rows of x have beyond k."""
    c = {"kind": "i8", "m": m, "k": k, "n": n, "dtype": dtype, "bias": bias, "act": act, "wide": wide}
    return dict(c, name=name) if name else c


def _rot(name, t, hq, hk, d, rot, far, axes=1, inter=False, dtype="bf16", fused=False):
    """t tokens of hq query and hk key heads (0: queries only), the first `rot` of d channels rotated by
    positions below `far`. fused: both lie in one projection's rows."""
    c = {"kind": "rot", "t": t, "hq": hq, "hk": hk, "d": d, "rot": rot, "far": far, "axes": axes, "inter": inter,
         "dtype": dtype, "fused": fused}
    return dict(c, name=name) if name else c


def _prefix(name, q_lens, prefix, kv_lens, hq, hkv, d, dtype="bf16", causal=True, fused=False):
    """Queries of q_lens tokens ("1x64" or "33,1,96") over `prefix` shared and kv_lens own tokens."""
    c = {"kind": "prefix", "q": q_lens, "p": prefix, "kv": kv_lens, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
         "causal": causal, "fused": fused}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token through a square projection: all latency.
        _i8("i8_step_1x2048x2048", 1, 2048, 2048),
        # One token of 16 streams through a feed-forward's gate and up weights: bytes of the weight.
        _i8("i8_step_16x2048x12288", 16, 2048, 12288),
        # The keys and values of 16 frames of 96 tokens.
        _i8("i8_tokens_1536x2048x4096", 1536, 2048, 4096, bias=True),
        # Queries of 16 frames of 64x64 latents, 320 channels to 10 heads of 64: rows in and out.
        _i8("i8_latents_65536x320x640", 65536, 320, 640),
        # The feed-forward of 16 frames of 320 tokens, the matrix cores' case.
        _i8("i8_feed_5120x2048x12288", 5120, 2048, 12288, act=True),
        # fp32 rows, sizes that are multiples of nothing.
        _i8("i8_f32_777x1001x1283", 777, 1001, 1283, dtype="f32", bias=True),
        # One token of each of 64 streams, far into their contexts.
        _rot("rot_step_64", 64, 16, 8, 128, 128, 131072),
        # Queries and keys of 16 frames of 320 tokens at (t, h, w) positions, in a fused projection's rows.
        _rot("rot_frames_5120", 5120, 16, 8, 128, 128, 4096, axes=3, fused=True),
        # 16 frames of 64x64 latents at (h, w) positions, interleaved pairs, part of the head.
        _rot("rot_latents_65536", 65536, 10, 10, 64, 32, 64, axes=2, inter=True),
        # A step of 64 streams that share a long context: one query each.
        _prefix("prefix_step_64", "1x64", 16384, "96x40,320x23,1", 16, 8, 128),
        # 16 frames' 32x32 latents over shared instruction tokens and the frame's own.
        _prefix("prefix_frames_16x1024", "1024x16", 480, "320x16", 10, 10, 64, causal=False, fused=True),
        # Chunks of unequal streams, fp32, odd lengths.
        _prefix("prefix_f32_ragged", "7,1,33,64,0,5", 1201, "7,60,33,50,9,200", 4, 2, 64, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    r = rng.random()
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if r < 0.45:
        k = rng.choice([320, 640, 1280, 2048, 4096]) if rng.random() < 0.5 else _log_int(rng, 17, 6144)
        n = rng.choice([320, 640, 1280, 2048, 4096]) if rng.random() < 0.4 else _log_int(rng, 17, 12288)
        # rows, results and products stay below the largest listed ones'
        top = min(65536, int(1.2e11 / (k * n)), int(4e7 / max(k, n)))
        m = rng.randint(1, 32) if rng.random() < 0.3 else _log_int(rng, 1, max(top, 1))
        return _i8("", min(m, max(top, 1)), k, n, dtype, rng.random() < 0.5, rng.random() < 0.3, rng.choice([0, 0, 0, 8, 3]))
    if r < 0.65:
        hq, hk = rng.choice([(8, 8), (10, 10), (16, 8), (4, 2), (16, 0), (8, 1), (5, 5)])
        d = rng.choice([64, 64, 128, 128, 40, 80])
        axes = rng.choice([1, 1, 2, 3])
        rot = d if rng.random() < 0.6 else 2 * rng.randint(axes, d // 2)
        t = _log_int(rng, 1, int(8e7 / ((hq + hk) * d)) if dtype == "bf16" else int(4e7 / ((hq + hk) * d)))
        return _rot("", min(t, 65536), hq, hk, d, rot, rng.choice([64, 4096, 131072, 1 << 20, 1 << 30]), axes,
                    rng.random() < 0.5, dtype, rng.random() < 0.3)
    hq, hkv = rng.choice([(8, 8), (10, 10), (16, 8), (4, 2), (16, 2), (8, 1), (12, 4), (5, 5)])
    d = rng.choice([64, 64, 128, 128, 40, 80])
    if rng.random() < 0.5:   # few queries a stream, a long prefix
        n = _log_int(rng, 1, 64)
        q = [rng.choice([1, 1, 1, 2, 4, 0, rng.randint(1, 24)]) for _ in range(n)]
        p = _log_int(rng, 64, 16384 if dtype == "bf16" else 4096)
        kv = [rng.choice([x, x + _log_int(rng, 1, 320), rng.randint(0, 320)]) for x in q]
    else:
        n = _log_int(rng, 1, 12)
        q = [_log_int(rng, 16, 1024 if dtype == "bf16" else 320) for _ in range(n)]
        p = _log_int(rng, 1, 800)
        kv = [rng.choice([x, x + rng.randint(0, 64), _log_int(rng, 1, 320)]) for x in q]
    if sum(q) == 0:
        q[0], kv[0] = 1, max(kv[0], 1)
    return _prefix("", ",".join(map(str, q)), p, ",".join(map(str, kv)), hq, hkv, d, dtype, rng.random() < 0.6,
                   rng.random() < 0.4)


def _lens(text):
    """"96x16" or "33,1,7x2" -> list of lengths."""
    parts = [p.split("x") for p in text.split(",")]
    return [int(p[0]) for p in parts for _ in range(int(p[1]) if len(p) > 1 else 1)]


def _start(lens):
    return [sum(lens[:i]) for i in range(len(lens))]


def _padded(lens):
    """Padded gather of packed rows: (row of [sequence, position], whether it is one, flat padded index of every row)."""
    n = torch.tensor(lens, device="cuda")
    s = torch.tensor(_start(lens), device="cuda")
    top = max(max(lens), 1)
    at = torch.arange(top, device="cuda").view(1, -1)
    valid = at < n.view(-1, 1)
    rows = torch.where(valid, s.view(-1, 1) + at, torch.zeros_like(at))
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n)
    return rows, valid, seq * top + torch.arange(sum(lens), device="cuda") - s[seq]


def _sections(pairs, axes):
    """Pairs of each axis: as even as they come, the first ones the larger."""
    return [pairs // axes + (i < pairs % axes) for i in range(axes)]


# ---- inputs -------------------------------------------------------------------------------------


def _quantized(x):
    """Scales [rows] and codes of x's rows (float64 quotients: a border decides a whole step)."""
    s = (x.float().abs().amax(1) / 127).clamp(min=2.0 ** -126)
    return torch.round(x.double() / s.double()[:, None]), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    dt = DT[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if kind == "i8":
        m, k, n = case["m"], case["k"], case["n"]
        # hidden states: a few channels far larger than the others, rows of unlike size
        full = k + case["wide"]
        x = randn(m, full) * torch.exp(0.7 * randn(full)) * torch.exp(0.5 * randn(m, 1))
        w = randn(n, k) * torch.exp(0.3 * randn(n, 1)) / math.sqrt(k)
        codes, scales = _quantized(w)
        pad = torch.zeros((n, (k + 127) // 128 * 128), dtype=torch.int8, device="cuda")
        pad[:, :k] = codes.to(torch.int8)
        return {"case": case, "x": x.to(dt)[:, :k], "codes": pad, "scales": scales,
                "bias": randn(n).to(dt) if case["bias"] else None}
    if kind == "rot":
        t, hq, hk, d = case["t"], case["hq"], case["hk"], case["d"]
        if case["fused"]:
            both = randn(t, hq + hk, d).to(dt)
            q, key = both[:, :hq], both[:, hq:]
        else:
            q, key = randn(t, hq, d).to(dt), randn(t, hk, d).to(dt)
        pairs = case["rot"] // 2
        # theta 5e6 and positions scaled to a quarter, as for contexts longer than trained
        freq = 0.25 * 5e6 ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
        shape = (case["axes"], t) if case["axes"] > 1 else (t,)
        pos = torch.randint(0, case["far"], shape, generator=g, device="cuda", dtype=torch.int32)
        return {"case": case, "q": q, "k": key if hk else None, "pos": pos, "freq": freq,
                "sections": _sections(pairs, case["axes"]) if case["axes"] > 1 else None}
    ql, kl, p = _lens(case["q"]), _lens(case["kv"]), case["p"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    q = (1.5 * randn(sum(ql), hq, d)).to(dt)

    def keys(rows):
        if case["fused"]:
            both = randn(rows, 2, hkv, d).to(dt)
            return both[:, 0], both[:, 1]
        return randn(rows, hkv, d).to(dt), randn(rows, hkv, d).to(dt)
    pk, pv = keys(p)
    k, v = keys(sum(kl))
    return {"case": case, "q": q, "pk": pk, "pv": pv, "k": k, "v": v, "q_lens": ql, "kv_lens": kl,
            "q_rows": _padded(ql), "k_rows": _padded(kl),
            "shift": torch.tensor([b - a for a, b in zip(ql, kl)], device="cuda")}


# ---- plain forms --------------------------------------------------------------------------------


def _plain_i8(st):
    x, k = st["x"], st["case"]["k"]
    codes, s = _quantized(x)
    y = codes.float() @ st["codes"][:, :k].float().t()
    y = y * s[:, None] * st["scales"][None]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if st["case"]["act"]:
        y = y / (1 + torch.exp(-y))
    return y.to(x.dtype)


def _plain_rot(st):
    c = st["case"]
    pairs, pos = c["rot"] // 2, st["pos"]
    if st["sections"] is not None:
        axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(st["sections"], device="cuda"))
        at = pos[axis].t()
    else:
        at = pos[:, None]
    a = at.double() * st["freq"]                       # far positions: 32 bits would lose the angle
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    f = 1.125

    def turn(x):
        y = x.float()
        r = y[..., :c["rot"]]
        if c["inter"]:
            a, b = r[..., 0::2], r[..., 1::2]
            out = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).reshape(r.shape)
        else:
            a, b = r[..., :pairs], r[..., pairs:]
            out = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([out * f, y[..., c["rot"]:]], -1).to(x.dtype)
    return turn(st["q"]), None if st["k"] is None else turn(st["k"])


def _plain_prefix(st):
    c = st["case"]
    q_rows, _, q_flat = st["q_rows"]
    k_rows, k_valid, _ = st["k_rows"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    rep, scale = hq // hkv, 1 / math.sqrt(d)
    n, lq = q_rows.shape
    q = st["q"].float()
    tq = q.shape[0]
    # shared keys: every query's rows at once
    s1 = q.view(tq, hkv, rep, d).permute(1, 0, 2, 3).reshape(hkv, tq * rep, d) @ \
        st["pk"].float().permute(1, 2, 0).contiguous() * scale
    # own keys: sequences padded
    k = st["k"].float() if st["k"].shape[0] else torch.zeros((1, hkv, d), device="cuda")
    v = st["v"].float() if st["v"].shape[0] else torch.zeros((1, hkv, d), device="cuda")
    k, v = (x[k_rows].transpose(1, 2).contiguous() for x in (k, v))
    qp = q[q_rows].view(n, lq, hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, lq * rep, d)
    s2 = (qp @ k.transpose(2, 3).contiguous() * scale).view(n, hkv, lq, rep, -1)
    see = k_valid[:, None]
    if c["causal"]:
        at = torch.arange(k_rows.shape[1], device="cuda")
        see = see & (at <= (st["shift"][:, None] + torch.arange(lq, device="cuda"))[..., None])
    s2 = torch.where(see[:, None, :, None], s2, torch.full_like(s2, -math.inf))
    # one softmax over both
    t1 = s1.amax(-1).view(hkv, tq, rep)
    t2 = s2.amax(-1).permute(0, 2, 1, 3).reshape(n * lq, hkv, rep)[q_flat].permute(1, 0, 2)
    top = torch.maximum(t1, t2)
    p1 = torch.exp(s1 - top.reshape(hkv, tq * rep, 1))
    padded = torch.zeros((n * lq, hkv, rep), device="cuda")
    padded[q_flat] = top.permute(1, 0, 2)
    p2 = torch.exp(s2 - padded.view(n, lq, hkv, rep).permute(0, 2, 1, 3)[..., None])
    o1 = (p1 @ st["pv"].float().transpose(0, 1).contiguous()).view(hkv, tq, rep, d).permute(1, 0, 2, 3)
    o2 = (p2.view(n, hkv, lq * rep, -1) @ v).view(n, hkv, lq, rep, d).permute(0, 2, 1, 3, 4)
    o2 = o2.reshape(n * lq, hkv, rep, d)[q_flat]
    l1 = p1.sum(-1).view(hkv, tq, rep).permute(1, 0, 2)
    l2 = p2.sum(-1).permute(0, 2, 1, 3).reshape(n * lq, hkv, rep)[q_flat]
    return ((o1 + o2) / (l1 + l2)[..., None]).reshape(tq, hq, d).to(st["q"].dtype)


def run(st):
    c = st["case"]
    if own:
        from paper_2606_05981_amd import conditioning as C
        from paper_2606_05981_amd import projections as P
        if c["kind"] == "i8":
            return P.i8_linear(st["x"], P.I8Rows(st["codes"], st["scales"], c["k"]), bias=st["bias"],
                               act="silu" if c["act"] else None)
        if c["kind"] == "rot":
            return P.rotary(st["q"], st["pos"], st["freq"], k=st["k"], interleaved=c["inter"], sections=st["sections"],
                            factor=1.125)
        return C.prefix_attention(st["q"], st["pk"], st["pv"], st["k"], st["v"], st["q_lens"], st["kv_lens"],
                                  causal=c["causal"])
    if c["kind"] == "i8":
        return _plain_i8(st)
    return _plain_rot(st) if c["kind"] == "rot" else _plain_prefix(st)


# ---- what it cannot do without ------------------------------------------------------------------


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "i8":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": m * k * es + n * k + 4 * n + m * n * es + (n * es if case["bias"] else 0), "flops": 2 * m * n * k}
    if case["kind"] == "rot":
        rows = case["t"] * (case["hq"] + case["hk"])
        return {"bytes": 2 * rows * case["d"] * es + case["t"] * case["axes"] * 4, "flops": 3 * rows * case["rot"]}
    q, kv, p = _lens(case["q"]), _lens(case["kv"]), case["p"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = 0
    for a, b in zip(q, kv):
        pairs += a * p
        if case["causal"]:
            pairs += sum(min(max(b - a + u + 1, 0), b) for u in range(a))
        else:
            pairs += a * b
    return {"bytes": 2 * sum(q) * hq * d * es + 2 * (p + sum(kv)) * hkv * d * es, "flops": 4 * hq * d * pairs}


# ---- 64 bits ------------------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "i8":
        x = st["x"].double()
        biggest = torch.maximum(x.max(1).values, -x.min(1).values)
        # the scale as it is held, in fp32: the fp32 quotient of two fp32 numbers is the float64 one, rounded
        s = (biggest / 127.0).float().double().clamp(min=2.0 ** -126)
        q = x / s.view(-1, 1)
        low = torch.floor(q)
        part = q - low
        odd = torch.remainder(low, 2.0)
        codes = low + ((part > 0.5) | ((part == 0.5) & (odd == 1))).double()
        w = st["codes"][:, :case["k"]].double()
        y = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        for a in range(0, case["m"], 8192):
            y[a:a + 8192] = torch.matmul(codes[a:a + 8192], w.T) * s[a:a + 8192].view(-1, 1)
        y *= st["scales"].double()
        if st["bias"] is not None:
            y += st["bias"].double()
        return y * torch.sigmoid(y) if case["act"] else y
    if case["kind"] == "rot":
        pairs = case["rot"] // 2
        sizes = st["sections"] or [pairs]
        pos = st["pos"].view(case["axes"], -1).double()
        a = torch.cat([pos[i].view(-1, 1) * st["freq"][sum(sizes[:i]):sum(sizes[:i + 1])] for i in range(len(sizes))], 1)
        turn = torch.polar(torch.full_like(a, 1.125), a).unsqueeze(1)

        def rotated(x):
            if x is None:
                return None
            y = x.double().clone()
            first, second = (slice(0, case["rot"], 2), slice(1, case["rot"], 2)) if case["inter"] else \
                (slice(0, pairs), slice(pairs, case["rot"]))
            z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y
        return rotated(st["q"]), rotated(st["k"])
    out, s, t = [], 0, 0
    hq, hkv = case["hq"], case["hkv"]
    if sum(_lens(case["q"])) * (case["p"] + max(st["kv_lens"])) * hq > 3e9:
        return None
    for n, m in zip(st["q_lens"], st["kv_lens"]):
        q = st["q"][s:s + n].double()
        k = torch.cat([st["pk"].double(), st["k"][t:t + m].double()])
        v = torch.cat([st["pv"].double(), st["v"][t:t + m].double()])
        at = torch.arange(case["p"] + m, device="cuda")[None]
        last = case["p"] + (m - n + torch.arange(n, device="cuda")[:, None] if case["causal"] else m)
        o = torch.zeros_like(q)
        for h in range(hq):
            e = torch.matmul(q[:, h], k[:, h // (hq // hkv)].T) / math.sqrt(case["d"])
            e = e.masked_fill((at > last) & (at >= case["p"]), -math.inf)
            o[:, h] = torch.matmul(torch.softmax(e, -1), v[:, h // (hq // hkv)])
        out.append(o)
        s, t = s + n, t + m
    return torch.cat(out)
