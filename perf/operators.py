"""Operator cases: normalisation, positions and attention over the pixels of feature maps.

Each case is one pass through an operator that a vision block runs between its
1x1 convolutions, on NHWC maps whose pixels are the tokens (several frames in a
row are a clip):

  op "norm"    group norm with an activation over [batch][pixels][channels]
  op "rotary"  rotary positions with one to three axes (time, height, width) on
               the query and key heads of a packed q|k|v map
  op "attn"    attention with optional score cap, distance bias, document mask,
               prefix mask, fewer key heads than query heads

`own` selects the framework's kernels; otherwise `run` is the plain form in
elementary torch operations, 32 bits inside (64 for angles), rounded once.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "f16": 2, "bf16": 2}


def _case(name, **kw):
    return dict(kw, name=name) if name else kw


def _norm(name, dtype, batch, h, w, c, groups, act):
    return _case(name, op="norm", dtype=dtype, batch=batch, h=h, w=w, c=c, groups=groups, act=act)


def _rotary(name, dtype, batch, t, h, w, heads, rest, d, nt, nh, nw, shared, adjacent, far):
    return _case(name, op="rotary", dtype=dtype, batch=batch, t=t, h=h, w=w, heads=heads,
                 rest=rest, d=d, nt=nt, nh=nh, nw=nw, shared=shared, adjacent=adjacent, far=far)


def _attn(name, dtype, batch, lq, lk, heads, kv_heads, d, cap=0.0, grid_w=0, docs=0,
          causal=False, prefix=False, ragged=False, layout=1):
    return _case(name, op="attn", dtype=dtype, batch=batch, lq=lq, lk=lk, heads=heads,
                 kv_heads=kv_heads, d=d, cap=cap, grid_w=grid_w, docs=docs, causal=causal,
                 prefix=prefix, ragged=ragged, layout=layout)


def listed():
    return [
        # one image's late map: the smallest call, launch latency counts
        _norm("norm_f16_b1_14x14x256", "f16", 1, 14, 14, 256, 32, "silu"),
        # a full batch of early maps: pure streaming
        _norm("norm_bf16_b64_56x56x256", "bf16", 64, 56, 56, 256, 32, "relu"),
        # odd maps, groups of ten channels, fp32
        _norm("norm_f32_b5_27x29x320", "f32", 5, 27, 29, 320, 32, "silu"),
        # two clips of eight frames, 16 query and 8 key heads of a packed map
        _rotary("rotary_clip_bf16", "bf16", 2, 8, 28, 28, 24, 8, 64, 8, 12, 12, True, False, 0),
        # one new token for each of 33 streams, far into them
        _rotary("rotary_single_f16", "f16", 33, 1, 1, 1, 40, 8, 128, 16, 24, 24, False, False,
                1000000),
        # odd fp32 images, two axes, neighbouring elements paired
        _rotary("rotary_image_f32", "f32", 3, 1, 57, 43, 16, 8, 80, 0, 20, 20, False, True, 0),
        # one small fp32 map batch: the smallest attention call
        _attn("attn_map_f32_b3_14x14", "f32", 3, 196, 196, 8, 8, 32, layout=2),
        # mid maps with a bias by the distance of two pixels
        _attn("attn_distance_bf16_b8_32x32", "bf16", 8, 1024, 1024, 16, 16, 64, grid_w=32),
        # nine images of different sizes packed into one row, capped scores, 3 query heads a key head
        _attn("attn_documents_f16_cap", "f16", 1, 8191, 8191, 12, 4, 128, cap=30.0, docs=9),
        # causal after a prefix that everybody sees, a head size between the powers of two
        _attn("attn_prefix_bf16", "bf16", 2, 4099, 4099, 16, 2, 80, docs=1, causal=True, prefix=True),
        # single tokens of 16 streams against caches of up to 16384 tokens
        _attn("attn_single_f16_b16", "f16", 16, 1, 16384, 32, 8, 128, ragged=True),
        # a batch of large maps: the most arithmetic
        _attn("attn_map_bf16_b4_64x64", "bf16", 4, 4096, 4096, 16, 16, 128),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    dtype = rng.choice(["f32", "f16", "bf16", "f16", "bf16"])
    op = rng.choice(["norm", "rotary", "attn", "attn"])
    if op == "norm":
        groups, per = rng.choice([1, 4, 8, 16, 32]), rng.choice([2, 4, 5, 8, 10, 16, 24, 32])
        c = groups * per
        while c % 8:
            c, per = c * 2, per * 2
        h, w = log(3, 112), log(3, 112)
        room = 60_000_000 // (h * w * c * ESZ[dtype])
        return _norm(None, dtype, min(log(1, 64), max(1, room)), h, w, c, groups,
                     rng.choice(["none", "relu", "relu6", "silu", "gelu"]))
    if op == "rotary":
        d = rng.choice([32, 40, 64, 80, 128, 160])
        nt, nh, nw = rng.choice([(d // 2, 0, 0), (0, d // 4, d // 4), (d // 8, d // 8, d // 8)])
        t, h, w = (rng.randint(1, 16), log(2, 56), log(2, 56)) if nt and nh else (
            (1, log(2, 80), log(2, 80)) if nh else (log(1, 4000), 1, 1))
        heads, rest = rng.choice([(8, 4), (24, 8), (40, 8), (6, 3), (2, 1)])
        room = 100_000_000 // (t * h * w * (heads + rest) * d * ESZ[dtype])
        return _rotary(None, dtype, min(log(1, 33), max(1, room)), t, h, w, heads, rest, d, nt, nh,
                       nw, rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice([0, 1000, 1000000]))
    d = rng.choice([32, 40, 64, 80, 96, 128, 160, 256])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8])
    heads = kv_heads * group
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    kind = rng.choice(["map", "docs", "prefix", "single"])
    layout = rng.choice([1, 2])
    if kind == "single":
        lk = log(64, 32768)
        batch = min(log(1, 32), max(1, 300_000_000 // (lk * kv_heads * d * ESZ[dtype])))
        return _attn(None, dtype, batch, rng.choice([1, 1, 2, 5]), lk, heads, kv_heads, d, cap,
                     ragged=True, layout=1)
    if kind == "map":
        h, w = log(5, 64), log(5, 64)
        batch = max(1, min(log(1, 16), 60_000_000 // (h * w * h * w * heads)))
        return _attn(None, dtype, batch, h * w, h * w, heads, kv_heads, d, cap,
                     grid_w=rng.choice([0, w]), layout=layout)
    n = log(40, 4500)
    batch = max(1, min(log(1, 8), 60_000_000 // (n * n * heads)))
    docs = 1 if kind == "prefix" else rng.randint(2, 12)
    return _attn(None, dtype, batch, n, n, heads, kv_heads, d, cap, docs=docs,
                 causal=kind == "prefix" or rng.random() < 0.5, prefix=kind == "prefix",
                 layout=layout)


# ---- what a case's sizes say, without its seed ----

def _documents(c):
    """[batch][docs + 1] offsets and [batch][docs] prefix lengths of an attn case."""
    r = random.Random(repr([c[k] for k in ("batch", "lq", "lk", "docs", "ragged", "prefix")]))
    offsets, prefix = [], []
    for _ in range(c["batch"]):
        if c["ragged"]:          # one document: the filled part of a cache
            end = max(c["lq"], int(c["lk"] * r.uniform(0.5, 1.0)))
            cuts = [0, end]
        else:
            inner = sorted(r.randint(0, c["lk"]) for _ in range(max(0, c["docs"] - 1)))
            cuts = [0] + inner + [c["lk"]]
        offsets.append(cuts)
        prefix.append([int((b - a) * r.uniform(0.1, 0.4)) if c["prefix"] else 0
                       for a, b in zip(cuts, cuts[1:])])
    return offsets, prefix


def _visible(c):
    """Visible (query, key) pairs of one head, all batch items."""
    if not (c["docs"] or c["ragged"]):
        return c["batch"] * c["lq"] * c["lk"]
    offsets, prefix = _documents(c)
    total = 0
    for cuts, pre in zip(offsets, prefix):
        for a, b, p in zip(cuts, cuts[1:], pre):
            n = b - a
            if c["ragged"]:
                total += c["lq"] * n
            elif c["causal"]:
                total += p * p + (n - p) * (n + p + 1) // 2 if p else n * (n + 1) // 2
            else:
                total += n * n
    return total


def work(case):
    c, e = case, ESZ[case["dtype"]]
    if c["op"] == "norm":
        n = c["batch"] * c["h"] * c["w"] * c["c"]
        return {"bytes": 2 * n * e + 8 * c["c"], "flops": 10 * n}
    if c["op"] == "rotary":
        n = c["batch"] * c["t"] * c["h"] * c["w"]
        axes = sum(1 for k in ("nt", "nh", "nw") if c[k])
        pairs = c["nt"] + c["nh"] + c["nw"]
        return {"bytes": n * (2 * c["heads"] * c["d"] * e + 4 * axes),
                "flops": n * pairs * (6 * c["heads"] + 4)}
    keys = sum(o[-1] for o in _documents(c)[0]) if c["ragged"] else c["batch"] * c["lk"]
    io = (2 * c["batch"] * c["lq"] * c["heads"] + 2 * keys * c["kv_heads"]) * c["d"] * e
    return {"bytes": io, "flops": 4 * c["d"] * c["heads"] * _visible(c)}


# ---- inputs ----

def prepare(case, seed):
    c, dt = case, TORCH[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = {"case": c, "op": c["op"]}
    if c["op"] == "norm":
        pixels, ch = c["h"] * c["w"], c["c"]
        x = normal(c["batch"], pixels, ch) * (0.5 + normal(ch).abs()) + normal(ch)
        s["x"] = x.to(dt)
        s["gamma"] = 1.0 + 0.2 * normal(ch)
        s["beta"] = 0.2 * normal(ch)
        s["eps"] = 1e-5
        s["y"] = torch.empty_like(s["x"])
        s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        return s
    if c["op"] == "rotary":
        n = c["t"] * c["h"] * c["w"]
        s["x"] = normal(c["batch"], n, c["heads"] + c["rest"], c["d"]).to(dt)
        s["y"] = torch.empty(c["batch"], n, c["heads"], c["d"], dtype=dt, device="cuda")
        i = torch.arange(n, device="cuda")
        axes = [i // (c["h"] * c["w"]), i // c["w"] % c["h"], i % c["w"]]
        pairs = [c["nt"], c["nh"], c["nw"]]
        start = torch.randint(0, c["far"] + 1, (c["batch"], 1, 1), device="cuda", generator=g)
        pos = torch.stack([a for a, p in zip(axes, pairs) if p], 1)[None] + start
        s["pos"] = pos.to(torch.int32).contiguous()
        s["pairs"] = tuple(p for p in pairs if p)
        return s
    b, lq, lk, h, hk, d = (c[k] for k in ("batch", "lq", "lk", "heads", "kv_heads", "d"))
    if c["layout"] == 2:         # q|k|v of one packed map
        x = normal(b, lq, h + 2 * hk, d).to(dt)
        s["q"], s["k"], s["v"] = x[:, :, :h], x[:, :, h:h + hk], x[:, :, h + hk:]
    else:
        s["q"] = normal(b, lq, h, d).to(dt)
        s["k"] = normal(b, lk, hk, d).to(dt)
        s["v"] = normal(b, lk, hk, d).to(dt)
    if c["cap"]:                 # scores that reach the cap
        s["q"] = s["q"] * 4
    s["out"] = torch.empty(b, lq, h, d, dtype=dt, device="cuda")
    s["scale"] = 1.0 / math.sqrt(d)
    s["spans"] = torch.empty(b, lq, 2, dtype=torch.int32, device="cuda")
    s["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    if c["docs"] or c["ragged"]:
        offsets, prefix = _documents(c)
        s["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda")
        ends = [o[-1] - lq if c["ragged"] else 0 for o in offsets]
        s["start"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if c["grid_w"]:
        i = torch.arange(lk, device="cuda")
        s["pos"] = torch.stack([i // c["grid_w"], i % c["grid_w"]], 1).to(torch.int32)[None].contiguous()
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(h, device="cuda") + 1) / h)
        s["slopes"] = s["slopes"].to(torch.float32) * (0.5 + torch.rand(h, device="cuda", generator=g))
    return s


# ---- one pass ----

def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "attn": _plain_attn}[s["op"]](s, c)


def _own(s, c):
    import paper_2507_18748_amd as lib
    stream = torch.cuda.current_stream().cuda_stream
    if s["op"] == "norm":
        lib.group_norm(s["x"].data_ptr(), s["y"].data_ptr(), c["dtype"], c["batch"],
                       c["h"] * c["w"], c["c"], c["groups"], s["gamma"].data_ptr(),
                       s["beta"].data_ptr(), s["eps"], c["act"], s["ws"].data_ptr(),
                       s["ws"].numel(), stream)
        return s["y"]
    if s["op"] == "rotary":
        x, y = s["x"], s["y"]
        lib.rotary(x.data_ptr(), y.data_ptr(), c["dtype"], c["batch"], x.shape[1], c["heads"],
                   c["d"], s["pairs"], s["pos"].data_ptr(), x.shape[1] * len(s["pairs"]),
                   x.stride()[:3], y.stride()[:3], 10000.0, c["shared"], c["adjacent"], stream)
        return y
    q, k, v, out = s["q"], s["k"], s["v"], s["out"]
    spans = 0
    if "offsets" in s:
        spans = s["spans"].data_ptr()
        lib.attention_spans(spans, c["batch"], c["lq"], c["lk"], s["offsets"].data_ptr(),
                            s["offsets"].shape[1] - 1, s["prefix"].data_ptr(), c["causal"],
                            s["start"].data_ptr(), stream)
    pos = s["pos"].data_ptr() if "pos" in s else 0
    lib.attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), c["dtype"],
                  c["batch"], c["lq"], c["lk"], c["heads"], c["kv_heads"], c["d"],
                  q.stride()[:3], k.stride()[:3], v.stride()[:3], out.stride()[:3],
                  s["scale"], c["cap"], s["slopes"].data_ptr() if pos else 0, pos, pos,
                  2 if pos else 0, 0, 0, spans, 2 * c["lq"], s["ws"].data_ptr(),
                  s["ws"].numel(), stream)
    return out


def _plain_norm(s, c):
    x = s["x"].float().view(c["batch"], c["h"] * c["w"], c["groups"], -1)
    mean = x.mean((1, 3), keepdim=True)
    var = (x - mean).square().mean((1, 3), keepdim=True)
    y = ((x - mean) * (var + s["eps"]).rsqrt()).view(c["batch"], -1, c["c"])
    y = y * s["gamma"] + s["beta"]
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "relu6":
        y = y.clamp(0, 6)
    elif c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    elif c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["x"].dtype)


def _frequencies(c, pairs):
    """Rotations per position of every pair, and its axis."""
    total = sum(pairs)
    f, axis = [], []
    for a, n in enumerate(pairs):
        for i in range(n):
            e = len(f) / total if c["shared"] else i / n
            f.append(10000.0 ** -e)
            axis.append(a)
    return f, axis


def _plain_rotary(s, c):
    x = s["x"][:, :, :c["heads"]].float()
    f, axis = _frequencies(c, s["pairs"])
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    angle = s["pos"].double()[:, :, torch.tensor(axis, device="cuda")] * f
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    n = len(axis)
    if c["adjacent"]:
        u, w = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        r = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)
    else:
        u, w = x[..., :n], x[..., n:2 * n]
        r = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
    return torch.cat([r, x[..., 2 * n:]], -1).to(s["x"].dtype)


def _plain_spans(s, c):
    """First and last visible key of every query, [batch][lq]."""
    p = s["start"][:, None] + torch.arange(c["lq"], device="cuda")
    doc = torch.searchsorted(s["offsets"][:, 1:].contiguous(), p.to(torch.int32), right=True)
    lo = s["offsets"].gather(1, doc)
    hi = s["offsets"].gather(1, doc + 1)
    if c["causal"]:
        hi = torch.minimum(hi, torch.maximum(p + 1, lo + s["prefix"].gather(1, doc)))
    return lo, hi


def _plain_attn(s, c):
    b, lq, lk, h, hk, d = (c[k] for k in ("batch", "lq", "lk", "heads", "kv_heads", "d"))
    q = s["q"].float().view(b, lq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    k = s["k"].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"].float().permute(0, 2, 1, 3).contiguous()
    sc = torch.matmul(q, k).mul_(s["scale"]).view(b, hk, h // hk, lq, lk)
    if c["cap"]:
        sc = sc.div_(c["cap"]).tanh_().mul_(c["cap"])
    if "pos" in s:
        dist = (s["pos"][:, :, None] - s["pos"][:, None]).abs().sum(-1).float()
        sc -= s["slopes"].view(1, hk, -1, 1, 1) * dist[:, None, None]
    if "offsets" in s:
        lo, hi = _plain_spans(s, c)
        j = torch.arange(lk, device="cuda")
        seen = (j >= lo[..., None]) & (j < hi[..., None])
        sc.masked_fill_(~seen[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True).clamp(min=-1e30)
    e = sc.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(b, hk, -1, lk), v).view(b, hk, -1, lq, d)
    o = o / total.clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(b, lq, h, d).to(s["q"].dtype)


# ---- from the definitions, in 64 bits ----

def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        out = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
        per = c["c"] // c["groups"]
        for n in range(c["batch"]):
            x = s["x"][n].double()
            sums = x.sum(0).view(c["groups"], per).sum(1) / (x.shape[0] * per)
            mu = sums.repeat_interleave(per)
            var = ((x - mu) ** 2).sum(0).view(c["groups"], per).sum(1) / (x.shape[0] * per)
            z = (x - mu) / torch.sqrt(var + s["eps"]).repeat_interleave(per)
            z = z * s["gamma"].double() + s["beta"].double()
            if c["act"] == "relu":
                z = torch.where(z > 0, z, torch.zeros_like(z))
            elif c["act"] == "relu6":
                z = torch.minimum(torch.maximum(z, torch.zeros_like(z)), torch.full_like(z, 6.0))
            elif c["act"] == "silu":
                z = z * torch.sigmoid(z)
            elif c["act"] == "gelu":
                z = z * torch.erfc(-z / math.sqrt(2.0)) / 2
            out[n] = z
        return out
    if c["op"] == "rotary":
        x = s["x"][:, :, :c["heads"]].double()
        out = x.clone()
        start, total = 0, sum(s["pairs"])
        for a, n in enumerate(s["pairs"]):
            for i in range(n):
                p = start + i
                f = math.exp(-math.log(10000.0) * (p / total if c["shared"] else i / n))
                t = s["pos"][:, :, a].double() * f
                i0, i1 = (2 * p, 2 * p + 1) if c["adjacent"] else (p, p + total)
                z = torch.complex(x[..., i0], x[..., i1]) * torch.polar(torch.ones_like(t), t)[:, :, None]
                out[..., i0], out[..., i1] = z.real, z.imag
            start += n
        return out
    b, lq, h, hk, d = (c[k] for k in ("batch", "lq", "heads", "kv_heads", "d"))
    out = torch.zeros(b, lq, h, d, dtype=torch.float64, device="cuda")
    j = torch.arange(c["lk"], device="cuda")
    offsets, prefix = _documents(c)
    for n in range(b):
        seen = torch.ones(lq, c["lk"], dtype=torch.bool, device="cuda")
        if c["docs"] or c["ragged"]:
            seen.zero_()
            for a, e, pre in zip(offsets[n], offsets[n][1:], prefix[n]):
                first = offsets[n][-1] - lq if c["ragged"] else 0
                for_rows = slice(max(a - first, 0), max(0, min(e - first, lq)))
                part = (j >= a) & (j < e)
                p = torch.arange(first, first + lq, device="cuda")[for_rows, None]
                seen[for_rows] = part & ((j <= p) | (j < a + pre)) if c["causal"] else part
        some = seen.any(1, keepdim=True)
        for m in range(h):
            q, k, v = (s[x][n, :, m if x == "q" else m // (h // hk)].double() for x in "qkv")
            z = (q @ k.t()) / math.sqrt(d)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if "pos" in s:
                xy = s["pos"][0].double()
                z -= s["slopes"][m].double() * torch.cdist(xy, xy, p=1.0)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            w = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
            out[n, :, m] = torch.where(some, torch.where(seen, w, torch.zeros_like(w)) @ v,
                                       torch.zeros_like(v[:1]))
    return out
