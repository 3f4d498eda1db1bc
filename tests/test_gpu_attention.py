"""Attention and its spans against a 64-bit reference on an MI355X."""
import math

import pytest

torch = pytest.importorskip("torch")

import operator_ref as R
from paper_2507_18748_amd import (PpipeError, attention, attention_desc, attention_spans,
                                  attention_workspace)

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "f16", "bf16"]


def call(q, k, v, out, dtype, scale, cap=0.0, slopes=None, qpos=None, kpos=None, span=None,
         stream=None, ws=None):
    n, lq, h, d = q.shape
    lk, hk = k.shape[1], k.shape[2]
    axes = 0 if slopes is None else qpos.shape[-1]
    bs = lambda t: 0 if t is None or t.shape[0] == 1 else t.stride(0)
    st = [t.stride()[:3] for t in (q, k, v, out)]
    desc = attention_desc(dtype, n, lq, lk, h, hk, d, *st, scale, cap, axes, bs(qpos), bs(kpos),
                          bs(span))
    need = attention_workspace(desc)
    own = ws is None
    if own:
        ws = torch.full((need + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    p = lambda t: 0 if t is None else t.data_ptr()
    s = stream or torch.cuda.current_stream()
    attention(q.data_ptr(), p(k), p(v), out.data_ptr(), dtype, n, lq, lk, h, hk, d, *st, scale,
              cap, p(slopes), p(qpos), p(kpos), axes, bs(qpos), bs(kpos), p(span), bs(span),
              ws.data_ptr(), need if own else ws.numel(), s.cuda_stream)
    if own:
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0x5A).all()), "wrote beyond its workspace"
    return out


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def tensors(dtype, n, lq, lk, h, hk, d, seed=0, packed=False, size=1.0, gap=0):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    if packed:
        x = r(n, lq, h + 2 * hk, d).to(R.TORCH[dtype])
        q, k, v = x[:, :, :h], x[:, :, h:h + hk], x[:, :, h + hk:]
    else:
        q = r(n, lq, h, d + gap).to(R.TORCH[dtype])[..., :d]
        k = r(n, hk, lk, d + gap).to(R.TORCH[dtype])[..., :d].transpose(1, 2)
        v = r(n, lk, hk, d + gap).to(R.TORCH[dtype])[..., :d]
    return q * size if size != 1.0 else q, k, v


def guarded(n, lq, h, d, dtype):
    """An output with a head and a token of guards behind each."""
    return torch.full((n, lq + 1, h + 1, d), 7.0, device="cuda").to(R.TORCH[dtype])[:, :lq, :h]


def case(dtype, n, lq, lk, h, hk, d, span=None, cap=0.0, slopes=None, qpos=None, kpos=None,
         seed=0, packed=False, size=1.0, gap=0):
    print(f"[attention] {dtype} {n}x{lq}x{lk} heads={h}/{hk} d={d} span={span is not None} "
          f"cap={cap} bias={slopes is not None}", flush=True)
    q, k, v = tensors(dtype, n, lq, lk, h, hk, d, seed, packed, size, gap)
    scale = 1.0 / math.sqrt(d)
    out = guarded(n, lq, h, d, dtype)
    call(q, k, v, out, dtype, scale, cap, slopes, qpos, kpos, span)
    ex = lambda t: None if t is None else t.expand(n, *t.shape[1:])
    ref, bound = R.attention(q, k, v, scale, cap, slopes, ex(qpos), ex(kpos), ex(span), dtype)
    R.check(out, ref, bound, dtype)
    whole = out._base
    assert bool((whole[:, lq:] == 7.0).all()) and bool((whole[:, :, h:] == 7.0).all())
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,lq,lk,h,hk,d", [
    (1, 1, 1, 1, 1, 8), (2, 1, 3, 2, 1, 16), (1, 5, 2, 3, 3, 24), (1, 31, 33, 2, 2, 32),
    (2, 64, 64, 1, 1, 64), (1, 65, 63, 4, 2, 40), (1, 129, 127, 2, 1, 80), (3, 49, 196, 6, 2, 96),
    (1, 196, 196, 8, 8, 32), (1, 300, 257, 4, 1, 128), (1, 33, 70, 3, 1, 136), (1, 40, 200, 2, 2, 160),
    (1, 70, 90, 2, 1, 192), (1, 100, 333, 2, 2, 256), (1, 37, 65, 5, 1, 248), (1, 513, 1025, 2, 2, 72),
    (1, 4, 100, 16, 1, 64), (2, 3, 70, 64, 2, 32), (1, 130, 64, 96, 1, 32), (1, 7, 0, 2, 1, 32),
])
def test_sizes(dtype, n, lq, lk, h, hk, d):
    case(dtype, n, lq, lk, h, hk, d)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,h,hk,lk,d", [
    (1, 1, 1, 1000, 64), (3, 8, 2, 4097, 128), (1, 32, 8, 20000, 128), (5, 4, 4, 777, 80),
    (2, 40, 1, 3000, 64), (1, 2, 1, 9999, 256), (17, 2, 2, 300, 32), (1, 16, 1, 70001, 40),
])
def test_single_tokens(dtype, n, h, hk, lk, d):
    """One query against a long cache, filled to different lengths, a shared
    span row and a batch item without any key among them."""
    g = torch.Generator().manual_seed(3)
    ends = torch.randint(0, lk + 1, (n,), generator=g)
    ends[0] = lk
    if n > 1:
        ends[n - 1] = 0
    span = torch.stack([torch.zeros_like(ends), ends], -1).to(torch.int32)[:, None].cuda().contiguous()
    case(dtype, n, 1, lk, h, hk, d, span)
    case(dtype, n, 2, lk, h, hk, d)


def bias(h, lq, lk, axes, seed=0, shared=True, n=1, step=1):
    g = gen(seed)
    slopes = (0.02 + 0.3 * torch.rand(h, device="cuda", generator=g)) * torch.sign(
        torch.randn(h, device="cuda", generator=g))
    slopes[0] = 0.0
    pos = lambda l: (torch.randint(-40, 40, (1 if shared else n, l, axes), device="cuda",
                                   generator=g, dtype=torch.int32) * step).contiguous()
    return slopes, pos(lq), pos(lk)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("axes", [1, 2, 3])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("lq,lk", [(70, 150), (1, 700)])
def test_bias_and_cap(dtype, axes, cap, lq, lk):
    n = 2
    slopes, qpos, kpos = bias(4, lq, lk, axes, shared=cap > 0, n=n)
    case(dtype, n, lq, lk, 4, 2, 64, None, cap, slopes, qpos, kpos, size=4.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [32, 128])
@pytest.mark.parametrize("cap", [1e-3, 20.0, 1e4])
def test_cap(dtype, d, cap):
    case(dtype, 1, 80, 130, 2, 1, d, cap=cap, size=6.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [-0.125, 0.0, 1e-15, 2.0])
@pytest.mark.parametrize("extra", ["none", "cap", "bias", "both"])
@pytest.mark.parametrize("lq", [1, 70])
def test_scales(dtype, scale, extra, lq):
    lk = 130
    q, k, v = tensors(dtype, 1, lq, lk, 2, 2, 64)
    slopes, qpos, kpos = bias(2, lq, lk, 2) if extra in ("bias", "both") else (None, None, None)
    cap = 7.0 if extra in ("cap", "both") else 0.0
    out = call(q, k, v, torch.empty_like(q, memory_format=torch.contiguous_format), dtype, scale,
               cap, slopes, qpos, kpos)
    ref, bound = R.attention(q, k, v, scale, cap, slopes, qpos, kpos, dtype=dtype)
    R.check(out, ref, bound, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("cap", [1000.0, 1e6, 1e30])
@pytest.mark.parametrize("biased", [False, True])
def test_large_caps_keep_the_scores(dtype, cap, biased):
    """A cap far above the scores leaves them as they are: within a few roundings of
    the score itself above 1024, and of the cap below."""
    lq, lk = 60, 300
    q, k, v = tensors(dtype, 1, lq, lk, 2, 1, 64, size=4.0)
    slopes, qpos, kpos = bias(2, lq, lk, 1) if biased else (None, None, None)
    out = call(q, k, v, torch.empty_like(q, memory_format=torch.contiguous_format), dtype, 0.125,
               cap, slopes, qpos, kpos)
    ref, bound = R.attention(q, k, v, 0.125, 0.0 if cap > 1024 else cap, slopes, qpos, kpos, dtype=dtype)
    if cap > 1024:      # x^3 / 3 of x = score / cap: below 1e-9 of the score from 1e6 on
        size = float((q.double().norm(dim=-1).max() * k.double().norm(dim=-1).max()) * 0.125)
        bound = bound + 2 * size * (size / 1e6) ** 2 * float(v.abs().max())
    R.check(out, ref, bound, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lk", [40, 900, 20000])
def test_nan_queries_and_keys(dtype, lk):
    """A NaN query gives NaN at any split of its keys, and so does one NaN among
    the keys it sees; other heads and items do not notice."""
    q, k, v = tensors(dtype, 2, 1, lk, 2, 2, 64)
    k, v = k.contiguous(), v.contiguous()
    clean = call(q, k, v, torch.empty_like(q, memory_format=torch.contiguous_format), dtype, 0.125)
    q2 = q.clone()
    q2[0, 0, 1, 3] = float("nan")
    out = call(q2, k, v, torch.empty_like(clean), dtype, 0.125)
    assert bool(torch.isnan(out[0, 0, 1]).all())
    assert torch.equal(out[1], clean[1]) and torch.equal(out[0, 0, 0], clean[0, 0, 0])
    k[1, lk // 3, 0, 0] = float("nan")
    out = call(q, k, v, torch.empty_like(clean), dtype, 0.125)
    assert bool(torch.isnan(out[1, 0, 0]).all())
    assert torch.equal(out[0], clean[0]) and torch.equal(out[1, 0, 1], clean[1, 0, 1])


@pytest.mark.parametrize("lk", [300, 40000])
def test_many_small_weights(lk):
    """One key of weight near one and thousands of e^-17 each: their sum is not
    lost to the small end of f16."""
    d = 32
    q = torch.zeros(1, 1, 1, d, device="cuda", dtype=torch.float16)
    k = torch.zeros(1, lk, 1, d, device="cuda", dtype=torch.float16)
    q[..., 0], k[0, 7, 0, 0] = 1.0, 17.0
    v = torch.ones(1, lk, 1, d, device="cuda", dtype=torch.float16)
    v[0, 7] = 0.0
    out = call(q, k, v, torch.empty_like(q), "f16", 1.0)
    # each weight is rounded once: 2^6 e^-17 = 2.6e-6 has steps of 2^-24, half of one is 0.0114 of it
    want = (lk - 1) * math.exp(-17) / (1 + (lk - 1) * math.exp(-17))
    assert float((out.double() / want - 1).abs().max()) <= 2.0 ** -25 / (64 * math.exp(-17)) + 4 * R.U["f16"] + 2.0 ** -25 / want


def test_far_positions_keep_their_distance():
    """Distances of 32-bit positions are exact before they are rounded to fp32."""
    slopes = torch.tensor([0.01, 1.0], device="cuda")
    base = (1 << 30) + 1
    qpos = torch.arange(base, base + 40, dtype=torch.int32, device="cuda").view(1, 40, 1)
    kpos = torch.arange(base - 5, base + 60, dtype=torch.int32, device="cuda").view(1, 65, 1)
    case("f32", 1, 40, 65, 2, 2, 32, None, 0.0, slopes, qpos.contiguous(), kpos.contiguous())


def make_spans(n, lq, lk, offsets=None, prefix=None, causal=False, start=None):
    t = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    off, pre, st = t(offsets), t(prefix), t(start)
    out = torch.full((n, lq + 1, 2), -5, dtype=torch.int32, device="cuda")
    p = lambda x: 0 if x is None else x.data_ptr()
    flat = torch.full((n * lq + 1, 2), -5, dtype=torch.int32, device="cuda")
    attention_spans(flat.data_ptr(), n, lq, lk, p(off), 1 if offsets is None else len(offsets[0]) - 1,
                    p(pre), causal, p(st), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert bool((flat[n * lq:] == -5).all())
    got = flat[:n * lq].view(n, lq, 2).contiguous()
    want = R.spans(n, lq, lk, offsets, prefix, causal, start)
    want = [[(0, 0) if lo >= hi else (lo, hi) for lo, hi in r] for r in want]
    mine = [[(0, 0) if lo >= hi else (lo, hi) for lo, hi in r] for r in got.tolist()]
    assert mine == want
    del out
    return got


SPAN_CASES = {
    "causal": dict(n=2, lq=150, lk=150, causal=True),
    "causal, later queries": dict(n=2, lq=70, lk=200, causal=True, start=[130, 17]),
    "prefix": dict(n=2, lq=200, lk=200, causal=True, offsets=[[0, 200], [0, 200]],
                   prefix=[[60], [0]]),
    "prefix longer than the document": dict(n=1, lq=90, lk=90, causal=True, offsets=[[0, 30, 90]],
                                            prefix=[[50, 10]]),
    "documents": dict(n=1, lq=333, lk=333, offsets=[[0, 1, 1, 64, 200, 201, 333]]),
    "documents, causal": dict(n=2, lq=260, lk=260, causal=True,
                              offsets=[[0, 100, 130, 260], [0, 0, 259, 260]]),
    "padding before and behind": dict(n=2, lq=180, lk=180, offsets=[[20, 60, 150], [0, 3, 90]]),
    "outside the keys": dict(n=1, lq=50, lk=40, offsets=[[-7, 10, 99]], start=[-4]),
    "no document": dict(n=1, lq=70, lk=70, offsets=[[0, 0]]),
    "no key": dict(n=1, lq=9, lk=0),
}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SPAN_CASES))
def test_masks(dtype, name):
    kw = SPAN_CASES[name]
    span = make_spans(**kw)
    case(dtype, kw["n"], kw["lq"], kw["lk"], 4, 2, 64, span)
    case(dtype, kw["n"], kw["lq"], kw["lk"], 2, 2, 40, span, cap=10.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_any_span(dtype):
    """Spans from elsewhere: reversed, negative, beyond the keys, one key, each row its own."""
    g = torch.Generator().manual_seed(5)
    span = torch.randint(-50, 400, (2, 170, 2), generator=g, dtype=torch.int32)
    span[0, 3] = torch.tensor([7, 8])
    span[0, 4] = torch.tensor([-(1 << 31), (1 << 31) - 1])
    span[1, 0] = torch.tensor([(1 << 31) - 1, -(1 << 31)])
    case(dtype, 2, 170, 350, 4, 1, 64, span.cuda())
    case(dtype, 2, 170, 350, 4, 4, 128, span[:1].cuda().contiguous())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lq,lk,d", [(130, 200, 64), (130, 200, 136), (1, 900, 128), (3, 100, 32)])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_hidden_keys_never_reach_an_output(dtype, lq, lk, d, what):
    """NaN and infinities in keys and values that a query does not see, in tiles
    that other queries of its block do see: its output keeps every bit."""
    q, k, v = tensors(dtype, 1, lq, lk, 4, 2, d, seed=8)
    k, v = k.contiguous(), v.contiguous()
    g = torch.Generator().manual_seed(9)
    lo = torch.randint(0, lk // 2, (1, lq), generator=g)
    span = torch.stack([lo, lo + torch.randint(0, lk // 2, (1, lq), generator=g)], -1)
    span = span.to(torch.int32).cuda().contiguous()
    scale = d ** -0.5
    clean = call(q, k, v, torch.empty(1, lq, 4, d, dtype=q.dtype, device="cuda"), dtype, scale, span=span)
    bad = float("nan") if what == "nan" else float("inf")
    at = [0, 5, lk // 3, lk // 2, lk - 1]
    k2, v2 = k.clone(), v.clone()
    for i, j in enumerate(at):
        k2[:, j, :, i % d] = bad
        v2[:, j, :, (i + 3) % d] = -bad
    got = call(q, k2, v2, torch.empty_like(clean), dtype, scale, span=span)
    j = torch.tensor(at, device="cuda")
    hit = ((j[None, None] >= span[..., :1]) & (j[None, None] < span[..., 1:])).any(-1)[0]
    if bool((~hit).any()):          # a few rows may all see one
        # the tiles may be added in another way: no more than a few roundings
        a, b = got[0, ~hit].double(), clean[0, ~hit].double()
        assert bool(torch.isfinite(a).all())
        assert float((a - b).abs().max()) <= 4 * R.U[dtype] * float(b.abs().max())
    else:
        assert lq < 4
    if lq > 1 and what == "nan" and bool(hit.any()):
        assert bool(torch.isnan(got[0, hit].float()).any(-1).all())
    # only the values bad: a query that sees them gets them in their element, no other
    got = call(q, k, v2, torch.empty_like(clean), dtype, scale, span=span)
    for i, jj in enumerate(at):
        e = (i + 3) % d
        sees = (span[0, :, 0] <= jj) & (jj < span[0, :, 1])
        if bool(sees.any()):
            assert not bool(torch.isfinite(got[0, sees][..., e].float()).any())
    fine = torch.ones(d, dtype=torch.bool, device="cuda")
    for i in range(len(at)):
        fine[(i + 3) % d] = False
    assert bool(torch.isfinite(got[..., fine].float()).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,lk,lo,hi", [(128, 900, 37, 500), (64, 70, 5, 6), (80, 5000, 3001, 4999),
                                        (32, 64, 0, 33), (256, 300, 299, 300)])
def test_rest_of_a_cache_is_not_read(dtype, d, lk, lo, hi):
    """One query; everything outside its span is NaN."""
    q, k, v = tensors(dtype, 2, 1, lk, 4, 2, d, seed=12)
    k, v = k.contiguous(), v.contiguous()
    span = torch.tensor([[[lo, hi]]], dtype=torch.int32, device="cuda")
    ref, bound = R.attention(q, k, v, d ** -0.5, span=span.expand(2, -1, -1), dtype=dtype)
    for t in (k, v):
        t[:, :lo] = float("nan")
        t[:, hi:] = float("nan")
    R.check(call(q, k, v, torch.empty_like(q), dtype, d ** -0.5, span=span), ref, bound, dtype)


# Grids beyond one round of 32-row blocks: the waves of a block share key tiles.
# 2100 queries of 8 key heads (a multiple of the XCDs) or 9 of them (not one).
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [24, 64, 80, 128, 160, 256])
@pytest.mark.parametrize("mask", ["none", "documents", "prefix", "any"])
def test_many_rows(dtype, d, mask):
    lq, lk, hk = 2100, 2100 if mask in ("documents", "prefix") else 333, 8 if d in (64, 128) else 9
    kw = dict(n=1, lq=lq, lk=lk)
    span = None
    if mask == "documents":
        span = make_spans(offsets=[[0, 7, 7, 300, 1111, 1500, 2090]], **kw)
    elif mask == "prefix":
        span = make_spans(causal=True, offsets=[[0, 900, 2100]], prefix=[[130, 500]], **kw)
    elif mask == "any":
        g = torch.Generator().manual_seed(11)
        span = torch.randint(-20, 360, (1, lq, 2), generator=g, dtype=torch.int32).cuda()
    case(dtype, 1, lq, lk, hk, hk, d, span)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [32, 72, 128, 200])
@pytest.mark.parametrize("axes,cap", [(0, 6.0), (1, 0.0), (2, 6.0), (3, 0.0), (2, 5000.0)])
def test_many_rows_with_bias_and_cap(dtype, d, axes, cap):
    lq, lk, h, hk = 1100, 190, 16, 8
    slopes, qpos, kpos = bias(h, lq, lk, axes) if axes else (None, None, None)
    g = torch.Generator().manual_seed(13)
    span = torch.stack([torch.zeros(1, lq), torch.randint(0, lk + 1, (1, lq), generator=g)], -1)
    for sp in (None, span.to(torch.int32).cuda().contiguous()):
        case(dtype, 1, lq, lk, h, hk, d, sp, cap, slopes, qpos, kpos, size=3.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 136])
def test_many_rows_do_not_see_hidden_values(dtype, d):
    lq, lk, hk = 2200, 300, 8
    q, k, v = tensors(dtype, 1, lq, lk, hk, hk, d, seed=21)
    k, v = k.contiguous(), v.contiguous()
    g = torch.Generator().manual_seed(22)
    lo = torch.randint(0, lk, (1, lq), generator=g)
    span = torch.stack([lo, lo + torch.randint(0, 90, (1, lq), generator=g)], -1)
    span = span.to(torch.int32).cuda().contiguous()
    bad = [3, 64, 130, 299]
    k[:, bad[1]], v[:, bad[0]], v[:, bad[2], :, 5], v[:, bad[3]] = (float(x) for x in ("nan", "nan", "inf", "-inf"))
    out = call(q, k, v, torch.empty(1, lq, hk, d, dtype=q.dtype, device="cuda"), dtype, d ** -0.5, span=span)
    j = torch.tensor(bad, device="cuda")
    hit = ((j >= span[0, :, :1]) & (j < span[0, :, 1:])).any(-1)
    clean = ~hit
    k2, v2 = k.clone(), v.clone()
    k2[:, bad], v2[:, bad] = 0.0, 0.0
    ref, bound = R.attention(q, k2, v2, d ** -0.5, span=span, dtype=dtype)
    R.check(out[:, clean], ref[:, clean], bound[:, clean], dtype)
    assert int(clean.sum()) > 100 and int(hit.sum()) > 100


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_scores(dtype):
    """All scores -inf: zeros; one +inf: NaN; some -inf: as if hidden."""
    q = torch.ones(1, 40, 1, 32, device="cuda").to(R.TORCH[dtype])
    k = torch.randn(1, 70, 1, 32, device="cuda").to(R.TORCH[dtype])
    v = torch.randn(1, 70, 1, 32, device="cuda").to(R.TORCH[dtype])
    out = torch.empty_like(q)
    k[0, 3, 0, 5] = float("-inf")
    call(q, k, v, out, dtype, 0.2)
    ref, bound = R.attention(q, torch.cat([k[:, :3], k[:, 4:]], 1), torch.cat([v[:, :3], v[:, 4:]], 1),
                             0.2, dtype=dtype)
    R.check(out, ref, bound, dtype)
    k[0, 3, 0, 5] = float("inf")
    assert bool(torch.isnan(call(q, k, v, out, dtype, 0.2)).all())
    k[..., 0] = float("-inf")
    k[0, 3, 0, 5] = 0.0
    assert bool((call(q, k, v, out, dtype, 0.2) == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(dtype):
    """Scores of several hundred: the running maximum moves far from tile to tile."""
    n, lk, d = 1, 300, 32
    q = torch.ones(n, 33, 1, d, device="cuda").to(R.TORCH[dtype])
    k = torch.randn(n, lk, 1, d, device="cuda", generator=gen(4))
    k = (k + torch.linspace(-20, 20, lk, device="cuda")[None, :, None, None]).to(R.TORCH[dtype])
    v = torch.randn(n, lk, 1, d, device="cuda", generator=gen(5)).to(R.TORCH[dtype])
    for kk in (k, k.flip(1).contiguous()):
        out = call(q, kk, v, torch.empty_like(q), dtype, 1.0)
        ref, bound = R.attention(q, kk, v, 1.0, dtype=dtype)
        R.check(out, ref, bound, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("packed,gap", [(True, 0), (False, 8), (False, 24)])
def test_layouts(dtype, packed, gap):
    case(dtype, 2, 77, 77, 4, 2, 64, packed=packed, gap=gap)
    case(dtype, 2, 140, 140, 6, 1, 72, packed=packed, gap=gap)


def test_batch_items_share_a_cache():
    """k and v with a batch stride of 0."""
    q, k, v = tensors("f16", 3, 50, 90, 4, 2, 64)
    k1, v1 = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    out = call(q, k1, v1, torch.empty(3, 50, 4, 64, dtype=torch.float16, device="cuda"), "f16", 0.125)
    ref, bound = R.attention(q, k1, v1, 0.125, dtype="f16")
    R.check(out, ref, bound, "f16")


def test_beyond_32_bit_offsets():
    """Keys whose byte offsets pass 2^32: a cache row of 2^21 elements."""
    d, lk, row = 64, 1100, 1 << 21
    big = torch.zeros(lk * row, dtype=torch.float16, device="cuda")
    g = gen(6)
    k, v = (big.as_strided((1, lk, 1, d), (0, row, d, 1), o) for o in (0, 4096))
    k.copy_(torch.randn(1, lk, 1, d, device="cuda", generator=g))
    v.copy_(torch.randn(1, lk, 1, d, device="cuda", generator=g))
    for lq in (1, 70):
        q = torch.randn(1, lq, 1, d, device="cuda", generator=g).half()
        out = call(q, k, v, torch.empty_like(q), "f16", 0.125)
        ref, bound = R.attention(q, k.contiguous(), v.contiguous(), 0.125, dtype="f16")
        R.check(out, ref, bound, "f16")
    del big, k, v


def test_workspace_too_small_is_refused():
    q, k, v = tensors("f16", 1, 1, 30000, 8, 1, 128)
    out = torch.empty_like(q)
    st = [t.stride()[:3] for t in (q, k, v, out)]
    need = attention_workspace(attention_desc("f16", 1, 1, 30000, 8, 1, 128, *st, 0.1))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for ptr, size in ((0, need), (ws.data_ptr(), need - 1), (ws.data_ptr() + 4, need)):
        with pytest.raises(PpipeError) as e:
            attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), "f16", 1, 1, 30000,
                      8, 1, 128, *st, 0.1, workspace_ptr=ptr, workspace_bytes=size)
        assert e.value.status == -1


@pytest.mark.parametrize("lq,lk", [(200, 200), (1, 5000)])
def test_captured_on_another_stream_and_repeatable(lq, lk):
    q, k, v = tensors("bf16", 2, lq, lk, 4, 2, 64)
    span = make_spans(2, lq, lk, causal=True, start=[lk - lq] * 2)
    want = call(q, k, v, torch.empty(2, lq, 4, 64, dtype=q.dtype, device="cuda"), "bf16", 0.125, span=span)
    ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    sp = torch.zeros_like(span)
    st = torch.tensor([lk - lq] * 2, dtype=torch.int32, device="cuda")
    out = torch.empty_like(want)
    s, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gr, stream=s):
        cs = torch.cuda.current_stream()
        attention_spans(sp.data_ptr(), 2, lq, lk, 0, 1, 0, True, st.data_ptr(), cs.cuda_stream)
        call(q, k, v, out, "bf16", 0.125, span=sp, stream=cs, ws=ws)
    for _ in range(4):
        out.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        assert float((q.float() * 2).abs().max()) > 0      # unrelated eager work
        assert torch.equal(out, want)
