"""Plain 64-bit references of the operators on device tensors, with bounds of
how far a correctly rounded fp32 computation may be from them.

Bounds count roundings: U is half a step of the storage type relative to the
value, F that of fp32 (2^-24)."""
import math

import torch

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
F = 2.0 ** -24
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}   # below the normal range


def activation(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "relu6":
        return z.clamp(0, 6)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z


def group_norm(x, groups, gamma, beta, eps, act):
    """(y, bound) of x [N][P][C]: the mean is off by at most a few dozen fp32
    roundings of the mean magnitude (sums run in partial sums, so their error
    grows with the depth, not the length), the deviation by as many of itself;
    every activation has slope at most 1.13, and its own fp32 evaluation takes a
    few roundings more."""
    n, p, c = x.shape
    v = x.double().view(n, p, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    var = (v - mean).square().mean((1, 3), keepdim=True)
    sd = (var + eps).sqrt()
    ga = torch.ones(c, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    be = torch.zeros(c, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    h = ((v - mean) / sd).view(n, p, c)
    z = h * ga + be
    level = (v.abs().mean((1, 3), keepdim=True) / sd).expand_as(v).reshape(n, p, c)
    size = (v.abs() / sd).reshape(n, p, c)
    dz = 64 * F * ((h.abs() + level + size) * ga.abs() + be.abs())
    return activation(z, act), 1.13 * dz + 16 * F * z.abs() + 1e-37


def rotary(x, pos, pairs, base, shared, adjacent):
    """(y, bound) of x [N][L][H][d] with pos [N][L][A]."""
    out = x.double().clone()
    bound = torch.zeros_like(out)
    total, p = sum(pairs), 0
    for a, n in enumerate(pairs):
        for i in range(n):
            f = base ** -(p / total if shared else i / n)
            t = (pos[:, :, a].double() * f)[:, :, None]
            i0, i1 = (2 * p, 2 * p + 1) if adjacent else (p, p + total)
            u, w = x[..., i0].double(), x[..., i1].double()
            out[..., i0] = u * t.cos() - w * t.sin()
            out[..., i1] = u * t.sin() + w * t.cos()
            # sine and cosine within a few roundings, two products, one sum; and the
            # turn: 64-bit products of the position, then 32 bits of a fraction
            b = (u.abs() + w.abs()) * (16 * F + pos[:, :, a].double().abs()[:, :, None] * f * 2.0 ** -50)
            bound[..., i0] = b
            bound[..., i1] = b
            p += 1
    return out, bound + 1e-37


def spans(batch, lq, lk, offsets=None, prefix=None, causal=False, start=None):
    """[batch][lq] lists of (first, end)."""
    out = []
    for b in range(batch):
        off = [0, lk] if offsets is None else [min(max(int(o), 0), lk) for o in offsets[b]]
        row = []
        for i in range(lq):
            p = i + (0 if start is None else int(start[b]))
            lo = hi = 0
            for d in range(len(off) - 1):
                if off[d] <= p < off[d + 1]:
                    lo, hi = off[d], off[d + 1]
                    if causal:
                        pre = 0 if prefix is None else int(prefix[b][d])
                        hi = min(hi, max(p + 1, lo + pre))
            row.append((lo, hi))
        out.append(row)
    return out


def attention(q, k, v, scale, cap=0.0, slopes=None, qpos=None, kpos=None, span=None, dtype="f32"):
    """(out, bound) of q [N][Lq][H][d], k, v [N][Lk][Hk][d], span [N][Lq][2] or None.

    Masked keys are left out by selection, so what they hold does not matter.
    A score is off by at most (d + 4) roundings of the sum of its products'
    magnitudes, a few of itself and of the bias; weights and sums take a few more
    and one for each key of the longest running sum.  In 16 bits the weights are rounded once
    to the storage type before the products with the values."""
    n, lq, h, d = q.shape
    lk, hk = k.shape[1], k.shape[2]
    out = torch.zeros(n, lq, h, d, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    j = torch.arange(lk, device=q.device)
    for b in range(n):
        seen = torch.ones(lq, lk, dtype=torch.bool, device=q.device)
        if span is not None:
            sp = span[b].to(q.device)
            seen = (j[None] >= sp[:, :1]) & (j[None] < sp[:, 1:])
        for m in range(h):
            Q, K, V = q[b, :, m].double(), k[b, :, m // (h // hk)].double(), v[b, :, m // (h // hk)].double()
            used = seen.any(0)
            K = torch.where(used[:, None], K, torch.zeros_like(K))
            s = Q @ K.t() * scale
            size = (Q.abs() @ K.abs().t()) * abs(scale)
            ds = (d + 4) * F * size
            if cap:
                s = cap * torch.tanh(s / cap)
                ds = ds + 8 * F * cap
            if slopes is not None:
                dist = (qpos[b].double()[:, None] - kpos[b].double()[None]).abs().sum(-1)
                s = s - float(slopes[m]) * dist
                ds = ds + 4 * F * abs(float(slopes[m])) * dist
            ds = ds + 8 * F * s.abs()
            s = torch.where(seen, s, torch.full_like(s, -math.inf))
            top = s.amax(1, keepdim=True) if lk else torch.zeros(lq, 1, device=q.device)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            p = torch.where(total > 0, p / total, torch.zeros_like(p))
            V0 = torch.where(used[:, None], V, torch.zeros_like(V))
            out[b, :, m] = p @ V0
            worst = torch.where(seen, ds, torch.zeros_like(ds)).amax(1, keepdim=True) if lk else 0.0
            rel = 2 * worst + (lk + 32) * F + (0 if dtype == "f32" else 2 * U[dtype])
            bound[b, :, m] = rel * (p @ V0.abs())
    return out, bound + 1e-30


def check(got, ref, bound, dtype):
    """got is ref rounded once to dtype, the value before that off by at most bound."""
    g, worst = got.double(), bound * (1 + U[dtype]) + U[dtype] * ref.abs() + TINY[dtype]
    off = (g - ref).abs()
    bad = ~(off <= worst)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float((off / worst)[bad].max() if bad.any() else 0):.3g} of its bound")
