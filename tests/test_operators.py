"""Argument checks of the operators on device tensors: every refusal comes from
the host before any device work, and sizes of zero launch nothing."""
import ctypes

import numpy as np
import pytest

import paper_2507_18748_amd as lib
from paper_2507_18748_amd import PpipeError, Partition
from workloads.zoo import Layer

P = 4096          # an aligned address that no refused call touches


def status(fn, *a, **kw):
    with pytest.raises(PpipeError) as e:
        fn(*a, **kw)
    assert str(e.value).split(": ", 1)[1], "a refusal says why"
    return e.value.status


def norm(x=P, y=2 * P, dtype="f16", batch=2, pixels=9, channels=64, groups=8, gamma=0, beta=0,
         eps=1e-5, act="silu", ws=4 * P, wb=1 << 40):
    lib.group_norm(x, y, dtype, batch, pixels, channels, groups, gamma, beta, eps, act, ws, wb)


@pytest.mark.parametrize("kw,want", [
    (dict(channels=60, groups=8), -1), (dict(channels=0), -1), (dict(groups=0), -1),
    (dict(batch=-1), -1), (dict(pixels=-1), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(x=0), -1), (dict(y=0), -1),
    (dict(x=P + 8), -1), (dict(y=P + 2), -1), (dict(gamma=P + 2), -1), (dict(beta=P + 1), -1),
    (dict(channels=12, groups=4), -3), (dict(channels=6, groups=2, dtype="f32"), -3),
    (dict(channels=1 << 17, groups=1), -3), (dict(batch=1 << 16, pixels=1 << 16), -3),
])
def test_group_norm_refusals(kw, want):
    assert status(norm, **kw) == want


def test_group_norm_of_nothing():
    norm(batch=0, x=0, y=0, ws=0, wb=0)
    norm(pixels=0, x=0, y=0, ws=0, wb=0)
    assert lib.group_norm_workspace("f16", 0, 9, 64, 8) == 0
    assert status(lib.group_norm_workspace, "f16", 1, 9, 64, 7) == -1


def rot(x=P, y=2 * P, dtype="f16", batch=2, tokens=9, heads=3, d=64, pairs=(8, 12, 12), pos=3 * P,
        ps=27, xs=None, ys=None, base=1e4, **kw):
    dense = (tokens * heads * d, heads * d, d)
    lib.rotary(x, y, dtype, batch, tokens, heads, d, pairs, pos, ps, xs or dense, ys or dense,
               base, **kw)


@pytest.mark.parametrize("kw,want", [
    (dict(pairs=(16, 17)), -1), (dict(pairs=(0, 0)), -1), (dict(pairs=(-1, 4)), -1),
    (dict(pairs=()), -1), (dict(pairs=(1, 1, 1, 1)), -1), (dict(base=0.0), -1),
    (dict(base=float("nan")), -1), (dict(base=float("inf")), -1), (dict(batch=-1), -1),
    (dict(heads=-1), -1), (dict(tokens=-2), -1), (dict(pos=0), -1), (dict(x=0), -1),
    (dict(y=0), -1), (dict(x=P + 8), -1), (dict(pos=P + 2), -1), (dict(ps=-27), -1),
    (dict(xs=(-1728, 192, 64)), -1), (dict(ys=(1728, 0, 64)), -1),
    (dict(ys=(1728, 192, 32)), -1), (dict(y=P, ys=(1728, 64, 576)), -1),
    (dict(d=60, pairs=(8,)), -3), (dict(d=0, pairs=(8,)), -3), (dict(d=264, pairs=(8,)), -3),
    (dict(xs=(1728, 196, 64)), -3), (dict(xs=(1 << 40, 1 << 22, 64)), -3),
    (dict(heads=1 << 17), -3), (dict(batch=1 << 16, tokens=1 << 16), -3),
    (dict(ps=1 << 60), -3), (dict(xs=(1 << 60, 192, 64)), -3),
])
def test_rotary_refusals(kw, want):
    assert status(rot, **kw) == want


def test_rotary_of_nothing():
    for kw in (dict(batch=0), dict(tokens=0), dict(heads=0)):
        rot(x=0, y=0, pos=0, **kw)


def att(q=P, k=2 * P, v=3 * P, out=4 * P, dtype="f16", batch=2, lq=5, lk=7, heads=4, kv=2, d=64,
        qs=None, ks=None, vs=None, os=None, scale=0.125, cap=0.0, slopes=0, qp=0, kp=0, axes=0,
        qps=0, kps=0, spans=0, ss=0, ws=8 * P, wb=1 << 40):
    lib.attention(q, k, v, out, dtype, batch, lq, lk, heads, kv, d,
                  qs or (lq * heads * d, heads * d, d), ks or (lk * kv * d, kv * d, d),
                  vs or (lk * kv * d, kv * d, d), os or (lq * heads * d, heads * d, d), scale, cap,
                  slopes, qp, kp, axes, qps, kps, spans, ss, ws, wb)


@pytest.mark.parametrize("kw,want", [
    (dict(heads=3), -1), (dict(heads=0), -1), (dict(kv=0), -1), (dict(batch=-1), -1),
    (dict(lq=-1), -1), (dict(lk=-1), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(cap=-1.0), -1), (dict(cap=float("nan")), -1),
    (dict(scale=2e30), -1), (dict(cap=2e30), -1), (dict(axes=4), -1), (dict(axes=-1), -1), (dict(slopes=P), -1),
    (dict(slopes=P, qp=P, kp=P, axes=0), -1), (dict(slopes=P, qp=P, axes=2), -1),
    (dict(qp=P, kp=P, axes=2), -1), (dict(q=0), -1), (dict(k=0), -1), (dict(v=0), -1),
    (dict(out=0), -1), (dict(q=P + 8), -1), (dict(out=P + 2), -1), (dict(spans=P + 4), -1),
    (dict(slopes=P + 2, qp=P, kp=P, axes=1), -1), (dict(out=P), -1), (dict(out=2 * P), -1),
    (dict(out=3 * P), -1), (dict(os=(1280, 0, 64)), -1), (dict(os=(1280, 256, 8)), -1),
    (dict(os=(0, 256, 64)), -1), (dict(ks=(896, -128, 64)), -1), (dict(ss=-2), -1),
    (dict(ss=3), -1), (dict(qps=-1), -1), (dict(kps=-1), -1),
    (dict(d=60), -3), (dict(d=264), -3), (dict(d=0), -3), (dict(qs=(1280, 260, 64)), -3),
    (dict(ks=(1 << 40, 1 << 22, 64)), -3), (dict(lk=(1 << 28) + 1), -3),
    (dict(heads=1 << 17, kv=1 << 17), -3), (dict(ss=1 << 60), -3),
])
def test_attention_refusals(kw, want):
    assert status(att, **kw) == want


def test_attention_of_nothing():
    att(batch=0, q=0, k=0, v=0, out=0, ws=0, wb=0)
    att(lq=0, q=0, k=0, v=0, out=0, ws=0, wb=0)
    d = lib.attention_desc("f16", 0, 5, 7, 4, 2, 64, (0, 0, 0), (0, 0, 0), (0, 0, 0), (0, 0, 0), 1.0)
    assert lib.attention_workspace(d) == 0
    d.heads = 3
    assert status(lib.attention_workspace, d) == -1


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), -1), (dict(q_len=-1), -1), (dict(kv_len=-1), -1), (dict(n_docs=0), -1),
    (dict(n_docs=2), -1), (dict(spans_ptr=0), -1), (dict(spans_ptr=P + 4), -1),
    (dict(doc_offsets_ptr=P + 2), -1), (dict(q_start_ptr=P + 2), -1),
    (dict(q_len=(1 << 28) + 1), -3), (dict(batch=1 << 10, q_len=1 << 22), -3),
])
def test_attention_spans_refusals(kw, want):
    a = dict(spans_ptr=P, batch=2, q_len=3, kv_len=4)
    a.update(kw)
    assert status(lib.attention_spans, **a) == want


def test_attention_spans_of_nothing():
    lib.attention_spans(0, 0, 3, 4)
    lib.attention_spans(0, 3, 0, 4)


def test_null_descriptions():
    L = lib.load_library()
    assert L.ppipe_rotary(None, None, None, None, None) == -1
    assert L.ppipe_attention(None, *([None] * 9), 0, None) == -1
    assert L.ppipe_attention_workspace(None) == -1


def block(cin=64, heads=4, kv=2, d=16, groups=8):
    return [Layer("norm", "groupnorm", -1, cin, cin, groups=groups, act="silu"),
            Layer("qkv", "conv", 0, cin, (heads + 2 * kv) * d, bias=True),
            Layer("att", "attention", 1, (heads + 2 * kv) * d, heads * d),
            Layer("proj", "conv", 2, heads * d, cin, bias=True, res_src=-1)]


def make(layers=None, attention=None, begin=0, end=4, dtype="f16", **kw):
    layers = layers or block()
    params = {1: {"weight": np.zeros((128, 64, 1, 1), np.float32)},
              3: {"weight": np.zeros((64, 64, 1, 1), np.float32)}}
    return Partition(layers, params, (64, 5, 5), begin, end, dtype, max_batch=2,
                     attention=attention, **kw)


def test_partition_refusals():
    ok = {2: dict(heads=4, kv_heads=2)}
    assert status(make) == -1                                        # no description
    assert status(make, attention={1: dict(heads=4)}) == -1          # no attention layer
    assert status(make, attention={7: dict(heads=4)}) == -1
    for bad in (dict(heads=4, kv_heads=4), dict(heads=0, kv_heads=2), dict(heads=4, kv_heads=0),
                dict(heads=4, kv_heads=2, prefix=3), dict(heads=4, kv_heads=2, causal=1, prefix=-1),
                dict(heads=4, kv_heads=2, rotary_pairs=(5, 4)),
                dict(heads=4, kv_heads=2, rotary_pairs=(-1, 4)),
                dict(heads=4, kv_heads=2, rotary_pairs=(4, 4), rotary_base=-1.0),
                dict(heads=4, kv_heads=2, softcap=-1.0),
                dict(heads=4, kv_heads=2, scale=float("inf"))):
        assert status(make, attention={2: bad}) == -1, bad
    assert status(make, attention=ok, cu_share_parts=9) == -1
    for i, change in ((0, dict(act="none", c_out=32)), (0, dict(groups=7)), (0, dict(groups=0)),
                      (2, dict(act="relu")), (2, dict(c_in=64)), (1, dict(act="silu"))):
        layers = block()
        for k, v in change.items():
            setattr(layers[i], k, v)
        assert status(make, layers, ok) == -1, (i, change)
    layers = block()
    layers[0].res_src = 0
    assert status(make, layers, ok) == -1                            # names no earlier layer
    layers[0].res_src = -1
    layers[2].res_src = 1
    assert status(make, layers, ok) == -3                            # residual on attention
    with pytest.raises(ValueError):
        make(attention={2: dict(heads=4, no_such_field=1)})
    with pytest.raises(ValueError):
        make(attention={2: dict(heads=4, kv_heads=2, slopes=[1.0])})
    with pytest.raises(ValueError):
        make(attention=ok, tuning={"no_pair": 1})


def test_description_twice():
    from paper_2507_18748_amd import binding as B
    arr = (B.LayerDesc * 1)()
    arr[0].op, arr[0].src, arr[0].res_src, arr[0].c_in, arr[0].c_out = 6, -1, -1, 48, 16
    desc = B.ModelDesc(1, arr, 48, 3, 3, 1)
    a = (B.AttentionLayer * 2)()
    for x in a:
        x.heads = x.kv_heads = 1
    L = lib.load_library()
    assert not L.ppipe_partition_create_attention(ctypes.byref(desc), 0, 1, 1, a, 2, 1)
    assert L.ppipe_last_status() == -1
    assert not L.ppipe_partition_create_attention(ctypes.byref(desc), 0, 1, 1, None, 1, 1)
    assert L.ppipe_last_status() == -1
    assert not L.ppipe_partition_create_attention(ctypes.byref(desc), 0, 1, 1, a, -1, 1)
    assert L.ppipe_last_status() == -1


def test_split_points_with_the_new_layers():
    layers = block()
    layers[3].res_src = 0
    assert lib.split_points(layers) == [1, 1, 0, 0, 1]
