"""Group norm, rotary and attention as layers of a partition, between the
convolutions that exist: against a chain of 64-bit references, eager, captured,
with static scratch, timed, profiled and split in two."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import operator_ref as R
from paper_2507_18748_amd import Partition
from workloads.zoo import Layer

pytestmark = pytest.mark.gpu

CIN, HEADS, KV, D, GROUPS, H, W = 96, 6, 2, 32, 8, 9, 11
ATT = dict(heads=HEADS, kv_heads=KV, softcap=8.0, slopes=np.linspace(0.0, 0.3, HEADS),
           rotary_pairs=(7, 8))
KINDS = {
    "all": ATT,
    "plain": dict(heads=HEADS, kv_heads=KV),
    "prefix": dict(heads=HEADS, kv_heads=KV, causal=1, prefix=20, rotary_pairs=(8, 8),
                   rotary_adjacent=1, rotary_shared=1, rotary_base=100.0, scale=0.3),
    "causal": dict(heads=HEADS, kv_heads=KV, causal=1, slopes=np.full(HEADS, 0.1)),
}


def layers():
    return [Layer("norm", "groupnorm", -1, CIN, CIN, groups=GROUPS, act="silu"),
            Layer("qkv", "conv", 0, CIN, (HEADS + 2 * KV) * D, bias=True),
            Layer("att", "attention", 1, (HEADS + 2 * KV) * D, HEADS * D),
            Layer("proj", "conv", 2, HEADS * D, CIN, bias=True, res_src=-1),
            Layer("norm2", "groupnorm", 3, CIN, CIN, groups=1, act="gelu")]


def params(dtype):
    r = np.random.default_rng(5)
    t = lambda a: torch.tensor(a).to(R.TORCH[dtype]).float().numpy()
    w = lambda o, i: t(r.standard_normal((o, i, 1, 1)) / np.sqrt(i))
    f = lambda n: (r.standard_normal(n) * 0.1).astype(np.float32)
    return {0: {"bn_gamma": 1 + f(CIN), "bn_beta": f(CIN)},
            1: {"weight": w((HEADS + 2 * KV) * D, CIN), "bias": f((HEADS + 2 * KV) * D)},
            3: {"weight": w(CIN, HEADS * D), "bias": f(CIN)}, 4: {}}


def reference(x, P, att, dtype):
    """The chain on the GPU in 64 bits, rounded to the storage type between layers."""
    n = x.shape[0]
    dt = R.TORCH[dtype]
    rnd = lambda t: t.to(dt)
    cu = lambda a: torch.tensor(a, device="cuda").double()
    m = x.reshape(n, H * W, CIN)
    y = rnd(R.group_norm(m, GROUPS, cu(P[0]["bn_gamma"]), cu(P[0]["bn_beta"]), 1e-5, "silu")[0])
    y = rnd(y.double().reshape(-1, CIN) @ cu(P[1]["weight"][..., 0, 0]).t().contiguous() + cu(P[1]["bias"]))
    y = y.reshape(n, H * W, HEADS + 2 * KV, D)
    i = torch.arange(H * W, device="cuda")
    pos = torch.stack([i // W, i % W], 1).to(torch.int32)[None].expand(n, -1, -1)
    qk, v = y[:, :, :HEADS + KV], y[:, :, HEADS + KV:]
    if "rotary_pairs" in att:
        qk = rnd(R.rotary(qk, pos, att["rotary_pairs"], att.get("rotary_base", 10000.0),
                          bool(att.get("rotary_shared")), bool(att.get("rotary_adjacent")))[0])
    span = None
    if att.get("causal"):
        hi = torch.clamp(i + 1, min=att.get("prefix", 0))
        span = torch.stack([torch.zeros_like(hi), hi], 1)[None].expand(n, -1, -1)
    sl = att.get("slopes")
    a, _ = R.attention(qk[:, :, :HEADS], qk[:, :, HEADS:], v, att.get("scale", D ** -0.5),
                       att.get("softcap", 0.0), sl, pos, pos, span, dtype)
    y = rnd(a).double().reshape(-1, HEADS * D) @ cu(P[3]["weight"][..., 0, 0]).t().contiguous() + cu(P[3]["bias"])
    y = rnd(y.reshape(n, H * W, CIN))
    return rnd(R.group_norm(y, 1, None, None, 1e-5, "gelu")[0]).reshape(n, H, W, CIN)


def run(part, x, out, stream=None):
    part.run(x.shape[0], x.data_ptr(), out.data_ptr(),
             (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return out


# roundings to the storage type along the chain: five layers, the weights of the
# softmax and the rotated heads, each passed on with a gain of at most about two
TOL = {k: 32 * u for k, u in R.U.items()}


def data(dtype, n, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, H, W, CIN, device="cuda", generator=g).to(R.TORCH[dtype])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", list(KINDS))
def test_block(dtype, kind):
    n = 3
    x, P = data(dtype, n), params(dtype)
    out = torch.empty_like(x)
    with Partition(layers(), P, (CIN, H, W), 0, 5, dtype, max_batch=4,
                   attention={2: KINDS[kind]}) as part:
        run(part, x, out)
        ref = reference(x, P, KINDS[kind], dtype).double()
        assert float((out.double() - ref).norm() / ref.norm()) <= TOL[dtype]
        eager = out.clone()
        for _ in range(2):
            assert torch.equal(run(part, x, out), eager)
        static = torch.empty_like(x)
        part.run_static_scratch(n, x.data_ptr(), static.data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(static, eager)
        part.capture(n, x.data_ptr(), out.data_ptr())
        for _ in range(3):
            out.zero_()
            assert torch.equal(run(part, x, out), eager)
        part.timing_setup(n, x.data_ptr(), out.data_ptr())
        out.zero_()
        part.run_timed(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        recs = part.timing_read()
        assert {r["layer"] for r in recs} == set(range(5)) and all(r["min_us"] > 0 for r in recs)
        assert sum(part.layer_info(i, n)["kernel_count"] for i in range(5)) == len(recs)
        table, whole = part.profile_layers([1, 3], warmup=1, reps=3)
        assert table.shape == (5, 2) and (table > 0).all() and (whole > 0).all()
        for r in part.profile_kernels(3, warmup=1, reps=3):
            assert r["median_us"] > 0 and r["bytes"] >= 0
        # one image of a batch alone gives the same as within it
        one = torch.empty(1, H, W, CIN, dtype=x.dtype, device="cuda")
        run(part, x[:1].contiguous(), one)
        r1 = reference(x[:1], P, KINDS[kind], dtype).double()
        assert float((one.double() - r1).norm() / r1.norm()) <= TOL[dtype]
        li = [part.layer_info(i, 1) for i in range(5)]
        assert li[0]["kernel"].startswith("group_norm") and li[2]["kernel"].startswith("attention")
        assert li[2]["out_c"] == HEADS * D and li[2]["flops_b1"] > 0


def test_two_partitions_in_a_row_and_on_a_share():
    dtype, n = "f16", 2
    x, P = data(dtype, n), params(dtype)
    whole, out = torch.empty_like(x), torch.empty_like(x)
    mid = torch.empty(n, H, W, (HEADS + 2 * KV) * D, dtype=x.dtype, device="cuda")
    L = layers()
    with Partition(L, P, (CIN, H, W), 0, 5, dtype, 2, attention={2: ATT}) as part:
        run(part, x, whole)
    with Partition(L, P, (CIN, H, W), 0, 2, dtype, 2) as a, \
            Partition(L, P, (CIN, H, W), 2, 5, dtype, 2, attention={2: ATT}) as b:
        run(a, x, mid)
        run(b, mid, out)
    assert torch.equal(out, whole)
    with Partition(L, P, (CIN, H, W), 0, 5, dtype, 2, attention={2: ATT}, cu_share_parts=4) as part:
        run(part, x, out)
    ref = reference(x, P, ATT, dtype).double()
    assert float((out.double() - ref).norm() / ref.norm()) <= TOL[dtype]
