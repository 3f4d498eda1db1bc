"""Group norm with an activation against a 64-bit reference on an MI355X."""
import pytest

torch = pytest.importorskip("torch")

import operator_ref as R
from paper_2507_18748_amd import PpipeError, group_norm, group_norm_workspace

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "relu6", "silu", "gelu"]


def run(x, groups, gamma=None, beta=None, eps=1e-5, act="none", dtype="f16", y=None, stream=None):
    n, p, c = x.shape
    y = torch.empty_like(x) if y is None else y
    need = group_norm_workspace(dtype, n, p, c, groups)
    ws = torch.full((need + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    s = stream or torch.cuda.current_stream()
    group_norm(x.data_ptr(), y.data_ptr(), dtype, n, p, c, groups,
               0 if gamma is None else gamma.data_ptr(), 0 if beta is None else beta.data_ptr(),
               eps, act, ws.data_ptr() if need else 0, need, s.cuda_stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0x5A).all()), "wrote beyond its workspace"
    return y


def case(dtype, n, p, c, groups, act="none", affine=True, eps=1e-5, seed=0, shift=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    print(f"[group-norm] {dtype} {n}x{p}x{c} groups={groups} {act}", flush=True)
    x = torch.randn(n, p, c, device="cuda", generator=g)
    x = (x + shift * torch.randn(c, device="cuda", generator=g)).to(R.TORCH[dtype])
    gamma = 1 + 0.3 * torch.randn(c, device="cuda", generator=g) if affine else None
    beta = 0.3 * torch.randn(c, device="cuda", generator=g) if affine else None
    ref, bound = R.group_norm(x, groups, gamma, beta, eps, act)
    got = run(x, groups, gamma, beta, eps, act, dtype)
    R.check(got, ref, bound, dtype)
    return x, got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,p,c,groups", [
    (1, 1, 8, 1), (1, 1, 64, 8), (3, 2, 32, 4), (2, 7, 40, 8), (1, 49, 320, 32), (5, 63, 24, 3),
    (2, 196, 256, 32), (3, 783, 320, 32), (1, 3136, 64, 4), (2, 4097, 8, 8), (1, 12544, 128, 32),
    (1, 5, 4096, 1), (2, 3, 8192, 32), (64, 1, 64, 32), (7, 64, 1280, 32), (1, 50000, 16, 1),
    (4, 2500, 512, 32), (1, 100, 65536, 16), (2, 33, 88, 11), (40, 400, 64, 1),
])
def test_sizes(dtype, n, p, c, groups):
    case(dtype, n, p, c, groups, act="silu")


@pytest.mark.parametrize("dtype,c,groups", [
    ("f32", 65536, 1), ("f16", 65536, 1), ("bf16", 65536, 2), ("f32", 65532, 2), ("f32", 65532, 1),
    ("f16", 65528, 2), ("f16", 65528, 8191), ("f32", 65536, 65536), ("bf16", 40000, 1),
])
@pytest.mark.parametrize("n,p", [(2, 1), (1, 5), (1, 700)])
def test_rows_longer_than_a_block(dtype, c, groups, n, p):
    case(dtype, n, p, c, groups, "relu")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("groups", [1, 3, 16, 48])
@pytest.mark.parametrize("n,p", [(1, 9000), (1, 60000), (30, 2000), (300, 9)])
def test_one_launch_and_two(dtype, groups, n, p):
    case(dtype, n, p, 48, groups, "gelu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("affine", [True, False])
@pytest.mark.parametrize("p", [30, 5000])
def test_activations(dtype, act, affine, p):
    case(dtype, 2, p, 64, 8, act, affine)


@pytest.mark.parametrize("p", [64, 6000])
def test_one_group_per_channel_and_constants(p):
    """Groups of one channel; a constant group has no deviation but eps."""
    case("f32", 2, p, 16, 16, "none")
    x = torch.full((2, p, 16), 3.5, device="cuda")
    got = run(x, 4, eps=1e-5, dtype="f32")
    # the mean of equal values is off by at most a few dozen roundings, over sqrt(eps)
    assert float(got.abs().max()) <= 64 * R.F * 3.5 / 1e-5 ** 0.5


@pytest.mark.parametrize("p", [50, 9000])
def test_far_mean_and_outlier(p):
    """A mean of a thousand deviations, and a first value far off the others:
    sums of squares would lose the variance."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(2, p, 32, device="cuda", generator=g) + 1000.0
    ref, bound = R.group_norm(x, 4, None, None, 1e-5, "none")
    R.check(run(x, 4, dtype="f32"), ref, bound, "f32")
    x = torch.randn(2, p, 32, device="cuda", generator=g)
    x[:, 0, 0] = 30000.0
    ref, bound = R.group_norm(x, 4, None, None, 1e-5, "none")
    R.check(run(x, 4, dtype="f32"), ref, bound, "f32")


@pytest.mark.parametrize("p", [40, 7000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_stay_in_their_group(p, bad):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn(3, p, 64, device="cuda", generator=g).half()
    clean = run(x, 8, act="silu")
    x[1, p // 2, 17] = bad                       # image 1, group 2
    got = run(x, 8, act="silu")
    hit = torch.zeros(3, p, 64, dtype=torch.bool, device="cuda")
    hit[1, :, 16:24] = True
    assert bool(torch.isnan(got[hit]).all())
    assert torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("act", ["relu", "relu6"])
def test_nan_passes_the_clamps(act):
    x = torch.randn(1, 30, 8, device="cuda").half()
    x[0, 3, 0] = float("nan")
    assert bool(torch.isnan(run(x, 1, act=act)).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("p", [100, 20000])
def test_in_place_gives_the_same_bits(dtype, p):
    x, got = case(dtype, 2, p, 96, 8, "gelu", affine=False)
    assert torch.equal(run(x, 8, act="gelu", dtype=dtype, y=x), got)


def test_large_activations():
    """silu and gelu of values far out: no overflow, the limits."""
    x = torch.zeros(1, 4, 8, device="cuda")
    x[0, :, 0] = torch.tensor([1.0, -1.0, 1.0, -1.0], device="cuda")
    gamma = torch.full((8,), 1e6, device="cuda")
    for act in ("silu", "gelu"):
        ref, bound = R.group_norm(x, 8, gamma, None, 1e-5, act)
        R.check(run(x, 8, gamma, None, act=act, dtype="f32"), ref, bound, "f32")


def test_workspace_too_small_is_refused():
    n, p, c, g = 2, 50000, 64, 8
    need = group_norm_workspace("f16", n, p, c, g)
    assert need > 0
    x = torch.zeros(n, p, c, dtype=torch.float16, device="cuda")
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for ptr, size in ((0, need), (ws.data_ptr(), need - 1)):
        with pytest.raises(PpipeError) as e:
            group_norm(x.data_ptr(), x.data_ptr(), "f16", n, p, c, g, 0, 0, 1e-5, "none", ptr, size)
        assert e.value.status == -1


@pytest.mark.parametrize("p", [196, 30000])
def test_captured_on_another_stream_and_repeatable(p):
    """Two graphs with workspaces of their own, replayed in turn and together with
    eager work, give the eager bits each time."""
    x = torch.randn(2, p, 64, device="cuda").half()
    x2 = torch.randn(2, p, 64, device="cuda").half()
    want, want2 = run(x, 8, act="silu"), run(x2, 8, act="silu")
    s = torch.cuda.Stream()
    got, graphs, keep = [torch.empty_like(x), torch.empty_like(x)], [], []
    for src, dst in ((x, got[0]), (x2, got[1])):
        ws = torch.empty(group_norm_workspace("f16", 2, p, 64, 8) + 16, dtype=torch.uint8, device="cuda")
        keep.append(ws)
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr, stream=s):
            group_norm(src.data_ptr(), dst.data_ptr(), "f16", 2, p, 64, 8, 0, 0, 1e-5, "silu",
                       ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        graphs.append(gr)
    for _ in range(4):
        for d in got:
            d.zero_()
        torch.cuda.synchronize()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert float((x.float() * 2).abs().max()) > 0     # unrelated eager work
        assert torch.equal(got[0], want) and torch.equal(got[1], want2)
