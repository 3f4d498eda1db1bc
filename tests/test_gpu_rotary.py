"""Rotary positions against a 64-bit reference on an MI355X."""
import pytest

torch = pytest.importorskip("torch")

import operator_ref as R
from paper_2507_18748_amd import rotary

pytestmark = pytest.mark.gpu


def positions(n, l, axes, far, gen):
    return torch.randint(-(far // 2), far + 1, (n, l, axes), device="cuda", generator=gen,
                         dtype=torch.int32)


def case(dtype, n, l, h, d, pairs, shared=False, adjacent=False, base=10000.0, far=100, extra=0,
         gap=0, in_place=False, shared_pos=False, seed=0):
    """extra: heads behind the rotated ones (a packed map); gap: unused elements behind each head."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    print(f"[rotary] {dtype} {n}x{l}x{h}x{d} pairs={pairs} shared={shared} adjacent={adjacent} "
          f"extra={extra} gap={gap} far={far}", flush=True)
    full = torch.randn(n, l, h + extra, d + gap, device="cuda", generator=g).to(R.TORCH[dtype])
    x = full[:, :, :h, :d]
    pos = positions(1 if shared_pos else n, l, len(pairs), far, g)
    ref, bound = R.rotary(x, pos.expand(n, -1, -1), pairs, base, shared, adjacent)
    if in_place:
        keep = full.clone()
        y = x
    else:
        y = torch.full((n, l, h + 1, d + 8), 7.0, device="cuda").to(R.TORCH[dtype])[:, :, :h, :d]
    rotary(x.data_ptr(), y.data_ptr(), dtype, n, l, h, d, pairs, pos.data_ptr(),
           0 if shared_pos else l * len(pairs), x.stride()[:3], y.stride()[:3], base, shared,
           adjacent, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    R.check(y, ref, bound, dtype)
    rest = 2 * sum(pairs)
    if in_place:        # what lies behind the rotated heads and elements is as it was
        assert torch.equal(full[:, :, h:], keep[:, :, h:])
        assert torch.equal(full[..., d:], keep[..., d:])
        assert torch.equal(full[:, :, :h, rest:d], keep[:, :, :h, rest:d])
    else:
        assert torch.equal(y[..., rest:], x[..., rest:])
        whole = y._base
        assert bool((whole[:, :, h:] == 7.0).all()) and bool((whole[..., d:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("n,l,h,d,pairs", [
    (1, 1, 1, 8, (4,)), (1, 1, 1, 8, (1,)), (2, 3, 1, 16, (3, 2)), (1, 7, 3, 40, (5, 5, 5)),
    (3, 50, 4, 64, (8, 12, 12)), (2, 33, 5, 80, (20, 20)), (1, 129, 2, 128, (16, 24, 24)),
    (2, 11, 3, 128, (0, 32, 32)), (1, 5, 2, 256, (64, 64)), (4, 9, 33, 96, (10, 9)),
    (1, 1000, 24, 64, (32,)), (33, 1, 40, 128, (16, 24, 24)), (1, 5, 1, 24, (7,)),
    (1, 3, 300, 32, (8, 8)), (2, 17, 7, 64, (4, 4, 0)),
])
def test_sizes(dtype, adjacent, n, l, h, d, pairs):
    case(dtype, n, l, h, d, pairs, shared=l % 2 == 0, adjacent=adjacent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("pairs", [(8, 12, 12), (7, 6), (16,)])
def test_packed_in_place_and_shared_positions(dtype, adjacent, pairs):
    case(dtype, 2, 21, 6, 64, pairs, adjacent=adjacent, extra=3, gap=8, in_place=True)
    case(dtype, 2, 21, 6, 64, pairs, adjacent=adjacent, extra=3, shared_pos=True)


@pytest.mark.parametrize("far", [1 << 20, 1 << 30])
@pytest.mark.parametrize("base", [10000.0, 1.0, 0.5, 1e6])
def test_far_positions(far, base):
    case("f32", 2, 40, 2, 64, (8, 8, 16), base=base, far=far, shared=True)


def test_extreme_positions_and_values():
    """The ends of 32 bits, and what is not a number, stay in their pair."""
    x = torch.randn(1, 2, 1, 16, device="cuda")
    pos = torch.tensor([[[-(1 << 31)], [(1 << 31) - 1]]], dtype=torch.int32, device="cuda")
    ref, bound = R.rotary(x, pos, (8,), 10000.0, False, False)
    y = torch.empty_like(x)
    call = lambda: rotary(x.data_ptr(), y.data_ptr(), "f32", 1, 2, 1, 16, (8,), pos.data_ptr(), 0,
                          x.stride()[:3], y.stride()[:3])
    call()
    torch.cuda.synchronize()
    R.check(y, ref, bound, "f32")
    clean = y.clone()
    x[0, 1, 0, 3] = float("inf")
    call()
    torch.cuda.synchronize()
    same = torch.ones(16, dtype=torch.bool, device="cuda")
    same[3] = same[11] = False
    assert torch.equal(y[0, 1, 0][same], clean[0, 1, 0][same])
    assert not bool(torch.isfinite(y[0, 1, 0][~same]).any())


def test_captured_and_replayed():
    x = torch.randn(2, 30, 4, 64, device="cuda").half()
    pos = torch.randint(0, 99, (2, 30, 2), dtype=torch.int32, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    args = ("f16", 2, 30, 4, 64, (16, 16), pos.data_ptr(), 60, x.stride()[:3], x.stride()[:3])
    rotary(x.data_ptr(), z.data_ptr(), *args)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        rotary(x.data_ptr(), y.data_ptr(), *args, stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        y.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, z)
