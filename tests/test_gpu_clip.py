"""som_clip against sums in 64 bits, on the GPU."""
import math

import pytest
import torch

import paper_2608_24067_amd.dense as dense
from dense_ref import check, wide

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def tensors(seed, sizes, dev, scale=1.0, types=TYPES, offset=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = torch.empty(n + offset, dtype=types[i % len(types)], device=dev)[offset:]
        out.append(t.copy_((torch.randn(n, generator=g) * scale).to(t.dtype)))
    return out


@pytest.mark.parametrize("sizes,offset", [([1], 0), ([0, 5, 0], 0), ([7, 1000, 65536, 65537], 0), ([3] * 130, 0),
                                          ([200001, 9, 131072], 1), ([1 << 20], 0)])
@pytest.mark.parametrize("limit", [1e-3, 1.0, 1e9])
def test_clip(dev, sizes, offset, limit):
    ts = tensors(41, sizes, dev, offset=offset)
    outs, norm = dense.clip(ts, limit, out=[torch.full_like(t, float("nan")) for t in ts])
    ref = math.sqrt(sum(float(wide(t).square().sum()) for t in ts))
    # squares and sums in 64 bits: only the rounding to fp32 is seen
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref
    c = min(1.0, limit / ref) if ref else 1.0
    for t, o in zip(ts, outs):
        if c == 1.0:
            assert torch.equal(t, o)
        else:
            check(o, wide(t) * c, 2.0 ** -23 * wide(t).abs() * c, "scaled")
    before = [t.clone() for t in ts]
    same, norm2 = dense.clip(ts, limit)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(same, outs))
    assert same[0] is ts[0] and len(before) == len(ts)


def test_large_and_small_values(dev):
    # squares beyond fp32's range, on both sides
    for v in (1e30, 1e-30):
        t = torch.full((1000,), v, device=dev)
        ref = math.sqrt(float(wide(t).square().sum()))
        _, norm = dense.clip([t], 1e-35)
        assert abs(float(norm) - ref) <= 2.0 ** -23 * ref
        check(t, torch.full((1000,), v, dtype=torch.float32).double() * (1e-35 / ref), 2.0 ** -100 * torch.ones(1000).double(), "scaled")


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_norm_that_is_no_number_scales_nothing(dev, bad):
    ts = tensors(42, [100, 5000], dev)
    ts[1][77] = bad
    before = [t.clone() for t in ts]
    outs, norm = dense.clip(ts, 1.0, out=[torch.empty_like(t) for t in ts])
    assert not math.isfinite(float(norm))
    for a, b, c in zip(before, ts, outs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(a.view(torch.uint8), c.view(torch.uint8))


def test_zeros_and_nothing(dev):
    t = torch.zeros(300, dtype=torch.bfloat16, device=dev)
    outs, norm = dense.clip([t], 1.0)
    assert float(norm) == 0 and not t.any()
    norm = torch.full((1,), 5.0, device=dev)
    assert float(dense.clip([], 1.0, norm=norm)[1]) == 0


def test_same_bits_on_repeats(dev):
    ts = tensors(43, [300001, 70000, 5], dev)
    runs = [dense.clip(ts, 0.5, out=[torch.empty_like(t) for t in ts]) for _ in range(3)]
    for outs, norm in runs[1:]:
        assert torch.equal(norm, runs[0][1]) and all(torch.equal(a, b) for a, b in zip(outs, runs[0][0]))


@pytest.mark.parametrize("count,each", [(4, 3), (300, 3), (2, 5_000_000)])
def test_norm_beyond_fp32_scales_nothing(dev, count, each):
    # finite values whose norm is none: two launches, three, and many chunks
    ts = [torch.full((each,), 3e38, device=dev) for _ in range(count)]
    outs, norm = dense.clip(ts, 1.0, out=[torch.empty_like(t) for t in ts])
    assert math.isinf(float(norm)) and all(torch.equal(t, o) for t, o in zip(ts, outs))
    before = ts[0].clone()
    dense.clip(ts, 1.0)
    assert all(torch.equal(t, before) for t in ts)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("count", [1, 60])
@pytest.mark.parametrize("limit", [1.0, 1e-3, 1e-5])
def test_scales_below_the_smallest_normal(dev, dtype, count, limit):
    # limit / norm is a subnormal fp32 value of few bits, or none; the results are ordinary values
    ts = tensors(44, [700] * count, dev, scale=1e36, types=[dtype])
    outs, norm = dense.clip(ts, limit, out=[torch.empty_like(t) for t in ts])
    ref = math.sqrt(sum(float(wide(t).square().sum()) for t in ts))
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref
    for t, o in zip(ts, outs):
        check(o, wide(t) * (limit / ref), 2.0 ** -23 * wide(t).abs() * (limit / ref), "scaled")
