"""som_linear and its gradients against 64-bit products, on the GPU."""
import pytest
import torch

import paper_2608_24067_amd.dense as dense
import paper_2608_24067_amd.som as som
from dense_ref import LIP, U, act, check, curve, slope, sums, wide

pytestmark = pytest.mark.gpu

HALVES = [torch.float16, torch.bfloat16]


def strided(shape, pad, dtype, dev, g, scale=1.0, offset=0):
    """A matrix whose rows are `pad` elements longer, filled with NaN around it, `offset` elements into its buffer."""
    buf = torch.full((shape[0] * (shape[1] + pad) + offset,), float("nan"), dtype=dtype, device=dev)
    t = buf[offset:].view(shape[0], shape[1] + pad)[:, :shape[1]]
    t.copy_((torch.randn(shape, generator=g) * scale).to(dtype))
    return t


def case(seed, N, K, M, dtype, dev, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    x = strided((N, K), pad, dtype, dev, g, offset=offset)
    W = strided((K, M), pad, dtype, dev, g, K ** -0.5, offset=offset)
    b = (torch.randn(M, generator=g) * 0.3).to(dev)
    r = strided((N, M), pad, dtype, dev, g, offset=offset)
    return x, W, b, r, g


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("N,K,M,pad,offset,a,f32", [
    (1, 64, 64, 0, 0, "none", True),
    (1, 1, 1, 0, 0, "gelu", False),          # a single product
    (1, 1024, 4096, 0, 0, "none", True),     # one row on a 64 x 64 map
    (2, 24, 8, 0, 0, "relu", False),         # less than a reduction step
    (3, 31, 33, 0, 0, "silu", False),        # odd everywhere
    (17, 96, 130, 6, 0, "gelu", False),      # widths that are no chunks, strided rows
    (16, 40, 72, 8, 8, "none", False),       # chunks in strided rows
    (33, 257, 129, 0, 1, "none", True),      # rows at any element
    (64, 128, 128, 0, 0, "silu", False),
    (100, 1003, 625, 0, 0, "none", True),    # a 25 x 25 map of odd width
    (128, 64, 4096, 0, 0, "relu", False),
    (300, 200, 1000, 0, 0, "gelu", False),   # ragged tiles of 128
    (257, 136, 40000, 0, 0, "none", False),  # ragged tiles of 256
    (5000, 72, 2600, 24, 0, "gelu", False),  # tiles of 256, a short reduction, strided rows
])
def test_linear(dev, dtype, N, K, M, pad, offset, a, f32):
    x, W, b, r, _ = case(11, N, K, M, dtype, dev, pad, offset)
    out = torch.full((N, M), float("nan"), dtype=torch.float32 if f32 else dtype, device=dev)
    pre = torch.empty(N, M, dtype=dtype, device=dev)
    dense.linear(x, W, b, residual=r, act=a, out=out, pre=pre)
    z = wide(x) @ wide(W) + wide(b)
    err = sums(K + 1, wide(x).abs() @ wide(W).abs() + wide(b).abs())
    check(pre, z, err, "pre")
    y = act(a, z) + wide(r)
    check(out, y, LIP * err + 2.0 ** -20 * (z.abs().clamp_min(1) if a != "none" else 0) + 2.0 ** -23 * (z.abs() + wide(r).abs()),
          "y")


def test_plain_product_bias_of_the_rows_type_and_residual_in_place(dev):
    x, W, b, r, _ = case(12, 70, 64, 96, torch.bfloat16, dev)
    err = sums(64, wide(x).abs() @ wide(W).abs())
    check(dense.linear(x, W), wide(x) @ wide(W), err, "product")
    b = b.to(torch.bfloat16)
    y = wide(x) @ wide(W) + wide(b) + wide(r)
    dense.linear(x, W, b, residual=r, out=r)
    check(r, y, err + 2.0 ** -22 * (y.abs() + wide(b).abs() + 10), "in place")


def test_infinities_and_nan_stay_in_their_rows(dev):
    # also where tiles reach past the last row and the last reduction step
    for N, K, M in ((40, 70, 30), (260, 72, 1000), (5, 8, 8)):
        x, W, b, r, _ = case(13, N, K, M, torch.float16, dev)
        clean = dense.linear(x, W, b)
        x = x.clone()
        x[N // 2, K - 1] = float("inf")
        x[N - 1, 0] = float("nan")
        got = dense.linear(x, W, b)
        rows = torch.ones(N, dtype=torch.bool, device=dev)
        rows[N // 2] = rows[N - 1] = False
        assert torch.equal(got[rows], clean[rows])
        assert not torch.isfinite(got[N // 2]).any() and torch.isnan(got[N - 1]).all()


def test_scores_rank_units_as_the_search_does(dev):
    # rows of a few ones, as dense rows: the highest score is the search's unit
    V, M, N = 96, 225, 64
    g = torch.Generator().manual_seed(14)
    W = (torch.randint(0, 256, (V, M), generator=g).float() / 256).half().to(dev)
    x = (torch.rand(N, V, generator=g) < 0.1)
    x[0] = False
    rp = torch.cat([torch.zeros(1, dtype=torch.int64), x.sum(1).cumsum(0)]).int().to(dev)
    ci = x.nonzero()[:, 1].int().to(dev)
    norms = som.codebook_norms(W, V, M)
    bmu, _ = som.bmu_search(W, norms, rp, ci, V, M)
    scores = dense.linear(x.half().to(dev), W, (-0.5 * norms).float(), out_dtype=torch.float32)
    idx, _ = dense.route(scores, 1)
    d = norms - 2 * (x.double().to(dev) @ W.double())
    picked = d.gather(1, idx.long())[:, 0]
    best = d.gather(1, bmu.long()[:, None])[:, 0]
    assert bool(((picked - best).abs() <= 2.0 ** -16 * (1 + norms.max())).all())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("N,K,M,pad,a,f32", [
    (1, 1, 1, 0, "silu", False),
    (1, 64, 128, 0, "gelu", False),
    (7, 31, 65, 0, "none", True),
    (33, 64, 40, 8, "relu", False),
    (100, 130, 257, 3, "gelu", True),
    (500, 264, 136, 0, "silu", False),
    (1000, 64, 72, 0, "none", False),
    (130, 4200, 4104, 0, "none", False),   # tiles of 256 in the weights' gradient
    (5001, 520, 2056, 0, "gelu", False),
])
def test_linear_gradients(dev, dtype, N, K, M, pad, a, f32):
    x, W, b, _, g = case(15, N, K, M, dtype, dev, pad)
    dy = strided((N, M), pad, dtype, dev, g)
    pre = torch.empty(N, M, dtype=dtype, device=dev)
    dense.linear(x, W, b, act=a, pre=pre)
    dx, dW, db = dense.linear_bwd(x, W, dy, pre=pre, act=a, bias_dtype=torch.float32 if f32 else None)
    # the formula on the pre that was kept; dz is rounded once
    dz = wide(dy) * slope(a, wide(pre))
    off = (U[dtype] * dz.abs() + 2.0 ** -20 * wide(dy).abs() * wide(pre).abs().clamp_min(1)) if a != "none" else 0 * dz
    mag = dz.abs() + off
    check(dx, dz @ wide(W).T, off @ wide(W).abs().T + sums(M, mag @ wide(W).abs().T), "dx")
    check(dW, wide(x).T @ dz, wide(x).abs().T @ off + sums(N, wide(x).abs().T @ mag), "dW")
    check(db, dz.sum(0), off.sum(0) + sums(N, mag.sum(0)), "db")
    assert db.dtype == (torch.float32 if f32 else dtype)


@pytest.mark.parametrize("a", ["none", "gelu", "silu", "relu"])
def test_linear_gradients_against_differences(dev, a):
    # <dy, y(x + h v) - y(x - h v)> / 2h in 64 bits against <dx, v>, and the same for W and b
    x, W, b, _, g = case(16, 12, 40, 24, torch.float16, dev)
    dy = torch.randn(12, 24, generator=g).half().to(dev)
    pre = torch.empty(12, 24, dtype=torch.float16, device=dev)
    dense.linear(x, W, b, act=a, pre=pre)
    grads = dense.linear_bwd(x, W, dy, pre=pre, act=a, bias_dtype=torch.float32)
    args = [wide(x), wide(W), wide(b)]
    h = 1e-6
    for i, grad in enumerate(grads):
        v = torch.randn(args[i].shape, generator=g, dtype=torch.float64)
        v /= v.norm()
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        f = lambda t: (wide(dy) * act(a, t[0] @ t[1] + t[2])).sum()  # noqa: E731
        diff = float(f(up) - f(down)) / (2 * h)
        # each gradient value is off by at most 2^-9 of its terms' magnitude (dz, pre and the result rounded)
        dz = wide(dy).abs() * LIP
        terms = [dz @ args[1].abs().T, args[0].abs().T @ dz, dz.sum(0)][i]
        assert abs(diff - float((wide(grad) * v).sum())) <= 2.0 ** -9 * float((terms * v.abs()).sum()) + 1e-5


def test_parts_of_the_gradient_and_no_rows(dev):
    x, W, b, _, g = case(17, 40, 48, 56, torch.bfloat16, dev)
    dy = torch.randn(40, 56, generator=g).bfloat16().to(dev)
    whole = dense.linear_bwd(x, W, dy)
    for i in range(3):
        out = [None, None, None]
        out[i] = torch.full_like(whole[i], float("nan"))
        assert torch.equal(dense.linear_bwd(x, W, dy, out=out)[i], whole[i])
    dx, dW, db = dense.linear_bwd(x[:0], W, dy[:0])
    assert dx.shape == (0, 48) and not dW.any() and not db.any()
    assert dense.linear(x[:0], W, b).shape == (0, 56)


def test_another_stream_and_repeats_give_the_same_bits(dev):
    x, W, b, r, g = case(18, 777, 520, 264, torch.bfloat16, dev)
    dy = torch.randn(777, 264, generator=g).bfloat16().to(dev)
    first = (dense.linear(x, W, b, residual=r),) + dense.linear_bwd(x, W, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = (dense.linear(x, W, b, residual=r),) + dense.linear_bwd(x, W, dy)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("N,K,M", [
    (300, 5, 200), (40, 7, 3), (5, 300, 50), (16, 64, 9), (9, 33, 130), (12, 7, 129), (3, 2048, 5), (1, 1000, 127),
    (17, 8, 8), (200, 9, 300), (130, 1001, 129), (1000, 33, 127), (2, 100, 1025), (16, 39, 7),
])
def test_linear_at_the_edges_of_tiles(dev, dtype, N, K, M):
    for pad, offset in ((0, 0), (3, 1)):
        x, W, b, r, _ = case(19, N, K, M, dtype, dev, pad, offset)
        out = dense.linear(x, W, b, residual=r, act="silu")
        z = wide(x) @ wide(W) + wide(b)
        err = sums(K + 1, wide(x).abs() @ wide(W).abs() + wide(b).abs())
        y = act("silu", z) + wide(r)
        check(out, y, LIP * err + 2.0 ** -20 * z.abs().clamp_min(1) + 2.0 ** -23 * (z.abs() + wide(r).abs()), "y")


@pytest.mark.parametrize("N,K,M,pad", [(20000, 40, 56, 0), (9001, 70, 91, 0), (30000, 264, 16, 8), (2000, 6, 7, 1),
                                       (1500, 129, 3, 0)])
def test_weights_gradient_of_many_rows(dev, N, K, M, pad):
    x, W, b, _, g = case(20, N, K, M, torch.float16, dev, pad)
    dy = strided((N, M), pad, torch.float16, dev, g)
    dx, dW, db = dense.linear_bwd(x, W, dy, bias_dtype=torch.float32)
    check(dW, wide(x).T @ wide(dy), sums(N, wide(x).abs().T @ wide(dy).abs()), "dW")
    check(db, wide(dy).sum(0), sums(N, wide(dy).abs().sum(0)), "db")
    check(dx, wide(dy) @ wide(W).T, sums(M, wide(dy).abs() @ wide(W).abs().T), "dx")
    part = dense.linear_bwd(x, W, dy, out=(None, None, torch.empty_like(db)))[2]
    assert torch.equal(part, db)


def test_rows_past_32_bit_offsets(dev):
    step = 1_200_000_000  # elements between rows: the third lies 4.8 GB in
    buf = torch.empty(2 * step + 64, dtype=torch.float16, device=dev)
    x = buf.as_strided((3, 64), (step, 1))
    g = torch.Generator().manual_seed(22)
    x.copy_(torch.randn(3, 64, generator=g).half())
    W = (torch.randn(64, 40, generator=g) / 8).half().to(dev)
    ref = wide(x) @ wide(W)
    check(dense.linear(x, W), ref, sums(64, wide(x).abs() @ wide(W).abs()), "few rows")
    many = buf.as_strided((40, 64), (2 * step // 39 // 8 * 8, 1))
    many.copy_(torch.randn(40, 64, generator=g).half())
    check(dense.linear(many, W), wide(many) @ wide(W), sums(64, wide(many).abs() @ wide(W).abs()), "tiles")
    dy = torch.randn(40, 40, generator=g).half().to(dev)
    dW = dense.linear_bwd(many, W, dy)[1]
    check(dW, wide(many).T @ wide(dy), sums(40, wide(many).abs().T @ wide(dy).abs()), "dW")
    del buf, x, many
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("N,K,M,pad,offset,a", [
    (96, 264, 1024, 0, 0, "silu"),   # one tile of 16 rows a CU at most
    (500, 130, 1003, 1, 1, "gelu"),
    (90, 72, 5504, 0, 0, "none"),    # 258 of them: tiles of 32 rows
    (600, 43, 1000, 3, 1, "gelu"),
    (1600, 40, 1280, 0, 0, "relu"),  # 500 of those
    (1640, 40, 1280, 0, 0, "silu"),  # 520: tiles of 128 rows
    (2050, 64, 3900, 8, 0, "none"),  # 527 of those: tiles of 256
])
def test_linear_where_the_tile_changes(dev, dtype, N, K, M, pad, offset, a):
    x, W, b, r, _ = case(21, N, K, M, dtype, dev, pad, offset)
    out = dense.linear(x, W, b, residual=r, act=a)
    z = wide(x) @ wide(W) + wide(b)
    err = sums(K + 1, wide(x).abs() @ wide(W).abs() + wide(b).abs())
    y = act(a, z) + wide(r)
    check(out, y, LIP * err + 2.0 ** -20 * (z.abs().clamp_min(1) if a != "none" else 0) + 2.0 ** -23 * (z.abs() + wide(r).abs()),
          "y")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("N,K,M", [(5, 5, 12), (3, 4, 64), (16, 7, 100), (1, 1, 8), (40, 3, 127), (300, 2, 31),
                                   (2, 6, 9), (17, 1, 128), (8, 7, 200)])
def test_fewer_than_eight_features(dev, dtype, N, K, M):
    # widths below a tile, whose last lanes' columns are read from further back
    for pad, offset in ((0, 0), (3, 1)):
        x, W, b, r, _ = case(23, N, K, M, dtype, dev, pad, offset)
        out = dense.linear(x, W, b, residual=r, act="silu")
        z = wide(x) @ wide(W) + wide(b)
        err = sums(K + 1, wide(x).abs() @ wide(W).abs() + wide(b).abs())
        y = act("silu", z) + wide(r)
        check(out, y, LIP * err + 2.0 ** -20 * z.abs().clamp_min(1) + 2.0 ** -23 * (z.abs() + wide(r).abs()), "y")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("a", ["gelu", "silu", "relu"])
@pytest.mark.parametrize("N,K,M", [(1, 8, 2048), (40, 8, 2000), (100, 9, 20001), (700, 8, 2048), (2100, 8, 4000)])
def test_activations_of_fp32_results(dev, dtype, a, N, K, M):
    # z = W's first row, exactly; erfc(x) moves by 2 x^2 = z^2 of its argument's rounding (two of 2^-24),
    # and the library functions are good to 16 units in the last place
    W = torch.zeros(K, M, dtype=dtype, device=dev)
    W[0] = torch.linspace(-12.5, 12.5, M).to(dtype)
    x = torch.zeros(N, K, dtype=dtype, device=dev)
    x[:, 0] = 1
    y = dense.linear(x, W, act=a, out_dtype=torch.float32)
    z = wide(W[0])
    ref = act(a, z)
    check(y, ref.expand(N, M), (2.0 ** -23 * (z * z + 16) * ref.abs()).expand(N, M), a)
