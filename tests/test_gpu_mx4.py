"""The 4-bit operators against 64 bits, on the GPU."""
import math

import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2608_24067_amd.dense as dense
from dense_ref import act, check, sums, wide, LIP

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def spread(seed, N, K, dtype):
    """Values over many sizes, with ties, zeros, and blocks of one value, of none, of subnormals and of the largest."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, K, generator=g) * torch.exp(2 * torch.randn(N, 1, generator=g))
    tie = torch.rand(N, K, generator=g) < 0.2
    x = torch.where(tie, torch.round(x * 4) / 4, x)
    x[torch.rand(N, K, generator=g) < 0.05] = 0.0
    x[torch.rand(N, K, generator=g) < 0.02] *= -0.0
    if N > 4:
        x[1, :32] = 0.0
        x[2, :32] = 2.0 ** -24 if dtype == F16 else 1e-40
        x[3, :32] = torch.finfo(dtype).max
        x[4] = 1.0
    return x.to(dtype)


def codes_equal(q, x):
    codes, scales = ref.codes4(wide(x))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("N,K,extra", [(1, 1, 0), (5, 31, 0), (7, 32, 0), (33, 33, 1), (64, 100, 4), (130, 1003, 0),
                                       (17, 2048, 8), (300, 64, 3)])
def test_quantise_and_values(dev, dtype, N, K, extra):
    x = spread(N + K, N, K, dtype)
    rows = torch.full((N, K + extra), float("nan"), dtype=dtype, device=dev)[:, :K].copy_(x)
    q = dense.mx4_quantise(rows)
    codes_equal(q, x)
    columns = torch.full((K, N + extra), float("nan"), dtype=dtype, device=dev)[:, :N].copy_(x.t())
    c = dense.mx4_quantise(columns, columns=True)
    assert torch.equal(c.codes, q.codes) and torch.equal(c.scales, q.scales)
    want = ref.values4(q.codes, q.scales, K)
    for t in (F32, BF16, F16):
        to = torch.full((N, K + extra), 7.0, dtype=t, device=dev)
        dense.mx4_values(q, out=to[:, :K])
        assert torch.equal(to[:, :K].cpu(), want.to(t)) and (to[:, K:] == 7.0).all()
        to = torch.full((K, N + extra), 7.0, dtype=t, device=dev)
        dense.mx4_values(q, columns=True, out=to[:, :N])
        assert torch.equal(to[:, :N].cpu(), want.t().to(t)) and (to[:, N:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_blocks_with_no_number(dev, dtype, bad):
    x = spread(3, 6, 100, dtype)
    x[2, 40] = bad
    x[5, 99] = bad
    for columns in (False, True):
        q = dense.mx4_quantise((x.t().contiguous() if columns else x).to(dev), columns=columns)
        v = dense.mx4_values(q, dtype=F32).cpu()
        spoiled = torch.zeros(6, 100, dtype=torch.bool)
        spoiled[2, 32:64] = spoiled[5, 96:] = True
        assert torch.equal(v.isnan(), spoiled)
        y = dense.mx4_quantise(torch.where(spoiled, torch.zeros_like(x), x).to(dev))
        keep = ~torch.tensor([[False] * 4, [False] * 4, [False, True, False, False], [False] * 4, [False] * 4,
                              [False] * 3 + [True]])
        assert torch.equal(q.scales.cpu()[keep], y.scales.cpu()[keep])


def matrix(seed, K, M, dev):
    g = torch.Generator().manual_seed(seed)
    return dense.mx4_quantise((torch.randn(K, M, generator=g) * torch.exp(torch.randn(1, M, generator=g)) * K ** -0.5).to(dev),
                              columns=True)


def product(dev, dtype, N, K, M, packed, a="none", res=False, bias=None, out=None, extra=0):
    g = torch.Generator().manual_seed(N + 7 * K + M)
    x = torch.full((N, K + extra), float("nan"), dtype=dtype, device=dev)[:, :K].copy_(torch.randn(N, K, generator=g))
    W = matrix(K + M, K, M, dev)
    rows = dense.mx4_quantise(x) if packed else x
    xv = ref.values4(rows.codes, rows.scales, K) if packed else wide(x)
    wv = ref.values4(W.codes, W.scales, K)
    b = torch.randn(M, generator=g).to(bias).to(dev) if bias is not None else None
    r = torch.full((N, M + extra), float("nan"), dtype=dtype, device=dev)[:, :M].copy_(torch.randn(N, M, generator=g)) if res else None
    z = xv @ wv.t() + (wide(b) if b is not None else 0)
    size = xv.abs() @ wv.abs().t() + (wide(b).abs() if b is not None else 0)
    # fp16 rows meet the matrix as two values each: twice the terms
    off = LIP * sums(2 * K + 4, size) + (2.0 ** -20 * z.abs().clamp_min(1) if a != "none" else 0)
    want = act(a, z)
    if r is not None:
        want, off = want + wide(r), off + 2.0 ** -24 * (want.abs() + wide(r).abs())
    to = torch.full((N, M + extra), 7.0, dtype=out or dtype, device=dev)
    y = dense.mx4_linear(rows, W, b, residual=r, act=a, out=to[:, :M], dtype=dtype if packed else None)
    check(y, want, off, "y")
    assert (to[:, M:] == 7.0).all()
    return y


SIZES = [(1, 1, 1), (1, 64, 64), (1, 1024, 4096), (2, 33, 17), (15, 100, 130), (16, 256, 257), (17, 1003, 70), (33, 2048, 300),
         (64, 96, 129), (65, 4096, 40), (100, 1000, 1000), (129, 160, 256), (257, 513, 515), (500, 257, 130), (1000, 640, 384)]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", SIZES)
def test_product(dev, dtype, packed, N, K, M):
    product(dev, dtype, N, K, M, packed, bias=dtype, out=F32)
    product(dev, dtype, N, K, M, packed, bias=F32)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("a", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype,out", [(F16, None), (BF16, None), (BF16, F32)])
@pytest.mark.parametrize("N", [3, 40, 300])
def test_epilogue_and_strides(dev, dtype, out, packed, a, N):
    product(dev, dtype, N, 200, 203, packed, a=a, res=True, bias=F32, out=out, extra=3)
    product(dev, dtype, N, 256, 256, packed, a=a, res=True, out=out, extra=8)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("N", [1, 20, 200])
def test_no_number_stays_in_its_row_and_column(dev, packed, N):
    K, M = 300, 150
    g = torch.Generator().manual_seed(9)
    x, w = torch.randn(N, K, generator=g).to(BF16).to(dev), torch.randn(K, M, generator=g).to(dev)
    clean = dense.mx4_linear(dense.mx4_quantise(x) if packed else x, dense.mx4_quantise(w, columns=True))
    x[N - 1, 299] = math.inf
    w[40, 5] = math.nan
    W = dense.mx4_quantise(w, columns=True)
    y = dense.mx4_linear(dense.mx4_quantise(x) if packed else x, W)
    spoiled = torch.zeros(N, M, dtype=torch.bool)
    spoiled[N - 1] = spoiled[:, 5] = True
    assert not y.isfinite().cpu()[spoiled].any()
    assert y[:, 5].isnan().all()
    assert torch.equal(y.cpu()[~spoiled], clean.cpu()[~spoiled])


@pytest.mark.parametrize("N", [2, 70, 300])
def test_fp16_rows_of_all_sizes(dev, N):
    # subnormal and largest fp16 values, and a matrix whose scales fp16 does not hold
    K, M = 128, 40
    g = torch.Generator().manual_seed(21)
    x = (torch.randn(N, K, generator=g) * torch.exp2(torch.randint(-24, 13, (N, K), generator=g).float())).clamp(-65504, 65504).half()
    w = torch.randn(K, M, generator=g) * torch.exp2(torch.randint(-60, 20, (K, M), generator=g).float())
    W = dense.mx4_quantise(w.to(dev), columns=True)
    wv = ref.values4(W.codes, W.scales, K)
    y = dense.mx4_linear(x.to(dev), W, out_dtype=F32)
    check(y, wide(x) @ wv.t(), sums(2 * K, wide(x).abs() @ wv.abs().t()), "y")


@pytest.mark.parametrize("packed", [False, True])
def test_scales_at_the_ends(dev, packed):
    # products of the smallest and of large blocks; sums stay within fp32
    K, M = 64, 33
    x = torch.full((3, K), 2.0 ** -100, device=dev)
    x[1] = 2.0 ** 100
    x[2, 32:] = 0.0
    w = torch.full((K, M), 2.0 ** -20, device=dev)
    w[:, 1] = 2.0 ** 20
    w[:, 2] = 2.0 ** -126
    W = dense.mx4_quantise(w, columns=True)
    rows = dense.mx4_quantise(x) if packed else x.to(BF16)
    y = dense.mx4_linear(rows, W, out_dtype=F32, dtype=BF16 if packed else None)
    want = wide(x) @ wide(w)
    assert ((wide(y) - want).abs() <= 2.0 ** -149 * 2 + 2.0 ** -22 * want.abs()).all()


def test_same_bits_on_repeats_and_on_another_stream(dev):
    x = torch.randn(300, 700, generator=torch.Generator().manual_seed(1)).to(BF16).to(dev)
    W = matrix(4, 700, 500, dev)
    for n in (1, 20, 300):
        for packed in (False, True):
            rows = dense.mx4_quantise(x[:n]) if packed else x[:n]
            first = dense.mx4_linear(rows, W)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                again = dense.mx4_linear(rows, W)
            torch.cuda.current_stream().wait_stream(side)
            assert torch.equal(first, again)


@pytest.mark.parametrize("N", [1, 40, 400])
def test_captured_and_replayed(dev, N):
    W = matrix(5, 512, 768, dev)
    x = torch.zeros(N, 512, dtype=BF16, device=dev)
    codes, scales = torch.empty(N, 256, dtype=torch.uint8, device=dev), torch.empty(N, 16, dtype=torch.uint8, device=dev)
    y, y4 = torch.empty(N, 768, dtype=BF16, device=dev), torch.empty(N, 768, dtype=BF16, device=dev)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=dev)

    def step(a, b):
        dense.mx4_linear(x, W, act="silu", out=a, workspace=ws)
        dense.mx4_linear(dense.mx4_quantise(x, out=(codes, scales)), W, residual=a, out=b, workspace=ws)

    step(y, y4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y, y4)
    for k in range(3):
        x.copy_(torch.randn(N, 512, generator=torch.Generator().manual_seed(k)).to(BF16))
        a, b = torch.empty_like(y), torch.empty_like(y)
        step(a, b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(b, y4)


def test_residual_in_place_and_no_rows(dev):
    W = matrix(6, 100, 90, dev)
    x = torch.randn(50, 100, generator=torch.Generator().manual_seed(2)).to(BF16).to(dev)
    r = torch.randn(50, 90, generator=torch.Generator().manual_seed(3)).to(BF16).to(dev)
    want = dense.mx4_linear(x, W, residual=r, act="gelu")
    dense.mx4_linear(x, W, residual=r, act="gelu", out=r)
    assert torch.equal(r, want)
    assert dense.mx4_linear(x[:0], W).shape == (0, 90)
    q = dense.mx4_quantise(x[:0])
    assert q.codes.shape == (0, 64) and dense.mx4_values(q).shape == (0, 100)
    assert dense.mx4_linear(q, W).shape == (0, 90)


# Every tile, and its edges: sizes on both sides of the rules' bounds.
TILES = [(16, 70, 4096), (16, 70, 4100), (16, 70, 8192), (16, 70, 8200), (33, 200, 3000), (128, 100, 1025), (60, 96, 5000),
         (31, 64, 16000), (20000, 70, 10), (9000, 200, 130), (40, 100, 33000), (300, 320, 2000), (1000, 33, 2000), (1500, 577, 2000), (2500, 96, 5000), (3300, 513, 3700), (2000, 100, 5600), (3800, 1090, 3000)]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", TILES)
def test_tiles(dev, dtype, packed, N, K, M):
    product(dev, dtype, N, K, M, packed, a="silu", bias=dtype, res=True, extra=1)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_copied_in_strips(dev, dtype):
    # 36 MB of padded rows, so two strips; the last one is short
    product(dev, dtype, 8200, 2113, 130, False, res=True, bias=F32, extra=1)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("K", [160, 544, 600, 1000])
@pytest.mark.parametrize("N,M", [(300, 1500), (2100, 2100), (4000, 3400)])
def test_no_number_in_the_last_block(dev, dtype, packed, K, N, M):
    # what stands behind the last block meets neither its infinities nor its scale for NaN
    g = torch.Generator().manual_seed(K)
    x, w = torch.randn(N, K, generator=g).to(dtype).to(dev), torch.randn(K, M, generator=g).to(dev)
    clean = dense.mx4_linear(dense.mx4_quantise(x) if packed else x, dense.mx4_quantise(w, columns=True))
    x[N - 2, K - 1] = math.inf
    w[K - 1, M - 3] = math.nan
    y = dense.mx4_linear(dense.mx4_quantise(x) if packed else x, dense.mx4_quantise(w, columns=True))
    spoiled = torch.zeros(N, M, dtype=torch.bool, device=dev)
    spoiled[N - 2] = spoiled[:, M - 3] = True
    assert not y[spoiled].isfinite().any()
    assert torch.equal(y[~spoiled], clean[~spoiled])


@pytest.mark.parametrize("packed", [False, True])
def test_operands_off_their_alignment(dev, packed):
    # scales that start on any byte and rows that start on any element have the same product
    K, N, M = 512, 700, 900
    W = matrix(8, K, M, dev)
    x = torch.randn(N, K, generator=torch.Generator().manual_seed(8)).to(BF16).to(dev)
    rows = dense.mx4_quantise(x) if packed else x

    def moved(s):
        return torch.empty(s.numel() + 5, dtype=torch.uint8, device=dev)[5:].view(s.shape).copy_(s)

    at = torch.empty(N * (K + 2) + 1, dtype=BF16, device=dev)[1:].view(N, K + 2)[:, :K].copy_(x)
    other = dense.Mx4(rows.codes, moved(rows.scales), K) if packed else at
    want = ref.values4(rows.codes, rows.scales, K) if packed else wide(x)
    wv = ref.values4(W.codes, W.scales, K)
    bound = sums(K, want.abs() @ wv.abs().t())
    for r, w in ((rows, W), (other, W), (rows, dense.Mx4(W.codes, moved(W.scales), K)), (other, dense.Mx4(W.codes, moved(W.scales), K))):
        y = dense.mx4_linear(r, w, out_dtype=F32, dtype=BF16 if packed else None)
        check(y, want @ wv.t(), bound, "y")


def codes_and_scales(seed, K, M, lowest, highest, dev):
    """A 4-bit matrix of random codes whose scale bytes are lowest ... highest, both among them, by column and block."""
    g = torch.Generator().manual_seed(seed)
    blocks = (K + 31) // 32
    codes = torch.randint(0, 256, (M, blocks * 16), generator=g, dtype=torch.uint8)
    if K % 32:
        codes[:, blocks * 16 - (32 - K % 32) // 2:] = 0
    scales = torch.randint(lowest, highest + 1, (M, blocks), generator=g).to(torch.uint8)
    scales[::7, 0], scales[::5, -1] = lowest, highest
    return codes, scales


@pytest.mark.parametrize("N,M", [(300, 1500), (700, 2100), (4000, 3400)])
@pytest.mark.parametrize("lowest,highest", [(120, 124), (100, 126), (100, 127), (60, 140), (1, 20), (190, 215), (215, 220)])
def test_fp16_rows_and_any_range_of_scales(dev, N, M, lowest, highest):
    # 2^26 and less within a tile, and more
    K = 160
    codes, scales = codes_and_scales(lowest + highest, K, M, lowest, highest, dev)
    W = dense.Mx4(codes.to(dev), scales.to(dev), K)
    g = torch.Generator().manual_seed(N)
    x = (torch.randn(N, K, generator=g) * torch.exp2(torch.randint(-22, 6, (N, K), generator=g).float())).half()
    b = torch.randn(M, generator=g)
    wv = ref.values4(codes, scales, K)
    size = wide(x).abs() @ wv.abs().t() + wide(b).abs()
    y = dense.mx4_linear(x.to(dev), W, b.to(dev), out_dtype=F32)
    check(y, wide(x) @ wv.t() + wide(b), sums(K + 4, size) + 2.0 ** -148, "y")


@pytest.mark.parametrize("N,M", [(300, 1500), (4000, 3400)])
@pytest.mark.parametrize("how", ["zeros", "smallest", "nan"])
def test_fp16_rows_and_scales_of_no_size(dev, N, M, how):
    # blocks of zeros have the scale 0, and so have blocks of the smallest values; 255 stands for NaN
    K = 544
    codes, scales = codes_and_scales(5, K, M, 128, 130, dev)
    g = torch.Generator().manual_seed(N + 1)
    some = torch.rand(scales.shape, generator=g) < 0.1
    scales[some] = 0
    if how != "smallest":
        codes.view(M, -1, 16)[some] = 0
    if how == "nan":
        scales[7, 3] = 255
    x = torch.randn(N, K, generator=g).half()
    if how == "smallest":
        x[5] = 0
        x.view(N, -1, 32)[5, some[9]] = 1.0  # nothing but the smallest of column 9
    W = dense.Mx4(codes.to(dev), scales.to(dev), K)
    y = dense.mx4_linear(x.to(dev), W, out_dtype=F32)
    wv = ref.values4(codes, scales, K)
    if how == "nan":
        assert y[:, 7].isnan().all()
        wv[7], y[:, 7] = 0, 0
    size = wide(x).abs() @ wv.abs().t()
    check(y, wide(x) @ wv.t(), sums(K, size) + 2.0 ** -148, "y")


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", [(40, 256, 300), (700, 320, 900), (1500, 577, 2000), (3300, 512, 3700)])
def test_residual_is_the_result(dev, dtype, packed, N, K, M):
    W = matrix(N, K, M, dev)
    g = torch.Generator().manual_seed(M)
    x, r = torch.randn(N, K, generator=g).to(dtype).to(dev), torch.randn(N, M + 2, generator=g).to(dtype).to(dev)
    rows = dense.mx4_quantise(x) if packed else x
    want = dense.mx4_linear(rows, W, residual=r[:, 1:M + 1], act="silu")
    sides = r[:, 0].clone(), r[:, M + 1].clone()
    dense.mx4_linear(rows, W, residual=r[:, 1:M + 1], act="silu", out=r[:, 1:M + 1])
    assert torch.equal(r[:, 1:M + 1], want) and torch.equal(r[:, 0], sides[0]) and torch.equal(r[:, M + 1], sides[1])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N", [3, 300])
def test_type_of_a_new_result_of_packed_rows(dev, dtype, N):
    W = matrix(9, 96, 130, dev)
    rows = dense.mx4_quantise(torch.randn(N, 96, generator=torch.Generator().manual_seed(9)).to(dev))
    want = dense.mx4_linear(rows, W, dtype=dtype)
    got = dense.mx4_linear(rows, W, out_dtype=dtype)
    assert got.dtype == dtype and torch.equal(got, want)
    b = torch.randn(130, generator=torch.Generator().manual_seed(10)).to(dtype).to(dev)
    assert torch.equal(dense.mx4_linear(rows, W, b, out_dtype=dtype), dense.mx4_linear(rows, W, b))
    with pytest.raises(TypeError):
        dense.mx4_linear(rows, W, b, out_dtype=F16 if dtype == BF16 else BF16)


@pytest.mark.parametrize("N,K,M", [(2, 544, 40), (16, 544, 4100), (40, 544, 3000), (33, 544, 9000), (300, 544, 1500), (1000, 544, 2000),
                                   (2011, 544, 5625), (4000, 544, 3400)])
def test_bf16_rows_and_the_smallest_scales(dev, N, K, M):
    # the scale 0 stands for 2^-127, under which the codes for 0.5 to 1.5 are subnormal in bf16
    codes, scales = codes_and_scales(6, K, M, 0, 2, dev)
    g = torch.Generator().manual_seed(N)
    x = (torch.randn(N, K, generator=g) * 2.0 ** 100).to(BF16)
    if N > 2:
        x[1] = 2.0 ** -100 * x[1]  # products that are subnormal in fp32
    W = dense.Mx4(codes.to(dev), scales.to(dev), K)
    wv = ref.values4(codes, scales, K)
    y = dense.mx4_linear(x.to(dev), W, out_dtype=F32)
    check(y, wide(x) @ wv.t(), sums(K, wide(x).abs() @ wv.abs().t()) + 2.0 ** -147, "y")
    # the four smallest sizes alone
    codes &= 0x33
    wv = ref.values4(codes, scales * 0, K)
    y = dense.mx4_linear(x.to(dev), dense.Mx4(codes.to(dev), (scales * 0).to(dev), K), out_dtype=F32)
    check(y, wide(x) @ wv.t(), sums(K, wide(x).abs() @ wv.abs().t()) + 2.0 ** -147, "y, the smallest")


@pytest.mark.parametrize("columns", [False, True])
def test_values_of_every_code_and_scale(dev, columns):
    # a row for each scale byte: its blocks hold every code at every place
    K = 64
    four = (torch.arange(256)[:, None] + torch.arange(K)[None, :] * 5) % 16
    codes = (four[:, 0::2] | four[:, 1::2] << 4).to(torch.uint8)
    scales = torch.arange(256)[:, None].expand(256, 2).to(torch.uint8).contiguous()
    want = ref.values4(codes, scales, K)
    q = dense.Mx4(codes.to(dev), scales.to(dev), K)
    for t in (F32, BF16, F16):
        v = dense.mx4_values(q, columns=columns, dtype=t).cpu()
        v = v.t() if columns else v
        assert torch.equal(v.isnan(), want.isnan())
        assert torch.equal(v[:255], want.to(t)[:255])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_codes_at_every_exponent(dev, dtype):
    # a block for each exponent of its largest value, subnormals too, and smaller values down to 2^-6 of it: ties, their
    # neighbours on either side, and any bits
    g = torch.Generator().manual_seed(31)
    kind, sign, last = {F32: (torch.int32, 1 << 31, 23), BF16: (torch.int16, 1 << 15, 7), F16: (torch.int16, 1 << 15, 10)}[dtype]
    most = (torch.tensor(torch.finfo(dtype).max, dtype=dtype).view(kind).item() >> last) + 1
    rows = []
    for e in range(most):
        for r in range(8):
            top = (e << last) + int(torch.randint(0, 1 << last, (1,), generator=g))
            low = max(0, top - (6 << last))
            bits = torch.randint(low, top + 1, (32,), generator=g)
            if r % 2:  # one bit behind the point, or two, and a step beside it
                bits = (bits >> (last - 2) << (last - 2)) + torch.randint(-1, 2, (32,), generator=g)
            bits = bits.clamp(0, top)
            bits[int(torch.randint(0, 32, (1,), generator=g))] = top
            bits = bits + sign * torch.randint(0, 2, (32,), generator=g)
            rows.append(bits)
    bits = torch.stack(rows)
    bits = torch.where(bits >= sign, bits - 2 * sign, bits).to(kind)
    x = bits.view(dtype)
    assert x.isfinite().all()
    codes_equal(dense.mx4_quantise(x.to(dev)), x)
    codes_equal(dense.mx4_quantise(x.t().contiguous().to(dev), columns=True), x)


# N, M: every tile for K = 96, by both kinds of rows
EVERY_TILE = [(3, 50), (16, 4200), (40, 3000), (33, 9000), (128, 2100), (300, 1500), (1000, 2000), (2011, 5625), (4000, 3400)]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,M", EVERY_TILE)
def test_blocks_for_nan_whose_codes_are_zeros(dev, dtype, packed, N, M):
    K = 96
    codes, scales = codes_and_scales(7, K, M, 126, 128, dev)
    codes[5, 16:32], scales[5, 1] = 0, 255
    codes[M - 1], scales[M - 1] = 0, 255
    W = dense.Mx4(codes.to(dev), scales.to(dev), K)
    spoiled = torch.zeros(N, M, dtype=torch.bool, device=dev)
    spoiled[:, 5] = spoiled[:, M - 1] = True
    if packed:
        x, xs = codes_and_scales(8, K, N, 126, 128, dev)
        x[N - 1, 32:48], xs[N - 1, 2] = 0, 255
        spoiled[N - 1] = True
        rows = dense.Mx4(x.to(dev), xs.to(dev), K)
    else:
        rows = torch.randn(N, K, generator=torch.Generator().manual_seed(N)).to(dtype).to(dev)
    for act_ in ("none", "relu", "silu", "gelu"):
        y = dense.mx4_linear(rows, W, act=act_, dtype=dtype if packed else None)
        assert torch.equal(y.isnan(), spoiled), act_


@pytest.mark.parametrize("N,M", EVERY_TILE)
def test_packed_rows_and_scales_from_end_to_end(dev, N, M):
    # a scale for each row and one for each column: their powers cancel, multiply beyond fp32's range, or below it
    K = 96
    g = torch.Generator().manual_seed(41)
    codes, scales = codes_and_scales(9, K, M, 127, 127, dev)
    x, xs = codes_and_scales(10, K, N, 127, 127, dev)
    ends = torch.tensor([0, 1, 2, 20, 60, 63, 64, 65, 100, 126, 127, 128, 150, 189, 190, 191, 220, 240, 250, 252], dtype=torch.uint8)
    scales[:] = ends[torch.randint(0, len(ends), (M, 1), generator=g)]
    xs[:] = ends[torch.randint(0, len(ends), (N, 1), generator=g)]
    y = wide(dense.mx4_linear(dense.Mx4(x.to(dev), xs.to(dev), K), dense.Mx4(codes.to(dev), scales.to(dev), K), out_dtype=F32))
    xv, wv = ref.values4(x, xs, K), ref.values4(codes, scales, K)
    want, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    inside = size < 2.0 ** 127
    off = sums(K, size) + K * 2.0 ** -149  # additions of subnormal sums round, too
    assert ((y - want).abs() <= off)[inside].all()
    beyond = want.abs() - sums(K, size) > 2.0 ** 128
    assert (~y.isfinite())[beyond].all()


@pytest.mark.parametrize("N,M", EVERY_TILE)
def test_bf16_rows_and_scales_from_end_to_end(dev, N, M):
    K = 96
    g = torch.Generator().manual_seed(43)
    codes, scales = codes_and_scales(11, K, M, 127, 127, dev)
    ends = torch.tensor([0, 1, 2, 20, 60, 64, 100, 126, 127, 128, 150, 190, 220, 240, 250, 252], dtype=torch.uint8)
    scales[:] = ends[torch.randint(0, len(ends), (M, 1), generator=g)]
    x = (torch.randn(N, K, generator=g) * torch.exp2(torch.randint(-130, 120, (N, 1), generator=g).float())).to(BF16)
    y = wide(dense.mx4_linear(x.to(dev), dense.Mx4(codes.to(dev), scales.to(dev), K), out_dtype=F32))
    wv = ref.values4(codes, scales, K)
    want, size = wide(x) @ wv.t(), wide(x).abs() @ wv.abs().t()
    inside = size < 2.0 ** 127
    assert ((y - want).abs() <= sums(K, size) + K * 2.0 ** -149)[inside].all()
    beyond = want.abs() - sums(K, size) > 2.0 ** 128
    assert (~y.isfinite())[beyond].all()
