"""Layer norm, AdamW and the 4-bit operators where offsets pass 32 bits: rows and elements on both sides of 2^31 and at the
end, against 64 bits."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2608_24067_amd.dense as dense
from dense_ref import check, sums, wide

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
N, D = 1050001, 2048  # 2^31 elements at row 1,048,576
ROWS = [0, 1, 524287, 524288, 1048575, 1048576, 1048577, 1049999, 1050000]


@pytest.fixture(scope="module")
def rows(dev):
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.empty(N, D, dtype=BF16, device=dev)
    for n in range(0, N, 1 << 17):
        x[n:n + (1 << 17)].normal_(generator=g)
    yield x
    del x
    torch.cuda.empty_cache()


def test_layer_norm(dev, rows):
    g = torch.Generator().manual_seed(2)
    w, b = (1 + 0.3 * torch.randn(D, generator=g)).to(dev), torch.randn(D, generator=g).to(dev)
    stats = torch.empty(N, 2, dtype=torch.float64, device=dev)
    y = dense.layer_norm(rows, w, b, stats=stats)
    want, bound, *_ = ref.norm(rows[ROWS], w, b, 1e-5)
    check(y[ROWS], want, bound, "y")
    dx, dw, db = dense.layer_norm_bwd(rows, y, stats, w, add=rows)  # any dy will do: the results
    (vx, off), *_ = ref.norm_grad(rows[ROWS], w, y[ROWS], 1e-5, rows[ROWS])
    check(dx[ROWS], vx, off, "dx")
    sw, sb = torch.zeros(2, D, dtype=torch.float64, device=dev), torch.zeros(2, D, dtype=torch.float64, device=dev)
    for n in range(0, N, 1 << 15):
        h = (rows[n:n + (1 << 15)].double() - stats[n:n + (1 << 15), :1]) * stats[n:n + (1 << 15), 1:]
        dy = y[n:n + (1 << 15)].double()
        sw[0] += (dy * h).sum(0)
        sw[1] += (dy * h).abs().sum(0)
        sb[0] += dy.sum(0)
        sb[1] += dy.abs().sum(0)
    check(dw, wide(sw[0]), (2 * (N + 2) + 8) * ref.E * wide(sw[1]), "dweight")
    check(db, wide(sb[0]), 2 * (N + 2) * ref.E * wide(sb[1]), "dbias")


def test_quantise_and_values(dev, rows):
    q = dense.mx4_quantise(rows)
    codes, scales = ref.codes4(wide(rows[ROWS]))
    assert np.array_equal(q.codes[ROWS].cpu().numpy(), codes) and np.array_equal(q.scales[ROWS].cpu().numpy(), scales)
    out = torch.empty_like(rows)
    v = dense.mx4_values(q, out=out)
    assert torch.equal(v[ROWS].cpu().double(), ref.values4(codes, scales, D))
    # the same memory as a feature-major matrix of 2,048 features
    columns = rows.view(D, N)
    c = dense.mx4_quantise(columns, columns=True)
    codes, scales = ref.codes4(wide(columns[:, ROWS]).t().contiguous())
    assert np.array_equal(c.codes[ROWS].cpu().numpy(), codes) and np.array_equal(c.scales[ROWS].cpu().numpy(), scales)
    v = dense.mx4_values(c, columns=True, out=out.view(D, N))
    assert torch.equal(v[:, ROWS].t().cpu().double(), ref.values4(codes, scales, D))


@pytest.mark.parametrize("packed", [False, True])
def test_product(dev, rows, packed):
    M = 2051  # the results pass 2^31, too
    g = torch.Generator().manual_seed(3)
    W = dense.mx4_quantise((torch.randn(D, M, generator=g) * D ** -0.5).to(dev), columns=True)
    x = dense.mx4_quantise(rows) if packed else rows
    y = dense.mx4_linear(x, W, act="gelu")
    xv = ref.values4(x.codes[ROWS], x.scales[ROWS], D) if packed else wide(rows[ROWS])
    wv = ref.values4(W.codes, W.scales, D)
    z = xv @ wv.t()
    off = 1.13 * sums(D, xv.abs() @ wv.abs().t()) + 2.0 ** -20 * z.abs().clamp_min(1)
    check(y[ROWS], z * 0.5 * torch.erfc(-z * 0.5 ** 0.5), off, "y")


@pytest.mark.parametrize("packed", [False, True])
def test_product_of_long_rows(dev, packed):
    # rows longer than what a tile's loads reach
    K, M = (1 << 22) + 40, 5
    g = torch.Generator().manual_seed(4)
    W = dense.mx4_quantise((torch.randn(K, M, generator=g) * K ** -0.5).to(dev), columns=True)
    for n in (2, 40):
        x = torch.randn(n, K, generator=g).to(BF16).to(dev)
        r = dense.mx4_quantise(x) if packed else x
        xv = ref.values4(r.codes, r.scales, K) if packed else wide(x)
        wv = ref.values4(W.codes, W.scales, K)
        y = dense.mx4_linear(r, W, out_dtype=F32)
        check(y, xv @ wv.t(), sums(K, xv.abs() @ wv.abs().t()), "y")


def test_adamw(dev):
    n = (1 << 31) + 70001
    p, g = torch.empty(n, dtype=BF16, device=dev), torch.empty(n, dtype=BF16, device=dev)
    gen = torch.Generator(device=dev).manual_seed(5)
    for at in range(0, n, 1 << 28):
        p[at:at + (1 << 28)].normal_(generator=gen)
        g[at:at + (1 << 28)].normal_(generator=gen)
    g.mul_(1e-2)
    parts = [(0, 1024), ((1 << 31) - 1024, (1 << 31) + 1024), ((n - 70001 % 256 - 1024), n)]  # whole blocks
    before = [p[a:b].clone() for a, b in parts]
    lr, betas, eps, decay = 1e-3, (0.9, 0.999), 1e-8, 0.01
    for bits in (8, 32):
        state = dense.adamw_state(p, bits)
        dense.adamw([p], [g], [state], 1, lr=lr, betas=betas, eps=eps, weight_decay=decay, seed=77)
        for (a, b), old in zip(parts, before):
            zero = torch.zeros(b - a, dtype=torch.float64)
            (want, off), (m, off_m), (v, off_v) = ref.adamw(old, g[a:b], zero, zero, 1, lr, betas, eps, decay)
            check(p[a:b], want, off, "p")
            if bits == 32:
                check(state.m[a:b], m, off_m, "m")
                check(state.v[a:b], v, off_v, "v")
                continue
            key = ref.mix(np.array([(77 + 0x9E3779B1) & 0xFFFFFFFF], dtype=np.uint32))
            with np.errstate(over="ignore"):
                random = ref.mix(np.arange(a, b, dtype=np.uint64).astype(np.uint32) * np.uint32(0x9E3779B1) + key)
            blocks = slice(a // 256, (b + 255) // 256)
            one, two = np.float32(1 - betas[0]), np.float32(1 - betas[1])
            grad = g[a:b].float().cpu().numpy()
            for name, x, codes, scales, signed, bit in (
                    ("m", grad * one, state.m, state.m_scales, True, random & np.uint32(0xFFFF)),
                    ("v", grad * grad * two, state.v, state.v_scales, False, random >> np.uint32(16))):
                c, s = ref.codes8(x, signed, bit)
                assert np.array_equal(scales[blocks].cpu().numpy(), s), name
                assert np.array_equal(codes[a:b].cpu().numpy(), c), name
        for (a, b), old in zip(parts, before):
            p[a:b] = old
        del state
    del p, g
    torch.cuda.empty_cache()
