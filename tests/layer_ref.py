"""Plain forms of layer norm, AdamW and the 4-bit operators (include/som_dense.h), on the CPU in 64 bits, and the bounds
the tests use. Every fp32 operation rounds by at most E = 2^-24 of its result."""
import numpy as np
import torch

from dense_ref import wide

E = 2.0 ** -24


# ------------------------------------------------------------------ layer norm

def norm(x, weight, bias, eps):
    """(y, bound of what fp32 adds before the last rounding, mean, 1 / std) of rows in 64 bits.

    h = ((x - hi) - lo) inv: two subtractions, a factor rounded once, a product: 4 E |h| and a little; lo itself is
    rounded to E^2 |mean|. y = h w + b in one rounding."""
    x = wide(x)
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    inv = 1 / torch.sqrt(var + eps)
    h = (x - mean) * inv
    w = wide(weight) if weight is not None else torch.ones(x.shape[1], dtype=torch.float64)
    b = wide(bias) if bias is not None else torch.zeros(x.shape[1], dtype=torch.float64)
    y = h * w + b
    return y, (6 * E * h.abs() + 2 * E * E * mean.abs() * inv) * w.abs() + E * y.abs(), mean, inv


def norm_grad(x, weight, dy, eps, add=None):
    """((dx, bound), (dweight, bound), (dbias, bound)) in 64 bits. fp32 sums over n terms in any order are off by at
    most (n + 2) E of the magnitudes' sum; twice that is taken, as for products."""
    N, D = x.shape
    _, _, mean, inv = norm(x, weight, None, eps)
    h = (wide(x) - mean) * inv
    g = wide(dy)
    w = wide(weight) if weight is not None else torch.ones(D, dtype=torch.float64)
    u = g * w
    s, q = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    dx = (u - s - h * q) * inv
    off_s = (2 * (D + 2) + 4) * E * u.abs().mean(1, keepdim=True)
    off_q = (2 * (D + 2) + 12) * E * (u * h).abs().mean(1, keepdim=True)
    bound = inv * (off_s + h.abs() * off_q + 16 * E * (u.abs() + s.abs() + (h * q).abs()))
    if add is not None:
        dx = dx + wide(add)
        bound = bound + E * (dx.abs() + wide(add).abs())
    dw, db = (g * h).sum(0), g.sum(0)
    return ((dx, bound), (dw, (2 * (N + 2) + 8) * E * (g * h).abs().sum(0)), (db, 2 * (N + 2) * E * g.abs().sum(0)))


# ------------------------------------------------------------------ AdamW

def adamw(p, g, m, v, step, lr, betas, eps, weight_decay, grad_scale=1.0):
    """((p, bound), (m, bound), (v, bound)) after a step, from values in 64 bits."""
    b1, b2 = betas
    g = wide(g) * grad_scale
    p, m, v = wide(p), wide(m), wide(v)
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    # each product has a rounded factor and rounds once, g rounds once, the sum once
    off_m = 5 * E * ((b1 * m).abs() + ((1 - b1) * g).abs()) + 2.0 ** -148
    off_v = 6 * E * v2 + 2.0 ** -148
    rate = lr / (1 - b1 ** step)
    den = torch.sqrt(v2 / (1 - b2 ** step)) + eps
    update = rate * m2 / den
    # the denominator: sqrt of a value off by 6 E (half of it), its rounding, the factor's, the product's and the sum's:
    # 8 E; the quotient, the rate and their product: 3 E more. Where v underflows, its absolute error counts.
    root_off = torch.sqrt((v2 + off_v) / (1 - b2 ** step)) - torch.sqrt((v2 - off_v).clamp_min(0) / (1 - b2 ** step))
    off = update.abs() * 12 * E + rate * off_m / den + update.abs() * root_off / den
    p2 = p * (1 - lr * weight_decay) - update
    return (p2, 4 * E * p.abs() + off), (m2, off_m), (v2, off_v)


def adamw_between(p, g, m, v, step, lr, betas, eps, weight_decay):
    """(low, high) of p after a step where v may underflow: any v that fp32 may hold instead is allowed, and nothing more.

    v is off by off_v at most, so the root lies between those of v - off_v (not below 0) and v + off_v. The root, its
    factor, eps, their fma, the reciprocal, its product with m and the rate round by 10 E together, p's decay by 3 E;
    what is subnormal on the way is off by 2^-149."""
    b1, b2 = betas
    _, (m2, off_m), (v2, off_v) = adamw(p, g, m, v, step, lr, betas, eps, weight_decay)
    rate = lr / (1 - b1 ** step)
    dens = [torch.sqrt(t / (1 - b2 ** step)) + eps for t in ((v2 - off_v).clamp_min(0), v2 + off_v)]
    updates = torch.stack([rate * t / d for t in (m2 - off_m, m2 + off_m) for d in dens])
    keep = wide(p) * (1 - lr * weight_decay)
    off = 3 * E * wide(p).abs() + (1 + rate) * 2.0 ** -148
    return (keep - (updates + 10 * E * updates.abs()).amax(0) - off,
            keep - (updates - 10 * E * updates.abs()).amin(0) + off)

BLOCK = 256
U32 = np.uint32


def mix(h):
    h = h ^ (h >> U32(16))
    h = h * U32(0xBB67AE85)
    h = h ^ (h >> U32(15))
    h = h * U32(0x6A09E667)
    return h ^ (h >> U32(16))


def random_bits(n, tensor, seed, step):
    """32 bits for each element, as the step draws them."""
    with np.errstate(over="ignore"):
        key = mix(U32([(seed + step * 0x9E3779B1 + tensor * 0x1F83D9AB) & 0xFFFFFFFF]))
        i = np.arange(n, dtype=np.uint64)
        low, high = (i & np.uint64(0xFFFFFFFF)).astype(U32), (i >> np.uint64(32)).astype(U32)
        return mix(low * U32(0x9E3779B1) + high * U32(0xA54FF53B) + key)


def _power(e):
    return np.ldexp(np.float32(1), e).astype(np.float32)


def codes8(x, signed, random):
    """(codes, scales) of fp32 values, by 16 random bits a value."""
    n = x.size
    x = np.pad(x.astype(np.float32), (0, -n % BLOCK)).reshape(-1, BLOCK)
    random = np.pad(random.astype(np.int64), (0, -n % BLOCK)).reshape(-1, BLOCK)
    top = (np.abs(x).view(np.int32) & 0x7FFFFFFF).max(1, keepdims=True).astype(np.int64)
    scale = np.minimum((top + 0xFFFFF) >> 23, 255)
    scale = np.where(scale < 27, 0, scale)
    with np.errstate(invalid="ignore", over="ignore"):
        # exact but for what falls below fp32's smallest values
        y = (np.abs(x).astype(np.float64) * np.ldexp(1.0, (127 - scale).astype(np.int32))).astype(np.float32)
        y = (y.astype(np.float64) * 2.0 ** (-112 if signed else -96)).astype(np.float32)
    c = (y.view(np.int32).astype(np.int64) + (random << 4)) >> 20
    if signed:
        c = np.minimum(c, 127) | np.where(x < 0, 128, 0)
    else:
        c = np.where(x > 0, np.clip(c, 1, 255), 0)
    return np.where(scale == 0, 0, c).astype(np.uint8).reshape(-1)[:n], scale.astype(np.uint8).reshape(-1)


def values8(codes, scales, signed):
    """What they stand for, in 64 bits, from the fields."""
    c = codes.astype(np.int64)
    size = c & 127 if signed else c
    field, last, low = size >> 3, (size & 7).astype(np.float64), -14 if signed else -30
    v = np.where(field > 0, (8 + last) * np.ldexp(1.0, (field + low - 4).astype(np.int32)), last * 2.0 ** (low - 3))
    v = np.where((c >= 128) & signed, -v, v)
    s = np.repeat(scales.astype(np.int64), BLOCK)[:c.size]
    v = v * np.ldexp(1.0, (s - 127).astype(np.int32))
    return np.where(s == 255, np.nan, np.where(s == 0, 0.0, v))


# ------------------------------------------------------------------ 4 bits

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def codes4(x):
    """(codes, scales) of rows, value by value in 64 bits: the nearest size, the even code of two equally near."""
    n, K = x.shape
    x = np.pad(wide(x).numpy() if isinstance(x, torch.Tensor) else x.astype(np.float64), ((0, 0), (0, -K % 32)))
    x = x.reshape(n, -1, 32)
    top = np.abs(x).max(2, initial=0.0)
    bad = ~np.isfinite(x).all(2)
    _, e = np.frexp(np.where(bad, 1.0, top))
    scale = np.where(bad, 255, np.where(top > 0, np.maximum(e - 1 - 2 + 127, 0), 0))
    y = np.abs(np.where(bad[..., None], 0.0, x)) * np.ldexp(1.0, (127 - np.where(bad, 127, scale)).astype(np.int32))[..., None]
    away = np.abs(y[..., None] - SIZES)  # ties: the even code is the lower one's neighbour either way
    code = np.zeros(y.shape, np.int64)
    best = away[..., 0]
    for k in range(1, 8):
        nearer = (away[..., k] < best) | ((away[..., k] == best) & (k % 2 == 0))
        code, best = np.where(nearer, k, code), np.where(nearer, away[..., k], best)
    code |= np.where(np.signbit(x), 8, 0)
    code = code.reshape(n, -1, 2)
    return (code[..., 0] | code[..., 1] << 4).astype(np.uint8), scale.astype(np.uint8)


def values4(codes, scales, K):
    c, s = (t.cpu().numpy().astype(np.int64) if isinstance(t, torch.Tensor) else t.astype(np.int64) for t in (codes, scales))
    four = np.stack((c & 15, c >> 4), 2).reshape(c.shape[0], -1)
    v = np.where(four >= 8, -SIZES[four % 8], SIZES[four % 8])
    s = np.repeat(s, 32, 1)
    v = np.where(s == 255, np.nan, v * np.ldexp(1.0, (s - 127).astype(np.int32)))
    return torch.from_numpy(v[:, :K])
