"""Inputs of layer norm's gradient and of the 4-bit products whose fp32 sums are exact in any order, so that results can be
compared for equality, and of which no row, unit or part can be left out without a difference.

Every term is a small multiple of a power of two, and the terms' magnitudes add up to less than 2^24 of that power: all
partial sums are then fp32 values, whatever order they are formed in.
"""
import numpy as np
import torch

import layer_ref as ref

UNIT = 128  # features of a step of the products' kernels at most


# ------------------------------------------------------------------ the gradients of layer norm's weight and bias

def gradient(N, D, x, y, seed, device="cpu"):
    """(x, dy, stats): rows of 1 and 2, gradients of 1, 2 and 3, mean 0 and 1 / std 1 for every row, so that the
    normalised rows are x itself. A row adds 1 to 6 to each of dweight's sums, 1 to 3 to dbias's."""
    g = torch.Generator(device=device).manual_seed(seed)
    rows, dy = torch.empty(N, D, dtype=x, device=device), torch.empty(N, D, dtype=y, device=device)
    for n in range(0, N, 1 << 16):  # in pieces: the random numbers are wider than the rows
        part = rows[n:n + (1 << 16)].shape
        rows[n:n + (1 << 16)] = torch.randint(1, 3, part, generator=g, device=device, dtype=torch.int32).to(x)
        dy[n:n + (1 << 16)] = torch.randint(1, 4, part, generator=g, device=device, dtype=torch.int32).to(y)
    stats = torch.zeros(N, 2, dtype=torch.float64, device=device)
    stats[:, 1] = 1.0
    return rows, dy, stats


def gradient_sums(x, dy):
    """(dweight, dbias) in whole numbers."""
    dw, db = (torch.zeros(x.shape[1], dtype=torch.int64, device=x.device) for _ in range(2))
    for n in range(0, x.shape[0], 1 << 15):
        a, b = x[n:n + (1 << 15)].to(torch.int64), dy[n:n + (1 << 15)].to(torch.int64)
        dw += (a * b).sum(0)
        db += b.sum(0)
    return dw, db


def gradient_bound(N, magnitude):
    """The bound of such a sum of any numbers: a part's sum runs over 256 rows at most (twice: the product with h rounds too),
    up to 64 of a workgroup's are added, then max(512, N / 256) parts in 32 stretches, and the stretches."""
    depth = 2 * min(N, 256) + 64 + max(512, -(-N // 256)) // 32 + 1 + 32
    return depth * ref.E * magnitude


# N, D, type of x, type of dy: every width of a row's threads, one workgroup and many, odd ends, rows longer than registers.
GRADIENTS = [(3, 7, "float32", "float32"), (120, 30, "bfloat16", "bfloat16"), (70000, 16, "bfloat16", "bfloat16"),
             (70000, 100, "float16", "float16"), (5000, 300, "bfloat16", "bfloat16"), (300001, 5, "float32", "float16"),
             (9001, 1003, "float32", "bfloat16"), (1201, 2048, "bfloat16", "bfloat16"), (3001, 4095, "bfloat16", "bfloat16"),
             (2000, 8190, "bfloat16", "bfloat16"), (700, 16000, "float16", "float16"), (801, 9001, "float32", "float32"),
             (601, 17003, "bfloat16", "bfloat16")]


# ------------------------------------------------------------------ products

def four(n, K, seed, sizes, lowest, highest):
    """(codes, scales, values in 64 bits): codes of the given sizes and either sign, zeros past feature K, scale bytes
    from lowest to highest."""
    g = torch.Generator().manual_seed(seed)
    blocks = (K + 31) // 32
    four = torch.randint(0, sizes, (n, 32 * blocks), generator=g, dtype=torch.uint8)
    four |= torch.randint(0, 2, four.shape, generator=g, dtype=torch.uint8) << 3
    four[:, K - 1] = 2  # the last feature counts, at 1
    four[:, K:] = 0
    codes = four[:, 0::2] | four[:, 1::2] << 4
    scales = torch.randint(lowest, highest + 1, (n, blocks), generator=g).to(torch.uint8)
    return codes, scales, ref.values4(codes, scales, K)


def factors(N, K, M, packed, seed=1):
    """((rows, their values), (codes, scales, their values)): rows are whole numbers from -3 to 3 (the last feature's 1), or
    in 4 bits; rows of more than 4,096 features hold smaller numbers."""
    short = K <= 4096
    W = four(M, K, seed, 8 if short else 4, 126 if short else 127, 128 if short else 127)
    if packed:
        *x, xv = four(N, K, seed + 1, 8 if short else 3, 126 if short else 127, 128 if short else 127)
        return (x, xv), W
    g = torch.Generator().manual_seed(seed + 1)
    most = 3 if short else 1
    x = torch.randint(-most, most + 1, (N, K), generator=g).float()
    x[:, K - 1] = 1.0
    return (x, x.double()), W


def multiply(xv, wv):
    """(the product, the terms' magnitudes added up, the smallest power of two that terms are multiples of), in 64 bits."""
    unit = min(float(t[t != 0].abs().min()) for t in (xv, wv))
    low = 2.0 ** np.floor(np.log2(unit))
    return xv @ wv.t(), xv.abs() @ wv.abs().t(), low * low


# N, K, M: both sides of the rules that choose a tile, of the widths whose scales and rows are copied, rows of more
# features than are copied (65,536), and rows longer than a tile's loads reach (2^22).
PRODUCTS = [(1, 1, 1), (1, 1024, 4096), (15, 100, 130), (17, 1003, 70), (33, 2048, 300), (31, 64, 16000), (40, 100, 33000), (64, 96, 129),
            (128, 100, 1025), (16, 70, 8200), (300, 320, 2000), (257, 513, 515), (1000, 33, 2000), (9000, 200, 130),
            (1500, 577, 2000), (2011, 1003, 5625), (3300, 513, 3700), (3800, 1090, 3000), (2100, 768, 2100), (300, 4096, 520)]
LONG = [(2, 65600, 300), (300, 65541, 200), (150, 70001, 260), (2, (1 << 22) + 40, 5), (40, (1 << 22) + 40, 5)]
