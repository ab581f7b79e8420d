"""The training operators from their definitions, in 64 bits with numpy, for
the tests (no code of the library)."""
import math

import numpy as np

EPS32 = 2.0 ** -24          # half a step of fp32, relative
HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
SMALLEST = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}
BLOCK = 128


def rounding(y, dtype):
    """Bound of one rounding of y to the type."""
    return np.abs(y) * HALF_STEP[dtype] + SMALLEST[dtype]


def gathered(table, ids):
    """Rows of the candidates, 0 for ids that are no entity."""
    inside = (ids >= 0) & (ids < table.shape[0])
    return np.where(inside[..., None], table[np.where(inside, ids, 0)], 0.0)


def valid_places(batch, n, n_valid=None, mask=None):
    if mask is not None:
        at = np.arange(n)
        return ((mask.view(np.uint32)[:, at // 32] >> (at % 32).astype(np.uint32)) & 1).astype(bool)
    limit = np.full(batch, n) if n_valid is None else n_valid
    return np.arange(n)[None, :] < limit[:, None]


def softplus(x):
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def preference(pos, neg, ref_pos, ref_neg, valid, kind, beta, smoothing):
    """loss [B], d loss / d pos [B], d loss / d neg [B, n], and z [B, n]."""
    if ref_pos is not None:
        pos, neg = pos - ref_pos, neg - ref_neg
    z = np.where(valid, beta * (pos[:, None] - np.where(valid, neg, 0.0)), 0.0)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "pairs":
            c = np.maximum(valid.sum(1), 1)[:, None]
            each = (1 - smoothing) * softplus(-z)
            if smoothing:
                each = each + smoothing * softplus(z)
            loss = (np.where(valid, each, 0.0) / c).sum(1)
            slope = np.where(valid, (smoothing - 1.0 / (1.0 + np.exp(z))) / c, 0.0)
        else:
            t = np.where(valid, -z, -np.inf)
            top = np.maximum(t.max(1, initial=0.0), 0.0)
            e = np.exp(t - top[:, None])
            s = e.sum(1)
            total = np.exp(-top) + s
            loss = np.where(top > 0, top + np.log(total), np.log1p(s))
            slope = -e / total[:, None]
    return loss, beta * slope.sum(1), -beta * slope, z


M32 = 0xFFFFFFFF


def mix(x):
    x = np.asarray(x, np.uint64)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x7FEB352D)) & np.uint64(M32)
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x846CA68B)) & np.uint64(M32)
    return x ^ (x >> np.uint64(16))


def draws(seed, step, index, row, dim):
    """The 32-bit words that round the elements of row `row` of a tensor."""
    k = mix(mix(seed & M32) ^ np.uint64(seed >> 32))
    k = mix(mix((int(k) + step) & M32) ^ np.uint64(step >> 32))
    key = int(mix((int(k) + index) & M32))
    at = np.arange(dim)
    block = row * (-(-dim // BLOCK)) + at // BLOCK
    base = mix((mix(np.uint64(key) ^ (block.astype(np.uint64) & np.uint64(M32))) + (block.astype(np.uint64) >> np.uint64(32)))
               & np.uint64(M32))
    return mix((base + (at % BLOCK).astype(np.uint64)) & np.uint64(M32))


def code_values():
    """Value of each e4m3 code, from its fields (NaN at 0x7F and 0xFF)."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, 2.0 ** (e - 7.0) * (1 + f / 8), f * 2.0 ** -9)
    v = np.where(c & 128, -v, v)
    return np.where((c & 127) == 127, np.nan, v)


def decode(codes, scale):
    """Values of one row's codes (uint8) with its blocks' scales."""
    return code_values()[codes] * scale[np.arange(len(codes)) // BLOCK]


def encode(x, share, least):
    """One row: scale of each block, the value (before the scale) of each
    element rounded up where its remainder plus share reaches 1 (share None:
    to nearest, ties to even), and how far the remainder is from that border."""
    blocks = -(-len(x) // BLOCK)
    at = np.arange(len(x)) // BLOCK
    top = np.array([np.abs(x[b * BLOCK:(b + 1) * BLOCK]).max() for b in range(blocks)])
    scale = top / 448.0
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.where(top[at] > 0, np.abs(x) * 448.0 / top[at], 0.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
    q = y / step
    if share is None:
        value, far = np.round(q), np.abs(q - np.floor(q) - 0.5)
    else:
        value, far = np.floor(q + share), np.abs(q + share - np.round(q + share))
    value = np.minimum(value * step, 448.0)
    if least:
        value = np.where(x != 0, np.maximum(value, 2.0 ** -9), value)
    return scale, np.copysign(value, x), far, step


def adamw(p, g, m, v, lr, betas, eps, decay, step):
    """New (p, m, v) in 64 bits."""
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    hat = (m / (1 - betas[0] ** step)) / (np.sqrt(v / (1 - betas[1] ** step)) + eps)
    return p * (1 - lr * decay) - lr * hat, m, v


def adamw_bounds(p, g, m, v, lr, betas, eps, decay, step):
    """Bounds of fp32's error of (p, m, v) for these inputs: m and v take
    products with rounded constants and a sum (each at most 4 roundings of
    their terms); the quotient's numerator and root carry those, and p adds
    its own product and sum and the bias corrections'."""
    dm = 5 * EPS32 * (np.abs(betas[0] * m) + np.abs((1 - betas[0]) * g))
    _, m1, v1 = adamw(p, g, m, v, lr, betas, eps, decay, step)
    dv = 6 * EPS32 * v1 + 2.0 ** -126
    root = np.sqrt(v1 / (1 - betas[1] ** step)) + eps
    c1 = 1 - betas[0] ** step
    # a root of a value off by r is off by r / 2 relatively
    hat = np.abs(m1) / c1 / root
    dp = 4 * EPS32 * np.abs(p) + lr * (dm / c1 / root + hat * 16 * EPS32) + 2.0 ** -126
    return dp, dm + 2.0 ** -126, dv
