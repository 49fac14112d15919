"""The 4-bit cache format and the treatment of new tokens, in numpy and 64 bits, from their definitions (include/eta.h)."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
# every finite non-negative e4m3 value, by code: 4 exponent bits (bias 7), 3 fraction bits
E4M3 = np.array([(c & 7) / 512 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)], np.float64)


def nearest(grid, x):
    """Code of the value of an ascending grid that is nearest to x >= 0: ties to the even code, saturating."""
    up = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    low, high = x - grid[up - 1], grid[up] - x
    return np.where((high < low) | ((high == low) & (up % 2 == 0)), up, up - 1)


def encode(x, g):
    """x [..., d] -> codes uint8 [..., d / 2], scales uint8 [..., d / 16]."""
    x = np.asarray(x, np.float64)
    g = np.float64(np.float32(g))
    groups = x.reshape(*x.shape[:-1], -1, 16)
    nan = np.isnan(groups).any(-1)
    with np.errstate(all="ignore"):
        want = (np.abs(groups).max(-1) / (6 * g)).astype(np.float32).astype(np.float64)
        scale = np.where(nan, 0x7f, nearest(E4M3, np.where(nan, 0, want)))
        unit = np.where(nan, 0, E4M3[np.minimum(scale, 126)]) * g
        y = np.where(unit[..., None] > 0, groups / np.where(unit > 0, unit, 1)[..., None], 0).astype(np.float32).astype(np.float64)
    y = np.where(nan[..., None], 0, y)
    code = nearest(E2M1, np.abs(y)) + 8 * np.signbit(y)
    code = code.reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.astype(np.uint8)


def decode(codes, scales, g):
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    s = np.where((scales & 0x7f) == 0x7f, np.nan, E4M3[np.minimum(scales & 0x7f, 126)]) * np.float64(np.float32(g))
    return E2M1[c & 7] * np.where(c & 8, -1.0, 1.0) * np.repeat(s, 16, -1)


def split(blocks, b, d):
    """Views of blocks uint8 [..., block bytes]: K codes, K scales, V codes, V scales, [..., b, d / 2] and [..., b, d / 16]."""
    c, s = b * d // 2, b * d // 16
    cuts = [(0, c), (c, c + s), (c + s, 2 * c + s), (2 * c + s, 2 * c + 2 * s)]
    return [blocks[..., i:j].reshape(*blocks.shape[:-1], b, -1) for i, j in cuts]


def pack(K, V, b, kg, vg):
    """K, V [..., n * b, d] -> blocks uint8 [..., n, block bytes]."""
    parts = []
    for x, g in ((K, kg), (V, vg)):
        x = x.reshape(*x.shape[:-2], -1, b, x.shape[-1])
        codes, scales = encode(x, g)
        parts += [codes.reshape(*codes.shape[:-2], -1), scales.reshape(*scales.shape[:-2], -1)]
    return np.concatenate(parts, -1)


def unpack(blocks, b, d, kg, vg):
    """-> K, V [..., n * b, d] in 64 bits"""
    kc, ks, vc, vs = split(blocks, b, d)
    join = lambda x: x.reshape(*x.shape[:-3], -1, d)  # noqa: E731
    return join(decode(kc, ks, kg)), join(decode(vc, vs, vg))


def norm(x, weight, eps):
    x = np.asarray(x, np.float64)
    return x if weight is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * np.asarray(weight, np.float64)


def rotate(x, positions, inv_freq, interleaved):
    """x [rows, heads, d], the first 2 * len(inv_freq) channels of it."""
    n = 2 * len(inv_freq)
    angle = (positions.astype(np.float64)[:, None] * inv_freq)[:, None]
    c, s = np.cos(angle), np.sin(angle)
    y = x.copy()
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def scatter(blocks, rng):
    """Blocks [B, Hkv, nb, bytes] as a paged pool [B * nb, Hkv, bytes] and its table."""
    B, Hkv, nb, size = blocks.shape
    perm = rng.permutation(B * nb).astype(np.int32)
    pool = np.empty((B * nb, Hkv, size), np.uint8)
    pool[perm] = blocks.transpose(0, 2, 1, 3).reshape(B * nb, Hkv, size)
    return pool, perm.reshape(B, nb)


def output_bound(q, K, V, beta, scale):
    """How far fp32 arithmetic may take an output.  A score is a sum of exact products in at most eight accumulation steps: off by 2^-20 of
    A = s |q| |k|.  The gate S sigmoid(beta (S - tau)) has a slope of at most 1 + beta |S| / 4 + 1, and adds 2^-21 of |S| by its own
    approximations.  A weight off by a factor 1 + e, and a sum of weights off as much, move an average of V by at most 2 e max|V|."""
    A = scale * np.sqrt((q ** 2).sum(-1).max()) * np.sqrt((K ** 2).sum(-1).max())
    e = (2 + beta * A / 4) * 2.0 ** -20 * A + 2.0 ** -21 * A + 2.0 ** -20
    return 2 * e * np.abs(V).max()
