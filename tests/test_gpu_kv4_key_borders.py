"""Rotated keys of a 4-bit cache whose quotients lie next to a border between two codes, where a sine or a cosine is small and the channel it is
multiplied with is all that a result consists of: an angle rounded to fp32 would be off by more than the result's own size allows.

Bytes, equal to the 64-bit definition's.  Every quotient is placed at a distance of 2^-8 to 2^-20 (relative) from its border, and the inputs it is
made of are rounded to at most 2^-24, so that 64 bits leave no doubt on which side it is."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu

BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
# positions (an angle of one radian each) next to multiples of pi or to odd multiples of pi / 2
NEAR = np.array([3, 11, 14, 19, 22, 33, 44, 52, 66, 88, 322, 333, 344, 355, 366, 710, 1065, 52174, 103638, 103993, 104348, 208341, 312689, 833719,
                 1146408, 4272943, 5419351, 80143857, 165707065, 245850922, 411557987, 1068966896])


def write(k, pos, inv, g, interleaved, weight=None, eps=0.0, block=32, dtype=torch.float32):
    """k [rows, heads, d] (fp64, exact in `dtype`) through the call -> (its K codes, scales), (the definition's)."""
    from paper_2609_20888_b200 import binding as eb
    rows, heads, d = k.shape
    pages = -(-rows // block)
    x = torch.from_numpy(k).to(dtype).cuda()
    assert np.array_equal(x.double().cpu().numpy(), k)
    pool = torch.zeros((pages, heads, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    desc, kv4 = eb.kv4_cache_desc(pool, heads, d, block, batch=1, t_cap=block, k_scale=g, v_scale=g)
    q_out = torch.empty((rows, heads, d), dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, x, x, x, torch.arange(rows, device="cuda"), torch.from_numpy(pos.astype(np.int32)).cuda(), q_out, pool,
                             inv_freq=torch.from_numpy(inv).cuda(), k_weight=None if weight is None else torch.from_numpy(weight).float().cuda(),
                             eps=eps, interleaved=interleaved)
    got = [v.transpose(0, 2, 1, 3).reshape(pages * block, heads, -1)[:rows] for v in ref.split(pool.cpu().numpy(), block, d)[:2]]
    y = ref.rotate(ref.norm(k, weight, eps), pos, inv, interleaved)
    return got, ref.encode(y, g)


def equal(got, want):
    assert np.array_equal(got[1], want[1]), "scales"
    off = got[0] != want[0]
    assert not off.any(), f"{off.sum()} bytes of codes, rows {np.unique(np.nonzero(off)[0])[:8]}"


def factor(pos, sine):
    return np.sin(pos.astype(np.float64)) if sine else np.cos(pos.astype(np.float64))


@pytest.mark.parametrize("sine", [True, False])
@pytest.mark.parametrize("d,g", [(64, 1.0), (128, 0.75), (128, 0.3711)])
def test_a_small_factor_alone_in_its_group(sine, d, g):
    """Channel 0 is partner * sine (or itself * cosine) and nothing else; channel 1, which does not turn, makes the group's scale 2^e g."""
    rng = np.random.default_rng(1)
    g = float(np.float32(g))
    f = factor(NEAR, sine)
    pos = NEAR[np.abs(f) < 0.5]
    f = f[np.abs(f) < 0.5]
    n = 12
    at = np.repeat(np.arange(len(pos)), n * len(BORDERS))
    border = np.tile(np.repeat(BORDERS, n), len(pos))
    rows, heads = len(at), 3
    k = np.zeros((rows, heads, d))
    for h in range(heads):
        off = rng.choice([-1, 1], rows) * 2.0 ** -rng.uniform(8, 20, rows)
        e = rng.integers(-3, 4, rows)
        size = border * (1 + off) * 2.0 ** e * g / np.abs(f[at])
        k[:, h, d // 2 if sine else 0] = (size * rng.choice([-1, 1], rows)).astype(np.float32)
        k[:, h, 1] = (6 * 2.0 ** e * g).astype(np.float32)
        k[:, h, 2:16] = (rng.uniform(-5, 5, (rows, 14)) * 2.0 ** e[:, None] * g).astype(np.float32)
    inv = np.zeros(d // 2)
    inv[0] = 1.0
    equal(*write(k, pos[at], inv, g, False))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads", [1, 4])
def test_partners_of_few_bits(dtype, heads):
    """The same with 16-bit inputs: of all partners of a power of two the ones that land closest to a border."""
    d, g = 64, 1.0
    bits = 8 if dtype == torch.bfloat16 else 11
    f = np.sin(NEAR.astype(np.float64))
    rows = []
    for p, s in zip(NEAR, f):
        m = 2.0 ** np.floor(np.log2(1 / abs(s))) * np.arange(1 << (bits - 1), 1 << bits) / (1 << (bits - 1))
        m = m[m < 60000]
        for scale in 2.0 ** np.arange(-9, 1.0):
            off = np.abs(m * abs(s) / scale / BORDERS[:, None] - 1)
            off[off < 2.0 ** -22] = 1
            b, j = np.unravel_index(np.argsort(off, None)[:2], off.shape)
            rows += [(p, scale, m[x]) for x in j]
    pos = np.array([r[0] for r in rows])
    scale, size = np.array([r[1] for r in rows]), np.array([r[2] for r in rows])
    k = np.zeros((len(rows), heads, d))
    k[:, :, 32] = size[:, None]
    k[:, :, 1] = 6 * scale[:, None]
    k[::2, :, 32] *= -1
    inv = np.zeros(32)
    inv[0] = 1.0
    equal(*write(k, pos, inv, g, False, dtype=dtype))


def test_interleaved_partners_in_one_group():
    """Neighbours as pairs: the group's scale is the partner's, which the sine has to be small against."""
    rng = np.random.default_rng(2)
    d, rows = 64, []
    p = np.arange(1, 40000)
    s = np.abs(np.sin(p.astype(np.float64)))
    for b in BORDERS[:3]:
        for j in np.nonzero(np.abs(s * np.sqrt(1 - np.minimum(s, 0.9) ** 2) ** -1 * 6 / b - 1) < 0.03)[0][:300]:
            # scale 1: partner = border / sine, a sixth of it times the cosine next to 1
            rows.append((p[j], b * (1 + rng.choice([-1, 1]) * 2.0 ** -rng.uniform(12, 20)) / s[j]))
    pos, size = np.array([r[0] for r in rows]), np.array([r[1] for r in rows])
    k = np.zeros((len(rows), 2, d))
    k[:, 0, 1] = size.astype(np.float32)
    k[:, 1, 0] = -size.astype(np.float32)
    inv = np.zeros(32)
    inv[0] = 1.0
    equal(*write(k, pos, inv, 1.0, True))


@pytest.mark.parametrize("spread", [1.0, 0.01])
def test_normed_keys(spread):
    """With a norm: z = x / rms is chosen, channel 0 again the sine's alone, and x = z / weight (eps: what is missing of a mean square of one)."""
    rng = np.random.default_rng(3)
    d, eps, s = 128, 2.0 ** -10, 2.0 ** -6
    p = np.arange(3, 30000)
    f = np.sin(p.astype(np.float64))
    ok = (np.abs(f) > 2.0 ** -9) & (np.abs(f) < 2.0 ** -6)
    pos = np.repeat(p[ok], 8)[:2500]
    f = np.sin(pos.astype(np.float64))
    w = np.ones(d)
    w[2:d // 2] = spread
    w = w.astype(np.float32).astype(np.float64)
    z = np.zeros((len(pos), 1, d))
    off = rng.choice([-1, 1], len(pos)) * 2.0 ** -rng.uniform(9, 17, len(pos))
    size = BORDERS[rng.integers(0, 4, len(pos))] * (1 + off) * s / np.abs(f)
    z[:, 0, d // 2] = size * (size < 9)
    z[:, 0, 1] = 6 * s
    z[:, 0, 2:16] = rng.uniform(-5, 5, (len(pos), 14)) * s * spread
    x = z / w
    left = d * (1 - eps) - (x ** 2).sum(-1)
    assert (left > 0).all()
    x[:, 0, 40] = np.sqrt(left[:, 0])
    x = x.astype(np.float32).astype(np.float64)
    inv = np.zeros(d // 2)
    inv[0] = 1.0
    got, want = write(x, pos, inv, 1.0, False, weight=w, eps=eps)
    equal(got, want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_sparse_keys_at_every_position(interleaved, normed):
    """Keys with three channels in ten at zero and groups of very different sizes, at usual frequencies and positions from 0 on."""
    rng = np.random.default_rng(4)
    rows, heads, d = 12000, 4, 64
    k = rng.standard_normal((rows, heads, d)) * 2.0 ** rng.integers(-10, 4, (rows, heads, 4)).repeat(16, -1)
    k[rng.random(k.shape) < 0.3] = 0
    k = k.astype(np.float32).astype(np.float64)
    inv = 10000.0 ** -(np.arange(d // 2) / (d // 2))
    w = (rng.random(d) + 0.5).astype(np.float32).astype(np.float64) if normed else None
    equal(*write(k, np.arange(rows), inv, 1.0, interleaved, weight=w, eps=2.0 ** -20 if normed else 0.0))
