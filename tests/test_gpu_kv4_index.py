"""The block index of a 4-bit cache against the oracle on the keys it stands for (bf16 numbers, at scales of a tensor of one or two bits)."""
import numpy as np
import pytest
import torch

from oracle import eta_oracle as orc
from tests import kv4_reference as ref
from tests.helpers import bf16_bits_from_f64, fp16_ulp_distance

pytestmark = pytest.mark.gpu


def cache(B, Hkv, nb, b, d, seed, kg=0.75, kind="normal"):
    rng = np.random.default_rng(seed)
    K = rng.standard_normal((B, Hkv, nb * b, d)) * np.exp(rng.standard_normal((1, Hkv, 1, d)))
    if kind == "offset":                     # a mean far from zero, and blocks of identical keys
        K = K * 0.05 + 3
        K.reshape(B, Hkv, nb, b, d)[:, :, 1::2] = K.reshape(B, Hkv, nb, b, d)[:, :, 1::2, :1]
    blocks = ref.pack(K, rng.standard_normal(K.shape), b, kg, 1.0)
    return blocks, ref.unpack(blocks, b, d, kg, 1.0)[0], rng


def run(blocks, table, lens, b, d, kg, newest=False, flags=0, fill=None, nb_cap=None):
    from paper_2609_20888_b200 import binding as eb
    B = len(lens)
    pool = torch.from_numpy(blocks).cuda()
    nb = blocks.shape[2] if table is None else table.shape[1]
    desc, kv4 = eb.kv4_cache_desc(pool, blocks.shape[1], d, b, batch=B, t_cap=nb * b, nb_cap=nb_cap, k_scale=kg)
    t = None if table is None else torch.from_numpy(table).cuda()
    musig, mnorm = fill or eb.alloc_summaries(desc, "cuda", packed=bool(flags & 2))
    call = eb.eta_append_summary_kv4 if newest else eb.eta_build_block_summaries_kv4
    call(desc, kv4, pool, torch.tensor(lens, dtype=torch.int32, device="cuda"), musig, mnorm, flags=flags,
         pages=None if t is None else eb.page_table(t, len(blocks)))
    torch.cuda.synchronize()
    return musig, mnorm


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b", [32, 64, 128])
@pytest.mark.parametrize("kind,paged,envelope", [("normal", False, False), ("normal", True, True), ("offset", True, False), ("offset", False, True)])
def test_build_matches_the_oracle(d, b, kind, paged, envelope):
    blocks, K, rng = cache(3, 2, 5, b, d, d + b, kind=kind)
    lens = np.array([5 * b, 3 * b + 7, b - 1], np.int32)
    bits = bf16_bits_from_f64(K)
    assert np.array_equal((bits.astype(np.uint32) << 16).view(np.float32), K)          # the keys are bf16 numbers
    want, wnorm = orc.block_summaries(orc.Cache(bits, bits, lens, b), envelope=envelope)
    pool, table = ref.scatter(blocks, rng) if paged else (blocks, None)
    musig, mnorm = run(pool, table, lens, b, d, 0.75, flags=1 if envelope else 0)
    got = musig.cpu().numpy().view(np.uint16)
    assert fp16_ulp_distance(got, want).max() <= 1
    assert (np.abs(mnorm.cpu().numpy() - wnorm) <= 4 * 2.0 ** -24 * wnorm).all()
    for i, n in enumerate(lens // b):                                                   # what is not full stays as it was
        assert not got[i, :, n:].any() and not mnorm[i, :, n:].any()
    if kind == "offset":
        assert not got[0, :, 1::2, 1].any() and got[0, :, 1::2, 0].all()                # identical keys: sigma is zero
    packed, pnorm = run(pool, table, lens, b, d, 0.75, flags=2 | int(envelope))
    w8, _ = orc.block_summaries_sigma8(orc.Cache(bits, bits, lens, b), envelope=envelope)
    p8 = packed.cpu().numpy()
    assert torch.equal(pnorm, mnorm) and np.array_equal(p8[..., :2 * d], musig[..., 0, :].cpu().contiguous().view(torch.uint8).numpy())
    assert np.abs(p8[..., 2 * d:].astype(int) - w8[..., 2 * d:]).max() <= 1


@pytest.mark.parametrize("d,b,flags", [(128, 64, 0), (64, 32, 0), (128, 32, 1), (64, 128, 2), (128, 128, 3)])
@pytest.mark.parametrize("paged", [False, True])
def test_append_writes_what_the_build_would_and_nothing_else(d, b, flags, paged):
    B, nb = 6, 4
    blocks, _, rng = cache(B, 3, nb, b, d, 7 * d + b)
    lens = [b, 3 * b, 4 * b, 2 * b + 1, 0, b - 1]
    pool, table = ref.scatter(blocks, rng) if paged else (blocks, None)
    built, bnorm = run(pool, table, lens, b, d, 1.5, flags=flags)
    fill = (torch.full_like(built, 3), torch.full_like(bnorm, 3))
    got, gnorm = run(pool, table, lens, b, d, 1.5, newest=True, flags=flags, fill=fill)
    for i, n in enumerate(lens):
        new = n // b - 1 if n and n % b == 0 else -1
        for j in range(nb):
            if j == new:
                assert torch.equal(got[i, :, j].view(torch.uint8), built[i, :, j].view(torch.uint8)) and torch.equal(gnorm[i, :, j], bnorm[i, :, j])
            else:
                assert (got[i, :, j] == 3).all() and (gnorm[i, :, j] == 3).all()


def test_lengths_beyond_the_cache_and_below_zero():
    b, d = 32, 64
    blocks, _, _ = cache(3, 1, 3, b, d, 1)
    full, norm = run(blocks, None, [3 * b] * 3, b, d, 1.0)
    got, gnorm = run(blocks, None, [5 * b, -4, 3 * b], b, d, 1.0)
    assert torch.equal(got[::2], full[::2]) and not got[1].any() and not gnorm[1].any()
    got, gnorm = run(blocks, None, [5 * b, -b, 0], b, d, 1.0, newest=True)
    assert not got.any() and not gnorm.any()


def test_a_nan_key_is_seen_in_its_channels_and_the_norm():
    b, d = 64, 128
    blocks, _, _ = cache(1, 2, 3, b, d, 2)
    c = b * d // 2
    blocks[0, 1, 1, c + 8 * 5 + 3] = 0x7f                     # token 5, channels 48 .. 63
    musig, mnorm = run(blocks, None, [3 * b], b, d, 1.0)
    nan = musig.isnan()
    assert nan[0, 1, 1, :, 48:64].all() and nan.sum() == 32
    assert mnorm.isnan().sum() == 1 and mnorm[0, 1, 1].isnan()
    packed, _ = run(blocks, None, [3 * b], b, d, 1.0, flags=2)
    assert (packed[0, 1, 1, 2 * d + 48:2 * d + 64] == 0x7f).all()
