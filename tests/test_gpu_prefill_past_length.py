"""Attention of more new tokens than a sequence has, or than its cache holds: rows before the first token are zeros, the others are attended, at capacities
below and above that from which parts of items are joined."""
import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_prefill import DENSE, call, check, make

pytestmark = pytest.mark.gpu


def many_rows(rows, lens, Hkv, G, d, b, paged, seed):
    """Sequences of lens[i] tokens with rows[i] new ones."""
    s = make(lens, [0] * len(lens), Hkv, G, d, b, paged, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    s["starts"] = [sum(rows[:i]) for i in range(len(rows) + 1)]
    s["q"] = torch.randn((sum(rows), Hkv * G, d), generator=gen, device="cuda").bfloat16()
    return s


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,lens,Hkv,G,d,paged", [([600], [512], 2, 4, 128, False), ([4096], [512], 8, 4, 64, True), ([5000], [300], 1, 4, 128, False),
                                                     ([2000], [512], 8, 2, 64, False), ([1000, 40], [64, 512], 2, 8, 128, True),
                                                     ([700, 3000, 1], [700, 40, 2000], 2, 4, 64, True)])
def test_rows_before_the_first_token(rows, lens, Hkv, G, d, paged, gated):
    s = many_rows(rows, lens, Hkv, G, d, 64, paged, seed=31)
    params, const = (eb.DecodeParams(), torch.full((Hkv * G,), 0.3, device="cuda")) if gated else (DENSE, None)
    out = check(s, params, const=const, status=eb.ETA_DEV_EMPTY_ROW)
    at = 0
    for n, T in zip(rows, lens):
        assert torch.all(out[at:at + max(0, n - T)] == 0)
        at += n
    if max(lens) == 512 and not paged:
        # lengths past the capacity of 512 are clamped to it
        s["lens"] = [1000]
        again, status = call(s, params, const=const)
        assert status == eb.ETA_DEV_EMPTY_ROW | eb.ETA_DEV_LEN_CLAMPED and torch.equal(again, out)
