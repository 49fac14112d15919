"""4-bit attention at scores near the ends of fp32, all of them negative among those: a softmax knows differences only."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [90, 104, 118])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("d,b,G,n", [(128, 64, 4, 1), (64, 32, 8, 31), (128, 32, 1, 700), (64, 128, 2, 129)])
def test_equal_scores_average_the_values(power, sign, d, b, G, n):
    from paper_2609_20888_b200 import binding as eb
    rng = np.random.default_rng(n)
    nb = -(-n // b)
    K = np.full((1, 1, nb * b, d), 1.5)
    V = rng.standard_normal((1, 1, nb * b, d))
    blocks = ref.pack(K, V, b, 1.0, 1.0)
    K, V = ref.unpack(blocks, b, d, 1.0, 1.0)
    # every score is a sum of d equal products: the same number, bit by bit, in every token
    q = torch.full((1, G, d), sign * 2.0 ** power, dtype=torch.bfloat16, device="cuda")
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, G, d, b)
    out, sel = torch.empty((1, G, d), device="cuda"), torch.zeros((1, 1, nb), dtype=torch.uint8, device="cuda")
    ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q, pool, torch.tensor([n], dtype=torch.int32, device="cuda"), None, None,
                      torch.zeros((1, G), device="cuda"), None, out, sel, ws)
    got, v = out[0].double().cpu().numpy(), V[0, 0, :n]
    # weights of one, exactly; sums cut off 2^-22 below their size, n / 16 times at most, and a few roundings
    tol = (n / 16 + 8) * 2.0 ** -22 * np.abs(v).mean(0)
    assert (np.abs(got - v.mean(0)) <= tol).all()


@pytest.mark.parametrize("G", [2, 8])
def test_the_largest_of_huge_scores_takes_all(G):
    from paper_2609_20888_b200 import binding as eb
    rng = np.random.default_rng(3)
    d, b, n = 64, 64, 300
    nb = -(-n // b)
    K, V = rng.standard_normal((2, 1, 1, nb * b, d))
    K[..., 0] = 3 + rng.random((1, 1, nb * b))
    blocks = ref.pack(K, V, b, 1.0, 1.0)
    K, V = ref.unpack(blocks, b, d, 1.0, 1.0)
    q64 = rng.standard_normal((1, G, d)) * 2.0 ** 100
    q64[..., 0] = -2.0 ** 112                                   # all scores below -1e33
    q = torch.from_numpy(q64).to(torch.bfloat16).cuda()
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, G, d, b)
    out, sel = torch.empty((1, G, d), device="cuda"), torch.zeros((1, 1, nb), dtype=torch.uint8, device="cuda")
    ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q, pool, torch.tensor([n], dtype=torch.int32, device="cuda"), None, None,
                      torch.zeros((1, G), device="cuda"), None, out, sel, ws)
    s = q.double().cpu().numpy()[0] @ K[0, 0, :n].T / 8
    assert (s < -1e33).all()
    got = out[0].double().cpu().numpy()
    for h in range(G):
        best = np.sort(s[h])[::-1]
        assert best[0] - best[1] > 2.0 ** -15 * abs(best[0])     # far more than fp32's rounding
        assert np.abs(got[h] - V[0, 0, s[h].argmax()]).max() <= 2.0 ** -21 * np.abs(V).max()
