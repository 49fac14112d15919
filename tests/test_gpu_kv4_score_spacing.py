"""4-bit attention at scores whose neighbours in fp32 are further apart than the slack that the running maximum leaves."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [22, 24, 25, 26, 27, 28])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("G,d,b", [(4, 64, 64), (8, 128, 32)])
def test_a_step_of_eight(power, odd, G, d, b):
    """Scores 2^power + 8 odd, then 8 (or one place of fp32, where that is more) above: products and sums are exact here, so weights are 1 and e^-8 or less."""
    from paper_2609_20888_b200 import binding as eb
    rng = np.random.default_rng(power)
    # enough tokens for every warp to see several runs of sixteen, low and high in turn
    n, step = 40960, max(8.0, 2.0 ** (power - 23))
    high = np.arange(n) // 16 % 2 == 1
    K, V = np.zeros((1, 1, n, d)), rng.standard_normal((1, 1, n, d))
    K[..., 0], K[..., 2] = 1.0, 6.0                             # channel 2, which no query looks at, makes the scale one
    K[0, 0, :, 1] = np.where(high, odd + 1, odd)
    blocks = ref.pack(K, V, b, 1.0, 1.0)
    K2, V = ref.unpack(blocks, b, d, 1.0, 1.0)
    assert np.array_equal(K, K2)
    q = torch.zeros((1, G, d), dtype=torch.bfloat16)
    q[..., 0], q[..., 1] = 2.0 ** power, step
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, G, d, b)
    out, sel = torch.empty((1, G, d), device="cuda"), torch.zeros((1, 1, n // b), dtype=torch.uint8, device="cuda")
    ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE, scale=1.0), q.cuda(), pool, torch.tensor([n], dtype=torch.int32, device="cuda"),
                      None, None, torch.zeros((1, G), device="cuda"), None, out, sel, ws)
    w = np.where(high, 1.0, np.exp(-step))
    want = w @ V[0, 0] / w.sum()
    got = out[0].double().cpu().numpy()
    # a weight to 2^-21, sums cut off 2^-22 below their size once a slab
    tol = (2.0 ** -20 + n / 16 * 2.0 ** -22) * (w @ np.abs(V[0, 0])) / w.sum()
    assert (np.abs(got - want) <= tol).all()
