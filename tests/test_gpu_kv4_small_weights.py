"""4-bit attention where one token has almost all of the weight and a value of zero, as a sequence's first token often has: the output is made of the other
tokens, whose weights are small against the largest.

A weight w (of a largest of one) is a score's exponential, off by the factor 1 + e that a score's error makes (2^-20 of A = s |q| |k| for its sum of products,
2^-21 of A for the exponent's own rounding) and by 2^-22 for the exponential; it is fed to the second product with 2^-24 of itself and 2^-45 of the
largest lost; what the product sums is cut off 2^-22 below its own size after every slab, at most 40 times here."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ahead", [6.0, 14.0, 18.0, 22.0, 26.0])
@pytest.mark.parametrize("d,b,G", [(128, 64, 4), (128, 32, 8), (64, 64, 8), (64, 128, 1), (128, 128, 2)])
@pytest.mark.parametrize("first", [True, False])
def test_a_token_without_a_value_holds_the_weight(ahead, d, b, G, first):
    from paper_2609_20888_b200 import binding as eb
    rng = np.random.default_rng(int(ahead) + d + b + G)
    B, Hkv, nb = 2, 1, 640 // b
    n = nb * b
    q = rng.standard_normal((B, G, d)) * 0.3
    q[..., 0] = 4.0
    K = rng.standard_normal((B, Hkv, n, d)) * 0.3
    K[..., 0] = 0.0
    V = rng.standard_normal((B, Hkv, n, d))
    sink = 0 if first else n // 2 + 3
    K[:, :, sink] = 0.0
    K[:, :, sink, 0] = ahead * np.sqrt(d) / 4.0
    V[:, :, sink] = 0.0
    blocks = ref.pack(K, V, b, 1.0, 1.0)
    K, V = ref.unpack(blocks, b, d, 1.0, 1.0)
    q = torch.from_numpy(q).to(torch.bfloat16)
    lens = torch.tensor([n, n - 5], dtype=torch.int32).cuda()
    pool = torch.from_numpy(blocks).cuda()
    desc, kv4 = eb.kv4_cache_desc(pool, G, d, b)
    out, sel = torch.empty((B, G, d), device="cuda"), torch.zeros((B, Hkv, nb), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(eb.eta_kv4_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    eb.eta_decode_kv4(desc, kv4, eb.DecodeParams(flags=eb.ETA_FLAG_DENSE), q.cuda(), pool, lens, None, None, torch.zeros((B, G), device="cuda"), None,
                      out, sel, ws, status=status)
    got, q = out.double().cpu().numpy(), q.double().numpy()
    assert status.item() == 0
    for i in range(B):
        m = n - 5 * i
        for h in range(G):
            s = K[i, 0, :m] @ q[i, h] / np.sqrt(d)
            w = np.exp(s - s.max())
            assert w[sink] == 1 and np.sort(w)[-2] < np.exp(4 - ahead)
            A = np.sqrt((q[i, h] ** 2).sum() * (K[i, 0, :m] ** 2).sum(-1).max() / d)
            each = w * (1.5 * 2.0 ** -20 * A + 2.0 ** -22 + 2.0 ** -24 + 40 * 2.0 ** -22) + 2.0 ** -45
            tol = 2 * (each @ np.abs(V[i, 0, :m])) / w.sum()
            want = w @ V[i, 0, :m] / w.sum()
            assert (np.abs(got[i, h] - want) <= tol).all(), (np.abs(got[i, h] - want).max(), np.abs(want).max(), tol.max())
