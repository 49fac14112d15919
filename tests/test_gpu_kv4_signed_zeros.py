"""A code keeps its number's sign, a zero's too (a group whose scale is zero excepted): whichever way a group is worked out, the same tokens give the same
bytes."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("g", [1.0, 0.75, 0.0123456789])         # the last has all of fp32's bits
@pytest.mark.parametrize("how", ["plain", "turned", "normed", "half"])
def test_zeros_of_both_signs(dtype, g, how):
    from paper_2609_20888_b200 import binding as eb
    rows, heads, d, block = 64, 3, 64, 32
    rng = np.random.default_rng(7)
    x = rng.standard_normal((rows, heads, d))
    x[rng.random(x.shape) < 0.3] = 0.0
    x[rng.random(x.shape) < 0.3] = -0.0
    x[5] = -0.0                                                   # whole groups: positive zeros
    t = torch.from_numpy(x).to(dtype).cuda()
    x = t.double().cpu().numpy()
    rotary = {"plain": 0, "turned": 64, "normed": 0, "half": 32}[how]
    inv = 10000.0 ** -(np.arange(rotary // 2) / max(1, rotary // 2))
    pos = np.arange(rows) * 37                                    # row 0 does not turn: its zeros keep their signs
    weight = (rng.random(d) + 0.5).astype(np.float32) if how == "normed" else None
    pool = torch.zeros((2, heads, eb.kv4_block_bytes(block, d)), dtype=torch.uint8, device="cuda")
    desc, kv4 = eb.kv4_cache_desc(pool, heads, d, block, batch=1, t_cap=block, k_scale=g, v_scale=g)
    q_out = torch.empty((rows, heads, d), dtype=torch.bfloat16, device="cuda")
    eb.eta_append_tokens_kv4(desc, kv4, t, t, t, torch.arange(rows, device="cuda"), torch.from_numpy(pos.astype(np.int32)).cuda(), q_out, pool,
                             inv_freq=torch.from_numpy(inv).cuda() if rotary else None,
                             k_weight=None if weight is None else torch.from_numpy(weight).cuda())
    got = [v.transpose(0, 2, 1, 3).reshape(rows, heads, -1) for v in ref.split(pool.cpu().numpy(), block, d)]
    y = ref.norm(x, weight, 1e-6)
    if rotary:
        y = ref.rotate(y, pos, inv, False)
    for at, want in ((0, y), (2, x)):
        codes, scales = ref.encode(want, g)
        assert np.array_equal(got[at + 1], scales)
        assert np.array_equal(got[at], codes), ("keys", "values")[at // 2]
