"""A row of prompt attention has the bits that its own query, threshold and the tokens up to its position give it, whatever a page held before."""
import math

import pytest
import torch

from paper_2609_20888_b200 import binding as eb
from test_gpu_prefill import DENSE, call, make

pytestmark = pytest.mark.gpu

MODES = {"softmax": DENSE, "constants": eb.DecodeParams(beta=3.0), "thresholds": eb.DecodeParams(beta=3.0, flags=eb.ETA_FLAG_UNGATE_LAST)}


def args(s, mode):
    gen = torch.Generator(device="cuda").manual_seed(61)
    tau = torch.randn((s["q"].shape[0], s["Hq"]), generator=gen, device="cuda") + 0.3
    return dict(tau=tau if mode == "thresholds" else None, const=tau[0].contiguous() if mode == "constants" else None)


def fill(x, what, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    noise = torch.randn(x.shape, generator=gen, device="cuda")
    x.copy_({"other": noise, "large": 30 * noise, "huge": 1e6 * noise, "nan": noise * math.nan, "inf": noise * math.inf, "zero": 0 * noise}[what])


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("what", ["other", "large", "huge", "nan", "inf", "zero"])
@pytest.mark.parametrize("paged", [False, True])
def test_what_a_page_held_before(mode, what, paged):
    """Behind the last token: of single tokens, of a chunk, of a share of a long one."""
    s = make([1, 77, 1], [170, 300, 2000], 2, 4, 64, 32, paged, seed=63)
    kw = args(s, mode)
    want, _ = call(s, MODES[mode], **kw)
    for i, T in enumerate(s["lens"]):
        for x in (s["K"], s["V"]):
            if paged:
                fill(x[s["table"][i, (T - 1) // 32].item(), :, (T - 1) % 32 + 1:], what, i)
            else:
                fill(x[i, :, T:], what, i)
    out, _ = call(s, MODES[mode], **kw)
    assert torch.equal(out, want)
