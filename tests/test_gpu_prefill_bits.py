"""A row of prompt attention has the bits that its own query, threshold and the tokens up to its position give it, whatever else stands in the call: tokens behind
it, what a page held before, other rows of the same tiles."""
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
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_behind_a_row(mode, what, d):
    s = make([300], [150], 1, 4, d, 64, False, seed=62)
    kw = args(s, mode)
    want, _ = call(s, MODES[mode], **kw)
    for t in (445, 383, 300, 231, 170):
        fill(s["K"][:, :, t:], what, t)
        if what in ("other", "large", "huge", "zero"):
            fill(s["V"][:, :, t:], what, t + 1)
        out, _ = call(s, MODES[mode], **kw)
        assert torch.equal(out[:t - 150], want[:t - 150]), (t, (out[:t - 150] != want[:t - 150]).any(2).sum().item())


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


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("what", ["other", "large", "huge", "nan", "inf", "zero"])
def test_other_rows(mode, what):
    """Queries and thresholds of every third row change, rows that do not count among them: the others' outputs stay."""
    s = make([50, 1, 21, 200], [100, 300, 7, 0], 2, 4, 128, 64, False, seed=64, pad=19, granted=[50, 1, 20, 200])
    kw = args(s, mode)
    want, _ = call(s, MODES[mode], **kw)
    rows = torch.arange(s["q"].shape[0], device="cuda")
    for k in range(3):
        t = {**s, "q": s["q"].clone()}
        x = torch.empty_like(t["q"][k::3])
        fill(x, what, k)
        t["q"][k::3] = x
        kept = dict(kw)
        if kw["tau"] is not None:
            kept["tau"] = kw["tau"].clone()
            kept["tau"][k::3] = x[..., 0].float()
        out, _ = call(t, MODES[mode], **kept)
        same = rows % 3 != k
        assert torch.equal(out[same], want[same]), (out[same] != want[same]).any(2).sum().item()
