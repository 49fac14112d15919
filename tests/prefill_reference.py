"""Attention of packed new tokens in 64 bits, row by row from the definition, with a bound on what a kernel that rounds its weights and its
output to bf16 and sums in fp32 may be off by."""
import torch

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def reference(q, K, V, starts, lens, granted, scale, beta=5.0, te=None, ungate=False):
    """q [rows, Hq, d]; K, V: lists of [Hkv, len, d] per sequence; te [rows, Hq] thresholds or None (softmax).
    -> out, bound [rows, Hq, d] in 64 bits, and which rows count."""
    rows, Hq, d = q.shape
    out = torch.zeros((rows, Hq, d), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    counts = torch.zeros(rows, dtype=torch.bool, device=q.device)
    for i, (k, v) in enumerate(zip(K, V)):
        n = starts[i + 1] - starts[i]
        n = n if granted is None else min(n, max(0, granted[i]))
        T = lens[i]
        k, v = k.double(), v.double()
        G = Hq // k.shape[0]
        for r in range(n):
            row, p = starts[i] + r, T - n + r
            counts[row] = True
            if p < 0:
                continue
            qr = q[row].double().view(-1, G, d)
            S = torch.einsum("hgd,htd->hgt", qr, k[:, :p + 1]) * scale
            # fp32 sums of d products: (d + 2) roundings of at most the sum of the magnitudes
            dS = (d + 2) * 2.0 ** -24 * torch.einsum("hgd,htd->hgt", qr.abs(), k[:, :p + 1].abs()) * scale
            slack = 2 * dS
            if te is not None:
                t = te[row].double().view(-1, G, 1)
                g = torch.sigmoid(beta * (S - t)) if beta else torch.full_like(S, 0.5)
                # the gate's slope, and a few roundings of its argument and of the reciprocal
                slack = slack * (1 + S.abs() * abs(beta) / 4) + S.abs() * (2.0 ** -20 + 2.0 ** -22 * (beta * (S - t)).abs().clamp(max=64))
                gated = S * g
                if ungate:
                    gated[..., -1] = S[..., -1]
                S = gated
            S = S.nan_to_num(nan=float("nan"), posinf=float("inf"), neginf=-float("inf"))
            w = torch.softmax(S, -1)
            rel = (slack + 2.0 ** -20 + S.abs().nan_to_num(0, 0, 0) * 2.0 ** -22).clamp(max=1)
            vv = v[:, :p + 1]
            o = torch.einsum("hgt,htd->hgd", w, vv)
            mass = torch.einsum("hgt,htd->hgd", w, vv.abs())
            off = torch.einsum("hgt,htd->hgd", w * rel, vv.abs()) + (w * rel).sum(-1, keepdim=True) * o.abs()
            out[row] = o.reshape(Hq, d)
            bound[row] = (HALF_STEP * (mass + o.abs()) * 1.01 + 1.1 * off + 1e-30).reshape(Hq, d)
    return out, bound, counts
