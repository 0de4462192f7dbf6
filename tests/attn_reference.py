"""Attention by its definition in float64 on the CPU, for the tests of the
attention operators, and the tolerances that the kernels' roundings imply."""
import math

import torch

# half a step of rounding to each type
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attention(q, k, v, seen, scale):
    """q [nq][Hq][d], k and v [nk][H][d], seen [nq][nk] or [Hq][nq][nk] (bool):
    (out, lse, bound) in float64.  Hidden keys take no part, whatever they hold.

    `bound` is what the kernels' roundings can make of out, element by element:
    the probabilities are rounded to the 16-bit type (half a step each, relative),
    the result once more, and the binary32 arithmetic moves each probability by
    the logit's error, at most 2 d + 64 roundings of sum |q k| scale, plus two
    units of the exponential and the sums' n + 64 roundings."""
    t = q.dtype
    nq, Hq, d = q.shape
    nk, H, _ = k.shape
    G = Hq // H
    out = torch.zeros(nq, Hq, d, dtype=torch.float64)
    bound = torch.zeros_like(out)
    lse = torch.full((nq, Hq), -math.inf, dtype=torch.float64)
    lse_bound = torch.zeros_like(lse)
    for h in range(Hq):
        s = seen if seen.dim() == 2 else seen[h]
        qh = q[:, h].double()
        kh, vh = k[:, h // G].double(), v[:, h // G].double()
        used = s.any(0)
        kh, vh, s = kh[used], vh[used], s[:, used]
        z = torch.where(s, qh @ kh.t() * scale, -math.inf)
        size = (qh.abs() @ kh.abs().t() * scale)
        rows = s.any(1)
        if not rows.any():
            continue
        lse[rows, h] = torch.logsumexp(z[rows], 1)
        p = torch.exp(z[rows] - lse[rows, h, None])
        p = torch.where(s[rows], p, 0.0)
        eps = 2.0 ** -24
        off = torch.where(s[rows], (2 * d + 64) * eps * size[rows] + 16 * eps, 0.0)  # of a logit, so relative to p
        n = s[rows].sum(1, keepdim=True).double()
        rel = HALF_STEP[t] + off + (n + 64) * eps
        each = [p[i] @ torch.where(s[rows][i][:, None], vh, 0.0) for i in range(p.shape[0])] if not torch.isfinite(vh).all() \
            else list(p @ vh)
        out[rows, h] = torch.stack(each)
        a = (p * (rel + (p * off).sum(1, keepdim=True))) @ torch.nan_to_num(vh, 0.0, 0.0, 0.0).abs()
        # a probability below the 16-bit type's normal range is rounded by an absolute step instead
        tiny = 2.0 ** -25 if t == torch.float16 else 0.0
        a = a + tiny * torch.nan_to_num(vh, 0.0, 0.0, 0.0).abs().sum(0)
        bound[rows, h] = a * (1 + HALF_STEP[t]) + out[rows, h].abs() * HALF_STEP[t] + 2.0 ** -25
        lse_bound[rows, h] = (off + 2 * eps).amax(1) + (n[:, 0] + 64) * eps + lse[rows, h].abs() * 4 * eps
    return out, lse, bound, lse_bound


def check(got, got_lse, want, name=""):
    out, lse, bound, lse_bound = want
    g, gl = got.cpu().double(), got_lse.cpu().double()
    fin = torch.isfinite(out)
    assert torch.equal(torch.isnan(g), torch.isnan(out)), name
    assert torch.equal(g[~fin & ~torch.isnan(out)], out[~fin & ~torch.isnan(out)]), name
    over = ((g - out).abs() - bound)[fin]
    assert over.numel() == 0 or over.max() <= 0, (name, over.max().item())
    fl = torch.isfinite(lse)
    assert torch.equal(torch.isnan(gl), torch.isnan(lse)), name
    assert torch.equal(gl[~fl & ~torch.isnan(lse)], lse[~fl & ~torch.isnan(lse)]), name
    over = ((gl - lse).abs() - lse_bound)[fl]
    assert over.numel() == 0 or over.max() <= 0, (name, "lse", over.max().item())


def causal(nq, nk):
    return torch.arange(nk)[None, :] <= torch.arange(nq)[:, None] + nk - nq
