"""What the attention kernels' roundings can make of a result where they are known more
closely than attn_reference assumes, and calls of the kernels on host tensors."""
import torch

from attn_reference import HALF_STEP
from paper_2606_08635_amd import skv

EPS = 2.0 ** -24  # half a step of binary32


def bound(q, k, v, seen, scale, out, half, tiny, dots=None):
    """Per element of out [nq][Hq][d] (float64, finite inputs): probabilities off by `half` relative or by `tiny` of
    the row's largest, logits by `dots` roundings (2 d + 64; a few where every product but one is 0: those of the scale, the product
    with it and the reference) of sum |q k| scale and the exponential by 16, sums by n + 64, the result by half a step
    of its type (and the type's own smallest step)."""
    nq, Hq, d = q.shape
    G = Hq // k.shape[1]
    tol = torch.zeros(nq, Hq, d, dtype=torch.float64)
    for h in range(Hq):
        qh, kh, vh = q[:, h].double(), k[:, h // G].double(), v[:, h // G].double()
        z = torch.where(seen, qh @ kh.t() * scale, -torch.inf)
        p = torch.softmax(z, 1)
        off = torch.where(seen, (2 * d + 64 if dots is None else dots) * EPS * (qh.abs() @ kh.abs().t() * scale) + 16 * EPS, 0.0)
        n = seen.sum(1, keepdim=True).double()
        each = torch.where(seen, p * (half + off + (p * off).sum(1, keepdim=True) + (n + 64) * EPS)
                           + tiny * p.amax(1, keepdim=True), 0.0)
        tol[:, h] = each @ vh.abs()
    return tol * (1 + HALF_STEP[q.dtype]) + out.abs() * HALF_STEP[q.dtype] + 2.0 ** -25


def within(got, want, tol, name=""):
    over = (got.cpu().double() - want).abs() - tol
    assert over.max() <= 0, (name, over.max().item(), (got.cpu().double() - want).abs().max().item())


def prompt(q, k, v, ql, kl, is_causal=True, split=False, scale=None):
    """attn_prompt on host tensors: (out, lse)."""
    q, k, v = (x.cuda() for x in (q, k, v))
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    ws = None
    if split:
        need = skv.attn_prompt_workspace_size(ql, kl, q.shape[1], k.shape[1], q.shape[2], causal=is_causal)
        assert need > 0
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    skv.attn_prompt(q, k, v, out, ql, kl, causal=is_causal, lse=lse, ws=ws, scale=scale)
    torch.cuda.synchronize()
    return out, lse


def decode(q, k, v, lens, prefix=0, tiers=None, scale=None, max_len=None, block=16):
    """attn_decode over requests whose tokens are given: q [B][Lq][Hq][d], k and v [B][n][H][d] (a common prefix in
    every row's first `prefix` tokens is stored once): (out, lse)."""
    B, n, H, d = k.shape
    width = -(-n // block)
    shared = prefix // block
    own = torch.arange(B * (width - shared)).view(B, width - shared) + shared
    tables = torch.cat([torch.arange(shared).expand(B, shared), own], 1).to(torch.int32).contiguous()
    blocks = shared + B * (width - shared)
    pools = []
    for x in (k, v):
        pool = torch.full((blocks * block, H, d), float("nan"), dtype=x.dtype)
        for b in reversed(range(B)):
            t = torch.arange(n)
            pool[tables[b, t // block].long() * block + t % block] = x[b]
        pools.append(pool.view(blocks, block, H, d).cuda())
    q = q.cuda()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    max_len = max(lens) if max_len is None else max_len
    need = skv.attn_decode_workspace_size(B, q.shape[1], q.shape[2], H, d, max_len, prefix)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    skv.attn_decode(q, *pools, tables.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, max_len,
                    prefix_len=prefix, tiers=None if tiers is None else tiers.cuda(), scale=scale, lse=lse, dev_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    return out, lse
