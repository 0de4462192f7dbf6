"""The attention and page operators around the codec, as measurable cases.

Each case is one pass of one of three operators of `paper_2606_08635_amd.skv`:

  prompt  attention over whole prompts: grouped heads, causal, sequences of
          different lengths in one call, K and V packed by token or in the
          codec's own [H][n][d] buffers (attn_prompt)
  decode  attention of a batch's next tokens over the paged cache, the prefix
          that the batch shares computed once, dropped tokens masked
          (attn_decode)
  fork, compact, copy
          pages of the cache: children of a request that share its pages and
          get room for their next tokens (pages_fork, pages_reserve,
          pages_free), requests rid of their dropped tokens (pages_compact,
          pages_free), pages moved to another pool (pages_copy)

With `own` false, `run` is the same arithmetic in elementary float32 torch;
`exact` is the definition in float64.
"""
import math

import torch

own = False
DEV = "cuda"
DROP = 3
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# query heads, KV heads, head dimension, layers: the models of the codec's workloads, a small one and one with
# ungrouped heads
MODELS = {
    "tiny": (4, 2, 64, 1),
    "qwen7b": (28, 4, 128, 28),
    "mistral7b": (32, 8, 128, 32),
    "gemma9b": (16, 8, 256, 42),
    "ungrouped": (8, 8, 32, 4),
}


def _prompt(model, count, nq, nk, dtype="f16", nq_min=None, causal=True, codec=False, **more):
    """count sequences of nq_min..nq queries, each over nk - nq more keys than it has queries."""
    return dict(kind="prompt", model=model, count=count, nq=nq, nk=nk, nq_min=nq if nq_min is None else nq_min,
                dtype=dtype, causal=causal, codec=codec, **more)


def _decode(model, count, prefix, n, n_min=None, queries=1, drop=0.0, block=16, dtype="f16", **more):
    """count requests of prefix + (n_min..n) tokens, the last `queries` of them new; `drop` of the older ones dropped."""
    return dict(kind="decode", model=model, count=count, prefix=prefix, n=n, n_min=n if n_min is None else n_min,
                queries=queries, drop=drop, block=block, dtype=dtype, **more)


def _pages(kind, model, count, n, n_min=None, block=16, **more):
    return dict(kind=kind, model=model, count=count, n=n, n_min=n if n_min is None else n_min, block=block, **more)


def listed():
    return [
        # the smallest prompt, the tests' shape: latency
        dict(_prompt("tiny", 1, 512, 512, codec=True), name="prompt_tiny"),
        # short prompts of many users in one call
        dict(_prompt("mistral7b", 24, 2300, 2300, nq_min=100), name="prompt_ragged_batch"),
        # one prompt of no round length, K and V in the buffers that the codec packs from
        dict(_prompt("mistral7b", 1, 8189, 8189, codec=True), name="prompt_mistral7b_8k"),
        # the last piece of a 32k prompt computed in pieces
        dict(_prompt("qwen7b", 1, 2048, 32768, dtype="bf16"), name="prompt_qwen7b_piece"),
        # head dimension 256
        dict(_prompt("gemma9b", 1, 8192, 8192, dtype="bf16"), name="prompt_gemma9b_8k"),
        # one request, one token: latency
        dict(_decode("qwen7b", 1, 0, 4096), name="decode_one"),
        # 64 continuations of one 16k prompt handed over at a tight budget
        dict(_decode("mistral7b", 64, 16384, 400, n_min=1, drop=0.4), name="decode_shared_16k"),
        # a batch of unrelated long requests
        dict(_decode("mistral7b", 4, 0, 32768, n_min=8189, drop=0.2), name="decode_long_batch"),
        # drafted tokens of 12 users behind one system prompt
        dict(_decode("gemma9b", 12, 2048, 1500, n_min=20, queries=5, dtype="bf16"), name="decode_drafts"),
        # a beam step: 8 children of one request
        dict(_pages("fork", "qwen7b", 1, 4001, children=8, grow=1), name="fork_beams"),
        # requests of different lengths rid of the tokens that their budgets dropped
        dict(_pages("compact", "mistral7b", 4, 16384, n_min=4095, drop=0.4), name="compact_batch"),
        # a preempted request's pages moved to another pool
        dict(_pages("copy", "mistral7b", 1, 8192), name="copy_request"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "decode", "decode", "decode", "fork", "compact", "copy"])
    model = rng.choice(list(MODELS))
    Hq, H, d, L = MODELS[model]
    dtype = rng.choice(list(TYPES))
    block = rng.choice([16, 16, 16, 32, 64, 8, 5, 1])
    if kind == "prompt":
        causal = rng.random() < 0.8
        c = _prompt(model, 1, 1, 1, dtype=dtype, causal=causal, codec=rng.random() < 0.5)
        while True:  # the plain form's logits stay below the largest listed case's
            c["count"] = _log(rng, 1, 32)
            c["nq"] = _log(rng, 1, 8000)
            c["nq_min"] = rng.randint(1, c["nq"])
            c["nk"] = c["nq"] + (rng.choice([0, _log(rng, 1, 30000)]))
            if 1000 < c["count"] * Hq * c["nq"] * c["nk"] < 1.8e9 and c["count"] * Hq * c["nk"] * d < 2.0e8:
                return c
    if kind == "decode":
        while True:
            count = _log(rng, 1, 96)
            prefix = rng.choice([0, _log(rng, 64, 20000) // block * block])
            n = _log(rng, 8, 30000)
            queries = rng.choice([1, 1, 1, rng.randint(2, 8)])
            n_min = rng.randint(queries, max(queries, n))
            if count * (prefix + max(n, queries)) * H * d < 1.0e9:
                return _decode(model, count, prefix, max(n, queries), n_min=n_min, queries=queries,
                               drop=rng.choice([0.0, rng.uniform(0.05, 0.9)]), block=block, dtype=dtype)
    while True:
        count = 1 if kind == "copy" else _log(rng, 1, 48)
        n = _log(rng, 1, 20000)
        n_min = rng.randint(1, n)
        children = rng.randint(1, 16)
        if count * n * L * H * d < 6e8 and count * children < 256:
            break
    c = _pages(kind, model, count, n, n_min=n_min, block=block)
    if kind == "fork":
        c.update(children=children, grow=rng.choice([1, 1, rng.randint(2, 40)]))
    if kind == "compact":
        c.update(drop=rng.uniform(0.05, 0.9))
    return c


def _spread(lo, hi, count):
    """count lengths over [lo, hi], both among them, in no order of size: a low-discrepancy sequence."""
    if count == 1:
        return [hi]
    mid = [lo + int((hi - lo + 1) * ((0.6180339887498949 * i) % 1.0)) for i in range(1, count - 1)]
    return [hi] + mid + [lo]


def _prompt_lens(c):
    q = _spread(c["nq_min"], c["nq"], c["count"])
    return q, [n + c["nk"] - c["nq"] for n in q]


def _decode_lens(c):
    return [c["prefix"] + max(n, c["queries"]) for n in _spread(c["n_min"], c["n"], c["count"])]


def _dropped(c, n):
    """How many of n tokens a map drops; a request keeps its first and last ones."""
    return int(c.get("drop", 0.0) * max(0, n - 1 - max(1, c.get("queries", 1))))


def _cdiv(a, b):
    return -(-a // b)


def _tier_map(c, n, g):
    """A tier map of n tokens as the codec makes it: 0..2 for kept tokens, DROP for the rest."""
    tier = torch.randint(0, 3, (n,), generator=g, device=DEV, dtype=torch.uint8)
    k = _dropped(c, n)
    if k:
        last = max(1, c.get("queries", 1))
        tier[1 + torch.randperm(n - 1 - last, generator=g, device=DEV)[:k]] = DROP
    return tier


def _heavy(shape, g, dtype):
    """N(0, 1) with a few channels eight times as large, as the caches of the codec's workloads."""
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., torch.randperm(shape[-1], generator=g, device=DEV)[:4]] *= 8
    return x.to(dtype)


def prepare(case, seed):
    c = case
    Hq, H, d, L = MODELS[c["model"]]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=c)
    if c["kind"] == "prompt":
        dtype = TYPES[c["dtype"]]
        ql, kl = _prompt_lens(c)
        s.update(q_lens=ql, kv_lens=kl, q=torch.randn(sum(ql), Hq, d, generator=g, device=DEV).to(dtype))
        if c["codec"]:
            for name in ("k", "v"):
                s[name] = [_heavy((H, n, d), g, dtype) for n in kl]
        else:
            for name in ("k", "v"):
                s[name] = _heavy((sum(kl), H, d), g, dtype)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(sum(ql), Hq, dtype=torch.float32, device=DEV)
        if own:
            from paper_2606_08635_amd import skv
            need = skv.attn_prompt_workspace_size(ql, kl, Hq, H, d, causal=c["causal"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return s
    block = c["block"]
    if c["kind"] == "decode":
        dtype = TYPES[c["dtype"]]
        lens = _decode_lens(c)
        shared = c["prefix"] // block
        width = _cdiv(max(lens), block)
        blocks = shared + c["count"] * (width - shared) + 7
        perm = torch.randperm(blocks, generator=g, device=DEV).to(torch.int32)
        tables = perm[shared:shared + c["count"] * (width - shared)].view(c["count"], width - shared)
        s["tables"] = torch.cat([perm[:shared].expand(c["count"], shared), tables], 1).contiguous()
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["max_len"] = max(lens)
        s["k"], s["v"] = (_heavy((blocks, block, H, d), g, dtype) for _ in range(2))
        s["q"] = torch.randn(c["count"], c["queries"], Hq, d, generator=g, device=DEV).to(dtype)
        s["tiers"] = None
        if c["drop"]:  # one map of the shared prefix, each request's own behind it
            top = torch.empty(c["count"], max(lens), dtype=torch.uint8, device=DEV)
            top[:, :c["prefix"]] = _tier_map(c, c["prefix"], g)
            for b, n in enumerate(lens):
                top[b, c["prefix"]:n] = _tier_map(c, n - c["prefix"], g)
                top[b, n:] = 0
            s["tiers"] = top
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(c["count"], c["queries"], Hq, dtype=torch.float32, device=DEV)
        if own:
            from paper_2606_08635_amd import skv
            need = skv.attn_decode_workspace_size(c["count"], c["queries"], Hq, H, d, s["max_len"], c["prefix"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return s
    # pages: a pool that the requests fill in part, in no order
    lens = _spread(c["n_min"], c["n"], c["count"])
    width = _cdiv(c["n"], block)
    used = c["count"] * width
    children = c["count"] * c.get("children", 0)
    out_width = width + _cdiv(c.get("grow", 0), block)
    spare = children * (1 + _cdiv(c.get("grow", 0), block)) if children else used
    blocks = used + spare + 5
    perm = torch.randperm(blocks, generator=g, device=DEV)[:used].to(torch.int32)
    s["tables"] = perm.view(c["count"], width)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV) < ((s["lens"] + block - 1) // block)[:, None]
    s["refs"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
    s["refs"][s["tables"][held].long()] = 1
    for name in ("k", "v"):
        t = torch.empty(L, blocks, block, H, d, dtype=torch.float16, device=DEV)
        for layer in t:
            layer.copy_(torch.randn(layer.shape, generator=g, device=DEV))
        s[name] = t
    s["status"] = torch.zeros(3, dtype=torch.int32, device=DEV)
    rows = children or c["count"]
    s["out_tables"] = torch.zeros(rows, out_width, dtype=torch.int32, device=DEV)
    s["out_lens"] = torch.zeros(rows, dtype=torch.int32, device=DEV)
    if c["kind"] == "fork":
        order = torch.randperm(children, generator=g, device=DEV)
        s["parents"] = (order % c["count"]).to(torch.int32)
        s["new_lens"] = s["lens"][s["parents"].long()] + c["grow"]
    if c["kind"] == "compact":
        s["tiers"] = torch.zeros(c["count"], c["n"], dtype=torch.uint8, device=DEV)
        for b, n in enumerate(lens):
            s["tiers"][b, :n] = _tier_map(c, n, g)
    if c["kind"] == "copy":
        s["src"] = s["tables"][held]
        s["dst"] = torch.randperm(blocks, generator=g, device=DEV)[:s["src"].numel()].to(torch.int32)
        s["k2"], s["v2"] = (torch.zeros_like(s[name]) for name in ("k", "v"))
    if own:
        from paper_2606_08635_amd import skv
        need = skv.pages_workspace_size(rows, blocks, c["n"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s


def _softmax_sum(z, seen, v):
    """Softmax of z over its last axis where `seen`, times v; its log-sum. Rows that see nothing give 0 and -inf."""
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out, (top + torch.log(total)).squeeze(-1)


def _padded(x, lens, size):
    """[sum(lens), ...] tokens as [sequence, size, ...] and which of its places hold one."""
    n = torch.tensor(lens, device=DEV)
    at = torch.arange(size, device=DEV)
    held = at < n[:, None]
    return x[torch.where(held, (n.cumsum(0) - n)[:, None] + at, 0)], held


def _plain_prompt(s):
    c = s["case"]
    Hq, H, d, _ = MODELS[c["model"]]
    G, B = Hq // H, c["count"]
    k, v = ((torch.cat([x.transpose(0, 1) for x in s[n]]) if c["codec"] else s[n]).float() for n in ("k", "v"))
    nq, nk = max(s["q_lens"]), max(s["kv_lens"])
    q, has_q = _padded(s["q"].float(), s["q_lens"], nq)
    k, has_k = _padded(k, s["kv_lens"], nk)
    v, _ = _padded(v, s["kv_lens"], nk)
    q = q.view(B, nq, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * nq, d)
    z = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, H, G, nq, nk) * (1.0 / math.sqrt(d))
    seen = has_k[:, None, :]
    if c["causal"]:
        more = torch.tensor(s["kv_lens"], device=DEV) - torch.tensor(s["q_lens"], device=DEV)
        last = torch.arange(nq, device=DEV) + more[:, None]
        seen = seen & (torch.arange(nk, device=DEV) <= last[..., None])
    seen = seen[:, None, None].expand(B, H, G, -1 if c["causal"] else nq, nk)
    out, lse = _softmax_sum(z, seen, v.permute(0, 2, 1, 3)[:, :, None])
    out = out.permute(0, 3, 1, 2, 4).reshape(B, nq, Hq, d)[has_q]
    return out.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, nq, Hq)[has_q]


def _plain_decode(s):
    c = s["case"]
    Hq, H, d, _ = MODELS[c["model"]]
    G, B, Lq, n, block = Hq // H, c["count"], c["queries"], s["max_len"], c["block"]
    at = torch.arange(n, device=DEV)
    page = s["tables"].long()[:, at // block]
    held = at < s["lens"][:, None]
    k, v = (s[name][torch.where(held, page, 0), at % block].float().transpose(1, 2) for name in ("k", "v"))
    q = s["q"].float().view(B, Lq, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * Lq, d)
    z = torch.matmul(q, k.transpose(2, 3)).view(B, H, G, Lq, n) * (1.0 / math.sqrt(d))
    last = s["lens"][:, None] - Lq + torch.arange(Lq, device=DEV)
    seen = at <= last[..., None]
    if s["tiers"] is not None:
        seen = seen & (s["tiers"] != DROP)[:, None]
    out, lse = _softmax_sum(z, seen[:, None, None], v[:, :, None])
    out = out.permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, d).to(s["q"].dtype)
    return out, lse.permute(0, 3, 1, 2).reshape(B, Lq, Hq)


def _plain_free(s, tables, lens):
    held = torch.arange(tables.shape[1], device=DEV) < _cdiv(lens, s["case"]["block"])[:, None]
    pages = tables[held].long()
    s["refs"].index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))


def _plain_take(s, need):
    """The lowest free pages for `need` [rows, places] (true: one page there), in order; held from now on."""
    pages = torch.nonzero(s["refs"] == 0).flatten()[:int(need.sum())]
    s["refs"][pages] = 1
    return pages


def _plain_rows(s, rows, src_page, src_slot, dst_page, dst_slot):
    for name in ("k", "v"):
        s[name][:, dst_page[rows], dst_slot[rows]] = s[name][:, src_page[rows], src_slot[rows]]


def _plain_fork(s):
    block, out = s["case"]["block"], s["out_tables"]
    tables, lens = s["tables"].long()[s["parents"].long()], s["lens"][s["parents"].long()]
    at = torch.arange(out.shape[1], device=DEV)
    full, part = (lens // block)[:, None], lens % block
    wide = torch.nn.functional.pad(tables, (0, out.shape[1] - tables.shape[1]))
    shared, last = at < full, (at == full) & (part > 0)[:, None]
    s["refs"].index_add_(0, wide[shared], torch.ones_like(wide[shared], dtype=torch.int32))
    pages = _plain_take(s, last)
    slot = torch.arange(block, device=DEV).expand(pages.numel(), block)
    _plain_rows(s, slot < part[part > 0][:, None], wide[last][:, None].expand_as(slot), slot,
                pages[:, None].expand_as(slot), slot)
    out[shared] = wide[shared].int()
    out[last] = pages.int()
    s["out_lens"].copy_(lens)
    # room for the children's next tokens
    more = (at >= _cdiv(lens, block)[:, None]) & (at < _cdiv(s["new_lens"], block)[:, None])
    out[more] = _plain_take(s, more).int()
    s["status"].zero_()
    _plain_free(s, out, s["new_lens"])


def _plain_compact(s):
    block, out, tables = s["case"]["block"], s["out_tables"], s["tables"].long()
    token = torch.arange(s["tiers"].shape[1], device=DEV).expand(s["tiers"].shape)
    keep = (token < s["lens"][:, None]) & (s["tiers"] != DROP)
    to = keep.cumsum(1) - 1
    kept = keep.sum(1, dtype=torch.int32)
    intact = torch.where(keep | (token >= s["lens"][:, None]), s["lens"][:, None], token).amin(1, keepdim=True)
    at = torch.arange(out.shape[1], device=DEV)
    shared = at < intact // block
    held = at < _cdiv(kept, block)[:, None]
    s["refs"].index_add_(0, tables[shared], torch.ones_like(tables[shared], dtype=torch.int32))
    out[shared] = tables[shared].int()
    out[held & ~shared] = _plain_take(s, held & ~shared).int()
    moved = keep & ~shared.gather(1, to.clamp(min=0) // block)
    _plain_rows(s, moved, tables.gather(1, token // block), token % block,
                out.long().gather(1, to.clamp(min=0) // block), to % block)
    s["out_lens"].copy_(kept)
    s["status"].zero_()
    _plain_free(s, out, kept)


def _pages_outputs(s):
    return dict(k=s["k"], v=s["v"], refs=s["refs"], tables=s["out_tables"], lens=s["out_lens"], status=s["status"])


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        if kind in ("prompt", "decode"):
            out, lse = (_plain_prompt if kind == "prompt" else _plain_decode)(s)
            return dict(out=out, lse=lse)
        if kind == "copy":
            for name in ("k", "v"):
                s[name + "2"][:, s["dst"].long()] = s[name][:, s["src"].long()]
            s["status"].zero_()
            return dict(k=s["k2"], v=s["v2"], status=s["status"])
        (_plain_fork if kind == "fork" else _plain_compact)(s)
        return _pages_outputs(s)
    from paper_2606_08635_amd import skv
    if kind == "prompt":
        skv.attn_prompt(s["q"], s["k"], s["v"], s["out"], s["q_lens"], s["kv_lens"], causal=c["causal"],
                        lse=s["lse"], ws=s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "decode":
        skv.attn_decode(s["q"], s["k"], s["v"], s["tables"], s["lens"], s["out"], s["ws"], s["max_len"],
                        prefix_len=c["prefix"], tiers=s["tiers"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if kind == "copy":
        skv.pages_copy(s["k"], s["v"], s["k2"], s["v2"], s["src"], s["dst"], s["status"][:1])
        return dict(k=s["k2"], v=s["v2"], status=s["status"])
    if kind == "fork":
        skv.pages_fork(s["k"], s["v"], s["refs"], s["tables"], s["lens"], s["parents"], s["out_tables"], s["out_lens"],
                       s["ws"], s["status"][:1])
        skv.pages_reserve(s["refs"], s["out_tables"], s["out_lens"], s["new_lens"], c["block"], s["ws"],
                          s["status"][1:2])
        skv.pages_free(s["refs"], s["out_tables"], s["new_lens"], c["block"], s["status"][2:])
    else:
        skv.pages_compact(s["k"], s["v"], s["refs"], s["tables"], s["lens"], s["tiers"], s["out_tables"], s["out_lens"],
                          s["ws"], s["status"][:1])
        skv.pages_free(s["refs"], s["out_tables"], s["out_lens"], c["block"], s["status"][1:2])
    return _pages_outputs(s)


def work(case):
    c = case
    Hq, H, d, L = MODELS[c["model"]]
    if c["kind"] == "prompt":
        ql, kl = _prompt_lens(c)
        pairs = sum(a * b - (a * (a - 1) // 2 if c["causal"] else 0) for a, b in zip(ql, kl))
        nbytes = 2 * d * (2 * Hq * sum(ql) + 2 * H * sum(kl)) + 4 * Hq * sum(ql)
        return {"bytes": nbytes, "flops": 4 * d * Hq * pairs}
    block = c["block"]
    if c["kind"] == "decode":
        lens, Lq = _decode_lens(c), c["queries"]
        prefix = c["prefix"] - _dropped(c, c["prefix"])
        tails = [n - c["prefix"] - _dropped(c, n - c["prefix"]) for n in lens]
        rows = prefix + sum(tails)
        masks = c["prefix"] + sum(n - c["prefix"] for n in lens) if c["drop"] else 0
        nbytes = 4 * d * H * rows + len(lens) * Lq * Hq * (4 * d + 4) + masks + 4 * sum(_cdiv(n, block) for n in lens)
        pairs = sum(Lq * (prefix + t) - Lq * (Lq - 1) // 2 for t in tails)
        return {"bytes": nbytes, "flops": 4 * d * Hq * pairs}
    lens = _spread(c["n_min"], c["n"], c["count"])
    row = 2 * L * H * d * 2  # K and V of a token in every layer
    if c["kind"] == "copy":
        pages = sum(_cdiv(n, block) for n in lens)
        return {"bytes": 2 * row * block * pages + 8 * pages, "flops": 0}
    if c["kind"] == "fork":
        moved = c["children"] * sum(n % block for n in lens)
        entries = c["children"] * sum(_cdiv(n + c["grow"], block) for n in lens)
        return {"bytes": 2 * row * moved + 16 * entries, "flops": 0}
    kept = [n - _dropped(c, n) for n in lens]
    return {"bytes": 2 * row * sum(kept) + sum(lens) + 16 * sum(_cdiv(n, block) for n in kept), "flops": 0}


def exact(case, seed):
    """Attention by its definition, one sequence and KV head at a time; the page operators only move values."""
    c = case
    if c["kind"] not in ("prompt", "decode"):
        return None
    Hq, H, d, _ = MODELS[c["model"]]
    G = Hq // H
    s = prepare(case, seed)
    outs, lses = [], []
    for b in range(c["count"]):
        if c["kind"] == "prompt":
            q0, k0 = sum(s["q_lens"][:b]), sum(s["kv_lens"][:b])
            nq, nk = s["q_lens"][b], s["kv_lens"][b]
            q = s["q"][q0:q0 + nq]
            k, v = (s[n][b].transpose(0, 1) if c["codec"] else s[n][k0:k0 + nk] for n in ("k", "v"))
            dropped = None
            limit = nk - nq if c["causal"] else nk
        else:
            nq, nk = c["queries"], int(s["lens"][b])
            q = s["q"][b]
            pages = s["tables"][b, :_cdiv(nk, c["block"])].long()
            k, v = (s[n][pages].reshape(-1, H, d)[:nk] for n in ("k", "v"))
            dropped = None if s["tiers"] is None else s["tiers"][b, :nk] == DROP
            limit = nk - nq
        out = torch.empty(nq, Hq, d, dtype=torch.float64, device=DEV)
        lse = torch.empty(nq, Hq, dtype=torch.float64, device=DEV)
        hidden = torch.triu(torch.ones(nq, nk, dtype=torch.bool, device=DEV), diagonal=limit + 1)
        if dropped is not None:
            hidden |= dropped
        for h in range(Hq):
            kh, vh = k[:, h // G].double(), v[:, h // G].double()
            z = (q[:, h].double() @ kh.t()).div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
            lse[:, h] = torch.logsumexp(z, 1)
            out[:, h] = torch.exp(z.sub_(lse[:, h, None])) @ vh
        outs.append(out)
        lses.append(lse)
    if c["kind"] == "prompt":
        return dict(out=torch.cat(outs), lse=torch.cat(lses))
    return dict(out=torch.stack(outs), lse=torch.stack(lses))
