"""Timed cases of decoding with several continuations of a request over the paged cache.

Four operators: attention of a tree of drafted tokens over the cache (all pages, or the pages selected per head), the
commit of accepted tokens to the cache with its page summaries, the re-layout of the cache when requests are forked,
reordered, freed or thinned out, and beam search's selection.  ``run`` computes them in elementary torch operations, or,
where ``own`` is true, through the library's entry points.

The layout of a case (lengths, trees, parents, kept pages) belongs to the case; the contents come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128                                     # head dimension of the library
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
POOL_BYTES = 4400 << 20                     # largest K/V pool of a case
SCORE_BYTES = 4400 << 20                    # largest fp32 score tensor of the plain attention


# ---- cases -------------------------------------------------------------------------------------------------------

def _tree(name, *, batch=1, q_heads=32, kv_heads=8, page=16, ctx=131072, ragged=False, draft=16, chain=False, top_k=0):
    """``draft``: drafted tokens a request; ``top_k``: pages selected per query head, 0 = the whole context."""
    return dict(name=name, op="tree", batch=batch, q_heads=q_heads, kv_heads=kv_heads, page=page, ctx=ctx, ragged=ragged,
                draft=draft, chain=chain, top_k=top_k)


def _append(name, *, batch, kv_heads=8, page=16, ctx=4096, new=16, path=0):
    """``path``: accepted tokens (1..path) out of ``new`` drafted ones; 0 = a prompt of up to ``new`` tokens."""
    return dict(name=name, op="append", batch=batch, kv_heads=kv_heads, page=page, ctx=ctx, new=new, path=path)


def _pages(name, *, batch, kv_heads=8, page=16, ctx=16384, mode="compact", beams=1):
    """``mode``: "compact" frees a third of the requests and a quarter of the others' pages inside one pool;
    "reorder" continues the surviving beams of every prompt in a second pool."""
    return dict(name=name, op="pages", batch=batch, kv_heads=kv_heads, page=page, ctx=ctx, mode=mode, beams=beams)


def _beam(name, *, batch, beams, vocab, keep, dtype="f32"):
    return dict(name=name, op="beam", batch=batch, beams=beams, vocab=vocab, keep=keep, dtype=dtype)


def listed():
    return [
        # a short chain of drafted tokens behind a short prompt: launches and hand-offs count
        _tree("tree_short_chain", ctx=777, draft=5, chain=True),
        # the headline layer (32 query heads, 8 KV heads, 128K tokens) with a small tree
        _tree("tree_128k_one_request"),
        # a serving batch: ragged contexts of up to 32K tokens, trees of up to 48 tokens
        _tree("tree_batch16_ragged", batch=16, ctx=32768, ragged=True, draft=48),
        # eight query heads per KV head, pages of 32, 64 drafted tokens over 256K: 512 rows per KV head
        _tree("tree_256k_wide", q_heads=64, page=32, ctx=262144, draft=64),
        # trees over the pages selected per head, 128K tokens a request
        _tree("tree_selected_batch8", batch=8, ctx=131072, draft=16, top_k=256),
        # the accepted tokens of a drafting step, 1..8 of 16, for 64 requests
        _append("append_accepted_batch64", batch=64, path=8),
        # prompts of up to 8191 tokens written to the cache
        _append("append_prompts", batch=8, ctx=40, new=8191),
        # requests that ended are freed, cold pages of the others dropped, the rest moved together inside the pool
        _pages("pages_compact_in_place", batch=24, ctx=16384),
        # a beam step of 4 prompts of 4 beams: every beam continues its parent in the second pool
        _pages("pages_reorder_beams", batch=16, ctx=8192, mode="reorder", beams=4),
        # one prompt, four beams, a small vocabulary
        _beam("beam_one_prompt", batch=1, beams=4, vocab=32000, keep=8),
        # a batch with an odd vocabulary in bf16
        _beam("beam_odd_vocab", batch=12, beams=5, vocab=50257, keep=10, dtype="bf16"),
        # a large batch over a large vocabulary
        _beam("beam_batch32_128k", batch=32, beams=16, vocab=131072, keep=32),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["tree", "tree", "tree", "selected", "append", "pages", "beam"])
    if op == "beam":
        batch, beams, vocab = log_int(1, 32), rng.choice([1, 2, 3, 4, 5, 8, 16]), log_int(1000, 131072)
        return _pure(_beam("", batch=batch, beams=beams, vocab=vocab, keep=min(64, beams * rng.choice([1, 2])),
                           dtype=rng.choice(list(DTYPES))))
    kv_heads, page = rng.choice([1, 2, 4, 8, 8]), rng.choice([16, 16, 32])
    if op == "append":
        if rng.random() < 0.5:
            return _pure(_append("", batch=log_int(1, 64), kv_heads=kv_heads, page=page, ctx=log_int(20, 4096),
                                 new=log_int(4, 64), path=rng.choice([1, 2, 3, 4])))
        return _pure(_append("", batch=log_int(1, 8), kv_heads=kv_heads, page=page, ctx=log_int(20, 4096), new=log_int(64, 8191)))
    if op == "pages":
        beams = rng.choice([2, 3, 4])
        mode = rng.choice(["compact", "reorder"])
        batch = beams * rng.randint(1, 5) if mode == "reorder" else rng.randint(3, 24)
        return _pure(_pages("", batch=batch, kv_heads=kv_heads, page=page, ctx=log_int(100, 8192), mode=mode, beams=beams))
    group = rng.choice([1, 2, 3, 4, 4, 8])
    batch, ctx, draft = log_int(1, 32), log_int(64, 131072), log_int(1, 128)
    while batch > 1 and batch * ctx * kv_heads * 4 * D > POOL_BYTES // 2:
        batch //= 2
    while draft > 1 and batch * kv_heads * group * draft * ctx * 4 > SCORE_BYTES:
        draft //= 2
    top_k = 0
    if op == "selected":
        draft = min(draft, 32)
        ctx = max(ctx, 1024)
        top_k = max(2, min(256, ctx // page // 8, 32768 // (batch * group * kv_heads // 4 + 1)) // 2 * 2)
    return _pure(_tree("", batch=batch, q_heads=kv_heads * group, kv_heads=kv_heads, page=page, ctx=ctx,
                       ragged=batch > 1 and rng.random() < 0.5 and not top_k, draft=draft, chain=rng.random() < 0.25, top_k=top_k))


def _pure(c):
    return {k: v for k, v in c.items() if k != "name"}


# ---- layouts of a case ------------------------------------------------------------------------------------------------

def _lengths(c):
    if c["op"] == "tree" and not c["ragged"]:
        return np.full(c["batch"], c["ctx"], dtype=np.int64)
    lens = np.random.default_rng(c["ctx"]).integers(max(1, c["ctx"] // 16), c["ctx"] + 1, size=c["batch"])
    if c["op"] == "pages" and c["mode"] == "reorder":                 # the beams of a prompt are equally long
        lens = np.repeat(lens[:: c["beams"]], c["beams"])
    return lens


def _drafts(c):
    """(drafted tokens of each request, which drafted tokens each of them attends: bool [B][T][T])."""
    batch, T = c["batch"], c["draft"]
    rng = np.random.default_rng(T)
    n = rng.integers(max(1, T // 2), T + 1, size=batch) if batch > 1 else np.full(1, T)
    sees = np.zeros((batch, T, T), dtype=bool)
    rows = np.arange(batch)
    for i in range(T):
        parent = np.full(batch, i - 1) if c["chain"] else rng.integers(-1, i, size=batch) if i else np.full(batch, -1)
        sees[:, i] = np.where((parent >= 0)[:, None], sees[rows, np.maximum(parent, 0)], False)
        sees[:, i, i] = True
    return n, sees


def _accepted(c):
    """(tokens that each request takes over, their places among the new ones)."""
    rng = np.random.default_rng(c["new"])
    if not c["path"]:
        return rng.integers(max(1, c["new"] // 4), c["new"] + 1, size=c["batch"]), None
    n = rng.integers(1, c["path"] + 1, size=c["batch"])
    path = np.sort(np.argsort(rng.random((c["batch"], c["new"])), axis=1)[:, : c["path"]], axis=1)
    return n, np.where(np.arange(c["path"]) < n[:, None], path, -1)


def _relayout(c):
    """(parents, spare pages, kept pages or None) of a re-layout."""
    rng = np.random.default_rng(c["ctx"] + 1)
    batch = c["batch"]
    lens = _lengths(c)
    pages = -(-lens // c["page"])
    if c["mode"] == "reorder":
        group = np.arange(batch) // c["beams"] * c["beams"]
        return group + rng.integers(0, c["beams"], size=batch), np.full(batch, 2), None
    parent = np.full(batch, -1)
    left = np.flatnonzero(rng.random(batch) >= 1 / 3)
    parent[: len(left)] = left
    keep = rng.random(int((pages + 1).sum())) >= 0.25
    return parent, np.ones(batch, dtype=np.int64), keep


def _moves(c):
    """Pages that a re-layout has to move."""
    parent, reserve, keep = _relayout(c)
    pages = -(-_lengths(c) // c["page"])
    base = np.concatenate([[0], np.cumsum(pages + 1)])
    at = n = 0
    for j, b in enumerate(parent):
        cnt = 0
        if b >= 0:
            src = np.arange(base[b], base[b] + pages[b])
            if keep is not None:
                src = src[keep[src]]
            cnt = len(src)
            n += int((src != at + np.arange(cnt)).sum()) if c["mode"] == "compact" else cnt
        at += cnt + int(reserve[j])
    return n


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x)).to(dtype).cuda()


def _normal(shape, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) * scale).contiguous()


def _pool(c, gen, spare=0):
    """A pool with ``spare`` pages behind the tokens of every request."""
    pages = -(-_lengths(c) // c["page"]) + spare
    base = np.concatenate([[0], np.cumsum(pages)])
    pool = _normal((int(base[-1]), c["kv_heads"], 2, c["page"], D), gen)
    return pool, base


def _handle(c, s, batch, q_heads, max_pages, top_k=1):
    """The ctx with its workspace that a program keeps beside its pool."""
    from paper_2603_17803_b200 import binding as B
    s["B"] = B
    s["shape"] = B.make_shape(batch=batch, n_q_heads=q_heads, n_kv_heads=c["kv_heads"], page_size=c["page"], top_k=top_k,
                              n_queues=1, max_pages_per_req=max_pages, max_clusters_total=1, n_pool_pages=s["pool"].shape[0])
    s["ctx"] = B.swarm_create(s["shape"])
    s["ctx_ws"] = torch.empty(B.swarm_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    B.swarm_set_workspace(s["ctx"], s["ctx_ws"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": case, "op": case["op"]}
    {"tree": _prepare_tree, "append": _prepare_append, "pages": _prepare_pages, "beam": _prepare_beam}[case["op"]](case, s, gen)
    return s


def _prepare_tree(c, s, gen):
    batch, T, hq, hkv, S = c["batch"], c["draft"], c["q_heads"], c["kv_heads"], c["page"]
    s["pool"], base = _pool(c, gen)
    lens = _lengths(c)
    n, sees = _drafts(c)
    s["page_base"], s["ctx_len"], s["n_draft"] = _dev(base, torch.int64), _dev(lens), _dev(n)
    s["q"] = _normal((batch, T, hq, D), gen, 2.0)
    s["k"], s["v"] = _normal((batch, T, hkv, D), gen), _normal((batch, T, hkv, D), gen)
    s["mask"] = None
    if not c["chain"]:
        words = -(-T // 32)
        bits = np.zeros((batch, T, words * 32), dtype=np.uint64)
        bits[:, :, :T] = sees
        packed = (bits.reshape(batch, T, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
        s["mask"] = torch.from_numpy(packed.view(np.int32)).cuda()
    s["sel"] = s["n_sel"] = None
    if c["top_k"]:
        # half of a head's pages are those of its whole group, half are its own
        g, k, P = hq // hkv, c["top_k"], -(-c["ctx"] // S)
        order = torch.rand((batch, hkv, P), generator=gen, device="cuda").argsort(-1)
        shared = order[:, :, None, : k // 2].expand(-1, -1, g, -1)
        single = order[:, :, k // 2: k // 2 + g * (k // 2)].reshape(batch, hkv, g, k // 2)
        s["sel"] = torch.cat([shared, single], -1).sort(-1).values.reshape(batch, hq, k).int().contiguous()
        s["n_sel"] = torch.full((batch, hq), k, dtype=torch.int32, device="cuda")
    s["out"] = torch.zeros((batch, T, hq, D), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((batch, T, hq), dtype=torch.float32, device="cuda")
    if own:
        _handle(c, s, batch, hq, int((-(-lens // S)).max()), max(1, c["top_k"]))
        B = s["B"]
        s["inputs"] = B.make_inputs(kv_pool=s["pool"], page_base=s["page_base"], ctx_len=s["ctx_len"])
        s["tree"] = B.make_tree(q=s["q"], k=s["k"], v=s["v"], n_draft=s["n_draft"], mask=s["mask"])
        s["ws"] = torch.empty(B.swarm_tree_attn_workspace_bytes(s["shape"], T), dtype=torch.uint8, device="cuda")


def _prepare_append(c, s, gen):
    batch, S = c["batch"], c["page"]
    n, path = _accepted(c)
    s["pool"], base = _pool(c, gen, -(-c["new"] // S) + 1)
    lens = _lengths(c)
    s["page_base"], s["ctx_len"], s["n_new"] = _dev(base, torch.int64), _dev(lens), _dev(n)
    s["path"] = None if path is None else _dev(path)
    s["k"], s["v"] = (_normal((batch, c["new"], c["kv_heads"], D), gen) for _ in range(2))
    # the summaries of the pages written so far
    s["ksum"] = torch.zeros((s["pool"].shape[0], c["kv_heads"], 2, D), dtype=torch.bfloat16, device="cuda")
    owner = np.repeat(np.arange(batch), np.diff(base))
    valid = np.clip(lens[owner] - (np.arange(base[-1]) - base[owner]) * S, 0, S)
    for lo in range(0, len(valid), 8192):                                 # (in slices: a pool in fp32 is large)
        v = _dev(valid[lo: lo + 8192])
        there = (torch.arange(S, device="cuda") < v[:, None])[:, None, :, None]
        K = s["pool"][lo: lo + 8192, :, 0]
        some = (v > 0)[:, None, None]
        s["ksum"][lo: lo + 8192, :, 0] = torch.where(some, K.masked_fill(~there, math.inf).amin(2), 0)
        s["ksum"][lo: lo + 8192, :, 1] = torch.where(some, K.masked_fill(~there, -math.inf).amax(2), 0)
    s["new_len"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
    if own:
        _handle(c, s, batch, c["kv_heads"], int(np.diff(base).max()))
        B = s["B"]
        s["inputs"] = B.make_inputs(page_base=s["page_base"], ctx_len=s["ctx_len"])
        s["tokens"] = B.make_new_tokens(k=s["k"], v=s["v"], n_new=s["n_new"], path=s["path"])


def _prepare_pages(c, s, gen):
    batch, hkv = c["batch"], c["kv_heads"]
    s["pool"], base = _pool(c, gen, 1)
    parent, reserve, keep = _relayout(c)
    n_pool = int(base[-1]) + 2 * batch                                   # room for the spare pages of the new layout
    s["pool"] = torch.cat([s["pool"], torch.zeros_like(s["pool"][: 2 * batch])])
    s["ksum"] = _normal((n_pool, hkv, 2, D), gen)
    s["p2c"] = torch.randint(0, 1 << 20, (n_pool,), generator=gen, device="cuda", dtype=torch.int32)
    s["page_base"], s["ctx_len"] = _dev(base, torch.int64), _dev(_lengths(c))
    s["parent"], s["reserve"] = _dev(parent), _dev(reserve)
    s["keep"] = None if keep is None else _dev(np.concatenate([keep, np.ones(n_pool - len(keep), dtype=bool)]), torch.uint8)
    s["to"] = (s["pool"], s["ksum"], s["p2c"])
    if c["mode"] == "reorder":
        s["to"] = tuple(torch.zeros_like(x) for x in s["to"])
    s["new_base"] = torch.zeros(batch + 1, dtype=torch.int64, device="cuda")
    s["new_len"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
    if own:
        _handle(c, s, batch, hkv, int(np.diff(base).max()) + 2)
        B = s["B"]
        i32 = dict(dtype=torch.int32, device="cuda")
        s["src"], s["dst"], s["n_moves"] = torch.empty(n_pool, **i32), torch.empty(n_pool, **i32), torch.empty(1, **i32)
        s["plan"] = B.make_page_plan(page_base=s["page_base"], ctx_len=s["ctx_len"], parent=s["parent"], reserve=s["reserve"],
                                     keep=s["keep"], in_place=c["mode"] == "compact", new_page_base=s["new_base"],
                                     new_ctx_len=s["new_len"], src=s["src"], dst=s["dst"], n_moves=s["n_moves"])
        s["moves"] = B.make_page_moves(src=s["src"], dst=s["dst"], n_moves=s["n_moves"], from_pool=s["pool"], to_pool=s["to"][0],
                                       from_ksum=s["ksum"], to_ksum=s["to"][1], from_page2cluster=s["p2c"],
                                       to_page2cluster=s["to"][2])
        s["ws"] = torch.empty(B.swarm_move_pages_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")


def _prepare_beam(c, s, gen):
    batch, beams, V = c["batch"], c["beams"], c["vocab"]
    # a language model's logits: a wide body and a few likely tokens
    x = torch.randn((batch, beams, V), generator=gen, device="cuda") * 2.5
    likely = torch.randint(0, V, (batch, beams, 16), generator=gen, device="cuda")
    x.scatter_add_(2, likely, torch.rand((batch, beams, 16), generator=gen, device="cuda") * 8)
    s["logits"] = x.to(DTYPES[c["dtype"]])
    s["score"] = -torch.rand((batch, beams), generator=gen, device="cuda") * 12
    s["new_score"] = torch.zeros((batch, c["keep"]), dtype=torch.float32, device="cuda")
    s["new_parent"], s["token"] = (torch.zeros((batch, c["keep"]), dtype=torch.int32, device="cuda") for _ in range(2))
    if own:
        from paper_2603_17803_b200 import binding as B
        s["B"] = B
        s["ws"] = torch.empty(B.swarm_beam_select_workspace_bytes(batch, beams, V, c["keep"]), dtype=torch.uint8, device="cuda")


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(state):
    op = state["op"]
    if own:
        return {"tree": _own_tree, "append": _own_append, "pages": _own_pages, "beam": _own_beam}[op](state)
    return {"tree": _plain_tree, "append": _plain_append, "pages": _plain_pages, "beam": _plain_beam}[op](state)


def _own_tree(s):
    s["B"].swarm_tree_attn(s["ctx"], s["inputs"], s["tree"], s["sel"], s["n_sel"], s["ws"], s["out"], s["lse"])
    return s["out"], s["lse"]


def _own_append(s):
    s["B"].swarm_append_tokens(s["ctx"], s["inputs"], s["tokens"], s["pool"], s["ksum"], s["new_len"])
    return s["pool"], s["ksum"], s["new_len"]


def _own_pages(s):
    s["B"].swarm_plan_pages(s["ctx"], s["plan"])
    s["B"].swarm_move_pages(s["ctx"], s["moves"], s["ws"])
    return s["to"], s["new_base"], s["new_len"]


def _own_beam(s):
    s["B"].swarm_beam_select(s["logits"], s["score"], s["ws"], s["new_score"], s["new_parent"], s["token"])
    return s["new_score"], s["new_parent"], s["token"]


def _plain_tree(s):
    c = s["c"]
    batch, T, hq, hkv, S = c["batch"], c["draft"], c["q_heads"], c["kv_heads"], c["page"]
    g, dev = hq // hkv, s["pool"].device
    scale = 1.0 / math.sqrt(D)
    t = torch.arange(T, device=dev)
    q = s["q"].float().view(batch, T, hkv, g, D).permute(0, 2, 3, 1, 4)              # [B][Hkv][g][T][d]
    # drafted tokens: the mask's bits, or a chain
    if s["mask"] is None:
        sees = (t[None, :] <= t[:, None])[None].expand(batch, T, T)
    else:
        sees = ((s["mask"][..., None] >> torch.arange(32, device=dev)) & 1).flatten(2)[:, :, :T].bool()
    sees = sees & (t < s["n_draft"][:, None])[:, None, :]
    kd, vd = (x.float().permute(0, 2, 3, 1).contiguous() if i == 0 else x.float().permute(0, 2, 1, 3).contiguous()
              for i, x in enumerate((s["k"], s["v"])))                               # [B][Hkv][d][T], [B][Hkv][T][d]
    own_scores = torch.matmul(q.reshape(batch, hkv, g * T, D), kd).view(batch, hkv, g, T, T) * scale
    own_scores = own_scores.masked_fill(~sees[:, None, None], -math.inf)
    # the context's tokens
    if s["sel"] is None:
        P = -(-int(_lengths(c).max()) // S)
        page = torch.arange(P, device=dev).expand(batch, P)
        at = (s["page_base"][:-1, None] + page).clamp(max=s["pool"].shape[0] - 1)
        there = (page[..., None] * S + torch.arange(S, device=dev) < s["ctx_len"][:, None, None]).view(batch, 1, 1, P * S)
        kv = s["pool"][at]                                                           # [B][P][Hkv][2][S][d]
        k = kv[:, :, :, 0].permute(0, 2, 1, 3, 4).float().reshape(batch, hkv, P * S, D)
        scores = torch.matmul(q.reshape(batch, hkv, g * T, D), k.transpose(-1, -2)).mul_(scale)
        del k
        scores = scores.masked_fill_(~there, -math.inf).view(batch, hkv, g, T, P * S)
        v = kv[:, :, :, 1].permute(0, 2, 1, 3, 4).float().reshape(batch, hkv, 1, P * S, D)
        v = v.masked_fill_(~there.view(batch, 1, 1, P * S, 1), 0)
        del kv
    else:
        k_sel = s["sel"].shape[-1]
        page = s["sel"].long()
        chosen = torch.arange(k_sel, device=dev) < s["n_sel"][..., None]
        at = (s["page_base"][:-1, None, None] + page).clamp(min=0)
        kv = s["pool"][at, (torch.arange(hq, device=dev) // g)[None, :, None]]       # [B][Hq][k][2][S][d]
        there = page[..., None] * S + torch.arange(S, device=dev) < s["ctx_len"][:, None, None, None]
        there = (there & chosen[..., None]).view(batch, hkv, g, 1, k_sel * S)
        k = kv[:, :, :, 0].float().reshape(batch, hkv, g, k_sel * S, D)
        scores = (torch.matmul(q, k.transpose(-1, -2)) * scale).masked_fill_(~there, -math.inf)
        v = kv[:, :, :, 1].float().reshape(batch, hkv, g, k_sel * S, D).masked_fill_(~there.transpose(-1, -2), 0)
    m = torch.maximum(scores.amax(-1, keepdim=True), own_scores.amax(-1, keepdim=True))
    ref = torch.where(m == -math.inf, 0.0, m)
    p = scores.sub_(ref).exp_()
    own_p = (own_scores - ref).exp()
    total = p.sum(-1, keepdim=True) + own_p.sum(-1, keepdim=True)
    if v.shape[2] == 1:
        rows = p.shape[-1]
        out = torch.matmul(p.view(batch, hkv, g * T, rows), v[:, :, 0]).view(batch, hkv, g, T, D)
    else:
        out = torch.matmul(p, v)
    out = out + torch.matmul(own_p.view(batch, hkv, g * T, T), vd).view(batch, hkv, g, T, D)
    out = torch.where(total > 0, out / total, 0.0)
    lse = (torch.log(total) + ref).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(batch, T, hq, D).to(torch.bfloat16)
    lse = lse.permute(0, 3, 1, 2).reshape(batch, T, hq)
    row = (t < s["n_draft"][:, None])[..., None]
    return torch.where(row[..., None], out, s["out"]), torch.where(row, lse, s["lse"])


def _plain_append(s):
    S = s["c"]["page"]
    batch, n_max = s["k"].shape[0], s["k"].shape[1] if s["path"] is None else s["path"].shape[1]
    dev = s["pool"].device
    i = torch.arange(n_max, device=dev)
    b, i = torch.nonzero(i < s["n_new"][:, None], as_tuple=True)
    from_ = i if s["path"] is None else s["path"][b, i].long()
    pos = s["ctx_len"][b].long() + i
    page, slot = s["page_base"][b] + pos // S, pos % S
    s["pool"][page, :, 0, slot] = s["k"][b, from_]
    s["pool"][page, :, 1, slot] = s["v"][b, from_]
    new_len = s["ctx_len"] + s["n_new"]
    # summaries of the pages touched
    p = torch.arange(-(-n_max // S) + 1, device=dev)
    first = s["ctx_len"].long() // S
    b, j = torch.nonzero((first[:, None] + p) * S < torch.where(s["n_new"] > 0, new_len, 0)[:, None], as_tuple=True)
    j = first[b] + j
    there = (j[:, None] * S + torch.arange(S, device=dev) < new_len[b][:, None])[:, None, :, None]
    K = s["pool"][s["page_base"][b] + j, :, 0]
    s["ksum"][s["page_base"][b] + j, :, 0] = K.masked_fill(~there, math.inf).amin(2)
    s["ksum"][s["page_base"][b] + j, :, 1] = K.masked_fill(~there, -math.inf).amax(2)
    return s["pool"], s["ksum"], new_len


def _plain_pages(s):
    S, dev = s["c"]["page"], s["pool"].device
    base, lens, parent = s["page_base"], s["ctx_len"].long(), s["parent"].long()
    batch, n_pool = lens.shape[0], s["pool"].shape[0]
    pages = (lens + S - 1) // S
    x = torch.arange(n_pool, device=dev)
    owner = (torch.searchsorted(base, x, right=True) - 1).clamp(max=batch - 1)
    kept = x < (base[:-1] + pages)[owner]
    if s["keep"] is not None:
        kept = kept & s["keep"].bool()
    before = torch.cumsum(kept, 0) - kept.long()                                     # kept pages in front of each page
    before = torch.cat([before, kept.sum().view(1)])
    first = before[base[:-1]]
    count = before[base[:-1] + pages] - first
    old = parent.clamp(min=0)
    n = torch.where(parent >= 0, count[old], 0)
    new_base = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), torch.cumsum(n + s["reserve"], 0)])
    # a partial last page that is kept ends the request as before
    tail = torch.where(kept[(base[:-1] + pages - 1).clamp(min=0)] & (pages > 0), pages * S - lens, 0)
    new_len = (n * S - torch.where(parent >= 0, tail[old], 0)).int()
    ids = torch.nonzero(kept).view(-1)
    j = torch.repeat_interleave(torch.arange(batch, device=dev), n)
    i = torch.arange(j.shape[0], device=dev) - (torch.cumsum(n, 0) - n)[j]
    src, dst = ids[first[old][j] + i], new_base[j] + i
    for a, b in zip((s["pool"], s["ksum"], s["p2c"]), s["to"]):                         # three tables of the cache
        b[dst] = a[src]
    return s["to"], new_base, new_len


def _plain_beam(s):
    batch, beams, V = s["logits"].shape
    keep = s["new_score"].shape[1]
    # in 64 bits: candidates of different beams lie close together
    x = s["logits"].double()
    m = x.amax(-1, keepdim=True)
    total = s["score"].double()[..., None] + (x - (m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))))
    value, at = torch.sort(total.view(batch, beams * V), dim=-1, descending=True, stable=True)
    value, at = value[:, :keep], at[:, :keep]
    none = value == -math.inf
    row = torch.arange(batch, device=x.device)[:, None] * beams
    return (value.float(), torch.where(none, -1, row + at // V).int(), torch.where(none, -1, at % V).int())


# ---- the floor ----------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "beam":
        n = c["batch"] * c["beams"] * c["vocab"]
        return {"bytes": n * (4 if c["dtype"] == "f32" else 2) + c["batch"] * (4 * c["beams"] + 12 * c["keep"]), "flops": 3 * n}
    row = c["kv_heads"] * 2 * D * 2                                                  # bytes of a token's K and V
    if c["op"] == "pages":
        return {"bytes": 2 * _moves(c) * (c["page"] * row + row + 4), "flops": 0}
    if c["op"] == "append":
        n, _ = _accepted(c)
        lens = _lengths(c)
        touched = int((-(-(lens + n) // c["page"]) - lens // c["page"]).sum())
        return {"bytes": int(n.sum()) * 2 * row + (touched + int((lens % c["page"] > 0).sum())) * row, "flops": int(n.sum()) * row // 2}
    n, sees = _drafts(c)
    group = c["q_heads"] // c["kv_heads"]
    lens = _lengths(c)
    if c["top_k"]:
        pages = c["top_k"] // 2 * (1 + group)
        kv = c["batch"] * min(pages * c["page"], c["ctx"]) * row
        seen = n * c["top_k"] * c["page"]
    else:
        kv = int(lens.sum()) * row
        seen = n * lens
    attended = int(seen.sum()) + sum(int(sees[b, : n[b], : n[b]].sum()) for b in range(c["batch"]))
    drafted = int(n.sum()) * (row + c["q_heads"] * (2 * D * 2 + 4))
    return {"bytes": kv + drafted, "flops": 4 * D * c["q_heads"] * attended}


# ---- in 64 bits, from the definitions ----------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"tree": _exact_tree, "append": _exact_append, "pages": _exact_pages, "beam": _exact_beam}[case["op"]](case, s)


def _exact_tree(c, s):
    S, g = c["page"], c["q_heads"] // c["kv_heads"]
    n, sees = _drafts(c)
    lens, base = _lengths(c), s["page_base"].tolist()
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(c["batch"]):
        L, nd = int(lens[b]), int(n[b])
        see = torch.from_numpy(sees[b, :nd, :nd]).cuda()
        for h in range(c["kv_heads"]):
            kv = s["pool"][base[b]: base[b + 1], h]                                  # [P][2][S][d]
            whole = [torch.cat([kv[:, i].reshape(-1, D)[:L], s["kv"[i]][b, :nd, h]]).double() for i in range(2)]
            for i in range(h * g, (h + 1) * g):
                K, V = whole
                if s["sel"] is not None:
                    pages = s["sel"][b, i].long()
                    at = (pages[:, None] * S + torch.arange(S, device="cuda")).view(-1)
                    at = torch.cat([at[at < L], torch.arange(L, L + nd, device="cuda")])
                    K, V = K[at], V[at]
                x = s["q"][b, :nd, i].double() @ K.T / math.sqrt(D)
                x[:, x.shape[1] - nd:][~see] = -math.inf
                lse[b, :nd, i] = torch.logsumexp(x, -1)
                out[b, :nd, i] = torch.softmax(x, -1) @ V
    return out, lse


def _exact_append(c, s):
    S = c["page"]
    n, path = _accepted(c)
    lens, base = _lengths(c), s["page_base"].tolist()
    for b in range(c["batch"]):
        L, nb = int(lens[b]), int(n[b])
        rows = torch.arange(nb, device="cuda") if path is None else torch.from_numpy(path[b, :nb]).cuda()
        for i, x in enumerate((s["k"], s["v"])):
            flat = s["pool"][base[b]: base[b + 1], :, i].transpose(1, 2).reshape(-1, c["kv_heads"], D)
            flat[L: L + nb] = x[b, rows]
            s["pool"][base[b]: base[b + 1], :, i] = flat.view(-1, S, c["kv_heads"], D).transpose(1, 2)
            if i == 0:
                for p in range(L // S, -(-(L + nb) // S)):
                    tokens = flat[p * S: min((p + 1) * S, L + nb)]
                    s["ksum"][base[b] + p, :, 0], s["ksum"][base[b] + p, :, 1] = tokens.amin(0), tokens.amax(0)
    return s["pool"], s["ksum"], _dev(lens + n)


def _exact_pages(c, s):
    parent, reserve, keep = _relayout(c)
    lens, S = _lengths(c), c["page"]
    pages = -(-lens // S)
    base = s["page_base"].tolist()
    old = [x.clone() for x in (s["pool"], s["ksum"], s["p2c"])]
    at, new_base, new_len = 0, [0], []
    for j, b in enumerate(parent):
        src = np.arange(base[b], base[b] + pages[b]) if b >= 0 else np.zeros(0, dtype=np.int64)
        length = int(lens[b]) if b >= 0 else 0
        if keep is not None and len(src):
            length = sum(min(S, length - S * p) for p in range(len(src)) if keep[src[p]])
            src = src[keep[src]]
        here = torch.from_numpy(src).cuda()
        for a, t in zip(old, s["to"]):
            t[at: at + len(src)] = a[here]
        at += len(src) + int(reserve[j])
        new_base.append(at)
        new_len.append(length)
    return s["to"], _dev(np.array(new_base), torch.int64), _dev(np.array(new_len))


def _exact_beam(c, s):
    rows = []
    for b in range(c["batch"]):
        p = torch.log_softmax(s["logits"][b].double(), -1) + s["score"][b].double()[:, None]
        rows.append(p.view(-1).topk(c["keep"]).values)
    return torch.stack(rows), None, None
