"""Decoding with several continuations, as a serving program runs it: drafted trees attended and committed through a Session, beams
selected, forked and compacted; on streams, in captured graphs, in pools beyond 32-bit offsets; and what is refused."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2603_17803_b200 import binding as B
from paper_2603_17803_b200 import workloads as W
from paper_2603_17803_b200.session import Session
from test_gpu_cache_pages import Layout, close, dev, handle, same
from test_gpu_tree import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def small(**kw):
    return W.scaled(W.CONFIGS["c2_128k"], **{**dict(batch=3, ctx_len=16 * 180 + 7, top_k=24, n_topics=8), **kw})


def rows_of(w, b, lo, hi):
    """K and V rows [tokens][Hkv][d] of tokens lo..hi-1 of request b."""
    S = w.cfg.page_size
    base = int(w.page_base[b])
    pos = torch.arange(lo, hi, device=w.kv_pool.device)
    kv = w.kv_pool[base + pos // S, :, :, pos % S]              # [n][Hkv][2][d]
    return kv[:, :, 0], kv[:, :, 1]


def test_drafted_rounds_rebuild_the_context_they_were_cut_from():
    """A context is cut short, then grown back by rounds of drafting: a tree whose accepted path is what was cut, attended over the
    selected pages, its path appended; the rest as a prompt.  Pool, summaries, lengths and the next step are then those of the
    whole context, bit for bit."""
    cfg = small()
    whole = W.generate(cfg, seed=5, device=DEV)
    ref = Session(whole)
    ref.step()
    torch.cuda.synchronize()
    cut = W.generate(cfg, seed=5, device=DEV)
    lens = cut.ctx_len.tolist()
    short = [lens[0] - 37, lens[1] - 1, lens[2] - 20]
    for b, n in enumerate(short):                               # what is cut is gone
        S, base = cfg.page_size, int(cut.page_base[b])
        pos = torch.arange(n, lens[b], device=DEV)
        cut.kv_pool[base + pos // S, :, :, pos % S] = float("nan")
    cut.ctx_len.copy_(dev(short))
    s = Session(cut)
    rng = np.random.default_rng(1)
    T, path_len = 9, 4
    gen = torch.Generator(device=DEV).manual_seed(2)
    for _ in range(12):
        left = [lens[b] - int(cut.ctx_len[b]) for b in range(3)]
        if max(left) == 0:
            break
        n_acc = [min(x, int(rng.integers(1, path_len + 1))) for x in left]
        q = torch.randn((3, T, cfg.n_q_heads, 128), generator=gen, device=DEV).to(torch.bfloat16)
        k, v = (torch.randn((3, T, cfg.n_kv_heads, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
        path = np.full((3, path_len), -1)
        sees = np.zeros((3, T, T), dtype=bool)
        for b in range(3):
            at = np.sort(rng.permutation(T)[: n_acc[b]])
            path[b, : n_acc[b]] = at
            if n_acc[b]:
                n0 = int(cut.ctx_len[b])
                k[b, at], v[b, at] = rows_of(whole, b, n0, n0 + n_acc[b])
            for t in range(T):
                sees[b, t, t] = True
                before = [x for x in at if x < t]
                if t in at and before:
                    sees[b, t] |= sees[b, before[-1]]
        bits = (sees.astype(np.uint64) << np.arange(T, dtype=np.uint64)).sum(-1).astype(np.uint32)
        mask = torch.from_numpy(bits.view(np.int32)[..., None].copy()).to(DEV)
        nd = dev([T, T - 1, T])
        s.select()
        out, lse = s.tree_attn(q, k, v, nd, mask, selected=True)
        # the attention itself, for one request and a head, against the formula
        b, h = 0, 5
        n0, S, kvh = int(cut.ctx_len[b]), cfg.page_size, 5 // cfg.group
        pages = s.o.sel[b, h, : int(s.o.n_sel[b, h])].long()
        pos = (pages[:, None] * S + torch.arange(S, device=DEV)).view(-1)
        pos = pos[pos < n0]
        kv = cut.kv_pool[int(cut.page_base[b]) + pos // S, kvh, :, pos % S].double()
        K, V = torch.cat([kv[:, 0], k[b, :, kvh].double()]), torch.cat([kv[:, 1], v[b, :, kvh].double()])
        x = q[b, :, h].double() @ K.T / math.sqrt(128)
        x[:, len(pos):][~torch.from_numpy(sees[b]).to(DEV)] = -math.inf
        w = torch.softmax(x, -1)
        want, W_ = w @ V, w @ V.abs()
        # half a step of bf16 for the weights and for the result (2^-8 each), and 2^-9 for all that is done in fp32
        tol = 2.0 ** -8 * (W_ + want.abs()) * 1.01 + 2.0 ** -9 * W_
        assert bool(((out[b, :, h].double() - want).abs() <= tol).all())
        assert (lse[b, :, h].double() - torch.logsumexp(x, -1)).abs().max().item() < 1e-3
        s.append(k, v, dev(n_acc), dev(path))
    left = [lens[b] - int(cut.ctx_len[b]) for b in range(3)]
    if max(left):                                               # the rest as a prompt
        n = max(left)
        k, v = (torch.zeros((3, n, cfg.n_kv_heads, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        for b, m in enumerate(left):
            if m:
                k[b, :m], v[b, :m] = rows_of(whole, b, lens[b] - m, lens[b])
        s.append(k, v, dev(left))
    assert cut.ctx_len.tolist() == lens
    for b in range(3):
        for a, c in zip(rows_of(whole, b, 0, lens[b]), rows_of(cut, b, 0, lens[b])):
            assert same(a.contiguous(), c.contiguous())
    assert torch.equal(s.ksum.float(), ref.ksum.float())
    s.step()
    torch.cuda.synchronize()
    for f in ("sel", "n_sel", "out", "lse", "queue_load"):
        assert torch.equal(getattr(s.o, f), getattr(ref.o, f)), f
    assert s.status() == 0 and ref.status() == 0
    s.close()
    ref.close()


def test_single_token_tree_is_the_step_over_all_pages():
    """With as many places as pages every page is selected: the step's attention and a tree of one token that sees only the
    context are the same sum, up to the rounding of the weights and of the result to bf16 (2^-8 each)."""
    cfg = small(ctx_len=16 * 40 + 3, top_k=64)
    w = W.generate(cfg, seed=9, device=DEV)
    s = Session(w)
    s.step()
    zero = torch.zeros((3, 1, cfg.n_kv_heads, 128), dtype=torch.bfloat16, device=DEV)
    mask = torch.zeros((3, 1, 1), dtype=torch.int32, device=DEV)
    for selected in (False, True):
        out, lse = s.tree_attn(w.q[:, None], zero, zero, dev([1, 1, 1]), mask, selected=selected)
        torch.cuda.synchronize()
        vmax = w.kv_pool[:, :, 1].abs().max().item()
        assert (out[:, 0].float() - s.o.out).abs().max().item() <= 2.0 ** -8 * 2 * vmax
        assert (lse[:, 0] - s.o.lse).abs().max().item() <= 1e-4
    s.close()


def test_beams_are_selected_forked_and_attended():
    """Two prompts of three beams: the selection's parents go into the plan, the moves into a second pool; every beam then attends
    exactly what its parent attended."""
    batch, beams, hkv, S = 6, 3, 2, 16
    gen = torch.Generator(device=DEV).manual_seed(3)
    lens, pages = [100] * 3 + [333] * 3, [8] * 3 + [22] * 3
    base = np.concatenate([[0], np.cumsum(pages)])
    n_pool = int(base[-1]) + 4
    pool = torch.randn((n_pool, hkv, 2, S, 128), generator=gen, device=DEV).to(torch.bfloat16)
    other = torch.full_like(pool, float("nan"))
    shape, ctx, ws = handle(batch, hkv, S, n_pool, max(pages))
    logits = torch.randn((2, beams, 777), generator=gen, device=DEV) * 3
    score = torch.tensor([[-1.0, -0.5, -2.0], [-0.1, -9.0, -0.2]], device=DEV)
    new, parent, token = torch.empty((2, beams), device=DEV), *(torch.empty((2, beams), dtype=torch.int32, device=DEV) for _ in range(2))
    bws = torch.empty(B.swarm_beam_select_workspace_bytes(2, beams, 777, beams), dtype=torch.uint8, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    src, dst, n_moves, new_len = torch.empty(n_pool, **i32), torch.empty(n_pool, **i32), torch.empty(1, **i32), torch.empty(batch, **i32)
    page_base, new_base, ctx_len = dev(base, torch.int64), torch.empty(batch + 1, dtype=torch.int64, device=DEV), dev(lens)
    mws = torch.empty(B.swarm_move_pages_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    B.swarm_beam_select(logits, score, bws, new, parent, token)
    plan = B.make_page_plan(page_base=page_base, ctx_len=ctx_len, parent=parent.view(-1), new_page_base=new_base, new_ctx_len=new_len,
                            src=src, dst=dst, n_moves=n_moves)
    B.swarm_plan_pages(ctx, plan)
    B.swarm_move_pages(ctx, B.make_page_moves(src=src, dst=dst, n_moves=n_moves, from_pool=pool, to_pool=other), mws)
    q = torch.randn((batch, 1, hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
    kv = torch.randn((2, batch, 1, hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
    tws = torch.empty(B.swarm_tree_attn_workspace_bytes(shape, 1), dtype=torch.uint8, device=DEV)
    outs = []
    up = parent.view(-1).long()
    assert sorted(set((up // 3).tolist())) == [0, 1] and up[:3].max() < 3 and up[3:].min() >= 3
    for p, pb, cl, qq, kk, vv in ((pool, page_base, ctx_len, q[up], kv[0][up], kv[1][up]), (other, new_base, new_len, q[up], kv[0][up], kv[1][up])):
        # the first run attends the parents where they were: request j's pages are those of parent j
        if p is pool:
            starts = torch.stack([page_base[up], page_base[up + 1]], 1)
            out = torch.empty((batch, 1, hkv, 128), dtype=torch.bfloat16, device=DEV)
            lse = torch.empty((batch, 1, hkv), device=DEV)
            for j in range(batch):                              # one request at a time, in its parent's place
                one_shape, one, one_ws = handle(1, hkv, S, n_pool, max(pages))
                held = [x[j: j + 1].contiguous() for x in (qq, kk, vv)] + [dev([1])]
                t1 = B.make_tree(q=held[0], k=held[1], v=held[2], n_draft=held[3])
                o1, l1 = torch.empty((1, 1, hkv, 128), dtype=torch.bfloat16, device=DEV), torch.empty((1, 1, hkv), device=DEV)
                pb1, cl1 = starts[j].contiguous(), cl[up[j]: up[j] + 1].clone()
                B.swarm_tree_attn(one, B.make_inputs(kv_pool=p, page_base=pb1, ctx_len=cl1), t1, None, None, tws, o1, l1)
                torch.cuda.synchronize()
                out[j], lse[j] = o1[0], l1[0]
                close(one)
        else:
            out = torch.empty((batch, 1, hkv, 128), dtype=torch.bfloat16, device=DEV)
            lse = torch.empty((batch, 1, hkv), device=DEV)
            held = [x.contiguous() for x in (qq, kk, vv)] + [dev([1] * batch)]
            tree = B.make_tree(q=held[0], k=held[1], v=held[2], n_draft=held[3])
            B.swarm_tree_attn(ctx, B.make_inputs(kv_pool=p, page_base=pb, ctx_len=cl), tree, None, None, tws, out, lse)
        outs.append((out.float(), lse))
    torch.cuda.synchronize()
    # the same tokens, cut differently over the CTAs: fp32 sums in another order, then a rounding to bf16 (2^-8 of the value)
    assert bool(((outs[0][0] - outs[1][0]).abs() <= 2.0 ** -7 * outs[0][0].abs() + 1e-3).all())
    assert (outs[0][1] - outs[1][1]).abs().max().item() < 1e-4
    assert B.swarm_device_status(ctx) == 0
    close(ctx)


def test_compaction_keeps_the_step():
    """A request is freed and the others moved together: their selection and attention stay what they were."""
    cfg = small(batch=4)
    w = W.generate(cfg, seed=6, device=DEV)
    s = Session(w)
    s.step()
    torch.cuda.synchronize()
    before = [x.clone() for x in (s.o.sel, s.o.out, s.o.lse)]
    base = w.page_base.tolist()
    s.compact(dev([-1, 0, 2, 3]), reserve=dev([1, 0, 2, 0]))
    assert s.status() == 0
    n = [base[1] - base[0], base[3] - base[2], base[4] - base[3]]
    assert w.page_base.tolist() == [0, 1, 1 + n[0], 3 + n[0] + n[1], 3 + sum(n)] and w.ctx_len.tolist()[0] == 0
    w.ctx_len[0] = 1                                            # (a step wants a token in every request)
    w.kv_pool[0] = 0
    s.ksum[0] = 0
    s.set_query(w.q[[0, 0, 2, 3]].contiguous())
    s.select()
    s.sparse_attn_paged()
    torch.cuda.synchronize()
    for got, was in zip((s.o.sel, s.o.out, s.o.lse), before):
        for new, old in ((1, 0), (2, 2), (3, 3)):
            assert torch.equal(got[new], was[old])
    s.compact(dev([3, 2, 1, 0]))                                # refused: not in order
    assert s.status() == B.DEV_BAD_PAGE and w.page_base.tolist()[-1] == 3 + sum(n)
    s.close()


def test_a_captured_round_replays():
    """Attention, commit, plan and moves, and a beam selection in one CUDA graph, replayed: each replay equals the calls by themselves."""
    c = Case(lens=[70, 300], T=6, n_draft=[6, 4], hq=8, hkv=2, S=16, seed=4, spare=3)
    n_pool = c.pool.shape[0]
    i32 = dict(dtype=torch.int32, device=DEV)
    new_len = torch.zeros(4, **i32)
    pool = torch.where(torch.isnan(c.pool), torch.zeros_like(c.pool), c.pool)
    ksum = torch.zeros((n_pool, 2, 2, 128), dtype=torch.bfloat16, device=DEV)
    B.swarm_build_summaries(c.ctx, B.make_inputs(kv_pool=pool, page_base=c.page_base, ctx_len=c.ctx_len), ksum)
    n_new, path = dev([2, 3]), dev([[0, 4, -1], [1, 2, 3]])
    tokens = B.make_new_tokens(k=c.k, v=c.v, n_new=n_new, path=path)
    t = dict(src=torch.zeros(n_pool, **i32), dst=torch.zeros(n_pool, **i32), n_moves=torch.zeros(4, **i32))
    nb, nl = torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(4, **i32)
    parent, reserve = dev([1, 0]), dev([1, 1])
    plan = B.make_page_plan(page_base=c.page_base, ctx_len=new_len[:2], parent=parent, reserve=reserve, new_page_base=nb,
                            new_ctx_len=nl[:2], src=t["src"], dst=t["dst"], n_moves=t["n_moves"])
    second = torch.zeros_like(pool)
    moves = B.make_page_moves(src=t["src"], dst=t["dst"], n_moves=t["n_moves"], from_pool=pool, to_pool=second)
    mws = torch.empty(B.swarm_move_pages_workspace_bytes(c.shape), dtype=torch.uint8, device=DEV)
    logits, score = torch.randn((1, 2, 900), device=DEV), torch.zeros((1, 2), device=DEV)
    bws = torch.empty(B.swarm_beam_select_workspace_bytes(1, 2, 900, 4), dtype=torch.uint8, device=DEV)
    beam = torch.empty((1, 4), device=DEV), torch.empty((1, 4), **i32), torch.empty((1, 4), **i32)
    inputs = B.make_inputs(kv_pool=pool, page_base=c.page_base, ctx_len=c.ctx_len)

    def once():
        B.swarm_tree_attn(c.ctx, inputs, c.tree, None, None, c.ws, c.out, c.lse)
        B.swarm_append_tokens(c.ctx, inputs, tokens, pool, ksum, new_len)
        B.swarm_plan_pages(c.ctx, plan)
        B.swarm_move_pages(c.ctx, moves, mws)
        B.swarm_beam_select(logits, score, bws, *beam)

    results = (c.out, c.lse, pool, ksum, new_len, nb, nl, second, *beam)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        once()
        st.synchronize()
        c.check()
        want = [x.clone() for x in results]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            once()
            once()
        for x in (c.out, c.lse):
            x.fill_(7.0)
        for x in (new_len, nb, nl, second, *beam):
            x.zero_()
        for _ in range(3):
            g.replay()
        st.synchronize()
    for x, y in zip(results, want):
        assert same(x, y)
    assert B.swarm_device_status(c.ctx) == 0
    c.close()


def test_two_streams_with_workspaces_of_their_own():
    """Two contexts, two streams, no order between them."""
    a = Case(lens=[900, 40, 0, 333], T=20, n_draft=[20, 3, 20, 11], hq=8, hkv=2, S=16, seed=11)
    b = Case(lens=[2000], T=70, n_draft=[66], hq=8, hkv=2, S=32, seed=12)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        a.run(sa)
        b.run(sb)
    torch.cuda.synchronize()
    a.check()
    b.check()
    a.close()
    b.close()


def test_calls_back_to_back_on_one_workspace():
    """Each call's kernels follow the last one's on the stream: nothing of one is left in the next."""
    c = Case(lens=[500, 77], T=12, n_draft=[12, 5], hq=16, hkv=2, S=16, seed=21)
    for _ in range(30):
        c.run()
    c.check()
    c.nd.copy_(dev([3, 0]))
    c.n_draft = [3, 0]
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.run()
    c.check()
    c.close()


def test_pools_beyond_32_bit_offsets():
    """A request at the end of a pool of 12 GB: attended, appended to, moved."""
    hkv, S, n_pool = 8, 16, 196608                              # 64 KB a page
    pool = torch.empty((n_pool, hkv, 2, S, 128), dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    first, n_pages, length = n_pool - 13, 11, 150
    pool[first:] = torch.randn((13, hkv, 2, S, 128), generator=gen, device=DEV).to(torch.bfloat16)
    shape, ctx, ws = handle(1, hkv, S, n_pool, n_pages)
    page_base, ctx_len = dev([first, first + n_pages], torch.int64), dev([length])
    inputs = B.make_inputs(kv_pool=pool, page_base=page_base, ctx_len=ctx_len)
    q = torch.randn((1, 2, hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn((1, 2, hkv, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty((1, 2, hkv), device=DEV)
    tws = torch.empty(B.swarm_tree_attn_workspace_bytes(shape, 2), dtype=torch.uint8, device=DEV)
    two = dev([2])
    B.swarm_tree_attn(ctx, inputs, B.make_tree(q=q, k=k, v=v, n_draft=two), None, None, tws, out, lse)
    for h in range(hkv):
        kv = pool[first: first + n_pages, h].transpose(1, 2).reshape(-1, 2, 128)[:length].double()
        K, V = torch.cat([kv[:, 0], k[0, :, h].double()]), torch.cat([kv[:, 1], v[0, :, h].double()])
        x = q[0, :, h].double() @ K.T / math.sqrt(128)
        x[0, -1] = -math.inf
        w = torch.softmax(x, -1)
        tol = 2.0 ** -8 * (w @ V.abs() + (w @ V).abs()) * 1.01 + 2.0 ** -9 * (w @ V.abs())
        assert bool(((out[0, :, h].double() - w @ V).abs() <= tol).all())
    new_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = pool[first:].clone()
    for i in range(2):
        p, slot = (length + i) // S, (length + i) % S
        want[p, :, 0, slot], want[p, :, 1, slot] = k[0, i], v[0, i]
    B.swarm_append_tokens(ctx, inputs, B.make_new_tokens(k=k, v=v, n_new=two), pool, None, new_len)
    torch.cuda.synchronize()
    assert same(pool[first:], want) and new_len.tolist() == [length + 2]
    mws = torch.empty(B.swarm_move_pages_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    src, dst = dev([first, first + 1]), dev([0, n_pool - 1])
    B.swarm_move_pages(ctx, B.make_page_moves(src=src, dst=dst, n_moves=two, from_pool=pool, to_pool=pool), mws)
    torch.cuda.synchronize()
    assert same(pool[0], want[0]) and same(pool[-1], want[1])
    assert B.swarm_device_status(ctx) == 0
    close(ctx)


@pytest.mark.parametrize("hq,hkv,T", [(128, 1, 3), (100, 1, 2), (65, 1, 4), (33, 33, 5)])
def test_wide_head_groups(hq, hkv, T):
    c = Case(lens=[200, 31], T=T, n_draft=[T, 1], hq=hq, hkv=hkv, S=16, seed=hq)
    c.run()
    c.check()
    c.close()


def test_lengths_that_do_not_fit_are_reported_and_left_alone():
    c = Case(lens=[100, 50, 30], T=4, n_draft=[4, 4, 4], hq=8, hkv=2, S=16, seed=2, spare=0)
    c.ctx_len.copy_(dev([100, 50 + 16 * 3, -2]))                # requests 1 and 2 do not fit
    c.nd.copy_(dev([9, 4, 4]))                                  # more than there are: clamped
    c.run()
    torch.cuda.synchronize()
    assert B.swarm_device_status(c.ctx) == B.DEV_BAD_LENGTH
    assert bool((c.out[1:] == 7.0).all()) and bool((c.lse[1:] == 7.0).all())
    c.n_draft, c.batch = [4], 1
    c.check()
    c.ctx_len.copy_(dev([100, 50, 30]))
    c.nd.copy_(dev([-1, 4, 4]))
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.run()
    assert B.swarm_device_status(c.ctx) == B.DEV_BAD_LENGTH
    c.n_draft, c.batch = [0, 4, 4], 3
    c.check()
    c.close()


def test_selections_with_bad_and_repeated_pages():
    c = Case(lens=[300, 100], T=3, n_draft=[3, 3], hq=4, hkv=2, S=16, seed=3, top_k=8)
    c.sel[0, 1, :3] = dev([5, 5, 5])                            # the same page again: counts once
    good = c.sel.clone()
    c.run()
    c.check()
    assert B.swarm_device_status(c.ctx) == 0
    c.sel[0, 0, 2] = 19                                         # behind the request's last page
    c.sel[1, 3, 0] = -4
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    c.run()
    assert B.swarm_device_status(c.ctx) == B.DEV_BAD_PAGE
    c.sel = good                                                # what is left: the list without those places
    sel, n = c.sel.clone(), c.n_sel.clone()
    keep = [x for i, x in enumerate(sel[0, 0, : int(n[0, 0])].tolist()) if i != 2]
    c.sel[0, 0, : len(keep)] = dev(keep)
    c.n_sel[0, 0] = len(keep)
    keep = sel[1, 3, 1: int(n[1, 3])].tolist()
    c.sel[1, 3, : len(keep)] = dev(keep)
    c.n_sel[1, 3] = len(keep)
    c.check()
    c.close()


def test_arguments_are_checked():
    c = Case(lens=[20], T=2, n_draft=[2], hq=4, hkv=2, S=16, seed=1)
    with pytest.raises(ValueError):
        B.make_tree(q=c.q, k=c.k, v=c.v.float(), n_draft=c.nd)
    with pytest.raises(ValueError):
        B.make_tree(q=c.q, k=c.k, v=c.v, n_draft=c.nd, mask=torch.zeros((1, 2, 2), dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        B.make_tree(q=c.q.transpose(1, 2), k=c.k, v=c.v, n_draft=c.nd)
    with pytest.raises(ValueError):
        B.swarm_tree_attn(c.ctx, c.inputs, c.tree, None, None, c.ws, c.out.float(), c.lse)
    for kw, code in ((dict(ws=c.ws[:256]), B.ERR_WORKSPACE_TOO_SMALL), (dict(sel=dev([0])), B.ERR_INVALID_ARG),
                     (dict(ws=c.ws_all[16:]), B.ERR_INVALID_ARG)):
        with pytest.raises(B.SwarmError) as e:
            B.swarm_tree_attn(c.ctx, c.inputs, c.tree, kw.get("sel"), None, kw.get("ws", c.ws), c.out, c.lse)
        assert e.value.code == code, kw
    bad = B.make_inputs(page_base=c.page_base, ctx_len=c.ctx_len)
    with pytest.raises(B.SwarmError) as e:
        B.swarm_tree_attn(c.ctx, bad, c.tree, None, None, c.ws, c.out, c.lse)
    assert e.value.code == B.ERR_INVALID_ARG
    tokens = B.make_new_tokens(k=c.k, v=c.v, n_new=c.nd)
    tokens.max_path = 3                                         # a path that is not there
    with pytest.raises(B.SwarmError) as e:
        B.swarm_append_tokens(c.ctx, c.inputs, tokens, c.pool, None, c.nd)
    assert e.value.code == B.ERR_INVALID_ARG
    lay = Layout([16], [1], 8)
    with pytest.raises(B.SwarmError) as e:                      # the new tables may not be the old ones
        lay.plan([0])
        p = B.make_page_plan(page_base=lay.page_base, ctx_len=lay.ctx_len, parent=lay.held[0], new_page_base=lay.page_base,
                             new_ctx_len=lay.new_len, src=lay.src, dst=lay.dst, n_moves=lay.n)
        B.swarm_plan_pages(lay.ctx, p)
    assert e.value.code == B.ERR_INVALID_ARG
    close(lay.ctx)
    c.close()


def test_captured_trees_keep_their_workspace():
    """A graph of short trees, then calls with longer ones, whose workspace is larger: the graph's is still its own."""
    cfg = small()
    w = W.generate(cfg, seed=12, device=DEV)
    s = Session(w)
    gen = torch.Generator(device=DEV).manual_seed(8)

    def drafts(T):
        make = lambda heads: torch.randn((3, T, heads, 128), generator=gen, device=DEV).to(torch.bfloat16)   # noqa: E731
        return make(cfg.n_q_heads), make(cfg.n_kv_heads), make(cfg.n_kv_heads), dev([T] * 3)

    few, many = drafts(2), drafts(40)
    want = s.tree_attn(*few)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out, lse = s.tree_attn(*few)
    first = s.tree_attn(*many)
    junk = [torch.full((1 << 20,), -1, dtype=torch.int32, device=DEV) for _ in range(64)]
    kept = [x.clone() for x in junk]
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert all(torch.equal(a, b) for a, b in zip(junk, kept))
    again = s.tree_attn(*many)
    torch.cuda.synchronize()
    assert torch.equal(first[0], again[0]) and s.status() == 0
    s.close()


def test_clusters_move_with_their_requests():
    """After a compaction the cluster tables are those of the requests that are left, and a resolution gives what it gave."""
    cfg = small(batch=4, ctx_len=16 * 90 + 5)
    w = W.generate(cfg, seed=31, device=DEV)
    left = W.generate(cfg, seed=31, device=DEV)
    s = Session(w)
    tables = [x.clone() for x in (w.cluster_base, w.cluster_replica_mask, w.cluster_size, w.page2cluster)]
    s.compact(dev([2, 1, 0, 3]))                                # refused: not in order
    assert s.status() == B.DEV_BAD_PAGE
    s.compact(dev([9, 1, 2, 3]))                                # refused: no such request
    assert s.status() == B.DEV_BAD_PAGE
    for now, was in zip((w.cluster_base, w.cluster_replica_mask, w.cluster_size, w.page2cluster), tables):
        assert torch.equal(now, was)
    s.compact(dev([1, -1, 2, 3]))
    assert s.status() == 0
    old = left.cluster_base.tolist()
    n = [old[b + 1] - old[b] for b in range(4)]
    base = [0, n[1], n[1], n[1] + n[2], n[1] + n[2] + n[3]]
    assert w.cluster_base.tolist() == base
    for j, b in ((0, 1), (2, 2), (3, 3)):
        for now, was in ((w.cluster_replica_mask, left.cluster_replica_mask), (w.cluster_size, left.cluster_size)):
            assert torch.equal(now[base[j]: base[j + 1]], was[old[b]: old[b + 1]])
        lo, hi, P = int(w.page_base[j]), int(left.page_base[b]), int(left.page_base[b + 1] - left.page_base[b])
        assert torch.equal(w.page2cluster[lo: lo + P], left.page2cluster[hi: hi + P])
    # resolution of hand-made selections: of old requests 1, 2, 3 before, of new requests 0, 2, 3 behind
    ref = Session(left)
    sel = torch.randint(0, 90, (4, cfg.n_q_heads, cfg.top_k), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV,
                        dtype=torch.int32)
    count = torch.full((4, cfg.n_q_heads), cfg.top_k, dtype=torch.int32, device=DEV)
    before, behind = count.clone(), count.clone()
    before[0] = 0
    behind[1] = 0
    ref.resolve(sel[[0, 1, 2, 3]].contiguous(), before)
    s.resolve(sel[[1, 0, 2, 3]].contiguous(), behind)
    torch.cuda.synchronize()
    assert s.status() == 0 and ref.status() == 0
    m = int(ref.o.n_uniq[0])
    assert int(s.o.n_uniq[0]) == m

    def routed(o, starts, requests):
        ids = [(r, c - starts[r], q) for c, q in zip(o.uniq[:m].tolist(), o.queue_of[:m].tolist())
               for r in requests if starts[r] <= c < starts[r + 1]]
        return {(requests.index(r), c): q for r, c, q in ids}

    assert set(routed(ref.o, old, [1, 2, 3])) == set(routed(s.o, base, [0, 2, 3]))
    assert sorted(routed(s.o, base, [0, 2, 3])) and torch.equal(ref.o.queue_load.sum(), s.o.queue_load.sum())
    s.close()
    ref.close()


def test_tables_are_not_changed_under_a_reader():
    cfg = small()
    w = W.generate(cfg, seed=13, device=DEV)
    s = Session(w, index_prefetch=True)
    kv = torch.zeros((3, 1, cfg.n_kv_heads, 128), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="index_prefetch"):
        s.append(kv, kv, dev([1, 1, 1]))
    with pytest.raises(ValueError, match="index_prefetch"):
        s.compact(dev([0, 1, 2]))
    s.close()
    # a resolution on a stream of its own is waited for
    tail = torch.cuda.Stream()
    a, b = Session(w), Session(W.generate(cfg, seed=13, device=DEV), tail_stream=tail)
    a.step()
    for _ in range(3):
        b.step()
        b.compact(dev([0, 1, 2]))
    b.tail_join()
    torch.cuda.synchronize()
    for f in ("sel", "out", "queue_load", "n_uniq"):
        assert torch.equal(getattr(a.o, f), getattr(b.o, f)), f
    with pytest.raises(ValueError, match="medoid"):
        a.enable_medoid_index(4)
        a.compact(dev([0, 1, 2]))
    a.close()
    b.close()


def test_counts_that_do_not_fit_are_refused():
    lay = Layout([16], [1], 40, hkv=2)
    src, dst, one = dev([1]), dev([2]), dev([1])
    ws = torch.empty(B.swarm_move_pages_workspace_bytes(lay.shape), dtype=torch.uint8, device=DEV)
    moves = B.make_page_moves(src=src, dst=dst, n_moves=one, from_pool=lay.pool, to_pool=lay.pool)
    for n, code in ((0, B.ERR_INVALID_ARG), ((1 << 31) - 1, B.ERR_UNSUPPORTED), (1 << 30, B.ERR_UNSUPPORTED), ((1 << 30) - 1, B.ERR_UNSUPPORTED)):
        moves.max_moves = n
        with pytest.raises(B.SwarmError) as e:
            B.swarm_move_pages(lay.ctx, moves, ws)
        assert e.value.code == code
    close(lay.ctx)


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16])
@pytest.mark.parametrize("top_k", [0, 4])
def test_the_largest_lengths_do_not_fit(length, top_k):
    """Their pages cannot be counted as (length + S - 1) / S in 32 bits: 2^31 - 16 is the last length that could."""
    c = Case(lens=[100, 50, 30], T=4, n_draft=[4, 4, 4], hq=8, hkv=2, S=16, seed=2, top_k=top_k)
    c.ctx_len.copy_(dev([100, length, 30]))
    c.run()
    torch.cuda.synchronize()
    bits = B.swarm_device_status(c.ctx)                         # (no page of a request without pages can be selected)
    assert bits == (B.DEV_BAD_LENGTH | B.DEV_BAD_PAGE if top_k else B.DEV_BAD_LENGTH)
    assert bool((c.out[1] == 7.0).all()) and bool((c.lse[1] == 7.0).all())
    c.n_draft = [4, 0, 4]                                       # the others are what they would be alone
    c.check()
    c.close()
    lay = Layout([20, 40, 5], [2, 4, 1], 8, hkv=1)
    lay.ctx_len.copy_(dev([20, length, 5]))
    lay.plan([0, 1, 2])
    assert B.swarm_device_status(lay.ctx) == B.DEV_BAD_LENGTH and int(lay.n) == -1
    assert lay.new_base.tolist() == lay.base and lay.new_len.tolist() == [20, length, 5]
    close(lay.ctx)


def test_selections_of_requests_with_more_pages_than_the_ctx_has():
    """Request 0 has 19 pages, in a ctx for 7: nothing can have been selected from it.  Over all pages it is attended all the same."""
    c = Case(lens=[300, 100], T=3, n_draft=[3, 3], hq=4, hkv=2, S=16, seed=3, top_k=5)
    B.swarm_destroy(c.ctx)
    c.shape = B.make_shape(batch=2, n_q_heads=4, n_kv_heads=2, page_size=16, top_k=5, n_queues=1, max_pages_per_req=7,
                           max_clusters_total=1, n_pool_pages=c.pool.shape[0])
    c.ctx = B.swarm_create(c.shape)
    B.swarm_set_workspace(c.ctx, c.ctx_ws)
    c.n_sel[0] = 0
    c.run()
    assert B.swarm_device_status(c.ctx) == B.DEV_BAD_LENGTH
    c.n_draft = [0, 3]
    c.check()
    c.sel = c.n_sel = None
    c.n_draft = [3, 3]
    c.run()
    assert B.swarm_device_status(c.ctx) == 0
    c.check()
    c.close()


@pytest.mark.parametrize("S", [16, 32])
def test_a_request_grows_past_its_configured_length(S):
    """Pages of one request are dropped, another gets them as spare ones and grows past the longest context that the workload began
    with: its steps and its trees are then those of a new session over the same tokens.  Without room in the session it stays as
    it was."""
    cfg = small(batch=2, ctx_len=S * 60 + 7, page_size=S)
    P = cfg.max_pages()
    gen = torch.Generator(device=DEV).manual_seed(3)
    T, more = 5 * S, [4 * S + 3, S // 2]
    k, v = (torch.randn((2, T, cfg.n_kv_heads, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    t = 6
    drafts = [torch.randn((2, t, h, 128), generator=gen, device=DEV).to(torch.bfloat16) for h in (cfg.n_q_heads, cfg.n_kv_heads, cfg.n_kv_heads)]
    for room in (None, P + 6):
        w = W.generate(cfg, seed=41, device=DEV)
        lens, base = w.ctx_len.tolist(), w.page_base.tolist()
        keep = torch.ones(w.n_pool_pages, dtype=torch.uint8, device=DEV)
        keep[base[1]: base[1] + 6] = 0
        s = Session(w, max_pages_per_req=room)
        s.compact(dev([0, 1]), reserve=dev([6, 0]), keep=keep)
        assert s.status() == 0
        at = int(w.page_base[0]) + P
        w.page2cluster[at: at + 6] = 0
        s.append(k, v, dev(more))
        if room is None:                                        # request 1 has lost pages, and grows inside its last one
            assert s.status() == B.DEV_BAD_LENGTH
            assert w.ctx_len.tolist() == [lens[0], lens[1] - 6 * S + more[1]]
            s.close()
            continue
        assert s.status() == 0 and w.ctx_len.tolist() == [lens[0] + more[0], lens[1] - 6 * S + more[1]]
        kept = rows_of(w, 0, lens[0], lens[0] + more[0])
        assert same(kept[0], k[0, : more[0]]) and same(kept[1], v[0, : more[0]])
        fresh = Session(w, max_pages_per_req=room)
        for x in (s, fresh):
            x.step()
        torch.cuda.synchronize()
        last = -(-(lens[0] + more[0]) // S) - 1
        assert int(s.o.n_sel[0].min()) == cfg.top_k and last >= P
        for f in ("sel", "n_sel", "out", "lse", "n_uniq", "queue_load"):
            assert same(getattr(s.o, f), getattr(fresh.o, f)), f
        for selected in (True, False):
            got, want = (x.tree_attn(*drafts, dev([t, t]), selected=selected) for x in (s, fresh))
            assert same(got[0], want[0]) and same(got[1], want[1])
        # the pages beyond the first length are attended: a query that points at the last one finds it
        q = w.q.clone()
        q[0] = (kept[0][-1].float() * 4).repeat_interleave(cfg.n_q_heads // cfg.n_kv_heads, 0).to(torch.bfloat16)
        s.set_query(q)
        s.select()
        assert bool((s.o.sel[0] == last).any(-1).all())
        assert s.status() == 0 and fresh.status() == 0
        s.close()
        fresh.close()


@pytest.mark.parametrize("in_stream", [False, True])
def test_the_medoid_index_follows_an_append(in_stream):
    """The index copies the summaries of the medoids' pages: one that gains tokens bounds them too, and the medoid step is that of a
    new session over the same tokens.  Here the medoid of the last page's cluster is that page."""
    cfg = small(ctx_len=16 * 60 + 3, top_k=24)
    w = W.generate(cfg, seed=14, device=DEV)
    s = Session(w)
    s.enable_medoid_index(4, keep_scores=True)
    lens, base, cbase = w.ctx_len.tolist(), w.page_base.tolist(), w.cluster_base.tolist()
    rows = []
    for b in range(3):
        last = -(-lens[b] // 16) - 1
        rows.append(cbase[b] + int(w.page2cluster[base[b] + last]))
        s.medoid_page[rows[-1]] = last
    B.swarm_build_medoid_index(s.ctx, s.inputs, s.medoid_page, s.medoid_ksum, s.cluster_ctx_len)
    before = s.medoid_ksum.clone()
    gen = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn((3, 5, cfg.n_kv_heads, 128), generator=gen, device=DEV).to(torch.bfloat16) * 8 for _ in range(2))
    more = [min(5, 16 - lens[b] % 16) if lens[b] % 16 else 0 for b in range(3)]
    assert max(more) > 0
    n_new = dev(more)
    stream = torch.cuda.Stream() if in_stream else None
    torch.cuda.synchronize()
    s.append(k, v, n_new, stream=stream)
    torch.cuda.synchronize()
    fresh = Session(w)
    fresh.enable_medoid_index(4, keep_scores=True)
    fresh.medoid_page.copy_(s.medoid_page)
    B.swarm_build_medoid_index(fresh.ctx, fresh.inputs, fresh.medoid_page, fresh.medoid_ksum, fresh.cluster_ctx_len)
    for x in (s, fresh):
        x.step_medoid()
    torch.cuda.synchronize()
    assert same(s.medoid_ksum, fresh.medoid_ksum) and torch.equal(s.cluster_ctx_len[:3], fresh.cluster_ctx_len[:3])
    for b in range(3):                                          # (the large new keys widen the bounds)
        assert same(s.medoid_ksum[rows[b]], before[rows[b]]) == (more[b] == 0)
    for a, b in ((s.cluster_scores, fresh.cluster_scores), (s.sel_clusters, fresh.sel_clusters), (s.o.out, fresh.o.out), (s.o.lse, fresh.o.lse)):
        assert same(a, b)
    assert s.status() == 0 and fresh.status() == 0
    s.close()
    fresh.close()


def test_nothing_is_compacted_under_a_cache_state():
    """Its arrays are indexed by global cluster ids, which a compaction changes."""
    cfg = small(ctx_len=16 * 60 + 7)
    w = W.generate(cfg, seed=15, device=DEV)
    s = Session(w)
    n = w.n_clusters + 16
    resident, freq = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    B.swarm_set_cache(s.ctx, resident=resident, freq=freq)
    tables = [x.clone() for x in (w.kv_pool, w.page_base, w.ctx_len, w.cluster_base, w.page2cluster)]
    with pytest.raises(ValueError, match="cache state"):
        s.compact(dev([1, -1, 2]))
    assert s.status() == 0
    assert all(same(a, b) for a, b in zip((w.kv_pool, w.page_base, w.ctx_len, w.cluster_base, w.page2cluster), tables))
    B.swarm_set_cache(s.ctx)
    s.compact(dev([1, -1, 2]))
    assert s.status() == 0 and w.ctx_len.tolist()[1] == 0
    s.close()


def refused(call, match):
    with pytest.raises(ValueError, match=match):
        call()


def test_tensors_that_are_too_small_or_of_another_type_are_refused():
    """What the kernels would read or write past the end of: refused by the binding, nothing is launched."""
    c = Case(lens=[60, 40], T=2, n_draft=[2, 2], hq=4, hkv=2, S=16, seed=1, top_k=3)

    def tree(tree=c.tree, sel=c.sel, n_sel=c.n_sel, out=c.out, lse=c.lse):
        B.swarm_tree_attn(c.ctx, c.inputs, tree, sel, n_sel, c.ws, out, lse)

    for kw, match in ((dict(out=c.out[:1]), "out"), (dict(out=c.out.float()), "out"), (dict(lse=c.lse[:, :1].contiguous()), "lse"),
                      (dict(lse=c.lse.half()), "lse"), (dict(sel=c.sel[..., :2].contiguous()), "sel"), (dict(sel=c.sel.long()), "sel"),
                      (dict(n_sel=c.n_sel[:1]), "n_sel"), (dict(n_sel=c.n_sel.long()), "n_sel")):
        refused(lambda: tree(**kw), match)
    for call in (lambda: tree(out=None), lambda: tree(lse=None), lambda: B.swarm_append_tokens(
            c.ctx, c.inputs, B.make_new_tokens(k=c.k, v=c.v, n_new=c.nd), None, None, c.nd.clone())):
        with pytest.raises(B.SwarmError) as e:                  # what is not there is the library's to refuse
            call()
        assert e.value.code == B.ERR_INVALID_ARG
    one = [x[:1].contiguous() for x in (c.q, c.k, c.v, c.nd)]   # drafts of fewer requests, of fewer heads
    refused(lambda: tree(tree=B.make_tree(q=one[0], k=one[1], v=one[2], n_draft=one[3])), "made for")
    few = [x[:, :, :1].contiguous() for x in (c.q, c.k, c.v)]
    refused(lambda: tree(tree=B.make_tree(q=few[0], k=c.k, v=c.v, n_draft=c.nd)), "made for")
    refused(lambda: tree(tree=B.make_tree(q=c.q, k=few[1], v=few[2], n_draft=c.nd)), "made for")

    tokens = B.make_new_tokens(k=c.k, v=c.v, n_new=c.nd)
    ksum = torch.zeros((c.pool.shape[0], 2, 2, 128), dtype=torch.bfloat16, device=DEV)
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)

    def append(tokens=tokens, pool=c.pool, ksum=ksum, lens=lens):
        B.swarm_append_tokens(c.ctx, c.inputs, tokens, pool, ksum, lens)

    for kw, match in ((dict(pool=c.pool[1:]), "kv_pool"), (dict(pool=c.pool.float()), "kv_pool"), (dict(ksum=ksum[1:]), "ksum"),
                      (dict(ksum=ksum.float()), "ksum"), (dict(lens=lens[:1]), "ctx_len_out"), (dict(lens=lens.long()), "ctx_len_out"),
                      (dict(tokens=B.make_new_tokens(k=one[1], v=one[2], n_new=one[3])), "made for"),
                      (dict(tokens=B.make_new_tokens(k=few[1], v=few[2], n_new=c.nd)), "made for")):
        refused(lambda: append(**kw), match)
    c.pool.nan_to_num_(0)
    before = c.pool.clone()
    tree()
    B.swarm_tree_attn(ctypes.c_void_p(c.ctx.value), c.inputs, c.tree, c.sel, c.n_sel, c.ws, c.out, c.lse)   # (a bare handle will do)
    torch.cuda.synchronize()
    assert B.swarm_device_status(c.ctx) == 0 and torch.equal(c.pool, before) and not bool(lens.any()) and not bool(ksum.any())
    c.close()

    lay = Layout([20, 40], [2, 4], 8)
    n, keep = dev([0]), torch.ones(8, dtype=torch.uint8, device=DEV)
    t = dict(page_base=lay.page_base, ctx_len=lay.ctx_len, parent=dev([0, 1]), new_page_base=torch.zeros_like(lay.page_base),
             new_ctx_len=torch.zeros_like(lay.ctx_len), src=torch.zeros(8, dtype=torch.int32, device=DEV),
             dst=torch.zeros(8, dtype=torch.int32, device=DEV), n_moves=n)
    refused(lambda: B.make_page_plan(**{**t, "n_moves": n.long()}), "n_moves")
    refused(lambda: B.make_page_plan(**{**t, "n_moves": n[:0]}), "n_moves")
    refused(lambda: B.swarm_plan_pages(lay.ctx, B.make_page_plan(**t, keep=keep[:7])), "keep")
    less = {**t, "parent": dev([0]), "page_base": lay.page_base[:2], "ctx_len": lay.ctx_len[:1], "new_page_base": t["new_page_base"][:2],
            "new_ctx_len": t["new_ctx_len"][:1]}
    refused(lambda: B.swarm_plan_pages(lay.ctx, B.make_page_plan(**less)), "made for")
    pairs = dict(src=t["src"], dst=t["dst"], n_moves=n)
    refused(lambda: B.make_page_moves(**{**pairs, "n_moves": n.long()}, from_pool=lay.pool, to_pool=lay.pool), "n_moves")
    refused(lambda: B.make_page_moves(**pairs, from_pool=lay.pool.view(torch.int16), to_pool=lay.pool.view(torch.int16)), "from_pool")
    wide = lay.p2c.long()
    for kw, match in ((dict(from_pool=lay.pool[1:], to_pool=lay.pool[1:]), "pool"),
                      (dict(from_pool=lay.pool, to_pool=lay.pool, from_ksum=lay.ksum[1:], to_ksum=lay.ksum[1:]), "ksum"),
                      (dict(from_pool=lay.pool, to_pool=lay.pool, from_page2cluster=lay.p2c[:4], to_page2cluster=lay.p2c[:4]), "page2cluster"),
                      (dict(from_pool=lay.pool, to_pool=lay.pool, from_page2cluster=wide, to_page2cluster=wide), "page2cluster")):
        refused(lambda: B.swarm_move_pages(lay.ctx, B.make_page_moves(**pairs, **kw), lay.ws), match)
    assert B.swarm_device_status(lay.ctx) == 0
    close(lay.ctx)
