"""swarm_append_tokens, swarm_plan_pages and swarm_move_pages: copies, compared bit for bit."""
import numpy as np
import pytest
import torch

from paper_2603_17803_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128


def handle(batch, hkv, S, n_pool, max_pages):
    shape = B.make_shape(batch=batch, n_q_heads=hkv, n_kv_heads=hkv, page_size=S, top_k=1, n_queues=1,
                         max_pages_per_req=max(1, max_pages), max_clusters_total=1, n_pool_pages=n_pool)
    ctx = B.swarm_create(shape)
    ws = torch.empty(B.swarm_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    B.swarm_set_workspace(ctx, ws)
    return shape, ctx, ws


def close(ctx):
    torch.cuda.synchronize()
    damaged = B.swarm_check_workspace(ctx)
    B.swarm_destroy(ctx)
    assert damaged == 0


def dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dtype).to(DEV)


def same(a, b):
    """Bit for bit, whatever the values mean."""
    kind = torch.int16 if a.dtype == torch.bfloat16 else a.dtype
    return torch.equal(a.view(kind), b.view(kind))


# ---- append ------------------------------------------------------------------------------------------------------------

def append_case(lens, owned, n_new, T, hkv, S, path, seed, with_ksum=True):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    batch = len(lens)
    base = np.concatenate([[0], np.cumsum(owned)])
    n_pool = int(base[-1]) + 2
    pool = torch.randn((n_pool, hkv, 2, S, D), generator=gen, device=DEV).to(torch.bfloat16)
    ksum = torch.randn((n_pool, hkv, 2, D), generator=gen, device=DEV).to(torch.bfloat16)
    for b, n in enumerate(lens):                                # summaries of the tokens so far
        for p in range(-(-n // S)):
            if 0 <= p < owned[b]:
                K = pool[base[b] + p, :, 0, : min(S, n - p * S)].float()
                ksum[base[b] + p, :, 0], ksum[base[b] + p, :, 1] = K.amin(1), K.amax(1)
    k, v = (torch.randn((batch, T, hkv, D), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    shape, ctx, ws = handle(batch, hkv, S, n_pool, max(owned))
    t = dict(page_base=dev(base, torch.int64), ctx_len=dev(lens), n_new=dev(n_new), path=None if path is None else dev(path))
    want_pool, want_sum, want_len = pool.clone(), ksum.clone(), list(lens)
    for b, n in enumerate(lens):
        m = n_new[b]
        places = T if path is None else len(path[b])
        if n < 0 or m < 0 or m > places or n + m > owned[b] * S:
            continue
        want_len[b] = n + m
        for i in range(m):
            src = i if path is None else path[b][i]
            p, slot = base[b] + (n + i) // S, (n + i) % S
            for z, x in enumerate((k, v)):
                want_pool[p, :, z, slot] = x[b, src] if 0 <= src < T else 0
        for p in range(n // S, -(-(n + m) // S) if m else 0):
            K = want_pool[base[b] + p, :, 0, : min(S, n + m - p * S)].float()
            want_sum[base[b] + p, :, 0], want_sum[base[b] + p, :, 1] = K.amin(1), K.amax(1)
    inputs = B.make_inputs(page_base=t["page_base"], ctx_len=t["ctx_len"])
    tokens = B.make_new_tokens(k=k, v=v, n_new=t["n_new"], path=t["path"])
    return dict(ctx=ctx, ws=ws, inputs=inputs, tokens=tokens, pool=pool, ksum=ksum if with_ksum else None, t=t, k=k, v=v,
                want=(want_pool, want_sum, want_len))


APPENDS = {
    "first_token": dict(lens=[0], owned=[1], n_new=[1], T=1, hkv=1, S=16, path=None),
    "decoded_tokens": dict(lens=[15, 16, 17, 31, 0], owned=[2, 2, 2, 2, 1], n_new=[1, 1, 1, 1, 1], T=1, hkv=8, S=16, path=None),
    "nothing_new": dict(lens=[15, 16], owned=[2, 2], n_new=[0, 1], T=4, hkv=2, S=16, path=None),
    "accepted_paths": dict(lens=[15, 32, 100], owned=[4, 4, 9], n_new=[3, 0, 5], T=16, hkv=4, S=16,
                           path=[[0, 4, 9, -1, -1], [-1] * 5, [1, 3, 3, 15, 2]]),
    "pages_of_32": dict(lens=[31, 33, 0], owned=[4, 4, 4], n_new=[70, 64, 96], T=96, hkv=2, S=32, path=None),
    "prompts": dict(lens=[0, 7, 300], owned=[70, 70, 90], n_new=[1000, 1113, 1001], T=1113, hkv=3, S=16, path=None),
    "pages_just_filled": dict(lens=[0, 1], owned=[2, 2], n_new=[32, 31], T=32, hkv=2, S=16, path=None),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", list(APPENDS))
def test_append_writes_rows_summaries_and_lengths(name, in_place):
    c = append_case(seed=len(name), **APPENDS[name])
    out = c["t"]["ctx_len"] if in_place else torch.full_like(c["t"]["ctx_len"], -5)
    B.swarm_append_tokens(c["ctx"], c["inputs"], c["tokens"], c["pool"], c["ksum"], out)
    torch.cuda.synchronize()
    pool, ksum, lens = c["want"]
    assert same(c["pool"], pool) and torch.equal(c["ksum"].float(), ksum.float()) and out.tolist() == lens
    assert B.swarm_device_status(c["ctx"]) == 0
    close(c["ctx"])


def test_append_without_summaries():
    c = append_case(lens=[20, 3], owned=[3, 3], n_new=[9, 2], T=9, hkv=2, S=16, path=None, seed=1, with_ksum=False)
    out = torch.zeros(2, dtype=torch.int32, device=DEV)
    B.swarm_append_tokens(c["ctx"], c["inputs"], c["tokens"], c["pool"], None, out)
    torch.cuda.synchronize()
    assert same(c["pool"], c["want"][0]) and out.tolist() == c["want"][2]
    close(c["ctx"])


def test_append_leaves_requests_without_room_as_they_were():
    c = append_case(lens=[30, 20, 32, -1, 5], owned=[2, 2, 2, 2, 2], n_new=[3, 12, 1, 1, 99], T=16, hkv=2, S=16, path=None, seed=2)
    out = torch.zeros(5, dtype=torch.int32, device=DEV)
    B.swarm_append_tokens(c["ctx"], c["inputs"], c["tokens"], c["pool"], c["ksum"], out)
    assert B.swarm_device_status(c["ctx"]) == B.DEV_BAD_LENGTH
    assert same(c["pool"], c["want"][0]) and same(c["ksum"], c["want"][1]) and out.tolist() == [30, 32, 32, -1, 5]
    close(c["ctx"])


def test_append_reports_tokens_that_are_not_there():
    c = append_case(lens=[4], owned=[2], n_new=[3], T=4, hkv=2, S=16, path=[[1, 4, -1]], seed=3)
    out = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.swarm_append_tokens(c["ctx"], c["inputs"], c["tokens"], c["pool"], c["ksum"], out)
    assert B.swarm_device_status(c["ctx"]) == B.DEV_BAD_TOKEN
    assert same(c["pool"], c["want"][0]) and torch.equal(c["ksum"].float(), c["want"][1].float()) and out.tolist() == [7]
    close(c["ctx"])


# ---- plan ----------------------------------------------------------------------------------------------------------------

def plan_reference(base, lens, parent, reserve, keep, S):
    new_base, new_len, src, dst = [0], [], [], []
    for j, b in enumerate(parent):
        pages, n = [], 0
        if b >= 0:
            P = -(-lens[b] // S)
            pages = [base[b] + p for p in range(P) if keep is None or keep[base[b] + p]]
            n = sum(min(S, lens[b] - (x - base[b]) * S) for x in pages)
        src += pages
        dst += [new_base[-1] + i for i in range(len(pages))]
        new_base.append(new_base[-1] + len(pages) + (reserve[j] if reserve is not None else 0))
        new_len.append(n)
    return new_base, new_len, src, dst


class Layout:
    def __init__(self, lens, owned, n_pool, hkv=2, S=16, seed=0, tables=True):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.S = lens, S
        self.base = [0] + np.cumsum(owned).tolist()
        self.n_pool = n_pool
        self.pool = torch.randint(-32768, 32768, (n_pool, hkv, 2, S, D), generator=gen, device=DEV, dtype=torch.int16).view(torch.bfloat16)
        self.ksum = torch.randint(-32768, 32768, (n_pool, hkv, 2, D), generator=gen, device=DEV, dtype=torch.int16).view(torch.bfloat16) if tables else None
        self.p2c = torch.arange(1000, 1000 + n_pool, device=DEV, dtype=torch.int32) if tables else None
        self.shape, self.ctx, self.ctx_ws = handle(len(lens), hkv, S, n_pool, max(owned))
        self.page_base, self.ctx_len = dev(self.base, torch.int64), dev(lens)
        n = B.swarm_move_pages_workspace_bytes(self.shape)
        self.ws = torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV)

    def plan(self, parent, reserve=None, keep=None, in_place=False, max_moves=None):
        i32 = dict(dtype=torch.int32, device=DEV)
        n = max_moves or self.n_pool
        self.src, self.dst, self.n = torch.full((n,), -7, **i32), torch.full((n,), -7, **i32), torch.zeros(1, **i32)
        self.new_base = torch.zeros(len(self.lens) + 1, dtype=torch.int64, device=DEV)
        self.new_len = torch.zeros(len(self.lens), **i32)
        self.held = [dev(parent), None if reserve is None else dev(reserve), None if keep is None else dev(keep, torch.uint8)]
        plan = B.make_page_plan(page_base=self.page_base, ctx_len=self.ctx_len, parent=self.held[0], reserve=self.held[1], keep=self.held[2],
                                new_page_base=self.new_base, new_ctx_len=self.new_len, src=self.src, dst=self.dst, n_moves=self.n,
                                in_place=in_place)
        B.swarm_plan_pages(self.ctx, plan)

    def moves(self, to=None, src=None, dst=None, n=None):
        to = to or (self.pool, self.ksum, self.p2c)
        if src is not None:
            self.src, self.dst = dev(src), dev(dst)
            self.n = dev([len(src) if n is None else n])
        self.to = to
        m = B.make_page_moves(src=self.src, dst=self.dst, n_moves=self.n, from_pool=self.pool, to_pool=to[0], from_ksum=self.ksum,
                              to_ksum=to[1], from_page2cluster=self.p2c, to_page2cluster=to[2])
        B.swarm_move_pages(self.ctx, m, self.ws)

    def expect(self, pairs, to=None):
        """Clones of the tables with the pairs moved, all sources read first."""
        out = []
        for a, b in zip((self.pool, self.ksum, self.p2c), to or (self.pool, self.ksum, self.p2c)):
            if a is None:
                out.append(None)
                continue
            new = b.clone()
            if pairs:
                s, d = (torch.tensor(x, device=DEV) for x in zip(*pairs))
                new.view(torch.int16 if new.dtype == torch.bfloat16 else new.dtype)[d] = a.view(torch.int16 if a.dtype == torch.bfloat16 else a.dtype)[s]
            out.append(new)
        return out

    def matches(self, want):
        torch.cuda.synchronize()
        return all(w is None or same(t, w) for t, w in zip(self.to, want))


def random_layout(seed, batch, S=16, most=40, empty=True):
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(0 if empty else 1, most * S, size=batch)]
    owned = [-(-n // S) + int(rng.integers(0, 3)) for n in lens]
    return rng, lens, owned


@pytest.mark.parametrize("seed", range(6))
def test_plan_matches_the_definition(seed):
    rng, lens, owned = random_layout(seed, 3 + 9 * seed, S=(16, 32)[seed % 2], most=(40, 3, 700)[seed % 3])
    S = (16, 32)[seed % 2]
    lay = Layout(lens, owned, sum(owned) * 2 + 200, hkv=1, S=S, tables=False)
    batch = len(lens)
    for trial in range(4):
        parent = rng.integers(-1, batch, size=batch)
        reserve = rng.integers(0, 3, size=batch) if trial % 2 else None
        keep = (rng.random(lay.n_pool) < 0.6).astype(np.uint8) * 3 if trial >= 2 else None
        want = plan_reference(lay.base, lens, parent, reserve, keep, S)
        if want[0][-1] > lay.n_pool:
            continue
        lay.plan(parent, reserve, keep)
        torch.cuda.synchronize()
        assert lay.new_base.tolist() == want[0] and lay.new_len.tolist() == want[1]
        n = int(lay.n)
        assert n == len(want[2]) and lay.src[:n].tolist() == want[2] and lay.dst[:n].tolist() == want[3]
        assert bool((lay.src[n:] == -7).all())
        assert B.swarm_device_status(lay.ctx) == 0
    close(lay.ctx)


def test_plan_refuses_as_a_whole():
    lay = Layout([20, 40, 5], [2, 4, 1], 8, hkv=1)
    for kw, bits in ((dict(parent=[0, 3, 1]), B.DEV_BAD_PAGE), (dict(parent=[0, -2, 1]), B.DEV_BAD_PAGE),
                     (dict(parent=[0, 0, 1], in_place=True), B.DEV_BAD_PAGE), (dict(parent=[1, -1, 0], in_place=True), B.DEV_BAD_PAGE),
                     (dict(parent=[1, 1, 1]), B.DEV_BAD_LENGTH), (dict(parent=[0, 1, 2], reserve=[0, 3, 0]), B.DEV_BAD_LENGTH),
                     (dict(parent=[0, 1, 2], reserve=[0, -1, 0]), B.DEV_BAD_LENGTH), (dict(parent=[0, 1, 2], max_moves=5), B.DEV_BAD_LENGTH)):
        lay.plan(**kw)
        assert B.swarm_device_status(lay.ctx) == bits, kw
        assert int(lay.n) == -1 and lay.new_base.tolist() == lay.base and lay.new_len.tolist() == lay.lens
        before = lay.expect([])
        lay.moves()                                             # a refused plan moves nothing
        assert lay.matches(before) and B.swarm_device_status(lay.ctx) == 0
    lay.ctx_len.copy_(dev([20, 400, 5]))                        # a length beyond its pages
    lay.plan([0, 1, 2])
    assert B.swarm_device_status(lay.ctx) == B.DEV_BAD_LENGTH and int(lay.n) == -1
    lay.plan([0, -1, 2])                                        # ... of a request that goes
    assert B.swarm_device_status(lay.ctx) == 0 and int(lay.n) == 3
    close(lay.ctx)


# ---- moves -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("hkv,S,tables", [(1, 16, True), (2, 32, True), (8, 16, True), (5, 32, False), (40, 16, True)])
def test_compaction_inside_the_pool(hkv, S, tables):
    """Freed requests, dropped pages, spare pages: moves down and up in one plan."""
    for seed in range(3):
        rng, lens, owned = random_layout(seed + 50, 12, S=S, most=12)
        lay = Layout(lens, owned, sum(owned) + 60, hkv=hkv, S=S, seed=seed, tables=tables)
        left = np.flatnonzero(rng.random(12) < 0.7)
        parent = np.full(12, -1)
        parent[12 - len(left):] = left
        reserve = rng.integers(0, 6, size=12)
        keep = (rng.random(lay.n_pool) < 0.8).astype(np.uint8)
        want = plan_reference(lay.base, lens, parent, reserve, keep, S)
        lay.plan(parent, reserve, keep, in_place=True)
        tables_after = lay.expect(list(zip(want[2], want[3])))
        lay.moves()
        assert lay.matches(tables_after)
        assert B.swarm_device_status(lay.ctx) == 0
        close(lay.ctx)


@pytest.mark.parametrize("by", [-1, 1, -7, 100])
def test_long_shifts_inside_the_pool(by):
    """Every page waits for a neighbour: 4000 pages of 32 KB moved by a few places, all at once."""
    n, room = 4000, 100
    lay = Layout([16], [1], n + 2 * room, hkv=4)
    src = np.arange(room, room + n)
    pairs = list(zip(src.tolist(), (src + by).tolist()))
    want = lay.expect(pairs)
    lay.moves(src=src, dst=src + by)
    assert lay.matches(want) and B.swarm_device_status(lay.ctx) == 0
    close(lay.ctx)


def test_forks_to_another_pool_and_to_free_pages():
    lay = Layout([40, 33], [3, 4], 40, hkv=3)
    other = tuple(torch.zeros_like(x) for x in (lay.pool, lay.ksum, lay.p2c))
    lay.plan([1, 1], reserve=[1, 0])
    want = lay.expect([(3, 0), (4, 1), (5, 2), (3, 4), (4, 5), (5, 6)], other)
    lay.moves(to=other)
    assert lay.matches(want)
    pairs = [(0, 30), (1, 31), (2, 32), (0, 20), (1, 21), (2, 39), (5, 5)]
    want = lay.expect(pairs)
    lay.moves(src=[p[0] for p in pairs], dst=[p[1] for p in pairs])
    assert lay.matches(want) and B.swarm_device_status(lay.ctx) == 0
    close(lay.ctx)


@pytest.mark.parametrize("name,pairs,done", [
    ("a swap", [(3, 4), (4, 3)], [(3, 4)]),                      # the downward move comes first and page 3 is read later
    ("a destination twice", [(10, 2), (11, 2), (12, 3)], [(10, 2), (12, 3)]),
    ("ids outside the pool", [(10, 40), (-1, 3), (40, 3), (11, 4)], [(11, 4)]),
    ("up in the wrong order", [(6, 7), (5, 6)], [(6, 7)]),       # the last upward pair comes first, and page 6 is read later
    ("up in order", [(5, 6), (6, 7)], [(5, 6), (6, 7)]),
    ("down in the wrong order", [(7, 6), (8, 7), (6, 5)], [(8, 7), (6, 5)]),
    ("onto a page that stays", [(9, 9), (12, 9)], [(9, 9)]),
    ("upward onto a page that stays", [(1, 9), (9, 9)], [(9, 9)]),
])
def test_pairs_out_of_order_are_found(name, pairs, done):
    lay = Layout([16], [1], 40, hkv=2)
    want = lay.expect(done)
    lay.moves(src=[p[0] for p in pairs], dst=[p[1] for p in pairs])
    assert lay.matches(want), name
    assert B.swarm_device_status(lay.ctx) == (0 if len(done) == len(pairs) else B.DEV_BAD_PAGE)
    close(lay.ctx)


def test_moves_count_and_refusals():
    lay = Layout([16], [1], 40, hkv=2)
    want = lay.expect([(10, 1)])
    lay.moves(src=[10, 11, 12], dst=[1, 2, 3], n=1)             # only the first
    assert lay.matches(want) and B.swarm_device_status(lay.ctx) == 0
    want = lay.expect([])
    for n in (0, -1):
        lay.moves(src=[10, 11, 12], dst=[1, 2, 3], n=n)
        assert lay.matches(want) and B.swarm_device_status(lay.ctx) == 0
    with pytest.raises(B.SwarmError) as e:                      # a pool of its own, but the same summaries
        lay.moves(to=(torch.zeros_like(lay.pool), lay.ksum, lay.p2c), src=[1], dst=[2])
    assert e.value.code == B.ERR_INVALID_ARG
    with pytest.raises(B.SwarmError) as e:
        lay.moves(to=(lay.pool, torch.zeros_like(lay.ksum), lay.p2c), src=[1], dst=[2])
    assert e.value.code == B.ERR_INVALID_ARG
    lay.ws = lay.ws[:256]
    with pytest.raises(B.SwarmError) as e:
        lay.moves(src=[1], dst=[2])
    assert e.value.code == B.ERR_WORKSPACE_TOO_SMALL
    close(lay.ctx)


def test_plan_and_moves_of_many_requests():
    """More requests than a plan's CTA has threads, freed, thinned out and grown inside the pool."""
    rng, lens, owned = random_layout(91, 700, most=4)
    lay = Layout(lens, owned, sum(owned) + 300, hkv=1, seed=9)
    left = np.flatnonzero(rng.random(700) < 0.8)
    parent = np.full(700, -1)
    parent[np.sort(rng.permutation(700)[: len(left)])] = left
    reserve = (rng.random(700) < 0.2).astype(int)
    keep = (rng.random(lay.n_pool) < 0.9).astype(np.uint8)
    want = plan_reference(lay.base, lens, parent, reserve, keep, 16)
    moved = lay.expect(list(zip(want[2], want[3])))
    lay.plan(parent, reserve, keep, in_place=True)
    torch.cuda.synchronize()
    assert lay.new_base.tolist() == want[0] and lay.new_len.tolist() == want[1] and int(lay.n) == len(want[2])
    lay.moves()
    assert lay.matches(moved) and B.swarm_device_status(lay.ctx) == 0
    close(lay.ctx)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("table", [[0, 2, 6, 12], [0, 2, 6, 1 << 40], [-3, -1, 1, 6], [0, 5, 9, 13]])
def test_append_writes_nothing_outside_the_pool(table, in_place):
    """Page tables that name pages behind the pool (8 pages of it) or in front of it; the tensors go on on both sides."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    hkv, S, n_pool, edge = 2, 16, 8, 8
    whole = torch.randn((edge + n_pool + edge, hkv, 2, S, D), generator=gen, device=DEV).to(torch.bfloat16)
    sums = torch.randn((edge + n_pool + edge, hkv, 2, D), generator=gen, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn((3, 8, hkv, D), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    shape, ctx, ws = handle(3, hkv, S, n_pool, 8)
    base, lens, n_new = dev(table, torch.int64), dev([10, 20, 3]), dev([8, 5, 7])
    want, want_sums, want_len = whole.clone(), sums.clone(), [10, 20, 3]
    for b, (n, m) in enumerate(zip([10, 20, 3], [8, 5, 7])):
        if table[b] < 0 or table[b + 1] > n_pool:
            continue
        want_len[b] = n + m
        for i in range(m):
            for z, x in enumerate((k, v)):
                want[edge + table[b] + (n + i) // S, :, z, (n + i) % S] = x[b, i]
        for p in range(n // S, (n + m - 1) // S + 1):
            at, lo = edge + table[b] + p, max(n - p * S, 0)
            K = want[at, :, 0, lo: min(S, n + m - p * S)].float()
            low, high = K.amin(1), K.amax(1)
            if lo:                                              # the page held tokens: their summary takes part
                low, high = torch.minimum(low, sums[at, :, 0].float()), torch.maximum(high, sums[at, :, 1].float())
            want_sums[at, :, 0], want_sums[at, :, 1] = low, high
    out = lens if in_place else torch.zeros_like(lens)
    B.swarm_append_tokens(ctx, B.make_inputs(page_base=base, ctx_len=lens), B.make_new_tokens(k=k, v=v, n_new=n_new),
                          whole[edge: edge + n_pool], sums[edge: edge + n_pool], out)
    torch.cuda.synchronize()
    assert same(whole, want) and same(sums, want_sums) and out.tolist() == want_len
    assert B.swarm_device_status(ctx) == B.DEV_BAD_LENGTH
    close(ctx)


@pytest.mark.parametrize("in_place", [False, True])
def test_append_stops_at_the_pages_that_a_step_can_use(in_place):
    """Requests of 4 pages in a ctx for 2: what fits 2 pages is written, what does not leaves the request as it was."""
    c = append_case(lens=[30, 30, 0, 32], owned=[4, 4, 4, 4], n_new=[2, 3, 33, 0], T=40, hkv=2, S=16, path=None, seed=6)
    B.swarm_destroy(c["ctx"])
    shape, ctx, ws = handle(4, 2, 16, 18, 2)
    before, sums, lens = c["pool"].clone(), c["ksum"].clone(), c["t"]["ctx_len"]
    out = lens if in_place else torch.full_like(lens, -5)
    B.swarm_append_tokens(ctx, c["inputs"], c["tokens"], c["pool"], c["ksum"], out)
    assert B.swarm_device_status(ctx) == B.DEV_BAD_LENGTH
    assert out.tolist() == [32, 30, 0, 32]
    assert same(c["pool"][:4], c["want"][0][:4]) and torch.equal(c["ksum"][:4].float(), c["want"][1][:4].float())
    assert same(c["pool"][4:], before[4:]) and same(c["ksum"][4:], sums[4:])
    close(ctx)


@pytest.mark.parametrize("pairs,done", [
    ([(9, 9), (9, 9)], [(9, 9)]), ([(9, 9), (3, 4), (9, 9)], [(9, 9), (3, 4)]), ([(9, 9), (9, 9), (5, 2)], [(9, 9), (5, 2)]),
    ([(9, 9), (8, 8), (3, 4)], [(9, 9), (8, 8), (3, 4)])])
def test_a_page_that_stays_twice_is_found(pairs, done):
    """A second pair with the same destination is one, whatever else moves."""
    lay = Layout([16], [1], 40, hkv=2)
    want = lay.expect(done)
    lay.moves(src=[p[0] for p in pairs], dst=[p[1] for p in pairs])
    assert lay.matches(want)
    assert B.swarm_device_status(lay.ctx) == (0 if len(done) == len(pairs) else B.DEV_BAD_PAGE)
    close(lay.ctx)
