"""swarm_tree_attn: drafted tokens over the paged context, against the formula in 64 bits.

Tolerances.  The weights are rounded to bf16 for the product with V and the result to bf16 on the way out: half a step of
2^-8 each, the first relative to W = sum_j w_j |v_j|, the second to the result.  Products of bf16 are exact in fp32;
a score is off by at most e = 128 * 2^-23 * sum |q k| / sqrt(d) (the accumulator may truncate), which moves a weight by a factor of
exp(2 e); exponentials and the running sums over L tokens in fp32 add 2^-18 + L * 2^-23 relative to W."""
import math

import numpy as np
import pytest
import torch

from paper_2603_17803_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128


class Case:
    """Requests in a pool whose unused slots (padding tokens, pages of nobody) and draft rows behind n_draft hold NaN."""

    def __init__(self, lens, T, n_draft, hq, hkv, S, seed, mask="tree", spare=1, top_k=0, q_scale=2.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.T, self.n_draft, self.hq, self.hkv, self.S, self.top_k = lens, T, n_draft, hq, hkv, S, top_k
        Bn = self.batch = len(lens)
        pages = [-(-n // S) + spare for n in lens]
        self.base = np.concatenate([[0], np.cumsum(pages)])
        n_pool = int(self.base[-1]) + 3
        self.pool = torch.full((n_pool, hkv, 2, S, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.K = []
        for b, n in enumerate(lens):
            kv = torch.randn((n, hkv, 2, D), generator=gen, device=DEV).to(torch.bfloat16)
            self.K.append(kv)
            pos = torch.arange(n, device=DEV)
            self.pool[int(self.base[b]) + pos // S, :, :, pos % S] = kv
        self.q, self.k, self.v = (torch.full((Bn, T, h, D), float("nan"), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
        for b, n in enumerate(n_draft):
            for x, f in ((self.q, q_scale), (self.k, 1.0), (self.v, 1.0)):
                x[b, :n] = (torch.randn(x[b, :n].shape, generator=gen, device=DEV) * f).to(torch.bfloat16)
        self.sees = np.zeros((Bn, T, T), dtype=bool)
        if mask == "tree":
            for b in range(Bn):
                for t in range(T):
                    parent = rng.integers(-1, t) if t else -1
                    if parent >= 0:
                        self.sees[b, t] = self.sees[b, parent]
                    self.sees[b, t, t] = True
        elif mask == "random":                                  # some rows see nothing, some what comes behind them
            self.sees = rng.random((Bn, T, T)) < 0.3
            self.sees[:, :: 3] = False
        elif mask == "chain":
            self.sees[:] = np.tril(np.ones((T, T), dtype=bool))
        words = -(-T // 32)
        bits = np.zeros((Bn, T, words * 32), dtype=np.uint64)
        bits[:, :, :T] = self.sees
        if T % 32 and mask != "chain":
            bits[:, :, T:] = 1                                  # bits behind T mean nothing
        packed = (bits.reshape(Bn, T, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
        self.mask = None if mask == "chain" else torch.from_numpy(packed.view(np.int32)).to(DEV)
        self.sel = self.n_sel = None
        if top_k:
            sel = np.full((Bn, hq, top_k), -1, dtype=np.int32)
            n_sel = np.zeros((Bn, hq), dtype=np.int32)
            for b, n in enumerate(lens):
                P = -(-n // S)
                for h in range(hq):
                    m = min(P, int(rng.integers(0, top_k + 1)) if h % 5 == 4 else top_k)
                    sel[b, h, :m] = np.sort(rng.permutation(P)[:m])
                    n_sel[b, h] = m
            self.sel, self.n_sel = torch.from_numpy(sel).to(DEV), torch.from_numpy(n_sel).to(DEV)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.page_base = torch.as_tensor(self.base, dtype=torch.int64, device=DEV)
        self.ctx_len, self.nd = torch.tensor(lens, **i32), torch.tensor(n_draft, **i32)
        self.shape = B.make_shape(batch=Bn, n_q_heads=hq, n_kv_heads=hkv, page_size=S, top_k=max(1, top_k), n_queues=1,
                                  max_pages_per_req=max(1, *pages), max_clusters_total=1, n_pool_pages=n_pool)
        self.ctx = B.swarm_create(self.shape)
        self.ctx_ws = torch.empty(B.swarm_workspace_bytes(self.shape), dtype=torch.uint8, device=DEV)
        B.swarm_set_workspace(self.ctx, self.ctx_ws)
        self.guard = 4096
        n_ws = B.swarm_tree_attn_workspace_bytes(self.shape, T)
        self.ws_all = torch.full((n_ws + self.guard,), 0xA5, dtype=torch.uint8, device=DEV)
        self.ws = self.ws_all[:n_ws]
        self.inputs = B.make_inputs(kv_pool=self.pool, page_base=self.page_base, ctx_len=self.ctx_len)
        self.tree = B.make_tree(q=self.q, k=self.k, v=self.v, n_draft=self.nd, mask=self.mask)
        self.out = torch.full((Bn, T, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((Bn, T, hq), 7.0, dtype=torch.float32, device=DEV)

    def run(self, stream=None):
        B.swarm_tree_attn(self.ctx, self.inputs, self.tree, self.sel, self.n_sel, self.ws, self.out, self.lse, stream)

    def check(self):
        torch.cuda.synchronize()
        assert bool((self.ws_all[-self.guard:] == 0xA5).all()), "wrote behind the workspace"
        g = self.hq // self.hkv
        for b in range(self.batch):
            n, L = self.n_draft[b], self.lens[b]
            assert bool((self.out[b, n:] == 7.0).all()) and bool((self.lse[b, n:] == 7.0).all())
            if n == 0:
                continue
            for h in range(self.hq):
                kv = self.K[b][:, h // g].double()
                K = torch.cat([kv[:, 0], self.k[b, :n, h // g].double()])
                V = torch.cat([kv[:, 1], self.v[b, :n, h // g].double()])
                see = torch.ones((n, L + n), dtype=torch.bool, device=DEV)
                see[:, L:] = torch.from_numpy(self.sees[b, :n, :n].copy()).to(DEV)
                if self.sel is not None:
                    see[:, :L] = False
                    for p in self.sel[b, h, : int(self.n_sel[b, h])].tolist():
                        see[:, p * self.S: min(L, (p + 1) * self.S)] = True
                q = self.q[b, :n, h].double()
                x = q @ K.T / math.sqrt(D)
                e = (q.abs() @ K.abs().T / math.sqrt(D)).masked_fill(~see, 0).amax(-1) * 128 * 2.0 ** -23
                x = x.masked_fill(~see, -math.inf)
                some = see.any(-1)
                m = torch.where(some, x.amax(-1), 0.0)
                w = torch.exp(x - m[:, None])
                total = w.sum(-1)
                w = torch.where(some[:, None], w / total[:, None], 0.0)
                ref = w @ V
                W = w @ V.abs()
                lse = torch.where(some, m + torch.log(total), -math.inf)
                got, got_lse = self.out[b, :n, h].double(), self.lse[b, :n, h].double()
                tol = 2.0 ** -8 * (W + ref.abs()) * 1.01 + (2 * e[:, None] + 2.0 ** -18 + (L + n) * 2.0 ** -23) * W
                assert bool(torch.isfinite(got).all())
                worst = ((got - ref).abs() - tol).max().item()
                assert worst <= 0, (b, h, worst, (got - ref).abs().max().item())
                assert torch.equal(got_lse == -math.inf, ~some)
                off = (got_lse - lse).abs()[some]
                lim = (e + 2.0 ** -19 + (64 + (L + n) / 128) * 2.0 ** -23 + lse.abs() * 2.0 ** -22)[some]
                assert bool((off <= lim).all()), (b, h, (off - lim).max().item())

    def close(self):
        torch.cuda.synchronize()
        damaged = B.swarm_check_workspace(self.ctx)
        B.swarm_destroy(self.ctx)
        assert damaged == 0


CASES = {
    "one_token": dict(lens=[1], T=1, n_draft=[1], hq=1, hkv=1, S=16),
    "one_token_no_context": dict(lens=[0], T=1, n_draft=[1], hq=4, hkv=1, S=16, spare=0),
    "single_token_gqa": dict(lens=[1000], T=1, n_draft=[1], hq=32, hkv=8, S=16),
    "borders_of_tiles": dict(lens=[127, 128, 129, 255, 256, 257, 15, 16, 17], T=3, n_draft=[3, 1, 2, 3, 3, 0, 1, 3, 2], hq=8, hkv=2, S=16),
    "pages_of_32": dict(lens=[31, 32, 33, 700, 1025], T=7, n_draft=[7, 7, 0, 5, 6], hq=16, hkv=4, S=32),
    "group_of_three": dict(lens=[530, 99], T=21, n_draft=[21, 13], hq=6, hkv=2, S=16),
    "rows_127_to_256": dict(lens=[400, 333], T=51, n_draft=[51, 30], hq=10, hkv=2, S=16),
    "two_streams_of_rows": dict(lens=[640, 1, 0], T=64, n_draft=[64, 40, 64], hq=8, hkv=2, S=16),
    "many_rows": dict(lens=[300, 50], T=100, n_draft=[100, 77], hq=16, hkv=2, S=32),
    "drafts_of_two_tiles": dict(lens=[200, 128], T=200, n_draft=[200, 129], hq=4, hkv=2, S=16),
    "random_masks": dict(lens=[77, 0, 0], T=40, n_draft=[40, 40, 17], hq=4, hkv=2, S=16, mask="random"),
    "random_masks_wide": dict(lens=[0, 300], T=90, n_draft=[90, 71], hq=8, hkv=2, S=16, mask="random"),
    "chain": dict(lens=[500, 20], T=33, n_draft=[33, 32], hq=8, hkv=4, S=16, mask="chain"),
    "chunk_of_a_prompt": dict(lens=[0, 64], T=300, n_draft=[300, 257], hq=4, hkv=2, S=16, mask="chain"),
    "long": dict(lens=[30011], T=9, n_draft=[9], hq=8, hkv=2, S=16),
    "many_small_requests": dict(lens=[(37 * i) % 300 for i in range(90)], T=4, n_draft=[i % 5 for i in range(90)], hq=8, hkv=4, S=16),
    "sharp": dict(lens=[2000], T=16, n_draft=[16], hq=8, hkv=2, S=16, q_scale=40.0),
    "selected": dict(lens=[1000, 333, 16], T=5, n_draft=[5, 3, 5], hq=8, hkv=2, S=16, top_k=12),
    "selected_32": dict(lens=[3000, 33], T=20, n_draft=[20, 20], hq=16, hkv=2, S=32, top_k=20),
    "selected_wide": dict(lens=[2500, 100], T=40, n_draft=[40, 33], hq=16, hkv=2, S=16, top_k=30),
    "selected_one": dict(lens=[5000], T=1, n_draft=[1], hq=4, hkv=4, S=16, top_k=1),
    "selected_no_draft_seen": dict(lens=[300, 0], T=9, n_draft=[9, 9], hq=10, hkv=2, S=16, top_k=3, mask="random"),
}


@pytest.mark.parametrize("name", list(CASES))
def test_tree_attention_matches_the_formula(name):
    c = Case(seed=len(name), **CASES[name])
    c.run()
    c.check()
    assert B.swarm_device_status(c.ctx) == 0
    c.close()


MANY = {
    # a thread looks after several units
    "units_beyond_threads": dict(lens=[(53 * i) % 200 for i in range(230)], T=3, n_draft=[(i * 7) % 4 for i in range(230)], hq=4, hkv=2, S=16),
    # a CTA works through several lists of units, some of them with nothing to do
    "lists_of_units": dict(lens=[(29 * i) % 50 for i in range(2600)], T=2, n_draft=[(i * 5) % 3 for i in range(2600)], hq=2, hkv=2, S=16),
    "lists_of_units_wide": dict(lens=[(29 * i) % 50 for i in range(1700)], T=130, n_draft=[(i * 11) % 131 for i in range(1700)], hq=3, hkv=3,
                                S=32, mask="chain"),
    # more selected pages of a KV head than its list kernel holds in registers
    "selected_thousands": dict(lens=[6405, 100], T=2, n_draft=[2, 1], hq=16, hkv=2, S=16, top_k=300),
    # more blocks of rows than SMs
    "row_blocks_beyond_sms": dict(lens=[70, 0], T=700, n_draft=[650, 700], hq=64, hkv=1, S=16, mask="chain"),
    "long_chunk": dict(lens=[1000], T=2100, n_draft=[2100], hq=8, hkv=2, S=16, mask="chain"),
}


@pytest.mark.parametrize("name", list(MANY))
def test_many_units_and_rows(name):
    c = Case(seed=len(name), **MANY[name])
    c.run()
    c.check()
    assert B.swarm_device_status(c.ctx) == 0
    c.close()
