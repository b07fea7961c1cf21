"""Host side of the operators for several continuations: sizes, refusals, and the order in which pages move (no GPU needed)."""
import ctypes
import random

import pytest
import torch

from paper_2603_17803_b200 import binding as B

SHAPE = dict(batch=2, n_q_heads=32, n_kv_heads=8, page_size=16, top_k=64, n_queues=4, max_pages_per_req=1024, max_clusters_total=16,
             n_pool_pages=2048)


@pytest.fixture(scope="module", autouse=True)
def library():
    from paper_2603_17803_b200 import build
    build.build()
    return B.load_library()


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(B.swarm_tree) == 5 * 8 + 2 * 4
    assert ctypes.sizeof(B.swarm_new_tokens) == 4 * 8 + 2 * 4
    assert ctypes.sizeof(B.swarm_page_plan) == 10 * 8 + 2 * 4
    assert ctypes.sizeof(B.swarm_page_moves) == 9 * 8 + 2 * 4


def test_workspace_sizes():
    shape = B.make_shape(**SHAPE)
    small, large = B.swarm_tree_attn_workspace_bytes(shape, 1), B.swarm_tree_attn_workspace_bytes(shape, 64)
    assert 0 < small <= large and small % 256 == 0 and large % 256 == 0
    assert B.swarm_move_pages_workspace_bytes(shape) >= 3 * 2048 * 4
    assert B.swarm_beam_select_workspace_bytes(1, 4, 32000, 8) > 0


@pytest.mark.parametrize("call,code", [
    (lambda s: B.swarm_tree_attn_workspace_bytes(s(), 0), B.ERR_INVALID_ARG),
    (lambda s: B.swarm_tree_attn_workspace_bytes(s(n_q_heads=129, n_kv_heads=1), 4), B.ERR_UNSUPPORTED),
    (lambda s: B.swarm_tree_attn_workspace_bytes(s(page_size=8), 4), B.ERR_UNSUPPORTED),
    (lambda s: B.swarm_move_pages_workspace_bytes(s(n_pool_pages=1 << 30)), B.ERR_UNSUPPORTED),
    (lambda s: B.swarm_move_pages_workspace_bytes(s(n_queues=0)), B.ERR_INVALID_ARG),
    (lambda s: B.swarm_beam_select_workspace_bytes(0, 4, 32000, 8), B.ERR_INVALID_ARG),
    (lambda s: B.swarm_beam_select_workspace_bytes(1, 4, 32000, 65), B.ERR_UNSUPPORTED),
    (lambda s: B.swarm_beam_select_workspace_bytes(1, 1 << 16, 1 << 16, 8), B.ERR_UNSUPPORTED),
])
def test_sizes_of_what_is_not_supported(call, code):
    with pytest.raises(B.SwarmError) as e:
        call(lambda **kw: B.make_shape(**{**SHAPE, **kw}))
    assert e.value.code == code


def test_a_null_ctx_is_refused(library):
    nothing = ctypes.c_void_p(0)
    assert library.swarm_tree_attn(nothing, nothing, nothing, nothing, nothing, nothing, ctypes.c_int64(0), nothing, nothing, nothing) == 1
    assert library.swarm_append_tokens(*[nothing] * 7) == 1
    assert library.swarm_plan_pages(*[nothing] * 3) == 1
    assert library.swarm_move_pages(nothing, nothing, nothing, ctypes.c_int64(0), nothing) == 1
    assert library.swarm_beam_select(nothing, ctypes.c_int32(0), ctypes.c_int64(1), nothing, *[ctypes.c_int32(1)] * 4, nothing,
                                     ctypes.c_int64(0), *[nothing] * 4) == 1


def test_tensors_have_to_be_on_the_gpu():
    bf16 = dict(dtype=torch.bfloat16)
    q, kv, n = torch.zeros((1, 2, 4, 128), **bf16), torch.zeros((1, 2, 1, 128), **bf16), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.make_tree(q=q, k=kv, v=kv, n_draft=n)
    with pytest.raises(ValueError, match="CUDA"):
        B.make_new_tokens(k=kv, v=kv, n_new=n)
    with pytest.raises(ValueError, match="shape"):
        B.make_new_tokens(k=kv, v=kv[:, :1], n_new=n)
    with pytest.raises(ValueError, match="CUDA"):
        B.swarm_beam_select(torch.zeros((1, 1, 8)), torch.zeros((1, 1)), n, torch.zeros((1, 1)), n[None], n[None])


def moved(pairs, pool):
    """The rule of swarm_move_pages inside one pool: downward moves first to last, then upward moves last to first; a pair is carried out
    iff no pair behind it in that order reads its destination and none in front writes it."""
    n = len(pairs)
    place = {i: (2 * n - 1 - i if d > s else i) for i, (s, d) in enumerate(pairs)}
    reads = {}
    for i, (s, d) in enumerate(pairs):
        if s != d:
            reads[s] = max(reads.get(s, -1), place[i])
    writer = {}
    for i, (s, d) in enumerate(pairs):
        writer[d] = min(writer.get(d, 1 << 60), place[i])
    new = list(pool)
    for i, (s, d) in enumerate(pairs):
        if writer[d] == place[i] and reads.get(d, -1) <= place[i]:
            new[d] = pool[s]
        elif s != d:
            return None
    return new


def test_every_plan_that_keeps_the_order_can_be_carried_out_in_place():
    """Random layouts: requests freed, pages dropped, spare pages added; requests move down, up and stay in one plan."""
    rng = random.Random(3)
    for _ in range(500):
        owned = [rng.randint(0, 6) for _ in range(rng.randint(1, 8))]
        base = [sum(owned[:i]) for i in range(len(owned) + 1)]
        pool = list(range(base[-1] + 40))
        pairs, at = [], 0
        for b, n in enumerate(owned):
            at += rng.choice([0, 0, 1, 5])
            if rng.random() < 0.7:
                for x in range(base[b], base[b + 1]):
                    if rng.random() < 0.8:
                        pairs.append((x, at))
                        at += 1
        want = list(pool)
        for s, d in pairs:
            want[d] = pool[s]
        assert moved(pairs, pool) == want


@pytest.mark.parametrize("vocab", [1 << 30, (1 << 31) - 1])
def test_rows_that_are_too_long_to_count_are_refused(vocab):
    with pytest.raises(B.SwarmError) as e:
        B.swarm_beam_select_workspace_bytes(1, 1, vocab, 1)
    assert e.value.code == B.ERR_UNSUPPORTED
    assert B.swarm_beam_select_workspace_bytes(1, 1, (1 << 30) - 1, 1) > 0
