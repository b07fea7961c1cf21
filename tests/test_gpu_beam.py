"""swarm_beam_select against the definition in 64 bits.

The values of a selection are compared with score + logit - log sum exp: every exponential in fp32 is off by at most 2^-21
relative, a chunk's sum adds at most 48 roundings of 2^-24: 2^-18 in all, plus the rounding of the result to fp32 (2^-24 of
its size).  The order is compared exactly wherever neighbours differ by more than twice that, or belong to one beam (where it is
the order of the logits, ties to the lower token)."""
import ctypes
import math

import pytest
import torch

from paper_2603_17803_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OFF = 2.0 ** -18


def reference(logits, score, keep):
    x = logits.double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    total = score.double()[..., None] + (x - torch.logsumexp(x, -1, keepdim=True))
    total = torch.where(torch.isnan(total), -math.inf, total)
    batch, beams, V = x.shape
    # inside a beam the logits decide: sort by (total of the beam's best, logit) is not needed, a stable sort keeps the lower index
    value, at = torch.sort(total.view(batch, -1), dim=-1, descending=True, stable=True)
    n = min(keep + 1, value.shape[1])
    return value[:, :n], at[:, :n]


def select(logits, score, keep):
    batch, beams, V = logits.shape
    n = B.swarm_beam_select_workspace_bytes(batch, beams, V, keep)
    ws = torch.full((n + 1024,), 0xA5, dtype=torch.uint8, device=DEV)
    new = torch.full((batch, keep), 7.0, device=DEV)
    parent, token = (torch.full((batch, keep), 7, dtype=torch.int32, device=DEV) for _ in range(2))
    B.swarm_beam_select(logits, score, ws[:n], new, parent, token)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xA5).all()), "wrote behind the workspace"
    return new, parent, token


def check(logits, score, keep):
    batch, beams, V = logits.shape
    new, parent, token = select(logits, score, keep)
    value, at = reference(logits, score, keep)
    for b in range(batch):
        n = int((value[b, :keep] > -math.inf).sum())
        assert bool((new[b, n:] == -math.inf).all()) and bool((parent[b, n:] == -1).all()) and bool((token[b, n:] == -1).all())
        v, a = value[b, :n], at[b, :n]
        got = new[b, :n].double()
        tol = OFF + v.abs() * 2.0 ** -24
        assert bool(((got - v).abs() <= tol).all()), (b, (got - v).abs().max().item())
        assert bool(((parent[b, :n] >= b * beams) & (parent[b, :n] < (b + 1) * beams)).all())
        index = (parent[b, :n].long() - b * beams) * V + token[b, :n]
        assert index.unique().numel() == n
        full = torch.cat([value[b], torch.full((1,), -math.inf, device=DEV, dtype=torch.float64)])
        ids = torch.cat([at[b], torch.full((1,), -1, device=DEV)])
        for i in range(n):
            # the place is certain where the neighbours are far, or are of the same beam
            near = [j for j in (i - 1, i + 1) if 0 <= j < len(ids) and abs((full[i] - full[j]).item()) <= 2 * OFF and ids[j] // V != ids[i] // V]
            if not near:
                assert int(index[i]) == int(a[i]), (b, i, int(index[i]), int(a[i]))


CASES = {
    "one_row": (1, 1, 1, 1, torch.float32),
    "vocabulary_below_keep": (2, 2, 3, 8, torch.float32),
    "one_prompt": (1, 4, 32000, 8, torch.float32),
    "odd_vocabulary": (3, 5, 50257, 10, torch.bfloat16),
    "odd_vocabulary_f16": (2, 3, 8191, 64, torch.float16),
    "odd_vocabulary_f32": (5, 2, 1001, 4, torch.float32),
    "line_borders": (2, 7, 8193, 20, torch.bfloat16),
    "many_rows": (40, 8, 10000, 16, torch.float32),
    "large_vocabulary": (1, 16, 200000, 32, torch.float16),
    "many_beams": (2, 64, 9000, 64, torch.bfloat16),
}


@pytest.mark.parametrize("name", list(CASES))
def test_selection_matches_the_definition(name):
    batch, beams, V, keep, dtype = CASES[name]
    gen = torch.Generator(device=DEV).manual_seed(V)
    logits = (torch.randn((batch, beams, V), generator=gen, device=DEV) * 3).to(dtype)
    score = -torch.rand((batch, beams), generator=gen, device=DEV) * 5
    check(logits, score, keep)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [4096, 5003])
def test_ties_go_to_the_lowest_index(dtype, V):
    """Whole-numbered logits, many of them equal; beams 0 and 2 (and 1 and 3) are the same row with the same score, at
    different places of a 16-byte line where the vocabulary is odd."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    logits = torch.randint(0, 4, (2, 4, V), generator=gen, device=DEV).to(dtype)
    logits[:, 2:] = logits[:, :2]
    score = torch.zeros((2, 4), device=DEV)
    keep = 40
    _, parent, token = select(logits, score, keep)
    for b in range(2):
        # beams 0 and 2 against 1 and 3: their sums of exponentials differ by far more than the tolerance, or not at all
        lse = torch.logsumexp(logits[b].double(), -1)
        assert abs((lse[0] - lse[1]).item()) > 1e-5
        order = sorted(((-(logits[b, k].max().double() - lse[k]).item()), k) for k in (0, 1))
        best = order[0][1]
        top = (logits[b, best] == logits[b, best].max()).nonzero().view(-1)[:keep].int()
        assert torch.equal(token[b, : len(top)], top)
        assert bool((parent[b, : len(top)] == b * 4 + best).all())


def test_masked_logits_and_beams():
    """Constrained decoding: -inf and NaN logits, a beam without any token left, beams that are not alive yet."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    logits = torch.randn((4, 3, 3001), generator=gen, device=DEV)
    logits[0, :, ::2] = -math.inf
    logits[1, 0] = -math.inf
    logits[1, 1, :] = math.nan
    logits[1, 1, 77] = 0.5                                      # a beam of one token
    logits[2] = -math.inf
    logits[2, 1, 5] = 1.0                                       # one continuation in all
    logits[3] = -math.inf                                       # none
    score = torch.tensor([[0.0, -math.inf, -math.inf], [-1.0, -2.0, -3.0], [0.0, 0.0, 0.0], [0.0, 0.0, 0.0]], device=DEV)
    check(logits, score, 12)
    new, parent, token = select(logits, score, 12)
    assert bool((parent[0] == 0).all()) and bool((token[0] % 2 == 1).all())
    assert int(token[2, 0]) == 5 and int(parent[2, 0]) == 7 and float(new[2, 0]) == 0.0 and int(token[2, 1]) == -1


def test_lowest_finite_logits_as_a_mask():
    logits = torch.full((2, 2, 700), torch.finfo(torch.float32).min, device=DEV)
    logits[:, 0, 123] = 2.0
    logits[:, 1, 600] = -3.0
    score = torch.tensor([[-1.0, -0.5], [-0.5, -1.0]], device=DEV)
    new, parent, token = select(logits, score, 2)
    assert token.tolist() == [[600, 123], [123, 600]] and parent.tolist() == [[1, 0], [2, 3]]
    assert torch.equal(new, torch.tensor([[-0.5, -1.0], [-0.5, -1.0]], device=DEV))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("order", ["rising", "falling", "late", "one_late"])
def test_logits_in_order(order, dtype):
    """Rows whose large logits come last (every chunk brings more candidates than there is room for), first, or behind tens of
    thousands of masked ones; long enough that a CTA goes through many chunks."""
    gen = torch.Generator(device=DEV).manual_seed(17)
    logits = torch.randn((90, 2, 70001), generator=gen, device=DEV).sort(-1, descending=order == "falling").values.to(dtype)
    if order in ("late", "one_late"):
        logits[..., : 60000] = -math.inf
    if order == "one_late":
        logits[..., : -1] = -math.inf
    check(logits, -torch.rand((90, 2), generator=gen, device=DEV), 24)


def test_padded_rows():
    gen = torch.Generator(device=DEV).manual_seed(3)
    whole = torch.full((2, 3, 1100), math.inf, device=DEV)
    whole[:, :, :1037] = torch.randn((2, 3, 1037), generator=gen, device=DEV)
    check(whole[:, :, :1037], torch.zeros((2, 3), device=DEV), 9)


def test_refusals():
    f = torch.zeros((1, 2, 64), device=DEV)
    score = torch.zeros((1, 2), device=DEV)
    i = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        B.swarm_beam_select(f.double(), score, ws, torch.zeros((1, 4), device=DEV), i, i.clone())
    with pytest.raises(ValueError):
        B.swarm_beam_select(f.transpose(1, 2), score, ws, torch.zeros((1, 4), device=DEV), i, i.clone())
    with pytest.raises(B.SwarmError) as e:
        B.swarm_beam_select(f, score, ws[:16], torch.zeros((1, 4), device=DEV), i, i.clone())
    assert e.value.code == B.ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("batch,beams,V,keep,dtype", [
    (1, 16, 131072, 64, torch.float32), (5, 16, 119450, 32, torch.bfloat16), (2, 7, 40001, 40, torch.float16), (3, 1, 250007, 64, torch.bfloat16)])
def test_many_candidates_for_a_prompt(batch, beams, V, keep, dtype):
    """Rows cut into many stretches: thousands to tens of thousands of candidates are left to the second kernel, many of equal value,
    once spread over the beams and once all of them in two."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    logits = (torch.randn((batch, beams, V), generator=gen, device=DEV) * 3).round().to(dtype)
    check(logits, torch.zeros((batch, beams), device=DEV), keep)
    logits = (torch.randn((batch, beams, V), generator=gen, device=DEV) * 3).to(dtype)
    score = torch.full((batch, beams), -30.0, device=DEV)
    score[:, -1] = -1.0
    score[:, 0] = -1.25
    check(logits, score, keep)


@pytest.mark.parametrize("order", ["rising", "falling", "random"])
def test_whole_rows_in_a_stretch(order):
    """More rows than the device holds CTAs: each is one stretch."""
    gen = torch.Generator(device=DEV).manual_seed(23)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn((330, 2, 36865), generator=gen, device=DEV) * 4
        if order != "random":
            x = x.sort(-1, descending=order == "falling").values
        check(x.to(dtype), -torch.rand((330, 2), generator=gen, device=DEV), 33)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch", [1, 20])
@pytest.mark.parametrize("lo,n", [(0, 2200), (0, 3100), (0, 3600), (0, 7000), (4096, 3600), (8192, 7000), (1, 20000)])
def test_blocks_of_nan_take_nothing_from_the_others(lo, n, batch, dtype):
    """A shard of the vocabulary that failed: threads with nothing but NaN beside threads with ordinary logits.  The best continuations
    stand right behind the block, in its chunk; with 1 and 20 prompts a chunk of 16-bit logits has 4096 and 8192 tokens.  Once with
    logits of both signs, once with log probabilities (all of them negative)."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    logits = torch.randn((batch, 3, 20011), generator=gen, device=DEV) * 3
    logits[:, :, lo + n: lo + n + 5] = torch.tensor([20.0, 24.0, 28.0, 22.0, 26.0], device=DEV)
    logits[:, :, lo: lo + n] = math.nan
    score = -torch.rand((batch, 3), generator=gen, device=DEV) * 5
    for keep in (4, 8, 40, 64):
        check(logits.to(dtype), score, keep)
        check((logits - 60).to(dtype), score, keep)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_blocks_of_nan_in_rising_rows(dtype):
    """Rows that bring more candidates than there is room for and are gone through once more, with blocks of NaN in several chunks."""
    gen = torch.Generator(device=DEV).manual_seed(29)
    x = (torch.randn((330, 2, 36865), generator=gen, device=DEV) * 4).sort(-1).values
    for lo, n in ((0, 3600), (8192, 7000), (20480, 3100), (32768, 3600)):
        x[:, :, lo: lo + n] = math.nan
    for keep, below in ((5, 0), (33, 60), (5, 60)):
        check((x - below).to(dtype), -torch.rand((330, 2), generator=gen, device=DEV), keep)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [50257, 8193, 37])
def test_the_logits_of_the_last_token(V, dtype):
    """A slice of a model's output: its first row starts anywhere in a 16-byte line.  What stands around it is +inf and NaN."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    for tokens in (2, 3, 4, 5):
        whole = torch.full((2, 3, tokens, V), math.inf, device=DEV, dtype=dtype)
        whole[:, :, : tokens - 2] = math.nan
        whole[:, :, -1] = (torch.randn((2, 3, V), generator=gen, device=DEV) * 3).to(dtype)
        logits = whole[:, :, -1]
        score = -torch.rand((2, 3), generator=gen, device=DEV)
        check(logits, score, 9)
        for a, b in zip(select(logits, score, 9), select(logits.contiguous(), score, 9)):
            assert torch.equal(a, b)
    rows = torch.zeros(4 * V + 64, device=DEV)
    out = torch.zeros((1, 1), device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for off in (1, 2, 3):                                        # not a whole number of elements
        assert B.load_library().swarm_beam_select(
            ctypes.c_void_p(rows.data_ptr() + off), 0, ctypes.c_int64(V), ctypes.c_void_p(out.data_ptr()), 1, 1, V, 1, ctypes.c_void_p(ws.data_ptr()),
            ctypes.c_int64(ws.numel()), *[ctypes.c_void_p(out.data_ptr())] * 3, ctypes.c_void_p(0)) == B.ERR_INVALID_ARG
