"""Beam selection where a slice of a row is several steps of 4096 logits long, against the definition in 64 bits: masked, banned, shifted, rising
and infinite logits at every place of a slice."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def sw():
    from paper_2603_17803_amd import binding
    s = binding.Swarm(0)
    yield s
    assert s.device_status() == 0
    s.close()


def reference(logits, scores, k):
    """Of each beam: all scores in 64 bits, its normaliser's allowance, and its best k tokens in order; of each group: (score, parent, token)."""
    B, K, V = logits.shape
    x = logits.double()
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.max(-1, keepdim=True).values
    w = (x - top).exp()
    z = w.sum(-1, keepdim=True)
    s = scores.double()[..., None] + (x - (top + z.log()))
    s = torch.where(s.isnan(), -math.inf, s)
    # The logarithm of a sum of exponentials in fp32: 2^-23 of each for the function, seven additions of half a step, and its argument, t octaves from
    # what it refers to, rounded twice.  t is at most 8 above that, and below it at most what the logit stands below the row's largest one.
    octaves = (torch.where(w > 0, w * (top - x), 0.0).sum(-1) / z[..., 0] / math.log(2)).nan_to_num(nan=0.0)
    tol = 2.0 ** -24 * (9 + 1.4 * (8 + octaves))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k]
    want = np.full((B, k), -np.inf), np.full((B, k), -1), np.full((B, k), -1)
    s_best, x_best = torch.gather(s, -1, order).numpy(), torch.gather(x, -1, order).numpy()
    order = order.numpy()
    for b in range(B):
        found = [(s_best[b, j, i], j, x_best[b, j, i], int(order[b, j, i])) for j in range(K) for i in range(order.shape[-1])]
        found.sort(key=lambda c: (-c[0], c[1], -c[2], c[3]))
        for i, c in enumerate(found[:k]):
            want[0][b, i], want[1][b, i], want[2][b, i] = c[0], b * K + c[1], c[3]
    return s.numpy().reshape(B * K, V), tol.numpy().reshape(B * K), want


def check(sw, logits, scores, k):
    B, K, V = logits.shape
    got = sw.beam_select(logits.cuda(), scores.cuda(), k)
    torch.cuda.synchronize()
    score, parent, token = (x.cpu().numpy() for x in got)
    s, tol, want = reference(logits, scores, k)
    assert (parent >= 0).all() and (token >= 0).all() and (token < V).all() and len({*zip(parent.ravel(), token.ravel())}) == B * k
    chosen, allowed = s[parent, token], tol[parent]
    same = (parent == want[1]) & (token == want[2])
    # beams whose scores are nearer than their normalisers are known may change places, nothing else
    near = np.isfinite(chosen) & np.isfinite(want[0]) & (np.abs(np.where(np.isfinite(chosen), chosen, 0) - np.where(np.isfinite(want[0]), want[0], 0)) <= 2 * allowed) & (parent != want[1])
    assert (same | near).all(), f"{int((~(same | near)).sum())} of {same.size} choices differ"
    full = np.isfinite(chosen)
    assert np.array_equal(score[~full], chosen[~full].astype(np.float32))
    off = np.abs(score[full].astype(np.float64) - chosen[full]) - 2.0 ** -24 * np.abs(chosen[full])
    assert (off <= allowed[full]).all(), f"scores off by {off.max():.3g}, {(off / allowed[full]).max():.3g} of what is allowed"


# rows and sizes whose slices are 3, 5, 3 and 2 steps long, the first two with rows that start off the vector alignment
SIZES = [(64, 8, 20001, 16), (16, 64, 20011, 5), (1, 2, 600000, 40), (2, 64, 60000, 128)]


def noise(seed, B, K, V, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, K, V), generator=g) * spread, torch.randn((B, K), generator=g) * 2 - 20


def leads(B, K, V):
    """Where a slice's first step stands, and a little behind it."""
    rows = B * K
    J = min(-(-1024 // rows), -(-(V + 8) // 4096), 64)
    at = torch.arange(V)
    return at % -(-V // J) < 4200


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,K,V,k", SIZES)
def test_plain(sw, dtype, B, K, V, k):
    logits, scores = noise(1, B, K, V)
    check(sw, logits.to(TYPES[dtype]), scores, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,K,V,k", SIZES)
def test_first_tokens_banned(sw, dtype, B, K, V, k):
    """Each slice starts with banned tokens; of the others some are allowed, far above."""
    logits, scores = noise(2, B, K, V)
    allowed = torch.rand(V, generator=torch.Generator().manual_seed(3)) < 0.02
    logits[..., leads(B, K, V) | ~allowed] = -100.0
    check(sw, logits.to(TYPES[dtype]), scores, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_rising_in_steps(sw, dtype):
    """Very low ones, a few high ones, then many between: these are no candidates, and far above what came first."""
    B, K, V, k = SIZES[0]
    logits, scores = noise(4, B, K, V, 0.5)
    logits += 5.0
    for low in (-1e4, -60000.0):
        for at in (0, -(-V // 2)):                                                         # the two slices of a row
            logits[..., at:at + 8200] = low
            logits[..., at + 5000:at + 5100] = 10.0 + 0.01 * torch.arange(100)
        check(sw, logits.to(TYPES[dtype]), scores, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("level", [-30.0, -100.0, -500.0, -1000.0, 200.0])
@pytest.mark.parametrize("size", [0, 2])
def test_first_tokens_masked_and_the_others_low(sw, dtype, level, size):
    """Nothing finite in a slice's first step, and what follows far from 0."""
    B, K, V, k = SIZES[size]
    logits, scores = noise(5, B, K, V, 1.0)
    logits += level
    logits[..., leads(B, K, V)] = -math.inf
    check(sw, logits.to(TYPES[dtype]), scores, k)
    # few tokens at all, in some slices none
    few = torch.rand(V, generator=torch.Generator().manual_seed(6)) < 2e-4
    few[-3:] = True
    logits[..., ~few] = -math.inf
    logits[..., :] = torch.where(few, torch.where(logits.isinf(), level, logits), logits)
    check(sw, logits.to(TYPES[dtype]), scores, 2)


@pytest.mark.parametrize("shift", [300.0, -3000.0, 30000.0])
def test_a_shift_of_all_logits_changes_no_score(sw, shift):
    for dtype in ("fp32", "fp16"):
        B, K, V, k = SIZES[0]
        logits, scores = noise(7, B, K, V)
        check(sw, (logits + shift).to(TYPES[dtype]), scores, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_rising_and_falling(sw, dtype):
    for size in (0, 3):
        B, K, V, k = SIZES[size]
        scores = noise(8, B, K, 1)[1]
        up = (torch.arange(V, dtype=torch.float32) * (400.0 / V) - 300).expand(B, K, V).contiguous().to(TYPES[dtype])
        check(sw, up, scores, k)
        check(sw, up.flip(-1).contiguous(), scores, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_equal_logits_below_one(sw, dtype):
    """One token above many alike: all of the sum's rounding points one way."""
    B, K, V, k = SIZES[0]
    for gap in (3.3, 9.7, 30.0):
        logits = torch.full((B, K, V), 12.3 - gap)
        logits[..., 15000], logits[..., 17] = 12.3, 12.2 - gap
        check(sw, logits.to(TYPES[dtype]), noise(9, B, K, 1)[1], k)


@pytest.mark.parametrize("size", [0, 2])
def test_values_that_are_not_numbers(sw, size):
    B, K, V, k = SIZES[size]
    logits, scores = noise(10, B, K, V)
    flat = logits.view(B * K, V)
    lead = leads(B, K, V)
    at = int(torch.nonzero(~lead)[100])
    flat[0, at] = math.nan
    flat[1, at] = math.inf
    check(sw, logits, scores, k)
    flat[0, lead], flat[1] = -math.inf, -math.inf
    check(sw, logits, scores, k)
    if B * K > 16:
        flat[2, at], flat[3, at] = 3e38, 1e30
        flat[4, lead], flat[5, lead], flat[6, lead] = -1e30, -3e38, 1e6
        flat[7], flat[8], flat[9] = 3e38, -3e38, -torch.finfo(torch.float32).max
        flat[10, ~lead] = math.nan
        flat[11, lead], flat[11, ~lead] = -math.inf, -3e38
        flat[12, lead], flat[12, ~lead] = -math.inf, -2.3e38
        flat[13, lead], flat[13, at] = -math.inf, math.inf
        scores[2] = math.inf
        scores[3, 1] = math.nan
        check(sw, logits, scores, k)


@pytest.mark.parametrize("B,K,V", [(3, 16, 300), (3, 17, 300), (64, 16, 5000), (2, 2, 30000), (1, 1, 68000)])
@pytest.mark.parametrize("k", [3, 4, 31, 128])
def test_sixteen_lists_and_seventeen(sw, B, K, V, k):
    """Either side of how many lists are merged at once."""
    logits, scores = noise(K + k, B, K, V)
    check(sw, logits, scores, k)
    check(sw, torch.round(logits), torch.zeros_like(scores), k)
    check(sw, logits[:, :1].expand(B, K, V).contiguous(), torch.zeros_like(scores), k)
    logits[0, K - 1], scores[0, 0] = -math.inf, -math.inf
    check(sw, logits, scores, k)
