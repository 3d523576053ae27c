"""Attention over a paged cache where small weights decide, and infinite values that are weighed: every stream's row holds the same pages, so that
one part of the work is a whole long context."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def sw():
    from paper_2603_17803_amd import binding
    s = binding.Swarm(0)
    yield s
    assert s.device_status() == 0
    s.close()


def shared_rows(k, v, B, page=16):
    """A cache of B rows that all hold the n keys k, v [n][d] of one head."""
    from paper_2603_17803_amd import binding
    n, d = k.shape
    pages = -(-n // page)
    pool = [torch.zeros((pages * page, d), dtype=k.dtype) for _ in range(2)]
    pool[0][:n], pool[1][:n] = k, v
    pool = [x.view(1, pages, 1, page, d).cuda() for x in pool]
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(B, pages).contiguous()
    return binding.Cache(pool[0], pool[1], table, torch.full((B,), n, dtype=torch.int32, device="cuda"))


def attend(sw, cache, q, **more):
    out, lse = sw.tree_attend(cache, 0, q.cuda(), scale=1.0, want_lse=True, **more)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 136])
@pytest.mark.parametrize("T,G", [(1, 4), (1, 16), (4, 8), (10, 4), (16, 8), (32, 8)])
@pytest.mark.parametrize("gap,spread", [(10.0, 0.0), (14.0, 0.0), (16.0, 0.0), (17.4, 0.0), (18.0, 1.5), (20.0, 0.0)])
def test_one_key_far_above_many(sw, dtype, d, T, G, gap, spread):
    """A key that nearly all weight goes to and whose value is small, as the first token of a text often is: what the many others bring counts.

    The error against 64 bits, in units of sum p |v|: half a step of the type for the result's rounding, and for the weights where they are
    rounded once (more than 32 rows, 16 of wide heads), else four half steps squared; for the score, one product, its rounding in units of ln 2, the
    difference and the exponential: 2^-24 of 3 s / ln 2 and 2^-22 at most; fp32 additions: of the weights a lane has a fourth, of the products the
    matrix cores add 32 at a time.  And fp16 ends at 2^-24, so that a weight may be off by half of that, or by all of it where it enters as two terms, the
    largest being 2^11 at least."""
    t, n, B = TYPES[dtype], 131072, 260 if T * G > 32 else 520
    g = torch.Generator().manual_seed(int(gap * 10) + T * G)
    k, v = torch.zeros((n, d), dtype=t), torch.ones((n, d), dtype=t)
    k[:, 0] = (torch.randn(n, generator=g) * spread).to(t)
    k[1::2, 1] = 0.001
    sink = 70001
    k[sink] = 0
    k[sink, 0] = gap
    v[sink] = 0.01
    v[:, 3] = torch.randn(n, generator=g).to(t)
    q = torch.zeros((B, T, G, d), dtype=t)
    q[..., 0] = 1.0
    q[..., 1] = torch.rand((B, T, G), generator=g).to(t)
    out, lse = attend(sw, shared_rows(k, v, B), q)
    half = torch.finfo(t).eps / 2
    one = T * G > (16 if d > 128 else 32)
    for b, i, h in [(0, 0, 0), (1, T - 1, G - 1), (B // 2, T // 2, 1), (B - 1, 0, G // 2)]:
        s = k.double() @ q[b, i, h].double()
        p = (s - s.max()).exp()
        w = p / p.sum()
        want, mass = w @ v.double(), w @ v.double().abs()
        e = 2.0 ** -24 * 3 * s.abs().max().item() / math.log(2) + 2.0 ** -22
        rel = 2 * e + (half if one else 4 * half * half) + (n / 4 + 64 + n / 32) * 2.0 ** -24
        flat = n * 2.0 ** (-36 if one else -35) * v.double().abs().max(0).values / p.sum() if dtype == "fp16" else 0.0
        tol = half * 1.01 * want.abs() + rel * mass + flat + torch.finfo(t).tiny * half
        bad = (out[b, i, h].double() - want).abs() / tol
        assert (bad <= 1).all(), f"off by {bad.max():.3g} tolerances, {((out[b, i, h].double() - want).abs() / want.abs()).max():.3g} of the value"
        assert abs(float(lse[b, i, h]) - (s.max() + p.sum().log()).item()) <= e + (n / 4 + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + gap)


def gaps(octaves, count, t):
    """Keys' first channel for scores between two numbers of octaves below 0, whole octaves among them."""
    g = torch.Generator().manual_seed(count)
    x = torch.rand(count, generator=g) * (octaves[1] - octaves[0]) + octaves[0]
    x[::4] = x[::4].round()
    return (-x * math.log(2)).to(t)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("T,G,d", [(1, 4, 64), (1, 32, 64), (10, 4, 64), (24, 8, 64), (1, 4, 256), (5, 4, 256)])
def test_infinite_values_of_the_context_that_weigh_little(sw, dtype, T, G, d):
    """An infinite value of a weight down to 2^-22 of the largest makes the result infinite: fp16 holds a weight from 2^-24 on, the largest being 2^11 at least."""
    from paper_2603_17803_amd import binding
    t, B, page = TYPES[dtype], 200, 16
    k = torch.zeros((1, B, 1, page, d), dtype=t)
    k[0, :, 0, 5, 0] = gaps((1, 22), B, t)
    v = torch.ones((1, B, 1, page, d), dtype=t)
    v[0, :, 0, 5, 2], v[0, :, 0, 5, 3] = math.inf, -math.inf
    q = torch.zeros((B, T, G, d), dtype=t)
    q[..., 0] = 1.0
    table = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    out, _ = attend(sw, binding.Cache(k.cuda(), v.cuda(), table, torch.full((B,), page, dtype=torch.int32, device="cuda")), q)
    assert (out[..., 2] == math.inf).all() and (out[..., 3] == -math.inf).all()
    assert ((out[..., 4].double() - 1.0).abs() <= 2 * torch.finfo(t).eps).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 200])
def test_infinite_values_of_drafted_tokens_that_weigh_little(sw, dtype, d):
    """Infinite from any weight that the type holds, never finite where it is seen, and nothing to those who do not see it."""
    t, B, T, G = TYPES[dtype], 200, 6, 3
    n = 40
    cache = shared_rows(torch.zeros((n, d), dtype=t), torch.ones((n, d), dtype=t), B)
    k_new, v_new = torch.zeros((B, T, 1, d), dtype=t), torch.ones((B, T, 1, d), dtype=t)
    q = torch.zeros((B, T, G, d), dtype=t)
    q[..., 0] = 1.0
    sees = torch.tensor([1 << i | (1 << 2 if i in (2, 4, 5) else 0) for i in range(T)], dtype=torch.int32).expand(B, T).contiguous().view(B, T, 1)
    for octaves, held in (((1, 22), True), ((22, 60), False), ((200, 300), False)):
        k_new[:, 2, 0, 0] = gaps(octaves, B, t)
        v_new[:, 2, 0, 2] = math.inf
        out, _ = attend(sw, cache, q, k_new=k_new.cuda(), v_new=v_new.cuda(), mask=sees.cuda())
        seen = out[:, [2, 4, 5], :, 2]
        assert (seen == math.inf).all() if held else ((seen == math.inf) | seen.isnan()).all()
        finite = out.clone()
        finite[:, [2, 4, 5], :, 2] = 1.0
        assert ((finite.double() - 1.0).abs() <= 2 * torch.finfo(t).eps).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("T,G,d", [(1, 4, 64), (10, 8, 64), (3, 2, 256), (70, 1, 64), (70, 2, 136)])
def test_infinite_values_among_weights_that_are_nothing(sw, dtype, T, G, d):
    """Keys of which 32 in a row weigh 2^-250 of the others, one with an infinite value: never finite, in the context or among the drafted tokens."""
    t, n = TYPES[dtype], 130
    far = -250 * math.log(2)
    k, v = torch.zeros((n, d), dtype=t), torch.ones((n, d), dtype=t)
    k[32:64, 0], v[40, 2] = far, math.inf
    q = torch.zeros((2, T, G, d), dtype=t)
    q[..., 0] = 1.0
    more = {}
    if T > 64:
        k_new, v_new = torch.zeros((2, T, 1, d), dtype=t), torch.ones((2, T, 1, d), dtype=t)
        k_new[:, 32:64, 0, 0], v_new[:, 50, 0, 3] = far, -math.inf
        more = dict(k_new=k_new.cuda(), v_new=v_new.cuda())
    for B in (1, 2):
        out, _ = attend(sw, shared_rows(k, v, B), q[:B].contiguous(), **{x: y[:B].contiguous() for x, y in more.items()})
        assert not out[..., 2].isfinite().any()
        if T > 64:
            assert out[:, :50, :, 3].isfinite().all() and not out[:, 50:, :, 3].isfinite().any()
        rest = out[..., [0, 1] + list(range(4, d))]
        assert ((rest.double() - 1.0).abs() <= 2 * torch.finfo(t).eps).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("T,G,d", [(1, 4, 64), (10, 8, 64), (3, 2, 256), (20, 4, 256)])
@pytest.mark.parametrize("where", ["context", "drafted", "both"])
def test_scores_of_minus_infinity_alone(sw, dtype, T, G, d, where):
    """What a token sees may all score -inf, values infinite or not: 0, and -inf for lse."""
    t, B = TYPES[dtype], 3
    low = torch.zeros((40, d), dtype=t)
    low[:, 0] = -math.inf
    v = torch.ones((40, d), dtype=t)
    v[7, 2], v[33, 5] = math.inf, math.nan
    cache = shared_rows(low, v, B)
    if where == "drafted":
        cache = cache._replace(length=torch.zeros_like(cache.length))
    q = torch.zeros((B, T, G, d), dtype=t)
    q[..., 0] = 1.0
    more = {}
    if where != "context":
        k_new, v_new = torch.zeros((B, T, 1, d), dtype=t), torch.ones((B, T, 1, d), dtype=t)
        k_new[..., 0], v_new[:, 0, 0, 2] = -math.inf, math.inf
        more = dict(k_new=k_new.cuda(), v_new=v_new.cuda())
    out, lse = attend(sw, cache, q, **more)
    assert (lse == -math.inf).all() and (out == 0).all()
