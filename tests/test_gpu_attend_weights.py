"""Attention over a paged cache where small weights decide, and where nothing is weighed: every stream's row holds the same pages, so that one part of
the work is a whole long context."""
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
