"""Beam search's selection against a plain implementation in 64 bits: choices exactly, scores within one rounding."""
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


def reference(logits, scores, k, finished=None, eos=-1):
    """(score, parent, token) of each group from all its candidates, sorted as the definition says."""
    B, K, V = logits.shape
    x = logits.double().numpy()
    x = np.where(np.isnan(x), -np.inf, x)
    out = np.full((B, k), -np.inf), np.full((B, k), -1, dtype=np.int64), np.full((B, k), -1, dtype=np.int64)
    for b in range(B):
        found = []
        for j in range(K):
            base = float(scores[b, j])
            if finished is not None and finished[b, j]:
                found.append((-np.inf if math.isnan(base) else base, j, 0.0, eos))
                continue
            row = x[b, j]
            with np.errstate(all="ignore"):
                m = row.max()
                z = m + np.log(np.exp(row - m).sum())
                s = base + (row - z)
            s = np.where(np.isnan(s), -np.inf, s)
            for t in np.lexsort((np.arange(V), -row))[:k]:
                found.append((s[t], j, row[t], int(t)))
        found.sort(key=lambda c: (-c[0], c[1], -c[2], c[3]))
        for i, c in enumerate(found[:k]):
            out[0][b, i], out[1][b, i], out[2][b, i] = c[0], b * K + c[1], c[3]
    return out


def check(sw, logits, scores, k, finished=None, eos=-1, vocab=None):
    got = sw.beam_select(logits.cuda(), scores.cuda(), k, finished=None if finished is None else finished.cuda(), eos=eos, vocab=vocab)
    torch.cuda.synchronize()
    score, parent, token = reference(logits[..., :vocab] if vocab else logits, scores, k, finished, eos)
    assert np.array_equal(got[1].cpu().numpy(), parent) and np.array_equal(got[2].cpu().numpy(), token)
    s = got[0].cpu().double().numpy()
    full = np.isfinite(score)
    assert np.array_equal(s[~full], score[~full])
    # one rounding to fp32 of the score, and a logarithm of a sum of exponentials good to 2^-22
    assert (np.abs(s - score)[full] <= 2.0 ** -24 * np.abs(score[full]) + 2.0 ** -22).all()
    return got


def random(seed, B, K, V, dtype, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((B, K, V), generator=g) * spread).to(TYPES[dtype]), torch.randn((B, K), generator=g) * 2 - 20


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,K,V,k", [(1, 1, 1, 1), (2, 3, 7, 4), (3, 4, 63, 8), (1, 2, 64, 5), (2, 5, 65, 10), (1, 8, 1023, 16), (2, 2, 1024, 2), (1, 3, 1025, 3), (3, 4, 4099, 8), (2, 8, 8192, 16),
                                     (1, 4, 8193, 8), (2, 3, 32001, 6), (1, 64, 500, 128), (1, 1, 70001, 128), (4, 2, 16385, 1)])
def test_ragged_vocabularies(sw, dtype, B, K, V, k):
    check(sw, *random(V + k, B, K, V, dtype), k)


@pytest.mark.parametrize("V", [100, 9000])
def test_ties_go_to_the_lower_beam_and_token(sw, V):
    logits, scores = random(1, 2, 4, V, "fp32")
    check(sw, torch.zeros_like(logits), torch.zeros_like(scores), 9)                       # all alike
    check(sw, torch.round(logits), torch.zeros_like(scores), 40)                           # few distinct values
    same = logits[:, :1].expand(2, 4, V).contiguous()
    check(sw, same, torch.zeros_like(scores), 8)                                           # beams alike
    check(sw, same, torch.tensor([[0.0, -math.inf, -math.inf, -math.inf]] * 2), 8)         # the first step: one beam counts
    signed = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0).expand(2, 4, V).contiguous()
    check(sw, signed, torch.zeros_like(scores), 8)                                         # -0 is 0


def test_ascending_and_descending_logits(sw):
    """All the best tokens in one place."""
    for V in (5000, 40000):
        up = torch.arange(V, dtype=torch.float32).mul(1e-3).expand(1, 2, V).contiguous()
        scores = torch.tensor([[-1.0, -1.003]])
        check(sw, up, scores, 100)
        check(sw, up.flip(-1).contiguous(), scores, 100)
        lump = torch.full((1, 2, V), -5.0)
        lump[..., 1000:1130] = torch.linspace(0, 3, 130)
        check(sw, lump, scores, 128)
        check(sw, torch.cat([lump[..., 4:], lump[..., :4]], -1).contiguous(), scores, 128)


def test_values_that_are_not_numbers(sw):
    for V in (300, 9000):
        logits, scores = random(V, 3, 4, V, "fp32")
        logits[0, 1, ::2] = math.nan
        logits[0, 2] = -math.inf                                                           # a beam without a token
        logits[1, 0, 5] = math.inf
        logits[1, 1] = math.nan
        scores[1, 3] = math.nan
        scores[2, :2] = -math.inf
        scores[2, 3] = math.inf
        logits[2, 2, :] = -math.inf
        logits[2, 2, V - 1] = 1e30
        check(sw, logits, scores, 12)
    every = torch.full((1, 2, 50), math.nan)
    check(sw, every, torch.zeros(1, 2), 20)
    check(sw, torch.full((1, 2, 50), 3e38), torch.zeros(1, 2), 3)


def test_finished_beams(sw):
    for dtype, V in (("fp32", 400), ("bf16", 20000)):
        logits, scores = random(V, 4, 5, V, dtype)
        done = torch.zeros((4, 5), dtype=torch.uint8)
        done[0, 1], done[1], done[2, [0, 4]] = 1, 1, 7
        scores[2, 4] = -math.inf
        scores[0, 1] = -2.0                                                                # finished and ahead
        got = check(sw, logits, scores, 10, done, eos=V - 1)
        assert (got[1][1, 5:] == -1).all() and (got[2][1, 5:] == -1).all() and (got[0][1, 5:] == -math.inf).all()


def test_padded_rows(sw):
    """A vocabulary padded to a longer row: the padding is not looked at."""
    for dtype in TYPES:
        for V, stride in ((50, 51), (1000, 1024), (8190, 8192), (20001, 20008)):
            logits, scores = random(V, 2, 3, stride, dtype)
            logits[..., V:] = 50.0
            check(sw, logits, scores, 6, vocab=V)


def test_rows_off_the_vector_alignment(sw):
    """Logits that start at any element, rows of odd length: nothing in front of them or behind is looked at."""
    for dtype, t in TYPES.items():
        for shift in (1, 3, 5):
            logits, scores = random(shift, 2, 3, 9001, dtype)
            flat = torch.full((logits.numel() + 16,), 60.0, dtype=t, device="cuda")
            view = flat[shift:shift + logits.numel()].view(logits.shape)
            view.copy_(logits)
            got = sw.beam_select(view, scores.cuda(), 7)
            want = sw.beam_select(logits.cuda(), scores.cuda(), 7)
            assert all(torch.equal(x, y) for x, y in zip(got, want))
            check(sw, logits, scores, 7)


@pytest.mark.parametrize("step", [0, 1, 63, 500, 1023])
def test_histories(sw, step):
    logits, scores = random(step, 2, 3, 700, "fp32")
    hist = torch.randint(0, 700, (2, 3, 1024), dtype=torch.int32)
    done = torch.zeros((2, 3), dtype=torch.uint8)
    done[1] = 1
    for k in (3, 6):
        out = torch.full((2, k, 1024), -5, dtype=torch.int32, device="cuda")
        _, parent, token = sw.beam_select(logits.cuda(), scores.cuda(), k, finished=done.cuda(), eos=2, hist=hist.cuda(), step=torch.tensor([step], dtype=torch.int32).cuda(), hist_out=out)
        parent, token = parent.cpu().long(), token.cpu()
        want = torch.full((2, k, 1024), -5, dtype=torch.int32)
        for b in range(2):
            for i in range(k):
                if parent[b, i] >= 0:
                    want[b, i, :step] = hist.view(6, 1024)[parent[b, i], :step]
                    want[b, i, step] = token[b, i]
        assert (parent[1, 3:] == -1).all()
        assert torch.equal(out.cpu(), want)


def test_a_step_outside_the_history(sw):
    from paper_2603_17803_amd import binding as b
    logits, scores = random(1, 1, 2, 50, "fp32")
    hist = torch.arange(16, dtype=torch.int32).view(1, 2, 8).cuda()
    for step, upto in ((-3, 0), (8, 8), (2 ** 31 - 1, 8)):
        out = torch.full((1, 2, 8), -5, dtype=torch.int32, device="cuda")
        _, parent, _ = sw.beam_select(logits.cuda(), scores.cuda(), 2, hist=hist, step=torch.tensor([step], dtype=torch.int32).cuda(), hist_out=out)
        assert sw.device_status() == b.SWARM_DEV_BAD_ENTRY
        assert (out[..., upto:] == -5).all()
        assert torch.equal(out[0, :, :upto], hist[0, parent[0].long(), :upto])


def test_refusals(sw):
    from paper_2603_17803_amd import binding as b
    logits, scores = (x.cuda() for x in random(2, 2, 3, 40, "fp32"))
    score, parent, token = (torch.zeros((2, 4), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32))
    done = torch.zeros((2, 3), dtype=torch.uint8, device="cuda")
    hist, step, hist_out = torch.zeros((6, 8), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((8, 8), dtype=torch.int32, device="cuda")
    names = ("logits", "dtype", "stride", "scores", "finished", "eos", "B", "K", "V", "k", "score", "parent", "token", "hist", "step", "cap", "hist_out")
    p = lambda x: x.data_ptr()  # noqa: E731
    base = dict(logits=p(logits), dtype=b.SWARM_FP32, stride=40, scores=p(scores), finished=None, eos=-1, B=2, K=3, V=40, k=4, score=p(score), parent=p(parent), token=p(token), hist=None, step=None,
                cap=0, hist_out=None)
    call = lambda **kw: b.swarm_beam_select(sw.ctx, *[{**base, **kw}[n] for n in names])  # noqa: E731
    full = dict(hist=p(hist), step=p(step), cap=8, hist_out=p(hist_out))
    assert call() == b.SWARM_OK and call(**full) == b.SWARM_OK and call(finished=p(done), eos=0) == b.SWARM_OK
    torch.cuda.synchronize()
    before = [x.clone() for x in (score, parent, token, hist_out)]
    for kw in [dict(logits=None), dict(scores=None), dict(score=None), dict(parent=None), dict(token=None), dict(dtype=3), dict(dtype=-1), dict(stride=39), dict(stride=1 << 41), dict(B=0), dict(K=0), dict(K=65),
               dict(V=0), dict(V=(1 << 24) + 1, stride=1 << 25), dict(k=0), dict(k=129), dict(B=1 << 20), dict(finished=p(done), eos=40), dict(finished=p(done), eos=-1), dict(logits=p(logits) + 2),
               dict(score=p(scores)), dict(parent=p(score)), dict(token=p(logits) + 64), {**full, "cap": 0}, {**full, "step": None}, {**full, "hist": None}, {**full, "hist_out": None}, {**full, "hist_out": p(hist)},
               {**full, "cap": 1 << 29}, dict(parent=p(parent) + 2)]:
        assert call(**kw) == b.SWARM_EINVAL, kw
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, (score, parent, token, hist_out)))
    for f in [lambda: sw.beam_select(logits[0], scores, 4), lambda: sw.beam_select(logits.double(), scores, 4), lambda: sw.beam_select(logits, scores[:1], 4), lambda: sw.beam_select(logits, scores, 4, finished=done.int()),
              lambda: sw.beam_select(logits, scores, 4, hist=hist.view(2, 3, 8)), lambda: sw.beam_select(logits, scores, 3, out=(score, parent, token))]:
        with pytest.raises(ValueError):
            f()


def test_recorded_calls_replay(sw):
    from paper_2603_17803_amd import binding as b
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s = b.Swarm(0, stream=stream)
        logits, scores = (x.cuda() for x in random(9, 2, 4, 20000, "bf16"))
        out = tuple(torch.zeros((2, 8), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32))
        s.beam_select(logits, scores, 8, out=out)
        stream.synchronize()
        s.capture_begin()
        s.beam_select(logits, scores, 8, out=out)
        graph = s.capture_end()
        for seed in range(4):
            x, y = (z.cuda() for z in random(seed, 2, 4, 20000, "bf16"))
            logits.copy_(x), scores.copy_(y)
            s.graph_launch(graph)
            stream.synchronize()
            got = [z.clone() for z in out]
            assert all(torch.equal(u, v) for u, v in zip(got, s.beam_select(x, y, 8)))
        b.swarm_graph_destroy(graph)
        s.close()


def test_a_generation_of_beams_over_a_cache(sw):
    """The calls as a program makes them: attention over the beams' rows, the token into the cache, the next tokens chosen, the rows
    reordered.  Checked against the same generation on plain lists of keys and values."""
    from paper_2603_17803_amd import binding as b
    rng = np.random.default_rng(5)
    K, H, G, d, page, P, cap, V, prompt = 4, 2, 2, 32, 4, 64, 12, 97, 9
    t = torch.bfloat16
    emb = [torch.randn((V, n, d), generator=torch.Generator().manual_seed(i)).to(t) for i, n in enumerate((H * G, H, H))]
    head = torch.randn((H * G * d, V), generator=torch.Generator().manual_seed(7))
    zero = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = b.Cache(torch.full((1, P, H, page, d), math.nan, dtype=t, device="cuda"), torch.full((1, P, H, page, d), math.nan, dtype=t, device="cuda"), zero(K, cap) - 1, zero(K), zero(P))
    first = torch.from_numpy(rng.integers(0, V, size=prompt))
    # the prompt goes into row 0, which every beam then starts from
    cache = sw.cache_fork(cache, torch.arange(K, dtype=torch.int32, device="cuda"), torch.tensor([prompt, 0, 0, 0], dtype=torch.int32, device="cuda"))
    cache = sw.cache_append(cache, emb[1][first][None, None].cuda(), emb[2][first][None, None].cuda())
    cache = sw.cache_fork(cache, zero(K), zero(K) + 1)
    rows = [[int(x) for x in first] for _ in range(K)]
    scores = torch.tensor([[0.0] + [-math.inf] * (K - 1)], device="cuda")
    token = torch.full((K,), 3, dtype=torch.int64)
    hist, step = zero(1, K, 16), 0
    for step in range(8):
        q, kn, vn = (e[token][:, None].contiguous().cuda() for e in emb)
        out, lse = sw.tree_attend(cache, 0, q, kn, vn, want_lse=True)
        for r in range(K):
            seq = rows[r] + [int(token[r])]
            for h in range(H * G):
                s = emb[1][seq, h // G].double() @ emb[0][int(token[r]), h].double() * d ** -0.5
                w = torch.softmax(s, 0)
                ref = w @ emb[2][seq, h // G].double()
                # half a step of bf16 of the result, and fp32 sums of at most 20 terms of a few units
                assert ((out[r, 0, h].cpu().double() - ref).abs() <= ref.abs() * 2.0 ** -8 + 2.0 ** -13 * (w @ emb[2][seq, h // G].double().abs())).all()
        cache = sw.cache_append(cache, kn[None], vn[None])
        logits = (out.float().cpu().reshape(K, -1) @ head * 0.05).reshape(1, K, V)
        nxt = zero(1, K, 16)
        new_scores, parent, chosen = sw.beam_select(logits.cuda(), scores, K, hist=hist, step=torch.tensor([step], dtype=torch.int32, device="cuda"), hist_out=nxt)
        want = reference(logits, scores.cpu(), K)
        assert np.array_equal(parent.cpu().numpy(), want[1]) and np.array_equal(chosen.cpu().numpy(), want[2])
        rows = [rows[p] + [int(token[p])] for p in want[1][0]]
        cache = sw.cache_fork(cache, parent.reshape(K), zero(K) + 1)
        scores, hist, token = new_scores, nxt, chosen.cpu().reshape(K).long()
        assert cache.length.tolist() == [len(r) for r in rows]
        held = [[int(x) for x in r if x >= 0] for r in cache.table.cpu().numpy()]
        counts = np.bincount([x for r in held for x in r], minlength=P)
        assert np.array_equal(cache.refs.cpu().numpy(), counts)
        for r in range(K):
            for i, tok in enumerate(rows[r]):
                assert torch.equal(cache.k[0, held[r][i // page], :, i % page].cpu(), emb[1][tok])
                assert torch.equal(cache.v[0, held[r][i // page], :, i % page].cpu(), emb[2][tok])
        if step == 4:
            cache, live = sw.cache_compact(cache)
            assert int(live) == int((counts > 0).sum())
    assert sw.device_status() == 0


def test_fewer_beams_are_recorded_after_more(sw):
    """No call with fewer groups, beams, tokens or candidates needs more scratch than the larger one before it."""
    from paper_2603_17803_amd import binding as b
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s = b.Swarm(0, stream=stream)
        s.beam_select(*(x.cuda() for x in random(1, 16, 64, 50000, "bf16")), 32)
        for B, K, V, k in [(15, 64, 50000, 32), (16, 63, 50000, 32), (1, 1, 50000, 32), (4, 64, 40000, 16), (16, 64, 300, 32)]:
            logits, scores = (x.cuda() for x in random(B + K, B, K, V, "bf16"))
            out = tuple(torch.zeros((B, k), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32))
            stream.synchronize()
            s.capture_begin()
            s.beam_select(logits, scores, k, out=out)
            graph = s.capture_end()
            for _ in range(2):
                s.graph_launch(graph)
                stream.synchronize()
                assert all(torch.equal(u, v) for u, v in zip(out, s.beam_select(logits, scores, k)))
                [x.zero_() for x in out]
            b.swarm_graph_destroy(graph)
        s.close()


@pytest.mark.parametrize("K,V", [(24, 300), (25, 300), (3, 30000), (6, 14000), (7, 14000), (1, 60000), (64, 100)])
@pytest.mark.parametrize("k", [3, 4, 7, 33, 128])
def test_lists_merged_at_once_and_in_rounds(sw, K, V, k):
    """Either side of the sizes that merge at once: plain, beams alike, some finished, some without a finite logit, NaN scores."""
    logits, scores = random(K + k, 2, K, V, "fp32")
    check(sw, logits, scores, k)
    same = logits[:, :1].expand(2, K, V).contiguous()
    check(sw, same, torch.zeros_like(scores), k)
    check(sw, torch.zeros_like(logits), torch.zeros_like(scores), k)
    done = (torch.arange(2 * K).reshape(2, K) % 3 == 1).to(torch.uint8)
    scores[0, 0], scores[1, K // 2] = math.nan, -math.inf
    logits[0, K - 1] = -math.inf
    logits[1, K - 1, 5:] = -math.inf
    check(sw, logits, scores, k, done, eos=17)
