"""Attention of drafted tokens over a paged cache against the formula in 64 bits, at the edges of tiles, pages, groups and masks."""
import math

import numpy as np
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


def random_tree(rng, B, T):
    """Ancestor masks as bits: every token sees itself, its parent (an earlier token or none) and what that one sees."""
    sees = np.zeros((B, T, T), dtype=bool)
    for b in range(B):
        for i in range(T):
            p = int(rng.integers(-1, i)) if i else -1
            if p >= 0:
                sees[b, i] = sees[b, p]
            sees[b, i, i] = True
    return sees


def words(sees):
    B, T, _ = sees.shape
    W = (T + 31) // 32
    out = np.zeros((B, T, W), dtype=np.uint32)
    for j in range(T):
        out[:, :, j // 32] |= sees[:, :, j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


class Problem:
    """Seeded inputs on the host: the pool's unused tokens are NaN, so that a kernel that lets one in shows it."""

    def __init__(self, seed, dtype, B, T, H, G, d, page, lens, sel=0, unit="page", tree=False, n_new=None, L=1, new=True, spare=2, wide=0, loud=1.0):
        rng = self.rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        t = TYPES[dtype]
        self.t, self.B, self.T, self.H, self.G, self.d, self.page, self.L, self.unit = t, B, T, H, G, d, page, L, unit
        self.lens = list(lens)
        held = [-(-n // page) for n in lens]
        cap = max(1, max(held)) + wide
        P = sum(held) + spare
        self.k = torch.full((L, P, H, page, d), math.nan).to(t)
        self.v = self.k.clone()
        ids = rng.permutation(P)
        self.table = np.full((B, cap), -1, dtype=np.int32)
        at = 0
        for b in range(B):
            self.table[b, :held[b]] = ids[at:at + held[b]]
            at += held[b]
            for j in range(held[b]):
                n = min(page, lens[b] - j * page)
                self.k[:, self.table[b, j], :, :n] = torch.randn((L, H, n, d), generator=g).mul(loud).to(t)
                self.v[:, self.table[b, j], :, :n] = torch.randn((L, H, n, d), generator=g).to(t)
        self.q = torch.randn((B, T, H * G, d), generator=g).to(t)
        self.k_new = torch.randn((B, T, H, d), generator=g).to(t) if new else None
        self.v_new = torch.randn((B, T, H, d), generator=g).to(t) if new else None
        self.n_new = None if n_new is None else np.asarray(n_new, dtype=np.int32)
        if self.n_new is not None and new:
            for b in range(B):
                self.k_new[b, self.n_new[b]:] = math.nan
                self.v_new[b, self.n_new[b]:] = math.nan
        self.sees = random_tree(rng, B, T) if tree else None
        self.sel = None
        if sel:
            self.sel = np.full((B, H, sel), -1, dtype=np.int32)
            for b in range(B):
                for h in range(H):
                    n = lens[b] if unit == "token" else held[b]
                    m = min(sel, n)
                    self.sel[b, h, :m] = np.sort(rng.choice(n, size=m, replace=False)) if m else []
        self.scale = d ** -0.5

    def context(self, b, h):
        """Positions that (stream, head) attends over."""
        n = self.lens[b]
        if self.sel is None:
            return list(range(n))
        if self.unit == "token":
            return [int(e) for e in self.sel[b, h] if 0 <= e < n]
        return [int(e) * self.page + o for e in self.sel[b, h] if e >= 0 for o in range(self.page) if int(e) * self.page + o < n]

    def reference(self, layer=0):
        """(out, lse, their tolerances) in 64 bits; rows behind n_new are NaN."""
        B, T, H, G, d = self.B, self.T, self.H, self.G, self.d
        out, lse = torch.full((B, T, H * G, d), math.nan, dtype=torch.float64), torch.full((B, T, H * G), math.nan, dtype=torch.float64)
        tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
        half = torch.finfo(self.t).eps / 2
        for b in range(B):
            n = T if self.n_new is None else int(self.n_new[b])
            for h in range(H):
                pos = self.context(b, h)
                pages = torch.tensor([int(self.table[b, p // self.page]) for p in pos], dtype=torch.long)
                off = torch.tensor([p % self.page for p in pos], dtype=torch.long)
                kc, vc = self.k[layer, pages, h, off].double(), self.v[layer, pages, h, off].double()
                for i in range(n):
                    vis = [] if self.k_new is None else [j for j in range(n) if (j <= i if self.sees is None else self.sees[b, i, j])]
                    kk = torch.cat([kc, self.k_new[b, vis, h].double()]) if vis else kc
                    vv = torch.cat([vc, self.v_new[b, vis, h].double()]) if vis else vc
                    for g in range(G):
                        q = self.q[b, i, h * G + g].double()
                        s = (kk @ q) * self.scale
                        m = s.max() if len(s) else torch.tensor(-math.inf, dtype=torch.float64)
                        if m == -math.inf:
                            out[b, i, h * G + g], lse[b, i, h * G + g] = 0, -math.inf
                            continue
                        p = (s - m).exp()
                        w = p / p.sum()
                        o = w @ vv
                        out[b, i, h * G + g], lse[b, i, h * G + g] = o, m + p.sum().log()
                        # a score: d products added in fp32 (each addition half a step of the partial sums, at most sum |q k|), one
                        # rounding for the scale, one for the difference to the maximum in units of ln 2, 2^-22 for the exponential itself
                        e = ((d + 2) * 2.0 ** -24 * (kk.abs() @ q.abs()).max() * abs(self.scale) + 4 * 2.0 ** -24 * s[s > -math.inf].abs().max() + 2.0 ** -22).item()
                        adds = (len(s) + 64) * 2.0 ** -24
                        # What the product with v takes of a weight w, the sum of weights being that of the unrounded ones.  Up to a wave's rows (32, 16
                        # of heads wider than 128) two terms: the second is the first one's error, rounded, so off by 2 half steps squared at most.
                        # Above, one term: w (1 + e) with |e| <= half a step, so that sum w v is off by half a step of sum w |v| at most.
                        # fp16 has terms below its smallest normal number, off by 2^-25; weights are below 2^8 (the maximum they refer to lags by
                        # as much) and their sum is that of the largest one at least
                        terms = (4 * half * half if T * G <= (16 if d > 128 else 32) else half) + (2.0 ** -25 * len(s) if self.t is torch.float16 else 0)
                        tol_o[b, i, h * G + g] = half * o.abs() * 1.01 + (2 * e + 2 * adds + terms) * (w @ vv.abs()) + torch.finfo(self.t).tiny * half
                        tol_l[b, i, h * G + g] = e + adds + 2.0 ** -22 * (1 + lse[b, i, h * G + g].abs())
        return out, lse, tol_o, tol_l

    def run(self, sw, layer=0, lse=True):
        from paper_2603_17803_amd import binding
        dev = lambda x: None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()  # noqa: E731
        B, T, HG, d = self.q.shape
        cache = binding.Cache(dev(self.k), dev(self.v), dev(self.table), dev(np.asarray(self.lens, dtype=np.int32)))
        flat = torch.full((B * T * HG * d + 64,), 77.0, dtype=self.t, device="cuda")
        out = flat[:B * T * HG * d].view(B, T, HG, d)
        flat_l = torch.full((B * T * HG + 64,), 77.0, device="cuda")
        l = flat_l[:B * T * HG].view(B, T, HG) if lse else None
        sw.tree_attend(cache, layer, dev(self.q), dev(self.k_new), dev(self.v_new), n_new=dev(self.n_new), mask=None if self.sees is None else dev(words(self.sees)),
                       sel=dev(self.sel), unit=self.unit, scale=self.scale, out=out, lse=l)
        torch.cuda.synchronize()
        assert (flat[B * T * HG * d:] == 77.0).all() and (flat_l[B * T * HG:] == 77.0).all(), "written behind the outputs"
        return out.cpu(), None if l is None else l.cpu()

    def check(self, sw, layer=0):
        out, lse, tol_o, tol_l = self.reference(layer)
        got, got_l = self.run(sw, layer)
        same(got, got_l, out, lse, tol_o, tol_l)
        return got, got_l



def same(got, got_l, out, lse, tol_o, tol_l):
    dead = out.isnan().all(-1)
    assert (got[dead] == 77.0).all() and (got_l[dead] == 77.0).all(), "tokens that a stream does not have were written"
    live = ~dead
    bad = ~((got.double() - out).abs() <= tol_o)[live]
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off, the worst by {((got.double() - out).abs() / tol_o)[live].nan_to_num(nan=1e30).max():.3g} tolerances"
    empty = live & (lse == -math.inf)
    assert (got_l[empty] == -math.inf).all() and (got[empty] == 0).all()
    full = live & ~empty
    assert ((got_l.double() - lse).abs() <= tol_l)[full].all(), f"lse off by {((got_l.double() - lse).abs() / tol_l)[full].max():.3g} tolerances"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens", [[0], [1], [15, 16, 17], [31, 32, 33], [63, 64, 65], [127, 128, 129], [255, 300, 0, 511], [640, 1, 513]])
def test_single_tokens_of_ragged_streams(sw, dtype, lens):
    Problem(len(lens) + lens[0], dtype, len(lens), 1, 2, 4, 128, 16, lens).check(sw)


@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 128, 256])
def test_page_sizes(sw, page):
    Problem(page, "bf16", 2, 3, 2, 2, 64, page, [301, 77], tree=True, wide=3).check(sw)


@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 80, 96, 112, 120, 128, 136, 160, 192, 200, 248, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_head_dimensions(sw, d, dtype):
    Problem(d, dtype, 2, 2, 2, 3, d, 16, [150, 33], tree=True).check(sw)


@pytest.mark.parametrize("T,G,H", [(1, 1, 1), (1, 7, 3), (2, 8, 1), (5, 3, 2), (15, 1, 2), (16, 1, 2), (17, 1, 1), (8, 4, 1), (33, 1, 1), (31, 2, 1), (64, 1, 2), (13, 5, 1),
                                   (64, 4, 1), (65, 2, 1), (129, 1, 1), (256, 1, 1), (3, 40, 1), (40, 8, 1), (200, 2, 1)])
def test_tokens_and_groups(sw, T, G, H):
    Problem(T * 100 + G, "bf16", 1, T, H, G, 64, 16, [201], tree=True).check(sw)


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 100])
def test_chains_and_padded_streams(sw, T):
    """Without a mask, and with fewer drafted tokens than T: the others are neither seen nor written."""
    Problem(T, "bf16", 4, T, 2, 2, 128, 16, [40, 0, 129, 7], n_new=[T, max(1, T // 2), 0, 1]).check(sw)
    Problem(T + 1, "fp16", 4, T, 1, 4, 128, 16, [40, 0, 129, 7], n_new=[0, T, 1, max(1, T - 1)], tree=True).check(sw)


@pytest.mark.parametrize("unit", ["page", "token"])
@pytest.mark.parametrize("page", [1, 8, 16, 64])
@pytest.mark.parametrize("T,G", [(1, 4), (6, 2), (20, 5)])
def test_selected_entries(sw, unit, page, T, G):
    """Selections of every stream and head: ragged, padded with -1, with the last, partly filled page among them."""
    for sel in (1, 5, 33, 130):
        Problem(sel + page, "bf16", 3, T, 2, G, 128, page, [400, 3, 131], sel=sel, unit=unit, tree=T > 1).check(sw)


def test_selections_of_the_scorer_are_what_is_attended_over(sw):
    """score_select's out_idx goes in as it is."""
    p = Problem(3, "bf16", 2, 1, 4, 2, 128, 16, [512, 512], sel=7)
    pages = p.k[0][torch.from_numpy(p.table[0]).long()].permute(1, 0, 2, 3)            # stream 0's keys [H][pages][16][d]
    summary = torch.stack([pages.amin(2), pages.amax(2)], 2).contiguous()
    idx, _ = sw.score_select("page", summary.cuda(), p.q[:, 0].contiguous().cuda(), 7, G=2)
    p.sel = idx.cpu().numpy()
    p.check(sw)


def test_positions_behind_a_row_and_repeats(sw):
    """A selected page behind the row's tokens adds nothing; one that is listed twice counts twice."""
    p = Problem(4, "bf16", 1, 2, 1, 2, 64, 16, [70], sel=6, wide=4)
    p.sel[0, 0] = [0, 2, 2, 4, 5, 8]
    p.check(sw)


def test_context_alone_and_nothing_at_all(sw):
    Problem(5, "bf16", 3, 4, 2, 2, 64, 16, [33, 0, 1], new=False).check(sw)
    p = Problem(6, "bf16", 2, 5, 1, 3, 64, 16, [0, 20], tree=True)
    p.sees[:, 2] = False                                                              # a token that sees no drafted one, itself included
    p.check(sw)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, "lowest"])
@pytest.mark.parametrize("T,lens", [(6, [40]), (40, [0]), (3, [0]), (70, [140])])
def test_what_a_token_does_not_see_never_reaches_it(sw, value, T, lens):
    """Keys and values of a drafted token are not numbers (or the type's lowest): only the tokens that see it may show that."""
    p = Problem(T, "bf16", 1, T, 2, 3, 128, 16, lens, tree=True)
    poison = T // 2
    x = torch.finfo(p.t).min if value == "lowest" else value
    p.sees[0, :, poison] = False
    out, lse, tol_o, tol_l = p.reference()
    p.v_new[0, poison] = x
    got, got_l = p.run(sw)
    same(got, got_l, out, lse, tol_o, tol_l)
    p.k_new[0, poison] = x
    got, got_l = p.run(sw)
    same(got, got_l, out, lse, tol_o, tol_l)


def test_one_token_sees_what_is_not_a_number(sw):
    p = Problem(11, "bf16", 1, 5, 1, 2, 64, 16, [50], tree=True)
    p.sees[0, :, 2] = False
    out, lse, tol_o, tol_l = p.reference()
    p.sees[0, 4, 2] = True
    p.v_new[0, 2, 0, 3] = math.inf
    p.v_new[0, 2, 0, 9] = math.nan
    got, got_l = p.run(sw)
    same(got[:, :4], got_l[:, :4], out[:, :4], lse[:, :4], tol_o[:, :4], tol_l[:, :4])
    assert (got[0, 4, :, 3] == math.inf).all() and got[0, 4, :, 9].isnan().all()
    assert torch.isfinite(got[0, 4][:, [c for c in range(64) if c not in (3, 9)]]).all()


def test_keys_of_minus_infinity_weigh_nothing(sw):
    """A score of -inf is a weight of 0, and a row of them is a row that sees nothing."""
    p = Problem(12, "bf16", 1, 1, 1, 2, 64, 16, [35], new=False)
    p.q[..., 0] = 1.0
    p.k[0, int(p.table[0, 1]), 0, 3, 0] = -math.inf
    p.check(sw)
    p.k[0, torch.from_numpy(p.table[0]).long(), :, :, 0] = -math.inf
    got, lse = p.run(sw)
    assert (got == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("loud", [30.0, 1e-3])
def test_sharp_and_flat_scores(sw, loud):
    """Weights from one key alone to all keys alike."""
    Problem(13, "bf16", 2, 3, 2, 2, 128, 16, [1000, 257], tree=True, loud=loud).check(sw)
    Problem(14, "fp16", 2, 3, 2, 2, 128, 16, [1000, 257], tree=True, loud=loud).check(sw)


def test_layers_of_a_pool(sw):
    p = Problem(15, "bf16", 2, 2, 2, 2, 64, 16, [50, 17], L=3)
    for layer in range(3):
        p.check(sw, layer)


def test_negative_and_zero_scale(sw):
    for scale in (-0.3, 0.0):
        p = Problem(16, "bf16", 1, 3, 2, 2, 64, 16, [90], tree=True)
        p.scale = scale
        p.check(sw)


def test_results_do_not_change_from_call_to_call(sw):
    p = Problem(17, "bf16", 5, 9, 2, 4, 128, 16, [3000, 17, 801, 0, 1500], tree=True)
    first, first_l = p.run(sw)
    for _ in range(3):
        again, again_l = p.run(sw)
        assert torch.equal(first, again) and torch.equal(first_l, again_l)
    assert torch.equal(p.run(sw, lse=False)[0], first)


def test_parts_join_by_their_lse(sw):
    """Attention over two halves of the selected pages, joined as the documentation says, is the attention over all."""
    p = Problem(18, "bf16", 2, 1, 2, 2, 128, 16, [900, 640], sel=24, new=False)
    whole, _, tol_o, _ = p.reference()
    every = p.sel
    parts = []
    for half in (every[:, :, :11], every[:, :, 11:]):
        p.sel = np.ascontiguousarray(half)
        parts.append(p.run(sw))
    lse = torch.stack([l.double() for _, l in parts])
    w = (lse - torch.logsumexp(lse, 0)).exp()[..., None]
    joined = (w * torch.stack([o.double() for o, _ in parts])).sum(0)
    # each part is rounded to the cache's type once: half a step of its own size
    slack = (torch.stack([o.double().abs() for o, _ in parts]) * w).sum(0) * torch.finfo(p.t).eps / 2
    assert ((joined - whole).abs() <= 2 * tol_o + slack).all()


def test_bad_data_is_dropped_and_flagged(sw):
    from paper_2603_17803_amd import binding as b
    p = Problem(19, "bf16", 2, 2, 2, 2, 64, 16, [100, 50], spare=0)
    assert sw.device_status() == 0
    good = p.table.copy()
    for bad in (-5, -1, p.k.shape[1], 2 ** 31 - 1):
        p.table = good.copy()
        p.table[0, 2] = bad
        got = p.run(sw)
        assert sw.device_status() == b.SWARM_DEV_BAD_PAGE
        # the same as a selection that leaves the page out
        p.table = good
        p.sel = np.array([[[0, 1, 3, 4, 5, 6]] * 2, [[0, 1, 2, 3, -1, -1]] * 2], dtype=np.int32)
        out, lse, tol_o, tol_l = p.reference()
        same(*got, out, lse, tol_o, tol_l)
        p.sel = None
    for unit, bad in (("page", [-2, 7, 2 ** 31 - 1]), ("token", [-7, 112, 2 ** 30])):
        p.unit = unit
        p.sel = np.array([[[1, 2] + bad] * 2] * 2, dtype=np.int32)
        got = p.run(sw)
        assert sw.device_status() == b.SWARM_DEV_BAD_ENTRY
        p.sel = np.ascontiguousarray(p.sel[:, :, :2])
        out, lse, tol_o, tol_l = p.reference()
        same(*got, out, lse, tol_o, tol_l)
    p.unit, p.sel = "page", None
    true = p.lens
    p.lens = [-3, 2 ** 30]
    p.run(sw)
    assert sw.device_status() & b.SWARM_DEV_BAD_LEN
    p.lens = true
    for n in ([-1, 2], [2, 3]):
        p.n_new = np.asarray(n, dtype=np.int32)
        got = p.run(sw)
        assert sw.device_status() == b.SWARM_DEV_BAD_LEN
        p.n_new = np.clip(p.n_new, 0, 2)
        out, lse, tol_o, tol_l = p.reference()
        same(*got, out, lse, tol_o, tol_l)


def test_refusals(sw):
    from paper_2603_17803_amd import binding as b
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, v, table, length = pool(1, 4, 2, 16, 64), pool(1, 4, 2, 16, 64), i32(2, 2), i32(2)
    q, new = pool(2, 3, 4, 64), pool(2, 3, 2, 64)

    def call(**kw):
        a = dict(dtype=b.SWARM_BF16, k=k.data_ptr(), v=v.data_ptr(), L=1, P=4, H=2, page=16, d=64, table=table.data_ptr(), len=length.data_ptr(), refs=None, rows=2, cap=2,
                 layer=0, q=q.data_ptr(), k_new=new.data_ptr(), v_new=new.data_ptr(), B=2, T=3, G=2, n_new=None, mask=None, sel=None, n_sel=0, unit=0, scale=1.0,
                 out=out.data_ptr(), lse=None)
        a.update(kw)
        c = b.swarm_cache(*[a[f] for f, _ in b.swarm_cache._fields_])
        return b.swarm_tree_attend(sw.ctx, c, *[a[f] for f in ("layer", "q", "k_new", "v_new", "B", "T", "G", "n_new", "mask", "sel", "n_sel", "unit", "scale", "out", "lse")])

    out = pool(2, 3, 4, 64)
    assert call() == b.SWARM_OK
    torch.cuda.synchronize()
    before = out.clone()
    sel = i32(2, 2, 2)
    for kw in [dict(dtype=2), dict(dtype=-1), dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(q=None), dict(out=None), dict(k_new=None), dict(v_new=None),
               dict(L=0), dict(P=0), dict(H=0), dict(rows=0), dict(cap=0), dict(page=0), dict(page=12), dict(page=512), dict(d=0), dict(d=60), dict(d=264), dict(P=1 << 27),
               dict(cap=1 << 27), dict(rows=65536), dict(layer=1), dict(layer=-1), dict(B=0), dict(B=3), dict(T=0), dict(T=257), dict(G=0), dict(G=1 << 20),
               dict(sel=sel.data_ptr(), n_sel=0), dict(sel=sel.data_ptr(), n_sel=1 << 28), dict(sel=sel.data_ptr(), n_sel=2, unit=2), dict(scale=math.nan), dict(scale=math.inf),
               dict(q=q.data_ptr() + 8), dict(out=out.data_ptr() + 2), dict(k=k.data_ptr() + 4), dict(lse=length.data_ptr() + 2), dict(mask=length.data_ptr() + 1),
               dict(out=q.data_ptr()), dict(out=k.data_ptr() + 1024), dict(lse=length.data_ptr()), dict(lse=out.data_ptr())]:
        assert call(**kw) == b.SWARM_EINVAL, kw
        assert b.swarm_last_error(sw.ctx)
    null = b.swarm_cache()
    assert b.load().swarm_tree_attend(sw.ctx, None, 0, 0, 0, 0, 1, 1, 1, 0, 0, 0, 0, 0, 1.0, 0, 0) == b.SWARM_EINVAL
    assert b.swarm_tree_attend(sw.ctx, null, 0, 0, 0, 0, 1, 1, 1, 0, 0, 0, 0, 0, 1.0, 0, 0) == b.SWARM_EINVAL
    torch.cuda.synchronize()
    assert torch.equal(out, before)
    cache = b.Cache(k, v, table, length)
    for bad in [dict(q=q.half()), dict(q=q[:, :, :3].contiguous()), dict(q=q.transpose(1, 2)), dict(k_new=new[:1]), dict(n_new=i32(3)), dict(mask=i32(2, 3, 2)), dict(sel=i32(2, 1, 2)),
                dict(unit="row"), dict(out=pool(2, 3, 4, 32)), dict(lse=pool(2, 3, 4)), dict(q=q.cpu())]:
        a = dict(q=q, k_new=new, v_new=new)
        a.update(bad)
        with pytest.raises(ValueError):
            sw.tree_attend(cache, 0, a.pop("q"), **a)
    with pytest.raises(ValueError):
        sw.tree_attend(b.Cache(k, v[:, :3].contiguous(), table, length), 0, q)
    with pytest.raises(ValueError):
        sw.tree_attend(b.Cache(k.float(), v.float(), table, length), 0, q.float())


def test_recorded_and_captured_calls_replay(sw):
    """Recorded by the library and captured by torch, replayed with new inputs and eager work in between."""
    from paper_2603_17803_amd import binding as b
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s = b.Swarm(0, stream=stream)
        p = [Problem(20 + i, "bf16", 3, 4, 2, 4, 128, 16, [2000, 5, 700], tree=True) for i in range(3)]
        dev = lambda x: (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()  # noqa: E731
        hold = [[dev(x) for x in (y.k, y.v, y.table, np.asarray(y.lens, dtype=np.int32), y.q, y.k_new, y.v_new, words(y.sees))] for y in p]
        use = [x.clone() for x in hold[0]]
        out, lse = torch.zeros_like(use[4]), torch.zeros(use[4].shape[:3], device="cuda")
        eager = []
        call = lambda t, o, l: s.tree_attend(b.Cache(*t[:4]), 0, t[4], t[5], t[6], mask=t[7], out=o, lse=l)  # noqa: E731
        for h in hold:
            o, l = torch.zeros_like(out), torch.zeros_like(lse)
            call(h, o, l)
            eager.append((o, l))
        stream.synchronize()
        s.capture_begin()
        call(use, out, lse)
        recorded = s.capture_end()
        captured = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(captured, stream=stream):
            call(use, out, lse)
        for replay in (lambda: s.graph_launch(recorded), captured.replay):
            for turn in (1, 2, 0, 1):
                for x, y in zip(use, hold[turn]):
                    x.copy_(y)
                out.zero_(), lse.zero_()
                replay()
                stream.synchronize()
                assert torch.equal(out, eager[turn][0]) and torch.equal(lse, eager[turn][1])
                call(hold[2], torch.zeros_like(out), None)
        b.swarm_graph_destroy(recorded)
        del captured
        stream.synchronize()
        s.close()


def test_long_cache_beyond_32_bit_offsets(sw):
    """A pool of more than 2^32 bytes on each side, the row's pages at its far end."""
    from paper_2603_17803_amd import binding as b
    P, H, page, d = 36000, 8, 64, 128
    free, _ = torch.cuda.mem_get_info()
    if free < 3 * P * H * page * d * 2:
        pytest.skip("needs 14 GB of device memory")
    p = Problem(23, "bf16", 1, 2, H, 1, d, page, [300], spare=0)
    k = torch.empty((1, P, H, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    n = p.k.shape[1]
    k[:, P - n:], v[:, P - n:] = p.k.cuda(), p.v.cuda()
    out, lse, tol_o, tol_l = p.reference()
    table = torch.from_numpy(p.table + (P - n)).int().cuda()
    got_l = torch.zeros((1, 2, H), device="cuda")
    got, _ = sw.tree_attend(b.Cache(k, v, table, torch.tensor(p.lens, dtype=torch.int32, device="cuda")), 0, p.q.cuda(), p.k_new.cuda(), p.v_new.cuda(), lse=got_l)
    torch.cuda.synchronize()
    same(got.cpu(), got_l.cpu(), out, lse, tol_o, tol_l)


@pytest.mark.parametrize("d", [136, 192, 256])
@pytest.mark.parametrize("T,G", [(16, 1), (17, 1), (11, 3), (13, 5), (25, 4), (43, 3), (257 // 8, 8), (130, 2)])
def test_many_rows_of_wide_heads(sw, d, T, G):
    Problem(d + T, "fp16" if T % 2 else "bf16", 2, T, 1, G, d, 16, [203, 40], tree=True).check(sw)


@pytest.mark.parametrize("T,G", [(3, 11), (13, 5), (32, 4), (43, 3), (75, 2), (49, 4), (65, 4), (97, 4)])
@pytest.mark.parametrize("d", [72, 128])
def test_many_rows_over_several_parts(sw, d, T, G):
    """Rows of one to eight waves and of two tiles, streams that end at every place of a part."""
    Problem(d + T, "bf16" if T % 2 else "fp16", 4, T, 2, G, d, 16, [385, 0, 64, 129], tree=True, n_new=[T, T, max(1, T - 3), 2]).check(sw)


@pytest.mark.parametrize("B", [63, 64, 65, 130, 256, 257, 600])
@pytest.mark.parametrize("T,G", [(1, 2), (20, 2)])
def test_many_streams(sw, B, T, G):
    """Streams that are found by one wave, by one pass and by two, among them empty ones and ones without drafted tokens."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.choice([0, 1, 20, 128, 129, 300], size=B)]
    Problem(B, "bf16", B, T, 1, G, 32, 16, lens, n_new=[int(x) for x in rng.choice([0, 1, T], size=B)]).check(sw)


def test_values_that_are_not_numbers_stay_in_their_stream(sw):
    """A token of the context is seen by its stream and head alone."""
    for T, G in ((2, 2), (20, 3)):
        p = Problem(24 + T, "bf16", 3, T, 2, G, 64, 16, [300, 200, 30], tree=True)
        out, lse, tol_o, tol_l = p.reference()
        p.v[0, int(p.table[1, 3]), 1, 5, 7] = math.nan
        p.v[0, int(p.table[1, 8]), 1, 2, 9] = math.inf
        got, got_l = p.run(sw)
        hit = got[1, :, G:]
        assert hit[..., 7].isnan().all() and (hit[..., 9] == math.inf).all()
        got[1, :, G:, 7], got[1, :, G:, 9] = 77.0, 77.0
        out[1, :, G:, 7], out[1, :, G:, 9] = 77.0, 77.0
        same(got, got_l, out, lse, tol_o, tol_l)
        p.k[0, int(p.table[1, 3]), 1, 5, 7] = math.nan
        got, got_l = p.run(sw)
        assert got[1, :, G:].isnan().all() and got_l[1, :, G:].isnan().all()
        keep = [0, 2]
        same(got[keep], got_l[keep], out[keep], lse[keep], tol_o[keep], tol_l[keep])


def test_smaller_calls_are_recorded_after_a_larger_one(sw):
    """No call with fewer streams, tokens or query heads, or narrower heads, needs more scratch than the larger one before it."""
    from paper_2603_17803_amd import binding as b
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for big, small in [((2, 48, 2, 4, 128), [(2, 32, 2, 4, 128), (1, 48, 2, 4, 128), (2, 16, 1, 4, 128), (2, 48, 2, 1, 128), (2, 1, 2, 4, 128), (2, 33, 2, 4, 64)]),
                           ((1, 65, 1, 4, 128), [(1, 64, 1, 4, 128), (1, 32, 1, 4, 128), (1, 8, 1, 4, 128)]),
                           ((1, 40, 1, 4, 256), [(1, 40, 1, 4, 192), (1, 33, 1, 4, 128), (1, 32, 1, 4, 256), (1, 8, 1, 2, 256), (1, 40, 1, 4, 64)])]:
            s = b.Swarm(0, stream=stream)
            Problem(1, "bf16", *big, 16, [5000] * big[0]).run(s)
            for shape in small:
                p = Problem(2, "bf16", *shape, 16, [5000] * shape[0])
                dev = [x.cuda() for x in (p.k, p.v, torch.from_numpy(p.table), torch.tensor(p.lens, dtype=torch.int32), p.q, p.k_new, p.v_new)]
                out = torch.zeros_like(dev[4])
                stream.synchronize()
                s.capture_begin()
                s.tree_attend(b.Cache(*dev[:4]), 0, *dev[4:], scale=p.scale, out=out)
                graph = s.capture_end()
                for _ in range(2):
                    out.zero_()
                    s.graph_launch(graph)
                    stream.synchronize()
                    assert torch.equal(out.cpu(), p.run(s)[0])
                b.swarm_graph_destroy(graph)
            s.close()


def test_contexts_on_two_streams_at_once(sw):
    from paper_2603_17803_amd import binding as b
    made = []
    for i, T in enumerate((1, 24)):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            p = Problem(30 + i, "bf16", 2, T, 2, 4, 128, 16, [4000, 900])
            dev = [x.cuda() for x in (p.k, p.v, torch.from_numpy(p.table), torch.tensor(p.lens, dtype=torch.int32), p.q, p.k_new, p.v_new)]
            made.append((b.Swarm(0, stream=stream), dev, [torch.zeros_like(dev[4]) for _ in range(20)], p.run(sw)[0]))
    torch.cuda.synchronize()
    for i in range(20):
        for s, dev, outs, _ in made:
            s.tree_attend(b.Cache(*dev[:4]), 0, *dev[4:], out=outs[i])
    torch.cuda.synchronize()
    for s, _, outs, want in made:
        assert all(torch.equal(o.cpu(), want) for o in outs)
        s.close()


def test_scale_that_fp32_does_not_hold_in_units_of_ln_2(sw):
    from paper_2603_17803_amd import binding as b
    p = Problem(40, "bf16", 1, 1, 1, 1, 64, 16, [3])
    p.scale = 3e38
    with pytest.raises(b.SwarmError):
        p.run(sw)


@pytest.mark.parametrize("T,G,H,n,d", [(4, 4, 1, 1100000, 8), (3, 2, 2, 700000, 16), (3, 9, 1, 1100000, 8), (33, 2, 1, 1100000, 8), (40, 4, 1, 600000, 8), (4, 4, 1, 600000, 136)])
def test_more_keys_of_a_pair_than_a_part_lists_at_a_time(sw, T, G, H, n, d):
    """Parts of more than 2048 keys, so that rows are looked up several times.  Few keys weigh nearly all, another set for each row."""
    p = Problem(T * G, "bf16", 1, T, H, G, d, 256, [n - 77], loud=8.0)
    p.check(sw)
