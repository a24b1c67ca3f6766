"""Eviction from KV pages: the choice and the move, exactly; positions given to the append; and the calls in a row as a
serving step makes them."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import DT, ULP, engine  # noqa: E402


def _say(*a):
    print("[case]", *a, flush=True)


def dev(x, t=None):
    x = torch.from_numpy(np.ascontiguousarray(x))
    return (x if t is None else x.to(t)).cuda()


def choice(score, budget, sink, recent):
    """Places that stay of one sequence's float32 scores, in order."""
    n = len(score)
    first = min(sink, budget)
    tail = min(recent, budget - first)
    middle = np.arange(first, n - tail)
    x = score[middle].astype(np.float64)
    x = np.where(np.isnan(x), -math.inf, x)
    low = np.isnan(score[middle])  # below minus infinity too
    order = middle[np.lexsort((middle, -x, low))]
    return np.sort(np.concatenate([np.arange(first), order[:budget - first - tail], np.arange(n - tail, n)]))


class Histories:
    """Sequences of given lengths with scattered pages and weights; entries between them that belong to nobody."""

    def __init__(self, block, lens, layers=2, heads=4, seed=0, gap=1, values=None):
        r = np.random.default_rng(seed)
        self.block, self.len, self.layers, self.heads = block, np.array(lens, np.int64), layers, heads
        pages = -(-self.len // block)
        self.off = np.concatenate([[0], np.cumsum(pages)]).astype(np.int64)
        self.pages = int(self.off[-1]) + 3
        self.page = r.permutation(self.pages)[:max(1, int(self.off[-1]))].astype(np.int32)
        self.rows = len(self.page) * block
        self.w = np.exp(3 * r.standard_normal((layers, heads, self.rows))).astype(np.float32)
        if values is not None:
            self.w = np.array(values, np.float32)[r.integers(0, len(values), size=self.w.shape)]

    def tables(self):
        return dev(self.off), dev(self.page), dev(self.len)

    def select(self, budget, sink=0, recent=0, share=1, room=None, eng=None):
        pk, e = engine(self.block)
        e = eng or e
        n = len(self.len)
        wide = torch.full((self.layers, self.heads, self.rows + 3), math.nan, device="cuda")
        wide[..., :self.rows] = dev(self.w)
        kept = torch.full((self.layers, self.heads // share, self.rows + 1), -7, dtype=torch.int32, device="cuda")
        keep, grow = torch.full((n,), -7, device="cuda"), torch.full((n,), -7, device="cuda")
        e.evict_select(self.tables(), wide[..., :self.rows], dev(np.array(budget, np.int64)),
                       None if room is None else dev(np.array(room, np.int64)), kept, keep, grow, sink=sink, recent=recent,
                       share=share)
        e.sync()
        return kept.cpu().numpy(), keep.cpu().numpy(), grow.cpu().numpy()

    def expected(self, budget, sink=0, recent=0, share=1):
        kept = np.full((self.layers, self.heads // share, self.rows + 1), -7, np.int32)
        for s, L in enumerate(self.len):
            if L <= budget[s]:
                continue
            a = int(self.off[s]) * self.block
            for layer in range(self.layers):
                for c in range(self.heads // share):
                    x = self.w[layer, c * share, a:a + L].copy()
                    for h in range(1, share):
                        x = x + self.w[layer, c * share + h, a:a + L]
                    kept[layer, c, a:a + budget[s]] = choice(x, budget[s], sink, recent)
        return kept

    def check(self, budget, room=None, **k):
        kept, keep, grow = self.select(budget, room=room, **k)
        past = self.len > np.array(budget)
        more = np.zeros(len(past), np.int64) if room is None else np.array(room)
        assert keep.tolist() == np.where(past, 0, self.len).tolist()
        assert grow.tolist() == (more + np.where(past, budget, 0)).tolist()
        assert np.array_equal(kept, self.expected(budget, **k))


LENS = [1, 2, 63, 64, 65, 100, 255, 256, 257, 511, 700, 1024, 1025, 1500]


@pytest.mark.parametrize("block", [4, 16, 64])
@pytest.mark.parametrize("share", [1, 2, 4])
@pytest.mark.parametrize("sink,recent", [(0, 0), (4, 32), (1, 0), (0, 77)])
def test_choice(block, share, sink, recent):
    _say("choice", block, share, sink, recent)
    b = Histories(block, LENS, seed=block + share)
    b.check([max(1, n // 3) for n in LENS], sink=sink, recent=recent, share=share, room=list(range(len(LENS))))


@pytest.mark.parametrize("values", [[0.0], [1.0, 2.0], [0.0, -0.0, 1e-45, -1e-45], [math.nan, 1.0, -math.inf, math.inf, -3.0],
                                    [math.nan], [1.0, 1.0 + 2.0 ** -23, 1.0 - 2.0 ** -24]])
def test_equals_and_odd_values(values):
    """Equal scores go to the earlier token; zeros of both signs are equal; NaN is below all."""
    _say("values", values)
    lens = [5, 64, 100, 900, 1300, 3000]
    b = Histories(16, lens, seed=3, values=values)
    b.check([1, 63, 50, 450, 1299, 7])
    b.check([3, 33, 99, 100, 640, 1501], sink=2, recent=3)


def test_budgets():
    """None, all but one, exactly the length, more; budgets below what always stays."""
    lens = [100, 100, 100, 100, 100, 100, 0, 100]
    b = Histories(16, lens, seed=4)
    b.check([0, 99, 100, 101, 1, 6, 0, 2 ** 40], sink=4, recent=8)
    b.check([0, 99, 100, 101, 1, 6, 5, 37], sink=0, recent=200)
    b.check([0, 99, 100, 101, 1, 6, 5, 37], sink=200, recent=200)


@pytest.mark.parametrize("lens", [[4096, 4097], [16_384, 16_385, 20], [70_001], [9000, 40_000, 3]])
def test_long_histories(lens):
    """Around the scores that are kept in registers, and past them."""
    _say("long", lens)
    b = Histories(64, lens, layers=1, heads=2, seed=5)
    b.check([n // 2 for n in lens], sink=4, recent=100)
    b.check([min(n, 1000) for n in lens], share=2)
    Histories(64, lens, layers=1, heads=2, seed=5, values=[0.5]).check([n // 2 for n in lens])


@pytest.mark.parametrize("share", [1, 2])
@pytest.mark.parametrize("lens", [[40_000], [24_577, 24_640, 30_001], [100_001, 12, 50_000, 0, 90_000], [150_000, 3]])
def test_choices_of_several_workgroups(lens, share):
    """Few and long choices: their parts' borders, equals that reach over them, short sequences between."""
    _say("split", lens, share)
    b = Histories(32, lens, layers=2, heads=2, seed=11)
    for budget in ([n // 2 for n in lens], [min(n, 777) for n in lens], [max(0, n - 1) for n in lens], [0 for _ in lens]):
        b.check(budget, sink=3, recent=65, share=share, room=list(range(len(lens))))
    for values in ([0.5], [0.0, -0.0], [1.0, 2.0, math.nan, math.inf, -math.inf]):
        Histories(32, lens, layers=1, heads=2, seed=12, values=values).check([n * 5 // 8 for n in lens], share=share)


def test_long_choices_of_one_workgroup():
    """Many of them, and one long among short ones."""
    _say("one workgroup")
    Histories(16, [26_000] * 4, layers=4, heads=16, seed=13).check([5000, 25_999, 1, 13_000], sink=1, recent=9)
    lens = [70_000] + [200] * 30
    for values in (None, [0.5]):
        Histories(16, lens, layers=1, heads=2, seed=14, values=values).check([n // 3 for n in lens], recent=5)


def test_malformed_tables_of_split_choices():
    """A length that its table cannot hold, a negative budget, offsets that decrease: reported; the others of the first two are
    chosen as ever, and so is a good call after them."""
    _say("split, malformed")
    pk, e = engine(32)
    b = Histories(32, [60_000, 50_000, 40_000], layers=2, heads=2, seed=17)
    budget = [7000, 800, 39_000]
    want = b.expected(budget)

    def run(off, length, budget):
        kept = torch.full((2, 2, b.rows + 1), -7, dtype=torch.int32, device="cuda")
        keep, grow = torch.full((3,), -7, device="cuda"), torch.full((3,), -7, device="cuda")
        e.evict_select((dev(off), dev(b.page), dev(length)), dev(b.w), dev(np.array(budget, np.int64)), None, kept, keep, grow)
        try:
            e.sync()
        except pk.DMError:
            return kept.cpu().numpy(), keep.tolist(), True
        return kept.cpu().numpy(), keep.tolist(), False

    others = want.copy()
    a = int(b.off[1]) * 32
    others[..., a:a + budget[1]] = -7
    for length, budgets, keep1 in ((np.array([60_000, 50_100, 40_000]), budget, 0), (b.len, [7000, -1, 39_000], 50_000)):
        kept, keep, told = run(b.off, length.astype(np.int64), budgets)
        assert told and np.array_equal(kept, others) and keep == [0, keep1, 0]
    _say("decreasing offsets")
    _, _, told = run(np.array([0, b.off[2], b.off[1], b.off[3]], np.int64), np.array([100_000, 9, 80_000], np.int64), budget)
    assert told
    kept, keep, told = run(b.off, b.len, budget)
    assert not told and np.array_equal(kept, want) and keep == [0, 0, 0]


def test_a_split_choice_in_a_graph():
    """Its work area is the context's: the same replays before and after a larger call has grown it."""
    _say("split graph")
    pk, _ = engine(64)
    b = Histories(64, [60_000, 30_000], layers=2, heads=2, seed=15)
    budget = [4000, 29_000]
    want = b.expected(budget)
    tables, w, bud = b.tables(), dev(b.w), dev(np.array(budget, np.int64))
    kept = torch.full((2, 2, b.rows + 1), -7, dtype=torch.int32, device="cuda")
    keep, grow = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")

    def run(eng):
        eng.evict_select(tables, w, bud, None, kept, keep, grow)

    st = torch.cuda.Stream()
    own = pk.DualMap(dict(block=64, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        run(own)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        run(own)
    for turn in range(4):
        kept.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(kept.cpu().numpy(), want), turn
        if turn == 1:
            more = Histories(64, [200_000, 100_000], layers=2, heads=2, seed=16)
            with torch.cuda.stream(st):
                got, _, _ = more.select([1000, 2000], eng=own)
            assert np.array_equal(got, more.expected([1000, 2000]))
            torch.cuda.synchronize()
    own.sync()
    own.close()


def test_many_short_histories():
    r = np.random.default_rng(1)
    lens = r.integers(0, 200, size=700)
    Histories(8, lens, layers=1, heads=2, seed=6).check(r.integers(0, 150, size=700).tolist(), sink=2, recent=5)


class Move:
    """Histories, their keys and values, and the next tables: fresh pages for sequences past their budgets."""

    def __init__(self, block, lens, budget, dim=64, dtype="bf16", layers=2, heads=4, share=1, seed=0, extra=0):
        self.h = h = Histories(block, lens, layers, heads, seed)
        self.budget = np.array(budget, np.int64)
        r, g = np.random.default_rng(seed + 1), torch.Generator().manual_seed(seed)
        past = h.len > self.budget
        to_len = np.where(past, self.budget, h.len) + r.integers(0, 9, size=len(lens))
        need = -(-to_len // block)
        old = -(-h.len // block)
        fresh = np.where(past, need, np.maximum(0, need - old))
        first = h.pages
        self.pages = first + int(fresh.sum()) + extra
        ids = first + r.permutation(int(fresh.sum()) + extra)
        rows, at = [], 0
        for s in range(len(lens)):
            kept = [] if past[s] else h.page[h.off[s]:h.off[s + 1]].tolist()
            rows.append(kept + ids[at:at + fresh[s]].tolist())
            at += fresh[s]
        self.to_off = np.concatenate([[0], np.cumsum([len(x) for x in rows])]).astype(np.int64)
        self.to_page = np.array(sum(rows, []) or [0], np.int32)
        self.to_len, self.past, self.share = to_len, past, share
        shape = (layers + 1, self.pages, heads, block, dim)
        self.k, self.v = (torch.randn(shape, generator=g).to(DT[dtype]) for _ in range(2))
        self.kept = h.expected(self.budget, sink=1, recent=2, share=share)[..., :h.rows]

    def expected(self):
        h, B = self.h, self.h.block
        k, v = self.k.clone(), self.v.clone()
        w = np.full((h.layers, h.heads, len(self.to_page) * B), -5, np.float32)
        for s in range(len(h.len)):
            a, b = int(h.off[s]) * B, int(self.to_off[s]) * B
            n = int(self.budget[s]) if self.past[s] else int(h.len[s])
            for layer in range(h.layers):
                for g in range(h.heads):
                    t = self.kept[layer, g // self.share, a:a + n] if self.past[s] else np.arange(n)
                    w[layer, g, b:b + n] = h.w[layer, g, a + t]
                    if self.past[s]:
                        i = np.arange(n)
                        p, q = h.page[h.off[s] + t // B].astype(np.int64), self.to_page[self.to_off[s] + i // B].astype(np.int64)
                        for x, y in ((self.k, k), (self.v, v)):
                            y[layer, q, g, i % B] = x[layer, p, g, t % B]
        return k, v, w

    def run(self, weights=True):
        pk, e = engine(self.h.block)
        h = self.h
        k, v = self.k.cuda(), self.v.cuda()
        kv = pk.KVPages(k[:h.layers], v[:h.layers])
        w_to = torch.full((h.layers, h.heads, len(self.to_page) * h.block), -5.0, device="cuda")
        to = (dev(self.to_off), dev(self.to_page), dev(self.to_len))
        e.kv_gather(kv, h.tables(), to, dev(self.budget), dev(self.kept), *((dev(h.w), w_to) if weights else ()))
        e.sync()
        return k.cpu(), v.cpu(), w_to.cpu().numpy()

    def check(self):
        k, v, w = self.expected()
        for weights in (True, False):
            k1, v1, w1 = self.run(weights)
            assert torch.equal(k1.view(torch.int16), k.view(torch.int16)) and torch.equal(v1.view(torch.int16), v.view(torch.int16))
            assert np.array_equal(w1, w) if weights else (w1 == -5).all()


@pytest.mark.parametrize("block", [4, 8, 16, 32, 64])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_move(block, dim):
    _say("move", block, dim)
    lens = [1, 90, 64, 65, 300, 17, 0, 130]
    Move(block, lens, [1, 30, 63, 80, 128, 1, 0, 0], dim=dim, dtype="f16" if dim == 64 else "bf16", seed=block).check()


@pytest.mark.parametrize("heads,share", [(1, 1), (3, 1), (6, 3), (8, 8), (2, 2)])
def test_move_of_heads(heads, share):
    _say("heads", heads, share)
    Move(16, [40, 200, 33], [20, 111, 32], heads=heads, share=share, seed=heads).check()


def test_long_move():
    Move(32, [5000, 900], [2500, 900], layers=1, heads=2, dim=128, seed=9).check()


def test_malformed_calls_are_reported():
    pk, e = engine(16)
    b = Histories(16, [100, 60], seed=1)
    n = b.len.copy()
    good = b.select([30, 30])
    # a length that its table cannot hold, offsets out of order, a negative budget
    b.len[0] = 500
    with pytest.raises(pk.DMError):
        b.select([30, 30])
    b.len = n
    with pytest.raises(pk.DMError):
        b.select([-1, 30])
    again = b.select([30, 30])
    assert all(np.array_equal(x, y) for x, y in zip(good, again))
    m = Move(16, [100, 60, 40], [30, 30, 20], seed=2)
    ref = m.expected()
    for where, what in ((0, 100), (1, -1), (29, 1 << 30)):
        bad = Move(16, [100, 60, 40], [30, 30, 20], seed=2)
        bad.kept[0, 1, where] = what
        with pytest.raises(pk.DMError):
            bad.run()
    bad = Move(16, [100, 60, 40], [30, 30, 20], seed=2)
    bad.to_page[0] = bad.pages
    with pytest.raises(pk.DMError):
        bad.run()
    bad = Move(16, [100, 60, 40], [30, 30, 20], seed=2)
    bad.budget[0] = 90  # no room for as many
    with pytest.raises(pk.DMError):
        bad.run()
    k, v, w = m.run()
    assert torch.equal(k, ref[0]) and torch.equal(v, ref[1]) and np.array_equal(w, ref[2])


def test_refusals():
    pk, e = engine(16)
    b = Histories(16, [100, 60], seed=1)
    t, w = b.tables(), dev(b.w)
    budget = dev(np.array([30, 30], np.int64))
    kept = torch.zeros((2, 4, b.rows), dtype=torch.int32, device="cuda")
    keep, grow = torch.zeros_like(budget), torch.zeros_like(budget)
    for bad in (w[0], w[..., 1:], w.double(), w.cpu(), w.transpose(1, 2), None):
        with pytest.raises(ValueError):
            e.evict_select(t, bad, budget, None, kept, keep, grow)
    for bad in (kept[:1], kept[:, :3].contiguous(), kept[..., 1:].contiguous(), kept.long()):
        with pytest.raises(ValueError, match="kept"):
            e.evict_select(t, w, budget, None, bad, keep, grow)
    for kw in (dict(share=3), dict(share=0), dict(sink=-1), dict(recent=1 << 31)):
        with pytest.raises(ValueError):
            e.evict_select(t, w, budget, None, kept, keep, grow, **kw)
    for bad in ((budget[:1], None, keep, grow), (budget, budget[:1], keep, grow), (budget, None, keep.int(), grow)):
        with pytest.raises(ValueError, match="entry for each|contiguous"):
            e.evict_select(t, w, bad[0], bad[1], kept, bad[2], bad[3])
    x = torch.zeros((2, b.pages, 4, 16, 64), dtype=torch.bfloat16, device="cuda")
    kv = pk.KVPages(x, x.clone())
    w_to = torch.zeros_like(w)
    for kw in (dict(kept=kept[0]), dict(kept=kept[:1]), dict(kept=kept[:, :3].contiguous()), dict(w=w), dict(w_to=w_to),
               dict(w=w, w_to=w_to[..., 1:]), dict(w=w[:1], w_to=w_to[:1]), dict(budget=budget[:1])):
        a = {**dict(budget=budget, kept=kept), **kw}
        with pytest.raises(ValueError):
            e.kv_gather(kv, t, t, **a)
    with pytest.raises(ValueError, match="first"):
        q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
        e.kv_append(kv, 0, t, dev(np.array([0, 1, 2], np.int64)), q, q.clone(), q.clone(), q, first=budget[:1])


def _turned(x, pos, cos, sin):
    half = cos.shape[1]
    c, s = cos[pos].double()[:, None], sin[pos].double()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def test_append_at_positions():
    """Rows go to their places, the rotation by the positions given; NULL positions are the places."""
    pk, e = engine(16)
    B, H, D, new = 16, 2, 64, [3, 1, 0, 40]
    lens = np.array([20, 7, 5, 90], np.int64)
    h = Histories(B, lens, seed=7)
    q_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    T = int(q_off[-1])
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((T, n, D), generator=g).bfloat16() for n in (4, H, H))
    angle = torch.arange(2000)[:, None] * 10000.0 ** -(torch.arange(D // 2) / (D // 2))
    cos, sin = angle.cos().float(), angle.sin().float()
    first = np.array([500, 0, 9, 1900], np.int64)

    def run(first):
        kv = pk.KVPages(*(torch.full((1, h.pages, H, B, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        out = torch.zeros_like(q, device="cuda")
        e.kv_append(kv, 0, h.tables(), dev(q_off), q.cuda(), k.cuda(), v.cuda(), out, cos=cos.cuda(), sin=sin.cuda(), first=first)
        e.sync()
        return out.cpu(), kv.k.cpu(), kv.v.cpu()

    out, pk_, pv = run(dev(first))
    pos = np.concatenate([first[s] + np.arange(new[s]) for s in range(4)])
    u = ULP["bf16"] * 1.02
    want = _turned(q.double(), pos, cos, sin)
    tol = u * want.abs() + 2.0 ** -20 * q.double().abs().amax(-1, keepdim=True)
    assert bool(((out.double() - want).abs() <= tol).all())
    key = _turned(k.double(), pos, cos, sin)
    for s in range(4):
        for i in range(new[s]):
            p = int(lens[s]) - new[s] + i
            page, t = int(h.page[h.off[s] + p // B]), int(q_off[s]) + i
            assert bool(((pk_[0, page, :, p % B].double() - key[t]).abs() <= u * key[t].abs() + 2.0 ** -20 * k[t].double().abs().max()).all())
            assert torch.equal(pv[0, page, :, p % B], v[t])
    plain = run(None)
    same = run(dev(lens - np.array(new)))
    assert all(torch.equal(a, b) for a, b in zip(plain, same))
    with pytest.raises(pk.DMError):  # past the rotation's tables
        run(dev(first + 90))


@pytest.mark.parametrize("paired", [False, True])
def test_calls_together(paired):
    """Prompts, then single tokens, in a bounded cache: append at positions, attention, weights, choice, tables, move. Each step
    against a plain model of it that keeps every sequence's rows by itself, in 64 bits from the same stored rows."""
    pk, e = engine(16)
    B, HQ, H, D, LAYERS, PAGES, MAX = 16, 8, 4, 64, 2, 120, 400
    g = torch.Generator().manual_seed(5)
    angle = torch.arange(MAX)[:, None] * 10000.0 ** -(torch.arange(D // 2) / (D // 2))
    cos, sin = angle.cos().float().cuda(), angle.sin().float().cuda()
    kv = pk.KVPages(*(torch.zeros((LAYERS, PAGES, H, B, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    lam = 0.3 + 0.1 * torch.arange(HQ // 2)
    norm = (1 + 0.1 * torch.randn(2 * D, generator=g)).bfloat16()
    i64 = dict(dtype=torch.int64, device="cuda")
    ref = torch.zeros(PAGES, dtype=torch.int32, device="cuda")
    tables = (torch.zeros(1, **i64), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, **i64))
    n, prompts, budget, sink, recent, share = 3, [70, 33, 120], 48, 2, 8, 2 if paired else 1
    new = list(prompts)
    seen = np.zeros(n, np.int64)  # positions so far
    src, keep, grow = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, **i64), torch.tensor(prompts, **i64)
    w, evicted = None, 0
    # the plain model: rows (positions, keys, values, weights) of [layer][sequence][head]
    rows = [[[dict(k=torch.zeros(0, D), v=torch.zeros(0, D), w=torch.zeros(0).double()) for _ in range(H)] for _ in range(n)]
            for _ in range(LAYERS)]
    for step in range(6):
        _say("step", step)
        cap = int((((keep + grow) + B - 1) // B).sum().item())
        old, fork = tables, e.pages_fork(tables, ref, src, keep, grow, max(cap, 1))
        e.pages_copy(kv, fork)
        tables, ref = (fork["off"], fork["page"], fork["len"]), fork["ref"]
        places = tables[1].numel() * B
        if w is not None:
            w_to = torch.full((LAYERS, H, places), 9.0, device="cuda")
            e.kv_gather(kv, old, tables, budgets, kept, w, w_to)
            prev = w_to
        else:
            prev = None
        w = torch.zeros((LAYERS, H, places), device="cuda")
        lens = tables[2].cpu().numpy()
        q_off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **i64)
        T = sum(new)
        plan = (e.diff_plan if paired else e.attn_plan)(kv, tables, q_off, T, HQ)
        for layer in range(LAYERS):
            q, k, v = (torch.randn((T, m, D), generator=g).bfloat16().cuda() * f for m, f in ((HQ, 2), (H, 1), (H, 1)))
            e.kv_append(kv, layer, tables, q_off, q, k, v, q, cos=cos, sin=sin, first=torch.tensor(seen, **i64))
            out, lse = torch.zeros_like(q), torch.zeros((T, HQ), device="cuda")
            if paired:
                e.diff_attn(plan, layer, q, D ** -0.5, lam.cuda(), out, lse, norm=norm.cuda())
            else:
                e.attn(plan, layer, q, D ** -0.5, out, lse)
            e.attn_weights(plan, layer, q, D ** -0.5, lse, w[layer], prev=None if prev is None else prev[layer], decay=0.5)
            e.sync()
            pages = [x[layer].cpu() for x in (kv.k, kv.v)]
            at, off, qh, w_now = tables[1].cpu().numpy(), tables[0].cpu().numpy(), q.cpu().double(), w[layer].cpu().double()
            turned = [_turned(x.cpu().double(), np.concatenate([seen[s] + np.arange(new[s]) for s in range(n)]), cos.cpu(),
                              sin.cpu()) for x in (k,)][0]
            for s in range(n):
                t0, t1, L = int(q_off[s]), int(q_off[s + 1]), int(lens[s])
                ids = at[off[s]:off[s] + -(-L // B)].astype(np.int64)
                maps = []
                for h in range(H):
                    m = rows[layer][s][h]
                    K, V = (x[ids, h].reshape(-1, D)[:L] for x in pages)
                    have = len(m["k"])
                    assert have + new[s] == L
                    # what was kept is there, bit for bit; what is new, to its rounding
                    assert torch.equal(K[:have].float(), m["k"]) and torch.equal(V[:have].float(), m["v"])
                    err = (K[have:].double() - turned[t0:t1, h]).abs()
                    assert bool((err <= ULP["bf16"] * 1.02 * turned[t0:t1, h].abs() + 1e-5).all())
                    assert torch.equal(V[have:], v[t0:t1, h].cpu())
                    m["k"], m["v"] = K.float(), V.float()
                    hidden = torch.arange(L) > (L - new[s] + torch.arange(new[s]))[:, None]
                    r = HQ // H
                    xs = [2 * (h // 2 * r + i) + h % 2 for i in range(r)] if paired else list(range(h * r, (h + 1) * r))
                    add = torch.zeros(L).double()
                    for x in xs:
                        z = torch.softmax((qh[t0:t1, x] @ K.double().T * D ** -0.5).masked_fill(hidden, -math.inf), -1)
                        add += z.sum(0)
                        maps.append((x, z, V.double()))
                    m["w"] = torch.cat([0.5 * m["w"], torch.zeros(new[s]).double()]) + add
                    got = w_now[h, off[s] * B:off[s] * B + L]
                    assert bool(((got - m["w"]).abs() <= 1e-4 * m["w"] + 1e-6).all()), (step, layer, s, h)
                    m["w"] = got.clone()
                by = {x: (z, V) for x, z, V in maps}
                for x in by:
                    if not paired:
                        want = by[x][0] @ by[x][1]
                        mean = by[x][0] @ by[x][1].abs()
                        err = (out[t0:t1, x].cpu().double() - want).abs()
                        assert bool((err <= ULP["bf16"] * 1.02 * (want.abs() + mean) + 1e-5).all())
                    elif x % 2 == 0:
                        V2 = torch.cat([by[x][1], by[x + 1][1]], 1)
                        o = by[x][0] @ V2 - float(lam[x // 2]) * (by[x + 1][0] @ V2)
                        d = (1.02 * ULP["bf16"] + 1e-5) * (by[x][0] @ V2.abs() + float(lam[x // 2]) * (by[x + 1][0] @ V2.abs()))
                        N, dn = torch.sqrt((o * o).sum(-1, keepdim=True) + 2 * D * 1e-5), d.norm(dim=-1, keepdim=True)
                        by_w = math.sqrt(2 * D) * norm.double()
                        tol = torch.where(dn < N, d / (N - dn) + o.abs() * dn / (N * (N - dn)), math.inf) * by_w.abs()
                        want = o / N * by_w
                        tol = tol + (ULP["bf16"] * 1.02 + 1e-5) * (want.abs() + tol)
                        assert bool(((out[t0:t1, x:x + 2].flatten(1).cpu().double() - want).abs() <= tol).all())
        seen += np.array(new)
        # the next step: a token or a few each
        new = [1, 2, 1]
        budgets = torch.full((n,), budget, **i64)
        kept = torch.zeros((LAYERS, H // share, places), dtype=torch.int32, device="cuda")
        src, keep, grow = torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros(n, **i64), torch.zeros(n, **i64)
        e.evict_select(tables, w, budgets, torch.tensor(new, **i64), kept, keep, grow, sink=sink, recent=recent, share=share)
        e.sync()
        for s in range(n):
            if lens[s] <= budget:
                assert int(keep[s]) == lens[s]
                continue
            evicted += 1
            a = int(off[s]) * B
            for layer in range(LAYERS):
                wl = w[layer].cpu().numpy()
                for c in range(H // share):
                    x = wl[c * share, a:a + lens[s]]
                    for h in range(1, share):
                        x = x + wl[c * share + h, a:a + lens[s]]
                    want = choice(x, budget, sink, recent)
                    assert kept[layer, c, a:a + budget].tolist() == want.tolist()
                    for h in range(c * share, (c + 1) * share):
                        m = rows[layer][s][h]
                        m["k"], m["v"], m["w"] = m["k"][want], m["v"][want], m["w"][want]
        live = int((ref > 0).sum().item())
        assert live == int(tables[0][-1].item())
    assert evicted >= 8


def test_choice_and_move_in_a_graph():
    """Captured and replayed with other weights and budgets, each replay equal to the eager result."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    m = Move(16, [300, 90, 64], [100, 40, 64], seed=3)
    h = m.h
    kv = pk.KVPages(m.k.cuda(), m.v.cuda())
    kv2 = pk.KVPages(kv.k[:h.layers], kv.v[:h.layers])
    t, to = h.tables(), (dev(m.to_off), dev(m.to_page), dev(m.to_len))
    w, budget = dev(h.w), dev(m.budget)
    kept = torch.zeros((h.layers, h.heads, h.rows), dtype=torch.int32, device="cuda")
    keep, grow = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    w_to = torch.zeros((h.layers, h.heads, len(m.to_page) * 16), device="cuda")

    def call():
        e.evict_select(t, w, budget, None, kept, keep, grow, sink=1, recent=2)
        e.kv_gather(kv2, t, to, budget, kept, w, w_to)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    r = np.random.default_rng(8)
    for i in range(4):
        h.w = np.exp(2 * r.standard_normal(h.w.shape)).astype(np.float32)
        m.budget = np.array([100 - 7 * i, 40 - i, 64], np.int64)
        m.kept = h.expected(m.budget, sink=1, recent=2)[..., :h.rows]
        w.copy_(torch.from_numpy(h.w))
        budget.copy_(torch.from_numpy(m.budget))
        kv.k.copy_(m.k)
        kv.v.copy_(m.v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        k, v, want = m.expected()
        assert torch.equal(kv.k.cpu().view(torch.int16), k.view(torch.int16))
        assert torch.equal(kv.v.cpu().view(torch.int16), v.view(torch.int16))
        got = w_to.cpu().numpy()
        assert np.array_equal(got[want != -5], want[want != -5])
    e.sync()
    e.close()


@pytest.mark.parametrize("lens,budget", [([100, 60, 200], [30, 30, 250]), ([60_000, 50_000, 40_000], [7000, 800, 41_000])])
@pytest.mark.parametrize("what", ["length", "room"])
def test_a_malformed_sequence_frees_nothing(lens, budget, what):
    """The fork that follows a choice at once, with these tables or with good ones, takes nothing of it: no page is freed, and
    what dm_sync reports comes in time. Whole choices and split ones."""
    pk, e = engine(32)
    b = Histories(32, lens, seed=5)
    n = len(lens)
    length, room = b.len.copy(), np.array([3, 4, 5], np.int64)
    if what == "length":
        length[1] += 4000
    else:
        room[1] = -1
    good, asked = b.tables(), (dev(b.off), dev(b.page), dev(length))
    ref = torch.zeros(b.pages + 4000, dtype=torch.int32, device="cuda")
    ref[torch.from_numpy(b.page.astype(np.int64)).cuda()] = 1
    src = torch.arange(n, dtype=torch.int32, device="cuda")

    def run(tables, room, then):
        kept = torch.full((2, 4, b.rows), -7, dtype=torch.int32, device="cuda")
        keep, grow = torch.full((n,), -7, device="cuda"), torch.full((n,), -7, device="cuda")
        out = e.alloc_pages_out(ref.numel(), n, 6000)
        for x in out.values():
            if x is not None:
                x.fill_(-5)
        e.evict_select(tables, dev(b.w), dev(np.array(budget, np.int64)), dev(room), kept, keep, grow)
        e.pages_fork_into(then, ref, src, keep, grow, out)
        try:
            e.sync()
        except pk.DMError:
            return keep.tolist(), grow.tolist(), out, True
        return keep.tolist(), grow.tolist(), out, False

    for then in (asked, good):
        _say("malformed", what, lens, "good" if then is good else "same")
        keep, grow, out, told = run(asked, room, then)
        assert told and int(out["moves"][0]) == 0 and bool((out["ref"] == -5).all()) and bool((out["len"] == -5).all())
        assert keep == [0, 0, lens[2]] and grow == [budget[0] + 3, -1, 5]
    keep, grow, out, told = run(good, np.array([3, 4, 5], np.int64), good)
    assert not told and keep == [0, 0, lens[2]] and grow == [budget[0] + 3, budget[1] + 4, 5]
    assert out["len"].tolist() == [budget[0] + 3, budget[1] + 4, lens[2] + 5]


def test_malformed_tables_without_entries_are_reported():
    """Sequences that the next tables have no entry of: freed ones have nothing moved, malformed ones are reported all the same."""
    pk, e = engine(16)
    h = Histories(16, [100, 60, 40], seed=2)
    k = torch.randn((2, h.pages + 4, 4, 16, 64)).bfloat16().cuda()
    kv, start = pk.KVPages(k, k.clone()), k.clone()
    kept = dev(np.zeros((2, 4, h.rows), np.int32))
    page = dev(np.array([h.pages, h.pages + 1], np.int32))

    def run(length, to_off, budget, page=page):
        to = (dev(np.array(to_off, np.int64)), page, dev(np.zeros(3, np.int64)))
        e.kv_gather(kv, (dev(h.off), dev(h.page), dev(np.array(length, np.int64))), to, dev(np.array(budget, np.int64)), kept)
        e.sync()

    _say("freed")
    run([100, 60, 40], [0, 0, 0, 0], [30, 30, 30])
    run([100, 60, 40], [0, 0, 0, 0], [30, 30, 30], page=page[:0])
    assert torch.equal(kv.k, start)
    for length, to_off, budget in (([100, 600, 40], [0, 0, 0, 0], [30, 30, 30]), ([100, 60, -1], [0, 0, 0, 0], [30, 30, 30]),
                                   ([100, 60, 40], [0, 0, 0, 0], [30, -1, 30]), ([100, 60, 40], [0, 0, -1, -1], [30, 30, 30]),
                                   ([100, 60, 40], [2, 0, 0, 0], [30, 30, 30]), ([100, 60, 40], [0, 0, 0, 5], [30, 30, 30])):
        for p in (page, page[:0]):
            _say("reported", length, to_off, budget, p.numel())
            with pytest.raises(pk.DMError):
                run(length, to_off, budget, page=p)
            # (a last sequence of more entries than there are is of this call's first ones: none of it is moved)
            assert torch.equal(kv.k, start)
    run([100, 60, 40], [0, 0, 0, 0], [30, 30, 30])
