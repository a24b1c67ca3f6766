"""Attention over KV pages against its definition in 64 bits.

Bounds, per element, from the roundings that the kernels make (u: half a unit in
the last place of the type, 2^-8 for bfloat16, 2^-11 for float16): the output is
rounded once, u |out|; every weight is rounded once before it meets the values,
u sum w|v| / sum w; a float16 weight below 2^-14 of the largest is off by up to
2^-25 of it, n 2^-25 max|v| over n keys; sums in 32 bits add some 2^-20 of sum
w|v| / sum w.  The log-sum-exp is in 32 bits: 2^-18 of the largest |score|, and of
itself.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
_ENG = {}


def engine(block):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_06502_amd as pk
    if block not in _ENG:
        _ENG[block] = pk.DualMap(dict(block=block, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1,
                                      index_log2_slots=4))
    return pk, _ENG[block]


class Batch:
    """Sequences with (new tokens, tokens of their own, run); a run's prefix is shared pages.  Pages are
    scattered; what no token fills holds NaN."""

    def __init__(self, block, seqs, prefixes=(), heads=(8, 2), dim=128, dtype="bf16", seed=0, layers=1,
                 layer=0, pad_q=0, spare=3, qscale=2.0):
        self.block, self.dim, self.dtype, self.layer = block, dim, dtype, layer
        self.hq, self.hkv = heads
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        B = block
        new = [s[0] for s in seqs]
        own = [s[1] for s in seqs]
        run = [s[2] if len(s) > 2 else -1 for s in seqs]
        pre = [prefixes[k] if k >= 0 else 0 for k in run]
        assert all(p % B == 0 for p in prefixes)
        self.len = np.array([p + o for p, o in zip(pre, own)], np.int64)
        own_pages = [-(-o // B) for o in own]
        total = sum(p // B for p in prefixes) + sum(own_pages)
        n_pages = total + spare
        ids = r.permutation(n_pages)[:total]
        at, pref = 0, []
        for p in prefixes:
            pref.append(ids[at:at + p // B])
            at += p // B
        page, off = [], [0]
        for k, n in zip(run, own_pages):
            row = (list(pref[k]) if k >= 0 else []) + list(ids[at:at + n])
            at += n
            page += row
            off.append(len(page))
        self.page, self.off = np.array(page + [0], np.int32)[:len(page)], np.array(off, np.int64)
        self.q_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        self.groups = None
        if prefixes:
            assert run == sorted(run)
            self.groups = np.concatenate([[0], np.flatnonzero(np.diff(run)) + 1, [len(run)]]).astype(np.int64)
        T = int(self.q_off[-1])
        shape = (layers, n_pages, self.hkv, B, dim)
        dt = DT[dtype]
        self.k = torch.randn(shape, generator=g).to(dt)
        self.v = torch.randn(shape, generator=g).to(dt)
        width = self.hq * dim + pad_q
        self.qrows = (qscale * torch.randn((T, width), generator=g)).to(dt)
        # stale places
        filled = np.zeros((n_pages, B), bool)
        for s in range(len(seqs)):
            for t in range(int(self.len[s])):
                filled[page[off[s] + t // B], t % B] = True
        stale = torch.from_numpy(~filled)
        for x in (self.k, self.v):
            x.permute(1, 3, 0, 2, 4)[stale] = float("nan")

    def dev(self, x):
        return None if x is None else torch.from_numpy(x).cuda()

    def tables(self):
        return self.dev(self.off), self.dev(self.page), self.dev(self.len)

    def run(self, lse=True, groups=True, eng=None, scale=None, reps=1):
        pk, e = engine(self.block)
        e = eng or e
        kv = pk.KVPages(self.k.cuda(), self.v.cuda())
        T = int(self.q_off[-1])
        q = self.qrows.cuda()[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim))
        out = torch.full((T, self.hq, self.dim), 7.0, dtype=DT[self.dtype], device="cuda")
        far = torch.full((T, self.hq), 7.0, device="cuda") if lse else None
        plan = e.attn_plan(kv, self.tables(), self.dev(self.q_off), T, self.hq,
                           groups=self.dev(self.groups) if groups else None)
        for _ in range(reps):
            e.attn(plan, self.layer, q, self.scale(scale), out, far)
        e.sync()
        return out.cpu(), None if far is None else far.cpu()

    def scale(self, s=None):
        return self.dim ** -0.5 if s is None else s

    def reference(self, scale=None):
        """(out, lse, bound of out, bound of lse) in 64 bits; a token sees the first position + 1 keys."""
        T = int(self.q_off[-1])
        out = torch.zeros((T, self.hq, self.dim), dtype=torch.float64)
        lse = torch.full((T, self.hq), -math.inf, dtype=torch.float64)
        tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
        u = ULP[self.dtype]
        q = self.qrows[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim)).double()
        for s in range(len(self.len)):
            L, t0, t1 = int(self.len[s]), int(self.q_off[s]), int(self.q_off[s + 1])
            if L == 0 or t0 == t1:
                continue
            at = torch.from_numpy(self.page[self.off[s]:self.off[s] - (-L // self.block)].astype(np.int64))
            for h in range(self.hkv):
                K = self.k[self.layer][at, h].reshape(-1, self.dim)[:L].double()
                V = self.v[self.layer][at, h].reshape(-1, self.dim)[:L].double()
                for t in range(t0, t1):
                    n = L - (t1 - t0) + (t - t0) + 1
                    if n <= 0:
                        continue
                    x = slice(h * self.hq // self.hkv, (h + 1) * self.hq // self.hkv)
                    sc = q[t, x] @ K[:n].T * self.scale(scale)
                    w = torch.softmax(sc, -1)
                    out[t, x] = w @ V[:n]
                    lse[t, x] = torch.logsumexp(sc, -1)
                    mean = w @ V[:n].abs()
                    tol[t, x] = u * (out[t, x].abs() + mean) * 1.02 + 2.0 ** -20 * mean + \
                        (n * 2.0 ** -25 * V[:n].abs().max() + 2.0 ** -25 if self.dtype == "f16" else 0.0)
                    ltol[t, x] = 2.0 ** -18 * (sc.abs().amax(-1) + lse[t, x].abs() + 1)
        return out, lse, tol, ltol

    def check(self, scale=None, **kw):
        out, lse = self.run(scale=scale, **kw)
        ref, rl, tol, ltol = self.reference(scale)
        err = (out.double() - ref).abs()
        bad = ~(err <= tol)
        assert not bool(bad.any()), ("out", int(bad.sum()), float((err / tol.clamp(min=1e-30)).nan_to_num(1e9).max()))
        if lse is not None:
            same = (lse.double() == rl) | ((lse.double() - rl).abs() <= ltol)
            assert bool(same.all()), ("lse", int((~same).sum()))


def _say(*a):
    print("[case]", *a, flush=True)


# one token each, lengths around tiles, pages and chunks
DECODE = [(1, n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 300, 511, 640)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (14, 2), (6, 2)])
def test_single_tokens(dtype, dim, heads):
    _say("decode", dtype, dim, heads)
    Batch(16, DECODE, heads=heads, dim=dim, dtype=dtype, seed=dim + heads[0]).check()


@pytest.mark.parametrize("block", [4, 8, 16, 32, 64])
def test_page_sizes(block):
    _say("block", block)
    Batch(block, [(1, 1), (3, 200), (40, 77), (1, 333), (90, 90), (7, 130)], heads=(8, 2), seed=block).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [(2, 2), (8, 2), (7, 1)])
def test_prompts(dtype, dim, heads):
    """Wide tiles: several new tokens with and without earlier ones, rows around tiles."""
    _say("prompts", dtype, dim, heads)
    Batch(16, [(33, 33), (1, 1), (128, 300), (64, 64), (65, 129), (200, 200), (17, 500)], heads=heads, dim=dim,
          dtype=dtype, seed=3).check()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_shared_prefixes(dim):
    """Runs that share, alone and not: single tokens, drafts and prompts, equal to the result without runs."""
    seqs = [(1, 1, 0), (1, 40, 0), (1, 17, 0), (3, 30, 1), (1, 1, 2), (1, 5, 2), (5, 5, 2), (1, 90, 2), (1, 2, 2),
            (1, 1, 2), (2, 33, 2), (40, 50, 3), (60, 60, 3)]
    b = Batch(16, seqs, prefixes=(256, 128, 640, 320), heads=(8, 2), dim=dim, seed=5)
    _say("shared", dim)
    b.check()
    b.check(groups=False)


def test_many_sequences_share():
    """A run whose rows fill wide tiles, odd ratio."""
    Batch(32, [(1, 1 + i % 70, 0) for i in range(45)] + [(1, 9, 1)], prefixes=(352, 160), heads=(14, 2), dim=64,
          dtype="f16", seed=6).check()


def test_runs_that_have_nothing_in_common():
    b = Batch(16, [(1, 100), (1, 200), (2, 300)], seed=7)
    b.groups = np.array([0, 3], np.int64)
    b.check()
    b.groups = np.array([0, 0, 2, 2, 3], np.int64)  # empty runs
    b.groups = b.groups[[0, 2, 3, 4]]
    b.check()


@pytest.mark.parametrize("n,runs", [(70, 3), (200, 100), (600, 5), (1300, 1100)])
def test_many_sequences_and_runs(n, runs):
    """More sequences than have a workgroup each in the plan, more units than it has threads, more runs than fit its LDS."""
    _say("many", n, runs)
    r = np.random.default_rng(n)
    run = np.sort(np.concatenate([np.arange(runs), r.integers(0, runs, size=n - runs)]))
    seqs = [(int(r.integers(1, 3)), int(r.integers(2, 40)), int(g)) for g in run]
    Batch(8, seqs, prefixes=[int(8 * r.integers(0, 30)) for _ in range(runs)], heads=(2, 1), dim=64, seed=n).check()


@pytest.mark.parametrize("tokens,keys,dim", [(96, 1500, 128), (200, 700, 64), (1, 3000, 128), (130, 900, 256)])
def test_same_bits_with_a_full_gpu(tokens, keys, dim):
    """A full GPU's worth of items, twelve times: nothing in a result goes by which wave or workgroup comes first."""
    _say("again", tokens, keys, dim)
    b = Batch(16, [(tokens, keys + 37 * i) for i in range(64)], heads=(16, 4), dim=dim, seed=3)
    pk, e = engine(16)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    t = tuple(torch.from_numpy(x).cuda() for x in (b.off, b.page, b.len))
    q_off, T = torch.from_numpy(b.q_off).cuda(), int(b.q_off[-1])
    q = b.qrows.unflatten(1, (16, dim)).contiguous().cuda()
    first = None
    for _ in range(12):
        out, lse = torch.full_like(q, 7), torch.full((T, 16), 7.0, device="cuda")
        e.attn(e.attn_plan(kv, t, q_off, T, 16), 0, q, dim ** -0.5, out, lse)
        e.sync()
        if first is None:
            first = out, lse
        assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])


def test_rows_around_tiles():
    """Rows of a unit around a narrow tile, the last narrow unit and a wide tile."""
    for ratio in (1, 3, 8):
        rows = sorted({x // ratio for x in (15, 16, 17, 32, 47, 48, 63, 64, 65, 66, 127, 128, 129, 256, 257)} - {0})
        _say("rows", ratio, rows)
        Batch(16, [(t, t + 90) for t in rows], heads=(ratio, 1), dim=64, seed=ratio).check()


def test_plan_and_attention_in_a_graph():
    """Captured, replayed with other lengths, tables and queries, each replay equal to the eager result's bits."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    sets = [Batch(16, [(1, 30 + 7 * i, 0), (1, 50, 0), (2, 9 + i, 0), (40, 60, 0), (1, 200 + i, 1), (1, 1, 1)],
                  prefixes=(256, 320), seed=30 + i, spare=9 - i) for i in range(3)]
    T = int(sets[0].q_off[-1])
    most = max(len(b.page) for b in sets)
    pages = max(b.k.shape[1] for b in sets)
    k = torch.zeros((1, pages) + tuple(sets[0].k.shape[2:]), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    kv = pk.KVPages(k, v)
    i64 = dict(dtype=torch.int64, device="cuda")
    off, page, length = torch.zeros(7, **i64), torch.zeros(most, dtype=torch.int32, device="cuda"), torch.zeros(6, **i64)
    q_off, grp = torch.zeros(7, **i64), torch.zeros(3, **i64)
    q = torch.zeros((T, 8, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((T, 8), device="cuda")

    def fill(b):
        off.copy_(torch.from_numpy(b.off))
        page[:len(b.page)].copy_(torch.from_numpy(b.page))
        length.copy_(torch.from_numpy(b.len))
        q_off.copy_(torch.from_numpy(b.q_off))
        grp.copy_(torch.from_numpy(b.groups))
        q.copy_(b.qrows.unflatten(1, (8, 128)))
        k[:, :b.k.shape[1]].copy_(b.k)
        v[:, :b.v.shape[1]].copy_(b.v)
        torch.cuda.synchronize()

    def call():
        e.attn(e.attn_plan(kv, (off, page, length), q_off, T, 8, groups=grp), 0, q, 128 ** -0.5, out, lse)

    fill(sets[0])
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for i in (1, 2, 0, 1):
        fill(sets[i])
        out.fill_(5)
        lse.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        with torch.cuda.stream(st):
            call()
        st.synchronize()
        assert torch.equal(got[0].view(torch.int16), out.view(torch.int16)) and torch.equal(got[1], lse)
        ref, rl, tol, ltol = sets[i].reference()
        assert bool(((out.cpu().double() - ref).abs() <= tol).all())
    e.sync()
    e.close()


def test_idle_places_and_empty_rows():
    """Length 0 with a new token (an idle place), no new token, fewer keys than new tokens: empty rows are zeros
    and -infinity, with and without runs."""
    seqs = [(1, 0), (1, 40), (5, 3), (0, 20), (3, 0), (70, 30), (1, 1), (0, 0), (1, 200)]
    _say("idle")
    Batch(16, seqs, seed=8).check()
    b = Batch(16, [(1, 60, 0), (1, 20, 0), (0, 5, 0), (1, 30, 0), (2, 9, 0)], prefixes=(192,), seed=9)
    b.len[1] = 0
    b.check()
    b.len[3] = 1  # shorter than the prefix
    b.check()
    b = Batch(16, [(2, 60, 0), (9, 20, 0), (1, 40, 0)], prefixes=(192,), seed=10)
    b.len[1] = 4  # fewer keys than new tokens, within the prefix
    b.check()


def test_long_rows_in_parts():
    _say("long")
    Batch(16, [(1, 9000), (1, 4097), (3, 6001)], heads=(4, 2), dim=64, seed=11).check()
    Batch(64, [(2, 12000)], heads=(4, 1), dim=128, seed=12).check()


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan"), "low"])
@pytest.mark.parametrize("shape", ["narrow", "wide", "run"])
def test_unseen_values_do_not_matter(what, shape):
    """Infinities, NaN and the type's lowest value in keys and values that a row does not see; the rows that see them
    get what the definition gives."""
    seqs, pre = {"narrow": ([(6, 80), (4, 33)], ()), "wide": ([(100, 100), (70, 200)], ()),
                 "run": ([(3, 20, 0), (2, 50, 0), (1, 1, 0)], (192,))}[shape]
    b = Batch(16, seqs, prefixes=pre, heads=(8, 2), seed=13)
    x = torch.finfo(torch.bfloat16).min if what == "low" else what
    places = set()
    for s in range(len(seqs)):
        t = int(b.len[s]) - 2
        p = int(b.page[b.off[s] + t // 16])
        b.v[0, p, :, t % 16, 5:9] = x
        if s % 2:
            b.k[0, p, :, t % 16, :] = x
        places.add((p, t % 16))
    # the rows that see one of the places (of a shared page: those of every sequence that holds it)
    later = []
    for s in range(len(seqs)):
        t0, t1 = int(b.q_off[s]), int(b.q_off[s + 1])
        for t in range(t0, t1):
            pos = int(b.len[s]) - (t1 - t0) + (t - t0)
            if any((int(b.page[b.off[s] + k // 16]), k % 16) in places for k in range(pos + 1)):
                later.append(t)
    out, lse = b.run()
    ref, rl, tol, ltol = b.reference()
    rows = [t for t in range(int(b.q_off[-1])) if t not in later]
    assert bool(((out[rows].double() - ref[rows]).abs() <= tol[rows]).all())
    assert bool(((lse[rows].double() - rl[rows]).abs() <= ltol[rows]).all())
    # rows that do see it: the same elements are finite, and NaN where NaN
    for t in later:
        if what != "low":
            assert torch.equal(out[t].isnan(), ref[t].isnan()), t
            assert torch.equal(out[t].isinf(), ref[t].isinf()), t


def test_large_scores():
    """Scores in the thousands: one key has all the weight; and sharp and flat scales."""
    Batch(16, [(4, 300), (80, 200)], heads=(4, 2), qscale=300.0, seed=14).check()
    Batch(16, [(4, 300), (80, 200)], heads=(4, 2), seed=15).check(scale=1e-4)


def test_rows_apart_and_layers():
    """Queries that are part of wider rows, the second of two layers, no lse, two passes on one plan."""
    Batch(16, [(3, 70), (40, 64), (1, 5)], heads=(6, 3), dim=64, pad_q=24 * 8, layers=2, layer=1, seed=16).check(
        lse=False, reps=2)


def test_another_stream():
    """A context on another stream than the tensors' own."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    b = Batch(16, [(1, 300), (70, 128)], seed=17)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        b.check(eng=e)
    e.close()


def test_plan_memory_goes_by_the_contexts_stream():
    """A plan that is dropped while its context's stream may still read it does not become another stream's tensor."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    b = Batch(16, [(1, 300), (70, 128)], seed=17)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    tb, qo = b.tables(), b.dev(b.q_off)
    torch.cuda.synchronize()
    plan = e.attn_plan(kv, tb, qo, 71, 8)
    at, size = plan.buf.data_ptr(), plan.buf.numel()
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert all(x.data_ptr() != at for x in others)
    e.sync()
    e.close()


def test_same_bits_every_time():
    """No order of atomics changes a result."""
    b = Batch(16, [(1, 3000, 0), (1, 200, 0), (2, 100, 0), (1, 1, 0), (1, 50, 0)], prefixes=(2048,), seed=18)
    first = b.run()
    for _ in range(3):
        again = b.run()
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16))
        assert torch.equal(first[1], again[1])


def test_refusals():
    pk, e = engine(16)
    b = Batch(16, [(1, 40), (2, 30)], seed=19)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    tb, qo = b.tables(), b.dev(b.q_off)
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    plan = e.attn_plan(kv, tb, qo, 3, 8)
    e.attn(plan, 0, q, 0.1, torch.empty_like(q))
    e.sync()
    with pytest.raises(pk.DMError, match="multiple of kv_heads"):
        e.attn_plan(kv, tb, qo, 3, 7)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pk.DMError, match="scale"):
            e.attn(plan, 0, q, scale, torch.empty_like(q))
    with pytest.raises(pk.DMError, match="layer"):
        e.attn(plan, 1, q, 0.1, torch.empty_like(q))
    with pytest.raises(ValueError):
        e.attn(plan, 0, q.half(), 0.1, torch.empty_like(q))
    with pytest.raises(ValueError):
        e.attn(plan, 0, q, 0.1, torch.empty_like(q)[:2])
    with pytest.raises(ValueError):
        pk.KVPages(b.k.cuda().float(), b.v.cuda().float())
    with pytest.raises(pk.DMError, match="unsupported"):
        e.attn_plan(pk.KVPages(b.k.cuda()[..., :32].contiguous(), b.v.cuda()[..., :32].contiguous()), tb, qo, 3, 8)
    with pytest.raises(pk.DMError, match="groups"):
        e.attn_plan(kv, tb, qo, 3, 8, groups=torch.tensor([0, 0, 1, 2], device="cuda"))
    rows = torch.zeros((3, 8 * 128 + 4), dtype=torch.bfloat16, device="cuda")[:, :1024].unflatten(1, (8, 128))
    with pytest.raises(pk.DMError, match="strides"):
        e.attn(plan, 0, rows, 0.1, torch.empty_like(q))


def test_malformed_input_is_reported():
    """Found on the device, reported by sync, other sequences unaffected where the documentation says so."""
    pk, e = engine(16)
    good = Batch(16, [(1, 40), (2, 30), (1, 64)], seed=20)
    ref, _, tol, _ = good.reference()

    def attempt(change, rows=None, groups=None):
        b = Batch(16, [(1, 40), (2, 30), (1, 64)], seed=20)
        change(b)
        b.groups = groups
        kv = pk.KVPages(b.k.cuda(), b.v.cuda())
        T = 4
        q = b.qrows.cuda().unflatten(1, (8, 128))
        out = torch.zeros((T, 8, 128), dtype=torch.bfloat16, device="cuda")
        plan = e.attn_plan(kv, b.tables(), b.dev(b.q_off), T, 8, groups=b.dev(b.groups))
        e.attn(plan, 0, q, b.scale(), out)
        with pytest.raises(pk.DMError) as x:
            e.sync()
        assert x.value.status == pk.DM_EINVAL
        for r in rows or []:
            assert bool(((out[r].cpu().double() - ref[r]).abs() <= tol[r]).all()), r

    def page(b):
        b.page[b.off[1]] = 1 << 30

    def length(b):
        b.len[1] = 1000

    def order(b):
        b.off[1] = 10 ** 12

    def tokens(b):
        b.q_off[2] = 99

    attempt(page, rows=[0, 3])
    attempt(length, rows=[0, 3])
    attempt(order)
    attempt(tokens)
    attempt(lambda b: None, rows=[0, 1, 2, 3], groups=np.array([0, 2], np.int64))
    attempt(lambda b: None, rows=[0, 1, 2, 3], groups=np.array([0, 50, 3], np.int64))
    # the plan of another batch
    kv = pk.KVPages(good.k.cuda(), good.v.cuda())
    other = Batch(16, [(1, 40), (2, 30)], seed=20)
    q = good.qrows.cuda().unflatten(1, (8, 128))
    out = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    mine = e.attn_plan(kv, good.tables(), good.dev(good.q_off), 4, 8)
    theirs = e.attn_plan(kv, other.tables(), other.dev(other.q_off), 3, 8)
    mine.buf = torch.cat([theirs.buf, torch.zeros(4096, dtype=torch.uint8, device="cuda")])
    e.attn(mine, 0, q, 0.1, out)
    with pytest.raises(pk.DMError):
        e.sync()
    assert not bool(out.any())
    good.check()  # and the context goes on


def test_pages_past_32_bits():
    """A store of more than 2^32 elements a side, read at its far end."""
    pk, e = engine(64)
    n = 2 ** 32 // (8 * 64 * 256) + 40
    k = torch.zeros((1, n, 8, 64, 256), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    b = Batch(64, [(1, 200), (40, 130)], heads=(8, 8), dim=256, seed=21)
    far = n - b.k.shape[1]
    k[0, far:] = b.k[0].cuda()
    v[0, far:] = b.v[0].cuda()
    b.page = b.page + far
    kv = pk.KVPages(k, v)
    q = b.qrows.cuda().unflatten(1, (8, 256))
    out = torch.empty((41, 8, 256), dtype=torch.bfloat16, device="cuda")
    e.attn(e.attn_plan(kv, b.tables(), b.dev(b.q_off), 41, 8), 0, q, b.scale(), out)
    e.sync()
    b.page = b.page - far
    ref, _, tol, _ = b.reference()
    assert bool(((out.cpu().double() - ref).abs() <= tol).all())
    del k, v, kv
    torch.cuda.empty_cache()


def test_store_without_pages_is_refused():
    """Through the C entry: a store of no pages has no place that a row could be read from."""
    pk, e = engine(16)
    b = Batch(16, [(1, 40), (2, 30)], seed=19)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    plan = e.attn_plan(kv, b.tables(), b.dev(b.q_off), 3, 8)
    kv.struct.n_pages = 0
    with pytest.raises(pk.DMError, match="n_pages"):
        e.attn(plan, 0, q, 0.1, torch.empty_like(q))
    kv.struct.n_pages = kv.pages
    e.attn(plan, 0, q, 0.1, torch.empty_like(q))
    e.sync()


def test_runs_without_bounds_are_refused():
    pk, e = engine(16)
    b = Batch(16, [(1, 40), (2, 30)], seed=19)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    with pytest.raises(ValueError, match="groups"):
        e.attn_plan(kv, b.tables(), b.dev(b.q_off), 3, 8, groups=torch.zeros(0, dtype=torch.int64, device="cuda"))
    e.sync()


@pytest.mark.parametrize("prefix", [0, 768])
@pytest.mark.parametrize("dtype,dim,heads", [("bf16", 64, (96, 96)), ("f16", 128, (96, 48)), ("bf16", 256, (64, 64))])
def test_many_rows_in_parts(dtype, dim, heads, prefix):
    """More rows in parts than the join has waves: of a run and of cut sequences, some that see nothing, some in one part."""
    seqs = [(9, 3400, 0), (3, 1, 0), (90, 300, 0), (33, 96, 1), (14, 0, 1), (20, 3100, 1), (1, 33, 1)]
    b = Batch(16, seqs if prefix else [s[:2] for s in seqs], prefixes=(prefix, prefix) if prefix else (), heads=heads, dim=dim,
              dtype=dtype, seed=43)
    _say("many rows", dtype, dim, heads, prefix)
    b.check()


@pytest.mark.parametrize("dtype,dim,heads", [("bf16", 64, (4, 2)), ("f16", 128, (14, 2)), ("bf16", 128, (16, 1)), ("f16", 256, (3, 3))])
def test_few_rows_on_few_keys(dtype, dim, heads):
    """Batches around the limits of the form without parts: rows, keys, sequences; idle places; a fault's report."""
    ratio = heads[0] // heads[1]
    most = {64: 1024, 128: 768, 256: 256}[dim]
    for keys in (1, 31, 32, 33, 127, 129, 255, 256, 257, 500, 752, 767, 768, 769, 1023, 1024, 1025):
        if keys <= most + 100:
            Batch(16, [(1, keys)], heads=heads, dim=dim, dtype=dtype, seed=keys).check()
    rows = 16 // ratio
    for seqs in ([(rows, most - 5)], [(rows + 1, most - 5)], [(rows, 2)], [(1, 100), (0, 40), (1, 3)][:rows + 1],
                 [(1, 0), (1, 77), (0, 0), (1, 1)][:rows + 1]):
        _say("few", dtype, dim, heads, seqs)
        Batch(16, seqs, heads=heads, dim=dim, dtype=dtype, seed=len(seqs) + 60).check()
    b = Batch(16, [(rows, 200)], heads=heads, dim=dim, dtype=dtype, seed=61)
    b.page = b.page.copy()
    b.page[3] = 10 ** 6
    pk, _ = engine(16)
    with pytest.raises(pk.DMError) as x:
        b.run()
    assert x.value.status == pk.DM_EINVAL


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_few_rows_and_unseen_values(what):
    """Infinities and NaN that some of a tile's rows do not see."""
    b = Batch(16, [(4, 300)], heads=(8, 2), dim=128, seed=62)
    out, lse = b.run()
    at = int(b.page[b.off[0] + 299 // 16])
    b.v[0, at, :, 299 % 16] = what
    b.k[0, at, :, 299 % 16] = what
    again, lse2 = b.run()
    assert torch.equal(out[:3].view(torch.int16), again[:3].view(torch.int16)) and torch.equal(lse[:3], lse2[:3])


@pytest.mark.parametrize("block", [4, 8, 64])
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 256), ("bf16", 128)])
def test_small_pages_and_heads(block, dtype, dim):
    """Pages smaller than the rows that a wave reads at once, in every form: few rows, narrow and wide tiles, a run."""
    _say("pages", block, dtype, dim)
    Batch(block, [(2, 150)], heads=(4, 2), dim=dim, dtype=dtype, seed=71).check()
    Batch(block, [(1, 900), (3, 70), (40, 333), (1, 2)], heads=(8, 2), dim=dim, dtype=dtype, seed=72).check()
    Batch(block, [(1, 30, 0), (2, 200, 0), (50, 77, 0), (9, 9, 0)], prefixes=(640,), heads=(8, 2), dim=dim, dtype=dtype, seed=73).check()
