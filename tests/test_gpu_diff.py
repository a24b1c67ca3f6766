"""Differential attention over KV pages against its definition in 64 bits.

Bounds, per element (u: half a unit in the last place of the type).  A map's result before the difference is off by
what a weight's rounding makes, u A with A = sum w |v| / sum w, by 2^-20 A for sums in 32 bits, and in float16 by n
2^-25 max |v| + 2^-25 for weights that lose bits (n keys); the difference by d = d1 + |lambda| d2 and some 2^-20 of its
terms.  A norm over x with N = sqrt(sum x^2 + D eps) turns d into at most d / (N - |d|) + |x| |d| / (N (N - |d|)), |d|
its length, times sqrt(D) |weight| gain; the result is rounded once, u, after some 2^-20 of 32-bit steps.  The
log-sum-exp is in 32 bits: 2^-18 of the largest |score|, and of itself.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import DECODE, DT, ULP, Batch, engine  # noqa: E402

EPS = 1e-5


def _say(*a):
    print("[case]", *a, flush=True)


class Pairs(Batch):
    """A batch whose query and KV heads are pairs, with a factor for each pair of query heads and weights of a norm."""

    def __init__(self, *a, heads=(8, 4), dim=64, norm=True, gain=0.5, seed=0, **kw):
        super().__init__(*a, heads=heads, dim=dim, seed=seed, **kw)
        g = torch.Generator().manual_seed(seed + 99)
        self.lam = 0.2 + 0.8 * torch.rand(heads[0] // 2, generator=g)
        self.norm = (1 + 0.2 * torch.randn(2 * dim, generator=g)).to(DT[self.dtype]) if norm else None
        self.gain = gain

    def run(self, lse=True, groups=True, eng=None, scale=None, reps=1, eps=EPS):
        pk, e = engine(self.block)
        e = eng or e
        kv = pk.KVPages(self.k.cuda(), self.v.cuda())
        T = int(self.q_off[-1])
        q = self.qrows.cuda()[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim))
        out = torch.full((T, self.hq, self.dim), 7.0, dtype=DT[self.dtype], device="cuda")
        far = torch.full((T, self.hq), 7.0, device="cuda") if lse else None
        plan = e.diff_plan(kv, self.tables(), self.dev(self.q_off), T, self.hq,
                           groups=self.dev(self.groups) if groups else None)
        for _ in range(reps):
            e.diff_attn(plan, self.layer, q, self.scale(scale), self.lam.cuda(), out, far,
                        norm=None if self.norm is None else self.norm.cuda(), eps=eps, gain=self.gain)
        e.sync()
        return out.cpu(), None if far is None else far.cpu()

    def reference(self, scale=None, eps=EPS):
        T, P, D = int(self.q_off[-1]), self.hq // 2, 2 * self.dim
        r = self.hq // self.hkv
        o, od = torch.zeros((T, P, D), dtype=torch.float64), torch.zeros((T, P, D), dtype=torch.float64)
        lse = torch.full((T, self.hq), -math.inf, dtype=torch.float64)
        ltol = torch.zeros_like(lse)
        u = ULP[self.dtype]
        q = self.qrows[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim)).double()
        for s in range(len(self.len)):
            L, t0, t1 = int(self.len[s]), int(self.q_off[s]), int(self.q_off[s + 1])
            if L == 0 or t0 == t1:
                continue
            at = torch.from_numpy(self.page[self.off[s]:self.off[s] - (-L // self.block)].astype(np.int64))
            rows = [[x[self.layer][at, h].reshape(-1, self.dim)[:L].double() for h in range(self.hkv)]
                    for x in (self.k, self.v)]
            n = L - (t1 - t0) + torch.arange(t1 - t0) + 1  # keys that a token sees
            hidden = torch.arange(L) >= n[:, None]
            for j in range(P):
                g = j // r
                V = torch.cat([rows[1][2 * g], rows[1][2 * g + 1]], 1)
                for m in (0, 1):
                    sc = (q[t0:t1, 2 * j + m] @ rows[0][2 * g + m].T * self.scale(scale)).masked_fill(hidden, -math.inf)
                    w = torch.softmax(sc, -1).masked_fill((n <= 0)[:, None], 0.0)
                    f = 1.0 if m == 0 else -float(self.lam[j])
                    o[t0:t1, j] += f * (w @ V)
                    mean = w @ V.abs()
                    d = u * mean * 1.02 + 2.0 ** -19 * mean
                    if self.dtype == "f16":
                        d = d + (n.clamp(min=0)[:, None] * 2.0 ** -25 * V.abs().max() + 2.0 ** -25)
                    od[t0:t1, j] += abs(f) * d
                    lse[t0:t1, 2 * j + m] = torch.logsumexp(sc, -1)
                    ltol[t0:t1, 2 * j + m] = 2.0 ** -18 * (sc.masked_fill(hidden, 0.0).abs().amax(-1) + lse[t0:t1, 2 * j + m].abs() + 1)
        out, tol = o * self.gain, od * self.gain
        if self.norm is not None:
            N = torch.sqrt((o * o).sum(-1, keepdim=True) + D * eps)
            dn = od.norm(dim=-1, keepdim=True)
            by = math.sqrt(D) * self.norm.double() * self.gain
            out = torch.where(N == 0, 0.0, o / N) * by
            tol = torch.where(dn < N, od / (N - dn) + o.abs() * dn / (N * (N - dn)), math.inf) * by.abs()
            tol = torch.where((o == 0).all(-1, keepdim=True) & (od == 0).all(-1, keepdim=True), 0.0, tol)
        tol = tol + (u * 1.02 + 2.0 ** -19) * (out.abs() + tol) + (2.0 ** -25 if self.dtype == "f16" else 0.0)
        tol = torch.where((out == 0).all(-1, keepdim=True), 0.0, tol)
        shape = (T, self.hq, self.dim)
        return out.reshape(shape), lse, tol.reshape(shape), ltol.nan_to_num(0.0, 0.0, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (16, 4), (14, 2), (6, 2)])
def test_single_tokens(dtype, dim, heads):
    _say("decode", dtype, dim, heads)
    Pairs(16, DECODE, heads=heads, dim=dim, dtype=dtype, seed=dim + heads[0]).check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 15, 33, 256, 300, 700])
def test_one_sequence(n, dim):
    """A few rows on a few keys: one kernel, nothing cut."""
    _say("one", n, dim)
    Pairs(16, [(1, n)], heads=(8, 4), dim=dim, seed=n).check()
    Pairs(16, [(2, n), (1, 3)], heads=(4, 2), dim=dim, norm=False, gain=1.0, seed=n).check()


@pytest.mark.parametrize("block", [4, 8, 16, 32, 64])
@pytest.mark.parametrize("dim", [64, 128])
def test_page_sizes(block, dim):
    _say("block", block, dim)
    Pairs(block, [(1, 1), (3, 200), (40, 77), (1, 333), (90, 90), (7, 130)], dim=dim, seed=block).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (16, 4), (14, 2)])
@pytest.mark.parametrize("norm", [True, False])
def test_prompts(dtype, dim, heads, norm):
    """Wide tiles: several new tokens with and without earlier ones, rows around tiles."""
    _say("prompts", dtype, dim, heads, norm)
    Pairs(16, [(33, 33), (1, 1), (128, 300), (64, 64), (65, 129), (200, 200), (17, 500)], heads=heads, dim=dim,
          dtype=dtype, norm=norm, seed=3).check()


@pytest.mark.parametrize("dim", [64, 128])
def test_shared_prefixes(dim):
    """Runs that share, alone and not: single tokens, drafts and prompts, joined from parts."""
    seqs = [(1, 1, 0), (1, 40, 0), (1, 17, 0), (3, 30, 1), (1, 1, 2), (1, 5, 2), (5, 5, 2), (1, 90, 2), (1, 2, 2),
            (1, 1, 2), (2, 33, 2), (40, 50, 3), (60, 60, 3)]
    b = Pairs(16, seqs, prefixes=(256, 128, 640, 320), dim=dim, seed=5)
    _say("shared", dim)
    b.check()
    b.check(groups=False)


@pytest.mark.parametrize("dim", [64, 128])
def test_batches_of_few_rows_a_sequence(dim):
    """A few rows a sequence on average, and one with many among them; the same with runs."""
    _say("few", dim)
    b = Pairs(16, [(1, 30 + 11 * i) for i in range(20)] + [(19, 300), (2, 2)], heads=(8, 4), dim=dim, seed=4)
    b.check()
    b.groups = np.array([0, 9, 22], np.int64)
    b.check()


def test_many_rows_in_parts():
    """More rows than waves, on shared prefixes: four rows joined by a wave."""
    _say("many")
    Pairs(32, [(20 + i % 30, 60 + i % 70, 0) for i in range(64)] + [(1, 9, 1)], prefixes=(352, 160), heads=(14, 2),
          dtype="f16", seed=6).check()
    Pairs(32, [(9 + i % 3, 40, 0) for i in range(160)], prefixes=(256,), heads=(12, 4), dim=128, norm=False,
          seed=7).check()


def test_long_rows_in_parts():
    _say("long")
    Pairs(16, [(1, 9000), (1, 4097), (3, 6001)], heads=(4, 2), seed=11).check()
    Pairs(64, [(2, 12000)], heads=(4, 2), dim=128, dtype="f16", seed=12).check()


def test_idle_places_and_empty_rows():
    """Rows that see nothing are zeros, with a norm too, and -infinity; also where eps is 0."""
    seqs = [(1, 0), (1, 40), (5, 3), (0, 20), (3, 0), (70, 30), (1, 1), (0, 0), (1, 200)]
    _say("idle")
    b = Pairs(16, seqs, seed=8)
    b.check()
    out, lse = b.run(eps=0.0)
    ref, rl, tol, _ = b.reference(eps=0.0)
    assert bool(((out.double() - ref).abs() <= tol).all())
    empty = rl[:, 0] == -math.inf
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all()) and int(empty.sum()) > 4
    b = Pairs(16, [(1, 60, 0), (1, 20, 0), (0, 5, 0), (1, 30, 0), (2, 9, 0)], prefixes=(192,), seed=9)
    b.len[1] = 0
    b.check()
    b.len[3] = 1  # shorter than the prefix
    b.check()


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("seqs", [[(1, 50), (2, 9)], [(40, 90), (33, 40)]])
def test_unseen_places_have_no_part(what, seqs):
    """Values and keys behind a sequence's end, and of later tokens, whatever they hold."""
    _say("unseen", what, seqs)
    b = Pairs(16, seqs, seed=4)
    ref, rl, tol, _ = b.reference()
    for s in range(len(seqs)):
        L = int(b.len[s])
        t = L - 1  # only the last token sees this one
        page, slot = int(b.page[b.off[s] + t // 16]), t % 16
        b.k[:, page, :, slot], b.v[:, page, :, slot] = what, what
    for x in (b.k, b.v):
        x[x.isnan()] = what
    out, lse = b.run()
    last = torch.zeros(len(out), dtype=torch.bool)
    last[torch.from_numpy(b.q_off[1:] - 1)] = True
    assert bool(((out[~last].double() - ref[~last]).abs() <= tol[~last]).all())


def test_large_scores_and_strides():
    """Scores of 2^14 and more; rows of q with room between them; a layer that is not the first."""
    b = Pairs(16, [(1, 300), (30, 90), (2, 700)], heads=(8, 2), seed=2, layers=3, layer=2, pad_q=24)
    _say("layers, strides")
    b.check()
    _say("large scores")
    b.check(scale=900.0)


def test_factors_of_zero_and_one():
    """lambda 0 is plain attention of the first heads; the two maps of one query cancel at 1."""
    _say("zero")
    b = Pairs(16, [(1, 200), (40, 60)], heads=(8, 4), norm=False, gain=1.0, seed=5)
    b.lam[:] = 0
    b.check()
    b.lam[:] = 1
    D = b.dim
    b.qrows = b.qrows.unflatten(1, (4, 2, D))[:, :, :1].expand(-1, -1, 2, -1).flatten(1).contiguous()
    b.k[:, :, 1::2] = b.k[:, :, 0::2]
    out, lse = b.run()
    assert bool((out == 0).all()) and torch.equal(lse[:, 0::2], lse[:, 1::2])


def test_same_bits_and_rows_behind_the_last():
    """Twice the same bits, with runs and cuts; rows past the last sequence's tokens are left as they were."""
    pk, e = engine(16)
    b = Pairs(16, [(1 + i % 3, 900 + 31 * i, 0) for i in range(24)], prefixes=(512,), heads=(8, 4), seed=3)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    T = int(b.q_off[-1])
    q = torch.zeros((T + 5, 8, 64), dtype=torch.bfloat16, device="cuda")
    q[:T] = b.qrows.unflatten(1, (8, 64)).cuda()
    first = None
    for _ in range(4):
        out, lse = torch.full_like(q, 7), torch.full((T + 5, 8), 7.0, device="cuda")
        plan = e.diff_plan(kv, b.tables(), b.dev(b.q_off), T + 5, 8, groups=b.dev(b.groups))
        e.diff_attn(plan, 0, q, 0.125, b.lam.cuda(), out, lse, norm=b.norm.cuda())
        e.sync()
        assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
        first = first or (out, lse)
        assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])


def test_in_a_graph():
    """Captured, replayed with other lengths, tables and queries, each replay equal to the eager result's bits."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    sets = [Pairs(16, [(1, 30 + 7 * i, 0), (1, 50, 0), (2, 9 + i, 0), (40, 60, 0), (1, 200 + i, 1), (1, 1, 1)],
                  prefixes=(256, 320), seed=30 + i, spare=9 - i) for i in range(3)]
    T, b0 = int(sets[0].q_off[-1]), sets[0]
    pages = max(b.k.shape[1] for b in sets)
    k = torch.zeros((1, pages) + tuple(b0.k.shape[2:]), dtype=torch.bfloat16, device="cuda")
    kv = pk.KVPages(k, torch.zeros_like(k))
    i64 = dict(dtype=torch.int64, device="cuda")
    off, length, q_off, grp = (torch.zeros(n, **i64) for n in (7, 6, 7, 3))
    page = torch.zeros(max(len(b.page) for b in sets), dtype=torch.int32, device="cuda")
    q = torch.zeros((T, 8, 64), dtype=torch.bfloat16, device="cuda")
    out, lse, lam, norm = torch.zeros_like(q), torch.zeros((T, 8), device="cuda"), b0.lam.cuda(), b0.norm.cuda()

    def fill(b):
        for to, x in ((off, b.off), (page[:len(b.page)], b.page), (length, b.len), (q_off, b.q_off), (grp, b.groups)):
            to.copy_(torch.from_numpy(x))
        q.copy_(b.qrows.unflatten(1, (8, 64)))
        kv.k[:, :b.k.shape[1]].copy_(b.k)
        kv.v[:, :b.v.shape[1]].copy_(b.v)
        lam.copy_(b.lam)
        norm.copy_(b.norm)
        torch.cuda.synchronize()

    def call():
        e.diff_attn(e.diff_plan(kv, (off, page, length), q_off, T, 8, groups=grp), 0, q, 0.125, lam, out, lse, norm=norm,
                    eps=EPS, gain=0.5)

    fill(b0)
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for i in (1, 2, 0, 1):
        fill(sets[i])
        out.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        with torch.cuda.stream(st):
            call()
        st.synchronize()
        assert torch.equal(got[0].view(torch.int16), out.view(torch.int16)) and torch.equal(got[1], lse)
        ref, _, tol, _ = sets[i].reference()
        assert bool(((out.cpu().double() - ref).abs() <= tol).all())
    e.sync()
    e.close()


def test_refusals():
    pk, e = engine(16)
    b = Pairs(16, [(1, 40), (2, 90)], heads=(8, 4), seed=1)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    q = b.qrows.cuda().unflatten(1, (8, 64)).contiguous()
    t, q_off, out, lam = b.tables(), b.dev(b.q_off), torch.zeros_like(q), b.lam.cuda()
    plan = e.diff_plan(kv, t, q_off, 3, 8)
    plain = e.attn_plan(kv, t, q_off, 3, 8)
    with pytest.raises(ValueError, match="attn_plan"):
        e.diff_attn(plain, 0, q, 0.125, lam, out)
    with pytest.raises(ValueError, match="diff_plan"):
        e.attn(plan, 0, q, 0.125, out)
    for bad in (lam[:3], lam.double(), lam.cpu(), None):
        with pytest.raises(ValueError, match="lam"):
            e.diff_attn(plan, 0, q, 0.125, bad, out)
    for bad in (b.norm.cuda()[:64], b.norm.cuda().float()):
        with pytest.raises(ValueError, match="norm"):
            e.diff_attn(plan, 0, q, 0.125, lam, out, norm=bad)
    with pytest.raises(ValueError, match="lse"):
        e.diff_attn(plan, 0, q, 0.125, lam, out, torch.zeros(3, 4, device="cuda"))
    for kw in (dict(scale=0.0), dict(scale=math.inf), dict(eps=-1.0), dict(eps=math.nan), dict(gain=math.inf), dict(gain=math.nan)):
        kw = dict(dict(scale=0.125), **kw)
        with pytest.raises(pk.DMError, match="scale must be"):
            e.diff_attn(plan, 0, q, kw.pop("scale"), lam, out, **kw)
    with pytest.raises(pk.DMError, match="layer"):
        e.diff_attn(plan, 1, q, 0.125, lam, out)
    for heads, dim in ((3, 64), (2, 256)):
        x = torch.zeros((1, 8, heads, 16, dim), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(pk.DMError, match="even number"):
            e.diff_plan(pk.KVPages(x, x.clone()), t, q_off, 3, heads)
    with pytest.raises(pk.DMError, match="multiple of kv_heads"):
        e.diff_plan(kv, t, q_off, 3, 6)
    # another batch's plan: reported, nothing written
    other = e.diff_plan(kv, (t[0][:2], t[1], t[2][:1]), q_off[:2], 3, 8)
    other.batch = plan.batch
    out.fill_(7)
    e.diff_attn(other, 0, q, 0.125, lam, out)
    with pytest.raises(pk.DMError):
        e.sync()
    assert bool((out == 7).all())
