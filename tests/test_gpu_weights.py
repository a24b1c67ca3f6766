"""The weight that cached keys collect, against its definition in 64 bits.

Bounds: the log-sum-exp is an input.  A score in 32 bits is off by some 2^-20 of sum |q| |k| scale (products of 16-bit
numbers are exact, their sum of D terms rounds), its product with log2(e) and the log-sum-exp's by 2^-23 of their sizes, an
exponential by 2^-22; a weight so by (2^-20 (A + |lse|) + 2^-21) of itself, A the sum of |q k| scale.  A sum of n of them
adds n 2^-24 of the sum at the most, the carried part 2^-22 of itself.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import DECODE, Batch, engine  # noqa: E402


def _say(*a):
    print("[case]", *a, flush=True)


class Collected(Batch):
    """A batch whose attention's log-sum-exps are inputs, and what was collected before."""

    def __init__(self, *a, paired=False, heads=(8, 2), last=0, decay=0.75, prev="fork", seed=0, **kw):
        super().__init__(*a, heads=heads, seed=seed, **kw)
        self.paired, self.last, self.decay, self.mode = paired, last, decay, prev
        r, g = np.random.default_rng(seed + 5), torch.Generator().manual_seed(seed + 5)
        n, B = len(self.len), self.block
        self.rows = len(self.page) * B
        new = np.diff(self.q_off)
        if prev == "fork":
            # the tables before: other sequences in another order; some carry less than all, one nothing
            self.keep = np.maximum(self.len - new, 0)
            self.keep[::3] //= 2
            self.src = r.permutation(n).astype(np.int32)
            before = np.empty(n, np.int64)
            before[self.src] = self.keep + r.integers(0, 40, size=n)
            self.prev_off = np.concatenate([[0], np.cumsum(-(-before // B))]).astype(np.int64)
            self.prev = torch.rand((self.hkv, int(self.prev_off[-1]) * B), generator=g) * 8
        elif prev == "same":
            self.prev = torch.rand((self.hkv, self.rows), generator=g) * 8

    def head_of(self, x):
        r = self.hq // self.hkv
        return 2 * (x // 2 // r) + x % 2 if self.paired else x // r

    def far(self):
        """Log-sum-exps of every query head, in 32 bits."""
        T = int(self.q_off[-1])
        lse = torch.full((T, self.hq), -math.inf, dtype=torch.float64)
        for s, t0, t1, q, K, hidden in self.each():
            for x in range(self.hq):
                sc = (q[:, x] @ K[self.head_of(x)].T * self.scale()).masked_fill(hidden, -math.inf)
                lse[t0:t1, x] = torch.logsumexp(sc, -1)
        return lse.float()

    def each(self):
        q = self.qrows[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim)).double()
        for s in range(len(self.len)):
            L, t0, t1 = int(self.len[s]), int(self.q_off[s]), int(self.q_off[s + 1])
            if L == 0 or t0 == t1:
                continue
            at = torch.from_numpy(self.page[self.off[s]:self.off[s] - (-L // self.block)].astype(np.int64))
            K = [self.k[self.layer][at, h].reshape(-1, self.dim)[:L].double() for h in range(self.hkv)]
            yield s, t0, t1, q[t0:t1], K, torch.arange(L) > (L - (t1 - t0) + torch.arange(t1 - t0))[:, None]

    def reference(self, lse):
        w = torch.zeros((self.hkv, self.rows), dtype=torch.float64)
        tol, written = torch.zeros_like(w), torch.zeros(self.rows, dtype=torch.bool)
        B, lse = self.block, lse.double()
        for s in range(len(self.len)):
            a, L = int(self.off[s]) * B, int(self.len[s])
            written[a:a + L] = True
            n, old = 0, 0
            if self.mode == "fork":
                n, old = min(int(self.keep[s]), L), int(self.prev_off[self.src[s]]) * B
            elif self.mode == "same":
                n, old = max(0, L - int(self.q_off[s + 1] - self.q_off[s])), a
            if n:
                w[:, a:a + n] = self.decay * self.prev[:, old:old + n].double()
                tol[:, a:a + n] = w[:, a:a + n].abs() * 2.0 ** -22
        for s, t0, t1, q, K, hidden in self.each():
            a, L = int(self.off[s]) * B, int(self.len[s])
            first = max(0, t1 - t0 - self.last) if self.last else 0
            for x in range(self.hq):
                h = self.head_of(x)
                far = lse[t0:t1, x][:, None]
                sc = q[:, x] @ K[h].T * self.scale()
                A = q[:, x].abs() @ K[h].abs().T * self.scale()
                z = torch.where(hidden | (far == -math.inf), 0.0, torch.exp(sc - far.clamp(min=-1e300)))
                e = z * (2.0 ** -20 * (A + far.clamp(min=-1e300).abs()) + 2.0 ** -21)
                w[h, a:a + L] += z[first:].sum(0)
                tol[h, a:a + L] += e[first:].sum(0)
        most = int(np.diff(self.q_off).max()) * (self.hq // self.hkv)
        return w, tol + (most + 2) * 2.0 ** -24 * w.abs() + 1e-37, written

    def run(self, lse, eng=None, groups=True, inplace=False):
        pk, e = engine(self.block)
        e = eng or e
        kv = pk.KVPages(self.k.cuda(), self.v.cuda())
        T = int(self.q_off[-1])
        q = self.qrows.cuda()[:, :self.hq * self.dim].unflatten(1, (self.hq, self.dim))
        plan = (e.diff_plan if self.paired else e.attn_plan)(kv, self.tables(), self.dev(self.q_off), T, self.hq,
                                                            groups=self.dev(self.groups) if groups else None)
        wide = torch.full((self.hkv, self.rows + 5), 7.0, device="cuda")
        w = wide[:, :self.rows]
        prev = None
        if self.mode == "fork":
            prev = (self.prev.cuda(), self.dev(self.prev_off), self.dev(self.src), self.dev(self.keep))
        elif self.mode == "same":
            prev = self.prev.cuda()
            if inplace:
                w.copy_(prev)
                prev = w
        e.attn_weights(plan, self.layer, q, self.scale(), lse.cuda(), w, last=self.last, prev=prev, decay=self.decay)
        e.sync()
        assert bool((wide[:, self.rows:] == 7).all())
        return w.cpu()

    def check(self, **kw):
        lse = self.far()
        w = self.run(lse, **kw)
        ref, tol, written = self.reference(lse)
        err = (w.double() - ref).abs()
        bad = ~(err <= tol) & written
        assert not bool(bad.any()), (int(bad.sum()), float((err / tol).nan_to_num(1e9)[:, written].max()))
        left = self.prev[:, ~written] if kw.get("inplace") else 7
        assert bool((w[:, ~written] == left).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (14, 2), (33, 3)])
def test_single_tokens(dtype, dim, heads):
    _say("decode", dtype, dim, heads)
    Collected(16, DECODE, heads=heads, dim=dim, dtype=dtype, seed=dim + heads[0]).check()


@pytest.mark.parametrize("block", [4, 8, 16, 32, 64])
@pytest.mark.parametrize("prev", ["fork", "same", None])
def test_page_sizes(block, prev):
    _say("block", block, prev)
    b = Collected(block, [(1, 1), (3, 200), (40, 77), (1, 333), (0, 50), (90, 90), (7, 130)], prev=prev, seed=block)
    b.check()
    if prev == "same":
        b.check(inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("last", [0, 1, 40])
def test_prompts(dtype, dim, last):
    _say("prompts", dtype, dim, last)
    Collected(16, [(33, 33), (1, 1), (128, 300), (64, 64), (65, 129), (200, 200), (17, 500)], dim=dim, dtype=dtype,
              last=last, seed=3).check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (12, 2), (16, 4)])
def test_pairs(dim, heads):
    """After differential attention: each head of a pair has its own map's weights."""
    _say("pairs", dim, heads)
    Collected(16, [(1, 100), (50, 90), (3, 700), (1, 1)], heads=heads, dim=dim, paired=True, seed=dim).check()
    Collected(32, [(1, 10, 0), (1, 45, 0), (2, 33, 0), (30, 40, 0)], prefixes=(256,), heads=heads, dim=dim, paired=True,
              seed=dim + 1).check()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_shared_prefixes(dim):
    """Runs that share, alone and not; one of them continues without new tokens."""
    seqs = [(1, 1, 0), (1, 40, 0), (1, 17, 0), (3, 30, 1), (1, 1, 2), (1, 5, 2), (5, 5, 2), (0, 90, 2), (1, 2, 2),
            (1, 1, 2), (2, 33, 2), (40, 50, 3), (60, 60, 3)]
    b = Collected(16, seqs, prefixes=(256, 128, 640, 320), dim=dim, seed=5)
    _say("shared", dim)
    b.check()
    b.check(groups=False)


def test_members_of_a_run_far_apart():
    """Between the sequences of a run that see its prefix, many that have no new token."""
    _say("far apart")
    seqs = [((1 if i % 37 == 5 else 0), 3 + i % 50, 0) for i in range(260)]
    Collected(16, seqs, prefixes=(192,), heads=(4, 2), dim=64, seed=4).check()
    Collected(16, [(n, 3 + i % 50, 0) for i, (n, _, _) in enumerate(seqs)], prefixes=(192,), heads=(16, 1), dim=64, prev="same",
              seed=5).check()


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (3, 1), (5, 1), (8, 1), (16, 1), (17, 1)])
def test_rows_of_a_run(heads):
    """One to seventeen rows a sequence, which share products by fours, eights and sixteens, or do not."""
    _say("rows", heads)
    Collected(16, [(1, 5 + 9 * i, 0) for i in range(21)], prefixes=(336,), heads=heads, dim=64, dtype="f16", seed=2).check()
    Collected(16, [(1 + i % 2, 5 + 9 * i, 0) for i in range(9)], prefixes=(336,), heads=heads, last=1, seed=3).check()


@pytest.mark.parametrize("heads", [(3, 1), (7, 1), (16, 1), (24, 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_many_rows_of_odd_ratios(heads, dim):
    """Rows that pass through LDS, where a step of them is not whole tokens, with room between rows of q."""
    _say("ratios", heads, dim)
    Collected(16, [(500, 700), (90, 90), (1, 300), (260, 900)], heads=heads, dim=dim, pad_q=40, last=0, seed=1).check()
    Collected(16, [(500, 700, 0), (90, 90, 0), (1, 300, 0)], prefixes=(320,), heads=heads, dim=dim, last=333, seed=1).check()


def test_no_new_tokens():
    """A batch without any: what was carried, decayed."""
    _say("none")
    Collected(16, [(0, 30), (0, 0), (0, 77)], prev="fork", seed=1).check()
    b = Collected(16, [(0, 30), (0, 77)], prev="same", seed=1)
    b.check(inplace=True)


def test_many_sequences_share():
    _say("many")
    Collected(32, [(1, 1 + i % 70, 0) for i in range(45)] + [(1, 9, 1)], prefixes=(352, 160), heads=(14, 2), dim=64,
              dtype="f16", seed=6).check()
    r = np.random.default_rng(1)
    run = np.sort(np.concatenate([np.arange(90), r.integers(0, 90, size=210)]))
    Collected(8, [(int(r.integers(0, 3)), int(r.integers(2, 40)), int(g)) for g in run],
              prefixes=[int(8 * r.integers(0, 30)) for _ in range(90)], heads=(2, 1), dim=64, seed=2).check()


def test_long_rows():
    _say("long")
    Collected(16, [(1, 9000), (1, 4097), (3, 6001)], heads=(4, 2), dim=64, seed=11).check()
    Collected(64, [(2, 12000)], heads=(4, 1), dim=128, seed=12).check()
    Collected(16, [(900, 1300), (1000, 1000)], heads=(4, 1), dim=64, seed=13).check()


def test_idle_places_and_empty_rows():
    """Length 0 with a new token, no new token, fewer keys than new tokens."""
    seqs = [(1, 0), (1, 40), (5, 3), (0, 20), (3, 0), (70, 30), (1, 1), (0, 0), (1, 200)]
    _say("idle")
    for prev in ("fork", "same", None):
        Collected(16, seqs, prev=prev, seed=8).check()
    b = Collected(16, [(1, 60, 0), (1, 20, 0), (0, 5, 0), (1, 30, 0), (2, 9, 0)], prefixes=(192,), prev="same", seed=9)
    b.len[0] = 0  # the run's first: its pages are still the run's
    b.check()
    b.len[3] = 1  # shorter than the prefix
    b.check()


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_unseen_places_have_no_part(what):
    """Keys behind a sequence's end and of later tokens, whatever they hold; a key that is NaN spoils its own place
    only."""
    b = Collected(16, [(1, 50), (40, 90), (33, 40)], seed=4)
    lse = b.far()
    ref, tol, written = b.reference(lse)
    seen = written.clone()
    for s in range(3):
        t = int(b.len[s]) - 1
        b.k[:, int(b.page[b.off[s] + t // 16]), :, t % 16] = what
        seen[int(b.off[s]) * 16 + t] = False
    w = b.run(lse)
    assert bool(((w.double() - ref).abs() <= tol)[:, seen].all())


def test_same_bits():
    """Results do not go by who comes first, with and without runs the same to rounding; a layer that is not the first, rows
    of q with room between them."""
    b = Collected(16, [(1 + 40 * (i % 3), 300 + 31 * i, 0) for i in range(24)], prefixes=(512,), layers=2, layer=1, pad_q=24,
                  seed=3)
    b.check()
    lse = b.far()
    first = b.run(lse)
    for _ in range(3):
        assert torch.equal(b.run(lse), first)


def test_in_a_graph():
    """Attention and the collecting of weights, captured and replayed, in place: a replay adds what an eager call adds."""
    pk, _ = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    b = Collected(16, [(1, 30, 0), (1, 50, 0), (2, 9, 0), (40, 60, 0), (1, 200, 1)], prefixes=(256, 320), prev="same", seed=30)
    kv, t, q_off, grp = pk.KVPages(b.k.cuda(), b.v.cuda()), b.tables(), b.dev(b.q_off), b.dev(b.groups)
    q = b.qrows.cuda().unflatten(1, (8, 128)).contiguous()
    T = len(q)
    out, lse = torch.zeros_like(q), torch.zeros((T, 8), device="cuda")
    w = torch.zeros((2, b.rows), device="cuda")

    def call():
        plan = e.attn_plan(kv, t, q_off, T, 8, groups=grp)
        e.attn(plan, 0, q, b.scale(), out, lse)
        e.attn_weights(plan, 0, q, b.scale(), lse, w, prev=w, decay=0.5)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        q.normal_(generator=g)
        start = torch.rand(w.shape, generator=g, device="cuda")
        w.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = w.clone()
        w.copy_(start)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            call()
        st.synchronize()
        assert torch.equal(got, w) and not torch.equal(got, start)
        b.prev, b.decay, b.qrows = start.cpu(), 0.5, q.cpu().flatten(1)
        ref, tol, written = b.reference(lse.cpu())
        assert bool(((got.cpu().double() - ref).abs() <= tol)[:, written].all())
    e.sync()
    e.close()


def test_refusals():
    pk, e = engine(16)
    b = Collected(16, [(1, 40), (2, 90)], seed=1)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    q = b.qrows.cuda().unflatten(1, (8, 128)).contiguous()
    t, q_off, lse = b.tables(), b.dev(b.q_off), b.far().cuda()
    w = torch.full((2, b.rows), 7.0, device="cuda")
    plan = e.attn_plan(kv, t, q_off, 3, 8)
    src, keep, off = b.dev(b.src), b.dev(b.keep), b.dev(b.prev_off)
    old = b.prev.cuda()
    for bad in (w[:1], w[:, :-1], w.double(), w.cpu(), w.t(), None):
        with pytest.raises(ValueError, match="w "):
            e.attn_weights(plan, 0, q, 0.1, lse, bad)
    for bad in (lse[:2], None):
        with pytest.raises(ValueError, match="lse"):
            e.attn_weights(plan, 0, q, 0.1, bad, w)
    with pytest.raises(ValueError, match="prev"):
        e.attn_weights(plan, 0, q, 0.1, lse, w, prev=w[:, :-1])
    with pytest.raises(ValueError, match="src and keep"):
        e.attn_weights(plan, 0, q, 0.1, lse, w, prev=(old, off, src[:1], keep))
    for kw in (dict(scale=0.0), dict(scale=math.nan), dict(decay=math.inf), dict(decay=math.nan)):
        kw = dict(dict(scale=0.1), **kw)
        with pytest.raises(pk.DMError, match="scale must be"):
            e.attn_weights(plan, 0, q, kw.pop("scale"), lse, w, **kw)
    with pytest.raises(pk.DMError, match="layer"):
        e.attn_weights(plan, 1, q, 0.1, lse, w)
    assert bool((w == 7).all())
    # found on the device: sources out of range carry nothing
    for bad in (torch.tensor([5, 0], dtype=torch.int32, device="cuda"), torch.tensor([-1, 0], dtype=torch.int32, device="cuda")):
        e.attn_weights(plan, 0, q, b.scale(), lse, w, prev=(old, off, bad, keep))
        with pytest.raises(pk.DMError):
            e.sync()
    # another batch's plan: reported, nothing written
    w.fill_(7)
    other = e.attn_plan(kv, (t[0][:2], t[1], t[2][:1]), q_off[:2], 3, 8)
    other.batch, other.n = plan.batch, plan.n
    e.attn_weights(other, 0, q, 0.1, lse, w)
    with pytest.raises(pk.DMError):
        e.sync()
    assert bool((w == 7).all())


def test_carried_in_place_by_other_tables():
    """w itself is what was carried by the same tables only: by others, places would be read after they are written."""
    pk, e = engine(16)
    b = Collected(16, [(1, 40), (2, 90)], seed=1)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    q = b.qrows.cuda().unflatten(1, (8, 128)).contiguous()
    plan = e.attn_plan(kv, b.tables(), b.dev(b.q_off), 3, 8)
    w = torch.full((2, b.rows), 7.0, device="cuda")
    with pytest.raises(ValueError, match="same"):
        e.attn_weights(plan, 0, q, 0.1, b.far().cuda(), w, prev=(w, b.dev(b.prev_off), b.dev(b.src), b.dev(b.keep)))
    e.sync()
    assert bool((w == 7).all())


def test_one_plan_for_attention_weights_and_other_layers():
    """Two layers' weights by one plan in turn, twice: the same bits, each its own layer's."""
    pk, e = engine(16)
    b = Collected(16, [(3, 70), (40, 90), (1, 200)], seed=6, layers=2)
    kv = pk.KVPages(b.k.cuda(), b.v.cuda())
    T = int(b.q_off[-1])
    q = b.qrows.cuda().unflatten(1, (8, 128)).contiguous()
    plan = e.attn_plan(kv, b.tables(), b.dev(b.q_off), T, 8)
    out, lse = torch.zeros_like(q), [torch.zeros((T, 8), device="cuda") for _ in range(2)]
    got = []
    for turn in range(2):
        for layer in (0, 1):
            e.attn(plan, layer, q, b.scale(), out, lse[layer])
            w = torch.zeros((2, b.rows), device="cuda")
            e.attn_weights(plan, layer, q, b.scale(), lse[layer], w)
            got.append(w)
    e.sync()
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3]) and not torch.equal(got[0], got[1])
    # every query gives a weight of 1 to the keys that it sees, each off by 2^-20 of the sum of its absolute products and of
    # its log-sum-exp, which are below 32 together
    for w in got[:2]:
        total = float(w.double().sum())
        assert abs(total - 8 * T) <= 8 * T * 2.0 ** -15, total


@pytest.mark.parametrize("paired", [False, True])
def test_runs_of_hundreds(paired):
    """Runs longer than a workgroup looks at a time, some of their sequences with nothing to do; the last group of a run short."""
    r = np.random.default_rng(4)
    seqs = [(int(r.integers(1, 3)), int(r.integers(2, 40)), 0) for _ in range(301)]
    seqs += [(1, 7, 1)] + [(1 if i % 5 else 0, 9 + i % 30, 2) for i in range(290)]
    b = Collected(16, seqs, prefixes=(160, 144, 320), heads=(8, 4) if paired else (4, 2), dim=64, paired=paired, seed=21)
    for i in (0, 3, 4, 260, 302, 303, 420):
        b.len[i] = 0
        b.keep[i] = 0
    _say("hundreds", paired)
    b.check()


def test_runs_with_malformed_arguments():
    """With runs: a source out of range carries nothing, a length that a table cannot hold counts as 0, another batch's plan writes
    nothing; each is reported, and the other sequences have theirs."""
    pk, e = engine(16)
    seqs = [(1, 30 + 7 * i, 0) for i in range(9)] + [(2, 20, 1), (1, 33, 1)]
    b = Collected(16, seqs, prefixes=(256, 192), heads=(4, 2), dim=64, seed=8)
    lse = b.far()
    kv, T = pk.KVPages(b.k.cuda(), b.v.cuda()), int(b.q_off[-1])
    q = b.qrows.cuda()[:, :4 * 64].unflatten(1, (4, 64)).contiguous()
    groups, q_off, keep, off = b.dev(b.groups), b.dev(b.q_off), b.dev(b.keep), b.dev(b.prev_off)

    def run(src, length=None, plan=None):
        tables = b.tables() if length is None else (b.tables()[0], b.tables()[1], b.dev(length))
        plan = plan or e.attn_plan(kv, tables, q_off, T, 4, groups=groups)
        w = torch.full((2, b.rows), 7.0, device="cuda")
        e.attn_weights(plan, 0, q, b.scale(), lse.cuda(), w, prev=(b.prev.cuda(), off, b.dev(src), keep), decay=b.decay)
        try:
            e.sync()
        except pk.DMError:
            return w.cpu(), True
        return w.cpu(), False

    good, told = run(b.src)
    assert not told
    ref, tol, written = b.reference(lse)
    assert bool(((good.double() - ref).abs() <= tol)[:, written].all())
    places = [slice(int(b.off[s]) * 16, int(b.off[s]) * 16 + int(b.len[s])) for s in range(len(seqs))]
    for bad in (-1, 5000):
        _say("source", bad)
        src = b.src.copy()
        src[4] = bad
        w, told = run(src)
        assert told
        for s, at in enumerate(places):
            if s != 4:
                assert torch.equal(w[:, at], good[:, at]), s
        n = int(b.keep[4])
        at = slice(places[4].start, places[4].start + n)
        old = b.decay * b.prev[:, int(b.prev_off[b.src[4]]) * 16:][:, :n].double()
        assert bool(((w[:, at].double() - (ref[:, at] - old)).abs() <= tol[:, at]).all())
    _say("length")
    length = b.len.copy()
    length[2] += 4000
    w, told = run(b.src, length)
    assert told and bool((w[:, places[2]] == 7).all())
    _say("plan")
    other = e.attn_plan(kv, b.tables(), q_off, T, 4, groups=b.dev(np.array([0, 11], np.int64)))
    mine = e.attn_plan(kv, b.tables(), q_off, T, 4, groups=groups)
    mine.buf = other.buf
    w, told = run(b.src, plan=mine)
    assert told and bool((w == 7).all())


@pytest.mark.parametrize("heads,dim,paired,new,dtype", [((8, 8), 64, False, [1], "bf16"), ((16, 8), 64, True, [1, 2], "f16"),
                                                        ((48, 8), 64, False, [1, 3, 1], "bf16"), ((14, 7), 64, False, [1, 0, 4], "f16"),
                                                        ((8, 8), 128, False, [2], "bf16"), ((8, 8), 256, False, [1], "f16")])
def test_waves_of_several_heads(heads, dim, paired, new, dtype):
    """So many places that a wave has several heads, the last set of them a short one: dealt to a run's sequences, which are
    not a whole number of fours; the same batch without runs; a sequence with many rows among them."""
    pages = 512 if dim < 256 else 256
    n = 45 if pages == 512 else 87
    seqs = [(new[i % len(new)], 5 + 3 * i % 47, 0) for i in range(n)]
    b = Collected(16, seqs, prefixes=(16 * pages,), heads=heads, dim=dim, dtype=dtype, paired=paired, seed=heads[0] + dim)
    a_wave = b.rows // 64 * heads[1] // (32 * torch.cuda.get_device_properties(0).multi_processor_count)
    assert 4 <= a_wave < heads[1] and heads[1] % a_wave, a_wave
    _say("several heads", heads, dim, paired, new, "a wave", a_wave)
    b.check()
    b.check(groups=False)


@pytest.mark.parametrize("n,heads", [(13, (16, 8)), (26, (16, 8)), (35, (8, 8)), (22, (6, 6))])
def test_waves_of_few_heads(n, heads):
    """Two to four heads a wave, below and at the number from which on they are dealt; one sequence with many rows."""
    seqs = [(1 if i != 2 else 300, 5 + 3 * i % 47 + (300 if i == 2 else 0), 0) for i in range(n)]
    b = Collected(16, seqs, prefixes=(16 * (512 if n != 13 else 700),), heads=heads, dim=64, seed=n)
    a_wave = b.rows // 64 * heads[1] // (32 * torch.cuda.get_device_properties(0).multi_processor_count)
    assert 2 <= a_wave <= 4, a_wave
    _say("few heads", n, heads, "a wave", a_wave)
    b.check()
    b.check(groups=False)
