"""Page tables of the next step, compaction and page copies against a plain implementation with lists and sets, entry
by entry (whole numbers: no tolerance)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

_ENG = {}


def engine(block):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_06502_amd as pk
    if block not in _ENG:
        _ENG[block] = pk.DualMap(dict(block=block, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1,
                                      index_log2_slots=4))
    return pk, _ENG[block]


def plain_fork(B, tables, lens, ref, src, keep, grow):
    """(tables, lengths, counts, moves) of the next step, one sequence after the other."""
    up = lambda n: -(-n // B)  # noqa: E731
    total = list(ref)
    for t in tables:
        for p in t:
            total[p] -= 1
    new = [list(tables[s][:up(k)]) if k else [] for s, k in zip(src, keep)]
    for t in new:
        for p in t:
            total[p] += 1
    writers = {}
    for j, (k, g) in enumerate(zip(keep, grow)):
        if k % B and g:
            writers.setdefault(new[j][-1], []).append(j)
    copies = set()
    for p, js in writers.items():
        copies |= set(js[1:] if total[p] == len(js) else js)
    free = iter([p for p, r in enumerate(ref) if r == 0])
    moves = []
    for j in range(len(new)):
        if j in copies:
            old, to = new[j][-1], next(free)
            new[j][-1] = to
            moves.append((old, to))
            total[old] -= 1
            total[to] += 1
        for _ in range(up(keep[j] + grow[j]) - up(keep[j])):
            to = next(free)
            new[j].append(to)
            total[to] += 1
    return new, [k + g for k, g in zip(keep, grow)], total, moves


def csr(tables):
    off = np.concatenate([[0], np.cumsum([len(t) for t in tables])]).astype(np.int64)
    return off, np.array([p for t in tables for p in t], np.int32)


def dev(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype).reshape(-1).copy()).cuda()


def make(r, B, n, pages, most, shared=4):
    """Tables in which pages are shared: some sequences begin with another's leading pages."""
    ids = list(r.permutation(pages))
    tables, lens = [], []
    for s in range(n):
        t = []
        if tables and r.random() < 0.6:
            o = tables[r.integers(max(0, s - shared), s)]
            t = list(o[:r.integers(0, len(o) + 1)])
        own = int(r.integers(0, most + 1))
        t += [int(ids.pop()) for _ in range(min(own, len(ids)))]
        tables.append(t)
        lens.append(int(r.integers(max(0, (len(t) - 1) * B + 1), len(t) * B + 1)) if t else 0)
    ref = np.zeros(pages, np.int64)
    for t in tables:
        for p in t:
            ref[p] += 1
    return tables, lens, ref


def check_fork(B, tables, lens, ref, src, keep, grow, room=0, entry0=0):
    pk, e = engine(B)
    want, wl, wr, wm = plain_fork(B, tables, lens, ref, src, keep, grow)
    off, page = csr(tables)
    wo, wp = csr(want)
    m = len(src)
    out = e.alloc_pages_out(len(ref), m, len(wp) + room)
    for x in out.values():
        x.fill_(-7)
    pad = np.full(entry0, 5, np.int32)  # entries that belong to no table
    e.pages_fork_into((dev(off + entry0, np.int64), dev(np.concatenate([pad, page, pad]), np.int32), dev(lens, np.int64)),
                      dev(ref, np.int32), dev(src, np.int32), dev(keep, np.int64), dev(grow, np.int64), out)
    e.sync()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert np.array_equal(got["off"], wo) and np.array_equal(got["len"], wl)
    assert np.array_equal(got["page"][:len(wp)], wp) and (got["page"][len(wp):] == -7).all()
    assert np.array_equal(got["ref"], wr)
    assert got["moves"][0] == len(wm)
    assert list(zip(got["move_src"][:len(wm)], got["move_dst"][:len(wm)])) == wm
    assert (got["move_src"][len(wm):] == -7).all()
    return want, wl, wr, wm


@pytest.mark.parametrize("B", [4, 16, 64])
@pytest.mark.parametrize("n,m", [(1, 1), (1, 5), (7, 0), (7, 3), (40, 90), (200, 150)])
def test_fork(B, n, m):
    """Random continuations, forks, ends, new sequences, cuts and pins, several steps on."""
    print("[case] fork", B, n, m, flush=True)
    r = np.random.default_rng([B, n, m])
    pages = 6000
    tables, lens, ref = make(r, B, n, 3000, 12)
    ref = np.concatenate([ref, np.zeros(pages - len(ref), np.int64)])
    ref[[t[0] for t in tables if t][:3]] += 1  # held by a cached prefix besides
    for step in range(3):
        src = r.integers(0, len(tables), size=m) if len(tables) else np.full(m, -1)
        keep = [int(lens[s] if r.random() < 0.5 else r.integers(0, lens[s] + 1)) if s >= 0 else 0 for s in src]
        grow = [int(g) for g in r.integers(0, 3 * B, size=m) * (r.random(m) < 0.7)]
        src = [int(s) if k else int(r.choice([-1, s, 10 ** 6])) for s, k in zip(src, keep)]
        tables, lens, ref, _ = check_fork(B, tables, lens, ref, src, keep, grow, room=step, entry0=step)
        ref = np.array(ref)


def test_fork_cases_by_hand():
    B = 16
    # one sequence of 20 tokens in pages 3, 1; three go on writing: the first keeps page 1
    t, n, r, mv = check_fork(B, [[3, 1]], [20], [0, 1, 0, 1, 0, 0], [0, 0, 0], [20, 20, 20], [1, 1, 1])
    assert t == [[3, 1], [3, 0], [3, 2]] and mv == [(1, 0), (1, 2)]
    # the page is held elsewhere too: all copy
    t, n, r, mv = check_fork(B, [[3, 1]], [20], [0, 2, 0, 1, 0, 0], [0, 0], [20, 20], [1, 1])
    assert t == [[3, 0], [3, 2]] and r[1] == 1
    # who does not write shares the page, and so the writer copies
    t, n, r, mv = check_fork(B, [[3, 1]], [20], [0, 1, 0, 1, 0, 0], [0, 0], [20, 20], [0, 1])
    assert t == [[3, 1], [3, 0]] and mv == [(1, 0)]
    # full pages are shared, whatever grows; a cut inside a full page copies it
    check_fork(B, [[3, 1]], [32], [0, 1, 0, 1, 0, 0], [0, 0], [32, 32], [5, 5])
    t, n, r, mv = check_fork(B, [[3, 1]], [32], [0, 1, 0, 1, 0, 0], [0, 0], [32, 20], [0, 5])
    assert mv == [(1, 0)]
    # everything ends; nothing there
    check_fork(B, [[3, 1]], [32], [0, 1, 0, 1, 0, 0], [], [], [])
    check_fork(B, [], [], [0, 0, 0], [-1, -1], [0, 0], [17, 0])
    # pages held past the length are let go
    check_fork(B, [[3, 1, 2]], [17], [0, 1, 1, 1, 0, 0], [0], [17], [1])


def test_fork_many_sequences():
    """More sequences than a workgroup scans at once, and more pages than one counts."""
    r = np.random.default_rng(5)
    tables, lens, ref = make(r, 8, 3000, 40_000, 10)
    ref = np.concatenate([ref, np.zeros(20_000, np.int64)])
    src = r.integers(0, 3000, size=2500)
    keep = [lens[s] for s in src]
    check_fork(8, tables, lens, ref, [int(s) for s in src], keep, [int(g) for g in r.integers(0, 12, size=2500)])


def test_fork_errors_write_nothing():
    pk, e = engine(16)
    tables, lens, ref = [[3, 1], [3, 2]], [20, 20], [0, 1, 1, 2, 0, 0]

    def attempt(status, tables=tables, lens=lens, ref=ref, src=(0, 0), keep=(20, 20), grow=(1, 1), cap=9, off=None,
                page=None):
        o, p = csr(tables)
        o = np.array(off, np.int64) if off is not None else o
        p = np.array(page, np.int32) if page is not None else p
        out = e.alloc_pages_out(len(ref), len(src), cap)
        for x in out.values():
            x.fill_(-7)
        e.pages_fork_into((dev(o, np.int64), dev(p, np.int32), dev(lens, np.int64)), dev(ref, np.int32),
                          dev(src, np.int32), dev(keep, np.int64), dev(grow, np.int64), out)
        with pytest.raises(pk.DMError) as x:
            e.sync()
        assert x.value.status == status
        assert out.pop("moves").item() == 0
        assert all(bool((v == -7).all()) for v in out.values())

    attempt(pk.DM_EFULL, cap=3)
    attempt(pk.DM_EFULL, ref=[1, 1, 1, 2, 1, 1])  # no free page
    attempt(pk.DM_EFULL, grow=(40, 40))
    attempt(pk.DM_EINVAL, src=(0, 2))
    attempt(pk.DM_EINVAL, src=(0, -1))
    attempt(pk.DM_EINVAL, keep=(21, 0))
    attempt(pk.DM_EINVAL, keep=(-1, 0))
    attempt(pk.DM_EINVAL, grow=(-1, 0))
    attempt(pk.DM_EINVAL, grow=(2 ** 40, 0))
    attempt(pk.DM_EINVAL, lens=[33, 20])
    attempt(pk.DM_EINVAL, lens=[-1, 20])
    attempt(pk.DM_EINVAL, off=[0, 9, 4])
    attempt(pk.DM_EINVAL, off=[-1, 2, 4])
    attempt(pk.DM_EINVAL, off=[0, 2, 5])
    attempt(pk.DM_EINVAL, page=[3, 6, 3, 2])
    attempt(pk.DM_EINVAL, page=[3, -1, 3, 2])
    attempt(pk.DM_EINVAL, ref=[0, 0, 1, 2, 0, 0])  # a page without a reference
    attempt(pk.DM_EINVAL, ref=[-1, 1, 1, 2, 0, 0])
    with pytest.raises(ValueError):
        e.pages_fork_into((dev([0], np.int64), dev([], np.int32), dev([], np.int64)), dev([0, 0], np.int64),
                          dev([], np.int32), dev([], np.int64), dev([], np.int64), e.alloc_pages_out(2, 0, 0))
    with pytest.raises(ValueError):
        e.pages_fork_into((dev([0], np.int64), dev([], np.int32), dev([], np.int64)), dev([0, 0], np.int32),
                          dev([], np.int32), dev([], np.int64), dev([], np.int64), e.alloc_pages_out(3, 0, 0))
    check_fork(16, tables, lens, ref, [0, 0], [20, 20], [1, 1])


def plain_compact(tables, ref):
    live = [p for p, r in enumerate(ref) if r > 0]
    L = len(live)
    holes = [p for p in range(L) if ref[p] == 0]
    movers = [p for p in live if p >= L]
    to = dict(zip(movers, holes))
    out = [0] * len(ref)
    for p in live:
        out[to.get(p, p)] = ref[p]
    return [[to.get(p, p) for p in t] for t in tables], out, list(zip(movers, holes)), L


@pytest.mark.parametrize("pages,share", [(1, 1.0), (5, 0.0), (64, 0.5), (1023, 0.9), (1024, 1.0), (1025, 0.01),
                                         (5000, 0.3), (40_000, 0.6)])
def test_compact(pages, share):
    print("[case] compact", pages, share, flush=True)
    pk, e = engine(16)
    r = np.random.default_rng(pages)
    live = [int(p) for p in r.permutation(pages)[:int(pages * share)]]
    cuts = sorted(int(x) for x in r.integers(0, len(live) + 1, size=6))
    tables = [live[a:b] for a, b in zip([0] + cuts, cuts + [len(live)])]
    tables.append(live[:len(live) // 3])
    ref = np.zeros(pages, np.int64)
    for t in tables:
        for p in t:
            ref[p] += 1
    if pages > 4:
        ref[r.integers(0, pages)] += 1  # held without a table
    wt, wr, wm, wl = plain_compact(tables, ref)
    off, page = csr(tables)
    out = e.alloc_pages_out(pages, 0, len(page) + 2)
    for x in out.values():
        x.fill_(-7)
    lens = np.zeros(len(tables), np.int64)
    e.pages_compact_into((dev(off, np.int64), dev(page, np.int32), dev(lens, np.int64)), dev(ref, np.int32), out)
    e.sync()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert got["live"][0] == wl and got["moves"][0] == len(wm)
    assert np.array_equal(got["page"][:len(page)], csr(wt)[1]) and (got["page"][len(page):] == -7).all()
    assert np.array_equal(got["ref"], wr)
    assert list(zip(got["move_src"][:len(wm)], got["move_dst"][:len(wm)])) == wm


def test_compact_errors_write_nothing():
    pk, e = engine(16)

    def attempt(status, off, page, ref, moves=None):
        out = e.alloc_pages_out(len(ref), 0, len(page))
        if moves is not None:
            out["move_src"], out["move_dst"] = out["move_src"][:moves].clone(), out["move_dst"][:moves].clone()
        for x in out.values():
            x.fill_(-7)
        e.pages_compact_into((dev(off, np.int64), dev(page, np.int32), dev([0] * (len(off) - 1), np.int64)),
                             dev(ref, np.int32), out)
        with pytest.raises(pk.DMError) as x:
            e.sync()
        assert x.value.status == status
        assert out.pop("moves").item() == 0
        assert all(bool((v == -7).all()) for v in out.values())

    attempt(pk.DM_EINVAL, [0, 2], [1, 9], [0, 1, 1, 0])
    attempt(pk.DM_EINVAL, [0, 2], [1, -1], [0, 1, 1, 0])
    attempt(pk.DM_EINVAL, [0, 2], [1, 3], [0, 1, 1, 0])
    attempt(pk.DM_EINVAL, [0, 3], [1, 2], [0, 1, 1, 0])
    attempt(pk.DM_EINVAL, [0, 2, 1], [1, 2], [0, 1, 1, 0])
    attempt(pk.DM_EINVAL, [0, 1], [1], [0, 1, -1, 0])
    attempt(pk.DM_EFULL, [0, 2], [2, 3], [0, 0, 1, 1], moves=1)


@pytest.mark.parametrize("where", [0, 0.5, 1])
@pytest.mark.parametrize("what", ["page past the pool", "negative page", "page without a reference", "negative count"])
def test_errors_in_large_calls_write_nothing(what, where):
    """One fault among many pages and entries, in the first, a middle or the last of them."""
    print("[case] large errors", what, where, flush=True)
    pk, e = engine(16)
    r = np.random.default_rng(41)
    n, pages = 1200, 40_000
    tables, lens, ref = make(r, 16, n, pages - 3000, 24)
    ref = np.concatenate([ref, np.zeros(3000, np.int64)])
    off, page = csr(tables)
    entry = int(where * (len(page) - 1))
    if what == "page past the pool":
        page[entry] = pages
    elif what == "negative page":
        page[entry] = -1
    elif what == "page without a reference":
        ref[page[entry]] = 0
    else:
        ref[int(where * (pages - 1))] = -1
    t = (dev(off, np.int64), dev(page, np.int32), dev(lens, np.int64))
    src = np.arange(n)
    for compact in (False, True):
        out = e.alloc_pages_out(pages, n, len(page) + 2 * n)
        for x in out.values():
            x.fill_(-7)
        if compact:
            e.pages_compact_into(t, dev(ref, np.int32), out)
        else:
            e.pages_fork_into(t, dev(ref, np.int32), dev(src, np.int32), dev(np.array(lens) // 2, np.int64),
                              dev(np.full(n, 9), np.int64), out)
        with pytest.raises(pk.DMError) as x:
            e.sync()
        assert x.value.status == pk.DM_EINVAL
        assert out.pop("moves").item() == 0
        assert all(bool((v == -7).all()) for v in out.values())


@pytest.mark.parametrize("B,heads,dim,layers,dtype", [(4, 1, 64, 1, "f16"), (16, 2, 64, 3, "bf16"), (32, 8, 128, 2, "bf16"),
                                                      (64, 3, 256, 2, "f16"), (16, 5, 128, 1, "bf16")])
def test_copy(B, heads, dim, layers, dtype):
    """Bits as they are (NaN too), every layer, keys and values; the list's rest is not read."""
    pk, e = engine(B)
    g = torch.Generator(device="cuda").manual_seed(B)
    pages = 50
    shape = (layers, pages, heads, B, dim)
    k = torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    v = torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    dt = dict(f16=torch.float16, bf16=torch.bfloat16)[dtype]
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(1))
    for count in (0, 1, 20):
        src, dst = perm[:20].int().cuda(), perm[20:40].int().cuda()
        wk, wv = k.clone(), v.clone()
        wk[:, dst[:count].long()] = k[:, src[:count].long()]
        wv[:, dst[:count].long()] = v[:, src[:count].long()]
        src[count:] = 10 ** 9
        e.pages_copy(pk.KVPages(k.view(dt), v.view(dt)), dict(move_src=src, move_dst=dst,
                                                              moves=torch.tensor([count], device="cuda")))
        e.sync()
        assert torch.equal(k, wk) and torch.equal(v, wv)


def test_copy_errors():
    pk, e = engine(16)
    k, v = (torch.randn((1, 8, 1, 16, 64), device="cuda").half() for _ in range(2))
    kv = pk.KVPages(k, v)
    i32 = dict(dtype=torch.int32, device="cuda")
    for src, dst, n, status in (([1, 8], [2, 3], 2, pk.DM_EINVAL), ([1, 4], [2, -1], 2, pk.DM_EINVAL),
                                ([1, 4], [2, 3], 3, pk.DM_EFULL)):
        want = k.clone()
        want[0, 2] = k[0, 1]
        if n == 3:
            want[0, 3] = k[0, 4]
        e.pages_copy(kv, dict(move_src=torch.tensor(src, **i32), move_dst=torch.tensor(dst, **i32),
                              moves=torch.tensor([n], device="cuda")))
        with pytest.raises(pk.DMError) as x:
            e.sync()
        assert x.value.status == status
        assert torch.equal(k, want)
    with pytest.raises(ValueError):
        pk.KVPages(k, v[:, :4])
    with pytest.raises(ValueError):
        engine(32)[1].pages_copy(kv, {})


def test_fork_then_copy_in_a_graph():
    """Captured, replayed with other inputs, each replay equal to the eager result."""
    pk, e0 = engine(16)
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    r = np.random.default_rng(3)
    n, pages = 20, 800
    tables, lens, ref = make(r, 16, n, 500, 8)
    ref = np.concatenate([ref, np.zeros(pages - len(ref), np.int64)])
    off, page = csr(tables)
    t = (dev(off, np.int64), dev(page, np.int32), dev(lens, np.int64))
    ref_d = dev(ref, np.int32)
    src, keep, grow = dev([0] * n, np.int32), dev([0] * n, np.int64), dev([0] * n, np.int64)
    k, v = (torch.randn((2, pages, 1, 16, 64), device="cuda").half() for _ in range(2))
    kv = pk.KVPages(k, v)
    out = e.alloc_pages_out(pages, n, 1000)
    for x in out.values():
        x.fill_(-7)
    k0 = k.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        e.pages_fork_into(t, ref_d, src, keep, grow, out)
        e.pages_copy(kv, out)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        e.pages_fork_into(t, ref_d, src, keep, grow, out)
        e.pages_copy(kv, out)
    for rep in range(4):
        s = r.integers(0, n, size=n)
        src.copy_(dev(s, np.int32))
        keep.copy_(dev([lens[x] for x in s], np.int64))
        grow.copy_(dev(r.integers(0, 20, size=n), np.int64))
        k.copy_(k0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, wl, wr, wm = plain_fork(16, tables, lens, ref, [int(x) for x in s], keep.tolist(), grow.tolist())
        assert out["page"][:len(csr(want)[1])].tolist() == csr(want)[1].tolist()
        assert out["ref"].tolist() == list(wr) and out["moves"].item() == len(wm)
        wk = k0.clone()
        for a, b in wm:
            wk[:, b] = k0[:, a]
        assert torch.equal(k, wk)
    e.close()
