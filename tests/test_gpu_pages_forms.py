"""Page tables around the sizes where a call goes from one workgroup to passes, entry by entry."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_pages import check_fork, csr, dev, engine, plain_compact  # noqa: E402


def tables_of(r, pages, n, entries, B):
    """n sequences of about entries / n pages among three quarters of the pages, shared as need be."""
    per = max(1, entries // n)
    ids = r.permutation(pages)[:max(1, min(pages * 3 // 4, entries))]
    tables = [[int(p) for p in np.resize(np.roll(ids, -int(r.integers(len(ids)))), min(per, len(ids)))] for _ in range(n)]
    lens = [int(r.integers((len(t) - 1) * B + 1, len(t) * B + 1)) for t in tables]
    ref = np.zeros(pages, np.int64)
    for t in tables:
        for p in t:
            ref[p] += 1
    return tables, lens, ref


# pages, sequences, entries: fork in one workgroup, at its limits, and in passes
SIZES = [(1100, 1024, 2900), (1200, 1024, 2900), (8000, 24, 4000), (8192, 24, 4000), (8192, 1, 30), (4096, 256, 6000),
         (4096, 256, 6200), (600, 300, 9000), (8193, 24, 1000), (1000, 1025, 1100)]


@pytest.mark.parametrize("pages,n,entries", SIZES)
def test_fork_of_either_form(pages, n, entries):
    print("[case] fork", pages, n, entries, flush=True)
    r = np.random.default_rng([pages, n])
    tables, lens, ref = tables_of(r, pages, n, entries, 8)
    src = [int(s) for s in r.integers(0, n, size=n)]
    keep = [lens[s] if r.random() < 0.7 else int(r.integers(0, lens[s] + 1)) for s in src]
    free = int((ref == 0).sum())
    grow = [int(g) for g in (r.integers(0, 9, size=n) if 2 * n < free else (r.random(n) < 0.1 * free / n) * 3)]
    check_fork(8, tables, lens, ref, src, keep, grow)


@pytest.mark.parametrize("pages,n,entries", SIZES + [(8192, 300, 8000), (8192, 300, 8400), (4096, 64, 16_000), (64, 3000, 3000)])
def test_compact_of_either_form(pages, n, entries):
    print("[case] compact", pages, n, entries, flush=True)
    pk, e = engine(8)
    r = np.random.default_rng([pages, n])
    tables, lens, ref = tables_of(r, pages, n, entries, 8)
    wt, wr, wm, wl = plain_compact(tables, ref)
    off, page = csr(tables)
    out = e.alloc_pages_out(pages, 0, len(page))
    e.pages_compact_into((dev(off, np.int64), dev(page, np.int32), dev(lens, np.int64)), dev(ref, np.int32), out)
    e.sync()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert got["live"][0] == wl and got["moves"][0] == len(wm)
    assert np.array_equal(got["page"], csr(wt)[1]) and np.array_equal(got["ref"], wr)
    assert list(zip(got["move_src"][:len(wm)], got["move_dst"][:len(wm)])) == wm
