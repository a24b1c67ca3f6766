"""What the calls on KV pages allocate, keep and refuse on the host, against the counted stand-in for the runtime
(fake_hip.c; see test_host_calls.py).  Every scenario runs in a child process."""
import ctypes as C
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from test_host_calls import Host, fake  # noqa: E402, F401


def _child(fake, scenario):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, scenario], cwd=ROOT, capture_output=True,
                       text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


class Pages:
    """Calls of given sizes on a context (arrays are addresses only: kernels do not run)."""

    def __init__(self, x, h):
        self.x, self.h, self.pk = x, h, x.pk
        self.p = (x.buf(4096) + 255) // 256 * 256

    def kv(self, kv_heads, dim):
        return self.pk.dm_kv_pages(self.p, self.p, 1 << 40, 1, 1000, kv_heads, dim, 0, 0)

    def batch(self, n, tokens, groups, entries):
        p = self.p
        return self.pk.dm_token_batch(self.pk.dm_page_tables(p, p, p, n, entries), p, tokens, p if groups else None, groups)

    def attn(self, tokens, heads=(8, 2), dim=128, n=1, groups=0, entries=1000):
        kv, b, p = self.kv(heads[1], dim), self.batch(n, tokens, groups, entries), self.p
        return self.x.L.dm_attn(self.h, C.byref(b), C.byref(kv), heads[0], p, 0, p, heads[0] * dim, 0.1, p, heads[0] * dim, None)

    def fork(self, n, m, n_pages, entries=1000, cap=1000):
        p = self.p
        t, o = self.pk.dm_page_tables(p, p, p, n, entries), self.pk.dm_pages_out(p, p, p, cap, p, p, p, 10, p, p)
        return self.x.L.dm_pages_fork(self.h, C.byref(t), p, n_pages, p, p, p, m, C.byref(o))

    def compact(self, n, n_pages, entries=1000):
        p = self.p
        t, o = self.pk.dm_page_tables(p, p, p, n, entries), self.pk.dm_pages_out(p, p, p, entries, p, p, p, 10, p, p)
        return self.x.L.dm_pages_compact(self.h, C.byref(t), p, n_pages, C.byref(o))


def scenario_captured_areas(x):
    """A work area that a captured call used is owned until the context goes, whatever call outgrows it; one that no
    capture used is given back when it is outgrown."""
    capturing, frees, held = x.word("fake_capturing", C.c_int), x.word("fake_frees"), x.word("fake_bytes")
    mallocs = x.word("fake_mallocs")
    calls = {
        "attn": lambda s, k: s.attn(512 * k, dim=64 if k < 100 else 256, groups=1),
        "fork": lambda s, k: s.fork(5000 * k, 5000 * k, 200_000 * k),
        "compact": lambda s, k: s.compact(5000 * k, 1_000_000 * k),
    }
    for name, call in calls.items():
        for outgrow in calls.values():
            for captured in (True, False):
                start = held.value
                h = x.create()
                s = Pages(x, h)
                assert call(s, 1) == x.pk.DM_OK, name
                capturing.value = int(captured)
                assert call(s, 1) == x.pk.DM_OK, ("capture", name)
                capturing.value = 0
                freed, made = frees.value, mallocs.value
                for k in (16, 400):
                    assert outgrow(s, k) == x.pk.DM_OK, name
                # captured: its area stays; one that no graph knows goes when it is outgrown
                grown = mallocs.value - made
                assert grown >= 1
                assert frees.value - freed == grown - captured, (name, captured, grown, frees.value - freed)
                x.L.dm_destroy(h)
                assert held.value == start, "everything is given back in the end"


def scenario_growth_under_capture(x):
    """A call that needs a larger area under capture is refused before it waits or allocates, and the context goes on."""
    capturing = x.word("fake_capturing", C.c_int)
    count = lambda: tuple(x.word(w).value for w in ("fake_mallocs", "fake_frees", "fake_syncs", "fake_launches"))  # noqa: E731
    calls = (lambda s, k: s.attn(4096 * k, groups=1), lambda s, k: s.fork(5000 * k, 5000 * k, 200_000 * k),
             lambda s, k: s.compact(5000 * k, 1_000_000 * k))
    for call in calls:
        for warm in (False, True):
            h = x.create()
            s = Pages(x, h)
            if warm:
                assert call(s, 1) == x.pk.DM_OK
            capturing.value = 1
            before = count()
            assert call(s, 16) == x.pk.DM_EDEVICE
            assert count() == before
            assert b"capture" in x.L.dm_last_error(h)
            if warm:
                assert call(s, 1) == x.pk.DM_OK
            capturing.value = 0
            assert call(s, 16) == x.pk.DM_OK
            x.L.dm_destroy(h)


def scenario_attention_area(x):
    """What attention's work area holds: 384 rows of parts a compute unit (256 of them here), and the batch's rows twice, up
    to 2^20, only if it has runs."""
    held = x.word("fake_bytes")
    for tokens in (300, 4096, 16_384):
        for dim in (64, 128, 256):
            for groups in (0, 1):
                h = x.create()
                s = Pages(x, h)
                before = held.value
                assert s.attn(tokens, heads=(32, 8), dim=dim, groups=groups) == x.pk.DM_OK
                rows = 384 * 256 + (min(2 * tokens * 32, 1 << 20) if groups else 0)
                assert rows * (dim + 2) * 4 <= held.value - before <= rows * (dim + 2) * 4 + 4096, (tokens, dim, groups)
                x.L.dm_destroy(h)


def test_attention_work_area(fake):  # noqa: F811
    _child(fake, "attention_area")


def scenario_small_calls(x):
    """Calls on page tables go in one workgroup where that is the faster, by pages, sequences and room for entries."""
    h, runs = x.create(), x.word("fake_launches")
    s = Pages(x, h)

    def launches(call, *a, **k):
        before = runs.value
        assert call(*a, **k) == x.pk.DM_OK
        return runs.value - before

    for pages, n, entries, one in ((767, 24, 600, True), (767, 24, 32_768, True), (2048, 256, 4096, True),
                                   (4096, 256, 4096, True), (4096, 256, 8192, False), (8192, 64, 8192, False),
                                   (8192, 1024, 8192, False), (8192, 256, 32_768, False), (8192, 1024, 32_768, False),
                                   (1000, 1025, 1000, False), (8193, 1, 1, False), (1, 1, 32_769, False), (1, 1, 0, True)):
        for rows, room in (((n, n), (entries, entries)), ((n, 1), (entries, 1)), ((1, n), (1, entries))):
            got = launches(s.fork, rows[0], rows[1], pages, entries=room[0], cap=room[1])
            assert got == (1 if one else 5), (pages, n, entries, got)
    for pages, n, entries, one in ((767, 24, 600, True), (767, 24, 32_768, True), (2048, 256, 4096, True), (8192, 256, 8192, True),
                                   (4096, 256, 16_384, True), (8192, 256, 16_384, False), (8192, 65_536, 4096, True),
                                   (8192, 256, 32_768, False), (8193, 1, 1, False), (1, 1, 32_769, False)):
        got = launches(s.compact, n, pages, entries=entries)
        assert got == (1 if one else 4), (pages, n, entries, got)


def test_page_table_calls_in_one_workgroup(fake):  # noqa: F811
    _child(fake, "small_calls")


def test_captured_work_areas_are_kept(fake):  # noqa: F811
    _child(fake, "captured_areas")


def test_growth_under_capture_is_refused(fake):  # noqa: F811
    _child(fake, "growth_under_capture")


if __name__ == "__main__":
    globals()["scenario_" + sys.argv[2]](Host(sys.argv[1], *sys.argv[3:]))
