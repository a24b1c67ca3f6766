"""What differential attention, the collecting of weights and eviction refuse on the host, and what they launch and
allocate, against the counted stand-in for the runtime (fake_hip.c; see test_host_calls.py)."""
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


class Calls:
    """The calls with arguments that are accepted, but for those given (arrays are addresses only)."""

    def __init__(self, x):
        self.x, self.pk, self.h = x, x.pk, x.create()
        self.p = (x.buf(4096) + 255) // 256 * 256

    def kv(self, **k):
        a = dict(k=self.p, v=self.p, layer_stride=1 << 40, layers=2, n_pages=1000, kv_heads=4, head_dim=64, dtype=0, reserved=0)
        return self.pk.dm_kv_pages(**{**a, **k})

    def tables(self, **k):
        return self.pk.dm_page_tables(**{**dict(off=self.p, page=self.p, len=self.p, n=3, entries=100), **k})

    def batch(self, tokens=5, groups=0, **k):
        return self.pk.dm_token_batch(self.tables(**k), self.p, tokens, self.p if groups else None, groups)

    def diff(self, heads=8, kv={}, batch={}, layer=0, plan=None, **k):
        p = self.p
        a = dict(q=p, out=p, q_stride=512, out_stride=512, lse=p, lambda_=p, norm=p, scale=0.1, eps=1e-5, gain=1.0, reserved=0)
        return self.x.L.dm_diff_attn(self.h, C.byref(self.batch(**batch)), C.byref(self.kv(**kv)), heads,
                                     p if plan is None else plan, layer, C.byref(self.pk.dm_diff_args(**{**a, **k})))

    def plan(self, heads=8, kv={}, batch={}, size=1 << 20):
        return self.x.L.dm_diff_plan(self.h, C.byref(self.batch(**batch)), C.byref(self.kv(**kv)), heads, self.p, size)

    def weights(self, heads=8, kv={}, batch={}, layer=0, plan=None, **k):
        p = self.p
        a = dict(q=p, q_stride=512, lse=p, w=p, w_stride=1600, prev=p, prev_stride=900, prev_room=800, prev_off=p, src=p,
                 keep=p, prev_n=2, scale=0.1, decay=0.5, last=0, paired=0)
        return self.x.L.dm_attn_weights(self.h, C.byref(self.batch(**batch)), C.byref(self.kv(**kv)), heads,
                                        p if plan is None else plan, layer, C.byref(self.pk.dm_weight_args(**{**a, **k})))

    def select(self, tables={}, **k):
        p = self.p
        a = dict(w=p, w_layer_stride=6400, w_stride=1600, budget=p, room=p, kept=p, kept_stride=1600, keep=p, grow=p,
                 layers=2, kv_heads=4, share=2, sink=4, recent=9, reserved=0)
        return self.x.L.dm_evict_select(self.h, C.byref(self.tables(**tables)), C.byref(self.pk.dm_select_args(**{**a, **k})))

    def gather(self, kv={}, tables={}, to={}, **k):
        p = self.p
        a = dict(budget=p, kept=p, kept_stride=1600, w=p, w_layer_stride=6400, w_stride=1600, w_to=p, to_layer_stride=6400,
                 to_stride=1600, share=2, reserved=0)
        return self.x.L.dm_kv_gather(self.h, C.byref(self.kv(**kv)), C.byref(self.tables(**tables)), C.byref(self.tables(**to)),
                                     C.byref(self.pk.dm_gather_args(**{**a, **k})))

    def append_at(self, first, **k):
        p = self.p
        a = dict(q=p, k=p, v=p, q_stride=512, k_stride=256, v_stride=256, q_out=p, q_out_stride=512, q_norm=p, k_norm=p, cos=p,
                 sin=p, max_pos=100, q_heads=8, rot_dim=64, interleaved=0, eps=1e-6)
        return self.x.L.dm_kv_append_at(self.h, C.byref(self.kv()), 0, C.byref(self.batch()),
                                        C.byref(self.pk.dm_append_args(**{**a, **k})), first)


NAN, INF = float("nan"), float("inf")
REFUSED = {
    "plan": [dict(kv=dict(kv_heads=3), heads=6), dict(kv=dict(head_dim=256)), dict(kv=dict(dtype=2)), dict(heads=6), dict(size=100),
             dict(batch=dict(tokens=1 << 31)), dict(batch=dict(groups=4))],
    "diff": [dict(kv=dict(kv_heads=3), heads=6), dict(kv=dict(head_dim=256)), dict(kv=dict(head_dim=96)), dict(heads=6), dict(heads=0),
             dict(layer=2), dict(plan=0), dict(plan=8), dict(lambda_=0), dict(lambda_=6), dict(norm=8), dict(lse=2), dict(q=0), dict(q=8),
             dict(out=0), dict(q_stride=504), dict(out_stride=516), dict(q_stride=-8), dict(scale=0.0), dict(scale=-1.0),
             dict(scale=INF), dict(scale=NAN), dict(eps=-1e-9), dict(eps=NAN), dict(gain=INF), dict(gain=NAN), dict(reserved=1),
             dict(batch=dict(off=0)), dict(batch=dict(tokens=1 << 28)), dict(kv=dict(k=0)), dict(kv=dict(layer_stride=1000))],
    "weights": [dict(paired=1, kv=dict(kv_heads=3), heads=6), dict(paired=1, kv=dict(head_dim=256), q_stride=4096), dict(paired=2),
                dict(heads=6), dict(layer=2), dict(plan=0), dict(w=0), dict(w=2), dict(w_stride=1599), dict(lse=0), dict(q=0),
                dict(q=8), dict(q_stride=508), dict(src=0), dict(keep=0), dict(prev_off=0), dict(prev_stride=799),
                dict(prev_room=-1), dict(prev_off=0, src=0, keep=0), dict(prev_n=1 << 31), dict(scale=0.0), dict(scale=NAN),
                dict(decay=INF), dict(decay=NAN), dict(batch=dict(tokens=1 << 28)), dict(batch=dict(page=0))],
    "select": [dict(share=0), dict(share=3), dict(share=8), dict(layers=0), dict(kv_heads=0, share=1), dict(kv_heads=5000, share=1),
               dict(w=0), dict(w=2), dict(w_stride=1599), dict(w_layer_stride=4000), dict(kept=0), dict(kept_stride=1599), dict(keep=0),
               dict(grow=4), dict(budget=0), dict(room=4), dict(reserved=1), dict(tables=dict(len=0)), dict(tables=dict(n=1 << 31)),
               dict(tables=dict(entries=1 << 40))],
    "gather": [dict(share=0), dict(share=3), dict(budget=0), dict(budget=4), dict(kept=0), dict(kept_stride=1599), dict(w=0),
               dict(w_to=0), dict(w_stride=1599), dict(to_stride=1599), dict(to_layer_stride=100), dict(w_layer_stride=-1),
               dict(reserved=1), dict(to=dict(n=2)), dict(to=dict(off=0)), dict(tables=dict(len=0)), dict(kv=dict(v=0)),
               dict(kv=dict(layers=0))],
}


OVERLAP = {  # layers of which one's last head would be another's first; with one head each, the same places
    "select": [dict(w_layer_stride=4800), dict(w_layer_stride=6399), dict(kv_heads=1, share=1, w_layer_stride=0),
               dict(kv_heads=1, share=1, w_layer_stride=1599), dict(w_layer_stride=6500, w_stride=2000), dict(w_layer_stride=-6400)],
    "gather": [dict(to_layer_stride=4800), dict(w_layer_stride=4800), dict(to_layer_stride=6399), dict(w_layer_stride=6399),
               dict(kv=dict(kv_heads=1), share=1, to_layer_stride=0), dict(kv=dict(kv_heads=1), share=1, w_layer_stride=0)],
}


def scenario_overlap(x):
    c = Calls(x)
    launches = x.word("fake_launches")
    for name, cases in OVERLAP.items():
        call = getattr(c, name)
        for bad in cases:
            before = launches.value
            assert call(**bad) == x.pk.DM_EINVAL, (name, bad)
            assert launches.value == before and x.L.dm_last_error(c.h), (name, bad)
    # one layer has no stride between layers; rows apart, the last one's end is what counts
    assert c.select(layers=1, w_layer_stride=0) == x.pk.DM_OK
    assert c.select(w_stride=2000, w_layer_stride=7600) == x.pk.DM_OK
    assert c.gather(kv=dict(layers=1), w_layer_stride=0, to_layer_stride=0) == x.pk.DM_OK
    assert c.gather(to_stride=(1 << 40) - 1, to_layer_stride=1 << 43) == x.pk.DM_OK


def scenario_refusals(x):
    c = Calls(x)
    launches = x.word("fake_launches")
    for name, cases in REFUSED.items():
        call = getattr(c, name)
        before = launches.value
        assert call() == x.pk.DM_OK, (name, x.L.dm_last_error(c.h))
        assert launches.value > before
        for bad in cases:
            # numbers that stand for places are off the arrays' base
            bad = {k: (c.p + v if v in (2, 4, 6, 8) and k in ("q", "w", "lse", "lambda_", "norm", "plan", "grow", "room", "budget")
                       else v) for k, v in bad.items()}
            before = launches.value
            assert call(**bad) == x.pk.DM_EINVAL, (name, bad)
            assert launches.value == before and x.L.dm_last_error(c.h), (name, bad)
        nothing = dict(batch=dict(n=0, entries=0, tokens=0)) if name in ("plan", "diff", "weights") else dict(tables=dict(n=0, entries=0))
        if name == "gather":
            nothing["to"] = dict(n=0, entries=0)
        assert call(**nothing) == x.pk.DM_OK, name
    assert c.append_at(None) == x.pk.DM_OK and c.append_at(c.p) == x.pk.DM_OK
    assert c.append_at(c.p + 4) == x.pk.DM_EINVAL
    assert c.append_at(c.p, q_norm=c.p + 8) == x.pk.DM_EINVAL and b"dm_kv_append_at" in x.L.dm_last_error(c.h)
    for f in ("dm_diff_plan", "dm_diff_attn", "dm_attn_weights", "dm_evict_select", "dm_kv_gather", "dm_kv_append_at"):
        fn = getattr(x.L, f)
        assert fn(None, *[0 if t in (C.c_uint32, C.c_uint64) else None for t in fn.argtypes[1:]]) == x.pk.DM_EINVAL, f


def scenario_areas(x):
    """Differential attention's work area is that of attention with heads twice as wide; the others have none."""
    c, held = Calls(x), x.word("fake_bytes")
    before = held.value
    assert c.weights() == x.pk.DM_OK and c.select() == x.pk.DM_OK and c.gather() == x.pk.DM_OK
    assert held.value == before
    assert c.diff(batch=dict(tokens=4096, entries=1000)) == x.pk.DM_OK
    rows = 384 * 256
    assert rows * 130 * 4 <= held.value - before <= rows * 130 * 4 + 4096


def scenario_weights_area(x):
    """Sums of stretches of rows: none for a few rows a sequence, up to 32 for a place otherwise, 2^24 floats or one for each
    place at the most; growth under capture is refused."""
    held, capturing = x.word("fake_bytes"), x.word("fake_capturing", C.c_int)
    for tokens, n, entries, last, parts in ((64, 64, 4000, 0, 0), (66, 64, 4000, 0, 0), (16_000, 2, 1000, 0, (2, 32)),
                                            (16_000, 2, 1000, 16, 0), (16_000, 2, 1000, 200, (1, 32)),
                                            (6400, 64, 32_768, 0, (1, 8)), (100_000, 4, 1 << 20, 0, (1, 1))):
        c = Calls(x)
        before = held.value
        kw = dict(batch=dict(tokens=tokens, n=n, entries=entries), w_stride=entries * 16, last=last)
        assert c.weights(**kw) == x.pk.DM_OK
        one = entries * 16 * 4 * 4
        got = held.value - before
        if parts == 0:
            assert got == 0, (tokens, n, got)
        else:
            assert one * parts[0] <= got <= one * parts[1] + 4096, (tokens, n, got / one)
            assert got <= max(4 << 24, one) + 4096
            capturing.value = 1
            assert c.weights(**kw) == x.pk.DM_OK
            kw["batch"]["entries"], kw["w_stride"] = 64 * entries, 64 * entries * 16
            assert c.weights(**kw) == x.pk.DM_EDEVICE and b"capture" in x.L.dm_last_error(c.h)
            capturing.value = 0
            assert c.weights(**kw) == x.pk.DM_OK
        x.L.dm_destroy(c.h)


def scenario_select_area(x):
    """Few and long choices: counts and a list, 2^29 bytes at the most; none for others; growth under capture is refused."""
    held, capturing = x.word("fake_bytes"), x.word("fake_capturing", C.c_int)
    for n, entries, layers, heads, some in ((4, 400, 2, 4, False), (4, 8000, 2, 4, True), (1, 1537, 1, 1, True), (1, 1536, 1, 1, False),
                                            (2, 65_536, 4, 8, True), (2, 65_536, 32, 8, False), (1, 1 << 22, 1, 2, False)):
        c = Calls(x)
        before = held.value
        rows = entries * 16
        kw = dict(tables=dict(n=n, entries=entries), w_stride=rows, w_layer_stride=rows * heads, kept_stride=rows, layers=layers,
                  kv_heads=heads, share=1)
        assert c.select(**kw) == x.pk.DM_OK
        got = held.value - before
        if some:
            assert layers * heads * rows * 4 < got <= (1 << 29) + 4096, (n, entries, got)
            capturing.value = 1
            assert c.select(**kw) == x.pk.DM_OK
            kw.update(tables=dict(n=n, entries=2 * entries), w_stride=2 * rows, w_layer_stride=2 * rows * heads, kept_stride=2 * rows)
            grown = c.select(**kw)
            capturing.value = 0
            assert grown == x.pk.DM_EDEVICE and b"capture" in x.L.dm_last_error(c.h)
        else:
            assert got == 0, (n, entries, got)
        x.L.dm_destroy(c.h)


def scenario_weights_runs_area(x):
    """With runs, 68 bytes a sequence, beside the sums of stretches where there are some."""
    held = x.word("fake_bytes")
    for tokens, n, groups, some in ((64, 64, 0, 0), (64, 64, 4, 68 * 64), (5000, 5000, 9, 68 * 5000)):
        c = Calls(x)
        before = held.value
        assert c.weights(batch=dict(tokens=tokens, n=n, entries=4000, groups=groups), w_stride=64_000) == x.pk.DM_OK
        assert some <= held.value - before <= (some + 4096 if some else 0), (n, groups, held.value - before)
        x.L.dm_destroy(c.h)


def test_weights_runs_work_area(fake):  # noqa: F811
    _child(fake, "weights_runs_area")


def test_select_work_area(fake):  # noqa: F811
    _child(fake, "select_area")


def test_weights_work_area(fake):  # noqa: F811
    _child(fake, "weights_area")


def test_refusals(fake):  # noqa: F811
    _child(fake, "refusals")


def test_layers_do_not_overlap(fake):  # noqa: F811
    _child(fake, "overlap")


def test_work_areas(fake):  # noqa: F811
    _child(fake, "areas")


if __name__ == "__main__":
    globals()["scenario_" + sys.argv[2]](Host(sys.argv[1], *sys.argv[3:]))
