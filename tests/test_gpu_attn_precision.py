"""How exactly attention's weights meet the values, against the definition in 64 bits.

Bounds, per element (u: half a unit in the last place of the type, 2^-8 for bfloat16, 2^-11 for float16): the output is
rounded once, u |out|; a weight that is rounded once before it meets the values is off by u of itself, u sum w|v| / sum
w; a float16 weight is raised by 2^7, so that one below 2^-21 of the row's largest is off by up to 2^-32 of that, n
2^-32 max|v| over n keys; sums in 32 bits add some 2^-20 of sum w|v| / sum w.  In narrow tiles (up to 16 rows a KV head) a weight
meets the values in two parts, the second what the first's rounding has left out: off by u^2 of itself.  The log-sum-exp is in 32 bits: 2^-18 of the largest |score|, and
of itself.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import DT, ULP, Batch, engine  # noqa: E402


def light_weights(dtype, heads, dim, where):
    """One key 17 above 131,072 others, which together have 0.0054 of the weight, 2^-24.5 of the largest each, for `heads`
    rows a KV head, of as many sequences as leave the keys uncut.  (out, lse, weights and values in 64 bits, lse in 64 bits)"""
    pk, e = engine(32)
    n, S, H = 131_073, 200, 4
    pages = -(-n // 32)
    one = {"first": 0, "middle": 70_001, "last": n - 1}[where]
    g = torch.Generator().manual_seed(dim + heads)
    k = torch.zeros((1, pages, H, 32, dim), dtype=DT[dtype])
    k[0, one // 32, :, one % 32] = 17 / (0.125 * dim)  # 17 at q = 1 and a scale of 1/8; a value of either type
    v = (1 + 0.25 * torch.randn((1, pages, 1, 32, dim), generator=g)).to(DT[dtype]).expand(1, pages, H, 32, dim).contiguous()
    v[0, one // 32, :, one % 32] = 0
    kd, vd = k.cuda(), v.cuda()
    i64 = dict(dtype=torch.int64, device="cuda")
    tables = (pages * torch.arange(S + 1, **i64), torch.arange(pages, dtype=torch.int32, device="cuda").repeat(S),
              torch.full((S,), n, **i64))
    q = torch.ones((S, H * heads, dim), dtype=DT[dtype], device="cuda")
    out, lse = torch.empty_like(q), torch.empty((S, H * heads), device="cuda")
    print("[case] light weights", dtype, heads, dim, where, flush=True)
    kv = pk.KVPages(kd, vd)
    e.attn(e.attn_plan(kv, tables, torch.arange(S + 1, **i64), S, H * heads), 0, q, 0.125, out, lse)
    e.sync()
    scores = (kd[0, :, 0].reshape(-1, dim)[:n].double() @ q[0, 0].double()) * 0.125
    assert float(scores.max()) == 17.0
    return out, lse, torch.softmax(scores, 0), vd[0, :, 0].reshape(-1, dim)[:n].double(), torch.logsumexp(scores, 0)


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 128), ("bf16", 256)])
@pytest.mark.parametrize("heads", [1, 32])
def test_many_light_weights_are_summed(heads, dtype, dim, where):
    """In a narrow tile (one row) and in a wide one (32)."""
    _, lse, _, _, far = light_weights(dtype, heads, dim, where)
    assert bool(((lse.double() - far).abs() <= 2.0 ** -18 * 36).all()), float((lse.double() - far).abs().max())


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [1, 32])
def test_many_light_float16_weights(heads, dim, where):
    """Weights of 2^-24.5 of the largest keep most of their bits."""
    out, _, w, vals, _ = light_weights("f16", heads, dim, where)
    want, mean = w @ vals, w @ vals.abs()
    tol = ULP["f16"] * (want.abs() + mean) * 1.02 + 2.0 ** -20 * mean + len(w) * 2.0 ** -32 * vals.abs().max() + 2.0 ** -25
    assert 0.005 < float(want.mean()) < 0.006 and float(tol.max()) < 1e-4
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


def magnitudes(b):
    """sum w|v| / sum w of each row, and the keys that each token sees."""
    T = int(b.q_off[-1])
    mean, keys = torch.zeros((T, b.hq, b.dim), dtype=torch.float64), torch.zeros((T, 1, 1), dtype=torch.float64)
    q = b.qrows.unflatten(1, (b.hq, b.dim)).double()
    ratio = b.hq // b.hkv
    for s in range(len(b.len)):
        L, t0, t1 = int(b.len[s]), int(b.q_off[s]), int(b.q_off[s + 1])
        at = torch.from_numpy(b.page[b.off[s]:b.off[s + 1]].astype("int64"))
        for t in range(t0, t1):
            n = L - t1 + t + 1
            keys[t] = n
            for h in range(b.hkv):
                K, V = (x[0][at, h].reshape(-1, b.dim)[:n].double() for x in (b.k, b.v))
                w = torch.softmax(q[t, h * ratio:(h + 1) * ratio] @ K.T * b.scale(), -1)
                mean[t, h * ratio:(h + 1) * ratio] = w @ V.abs()
    return mean, keys


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,heads", [(64, (14, 2)), (128, (32, 8)), (256, (4, 4))])
def test_few_rows_are_rounded_once(dtype, dim, heads):
    """Single tokens and drafts have the output's own rounding, and next to nothing of the weights'."""
    u = ULP[dtype]
    for seqs in ([(1, 300)], [(1, 100 + 331 * i) for i in range(17)] + [(2, 5), (2, 1400), (1, 9000)]):
        print("[case] rounded once", dtype, dim, heads, len(seqs), flush=True)
        b = Batch(16, seqs, heads=heads, dim=dim, dtype=dtype, seed=dim)
        out, _ = b.run()
        ref = b.reference()[0]
        mean, keys = magnitudes(b)
        tol = 1.02 * u * ref.abs() + (1.02 * u * u + 2.0 ** -20) * mean
        if dtype == "f16":
            tol = tol + keys * 2.0 ** -32 * float(b.v[~b.v.isnan()].abs().max()) + 2.0 ** -25
        err = (out.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())


def exact_scores(dtype, dim, heads, seqs, power, r):
    """A batch whose scores are 2^power times whole numbers from -3 to 3, so that they are exact in 32 bits: the keys of the
    largest share the weight (at 2^10 and above, whatever a row's largest is)."""
    b = Batch(16, seqs, heads=heads, dim=dim, dtype=dtype, seed=dim)
    b.qrows.zero_()
    b.qrows.unflatten(1, (b.hq, dim))[:, :, 0] = 2.0 ** (power // 2)
    b.k[~b.k.isnan()] = 0
    small = torch.from_numpy(r.integers(-3, 4, size=tuple(b.k.shape[:4]))).double()
    b.k[..., 0] = torch.where(b.k[..., 0].isnan(), math.nan, small * 2.0 ** (power - power // 2)).to(DT[dtype])
    return b


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,heads", [(64, (4, 2)), (128, (16, 1)), (256, (6, 3))])
def test_rows_in_parts_with_large_scores(dtype, dim, heads):
    """Parts of a row whose largest scores are equal count by their sums, however large the scores are."""
    r = np.random.default_rng(dim)
    for seqs in ([(3, 200), (1, 33), (40, 130), (70, 70)], [(1, 2500), (2, 4000), (1, 16)]):
        for power in (10, 14, 18):
            print("[case] parts, scores of 2 to the", power, dtype, dim, heads, len(seqs), flush=True)
            exact_scores(dtype, dim, heads, seqs, power, r).check(scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,heads", [(64, (4, 2)), (128, (16, 1)), (256, (6, 3))])
def test_scores_of_any_size(dtype, dim, heads):
    """Finite scores from 2^10 to 2^60 (bfloat16) or 2^26 (float16): drafts in narrow tiles, a prompt in wide ones, few rows."""
    r = np.random.default_rng(dim)
    for seqs in ([(2, 90)], [(3, 200), (1, 33), (40, 130), (70, 70)]):
        for power in range(10, (26 if dtype == "f16" else 60) + 1, 4):
            print("[case] scores of 2 to the", power, dtype, dim, heads, len(seqs), flush=True)
            exact_scores(dtype, dim, heads, seqs, power, r).check(scale=1.0)
