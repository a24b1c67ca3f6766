"""Queries and keys of new tokens normed, rotated and written to their pages, against the definition in 64 bits.

Bound, per element: one rounding to the type (half a unit in the last place: 2^-8 for bfloat16, 2^-11 for float16, and
half of float16's least step 2^-24) of a value that is computed in 32 bits from at most 256 squares, a reciprocal root and
a rotation: 2^-17 of the rotated pair's magnitude |a| + |b|.  Values are copied: equal in every bit.
"""
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


def turned(x, w, eps, cos, sin, pos, interleaved):
    """(result, pair magnitudes) in 64 bits."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + eps) * w.double()
    size = y.abs()
    if cos is not None:
        R = 2 * cos.shape[1]
        c, s = cos[pos].double()[:, None], sin[pos].double()[:, None]
        out, size = y.clone(), size.clone()
        if interleaved:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            out[..., 0:R:2], out[..., 1:R:2] = a * c - b * s, b * c + a * s
            size[..., 0:R:2] = size[..., 1:R:2] = a.abs() + b.abs()
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            out[..., :R // 2], out[..., R // 2:R] = a * c - b * s, b * c + a * s
            size[..., :R // 2] = size[..., R // 2:R] = a.abs() + b.abs()
        y = out
    return y, size


def case(dtype="bf16", dim=128, heads=(8, 2), block=16, rot=None, interleaved=False, norm="both", seqs=((3, 10), (1, 1)),
         layers=1, layer=0, in_place=False, packed=True, seed=0, lens=None):
    """seqs: (new tokens, tokens before them)."""
    pk, e = engine(block)
    g = torch.Generator().manual_seed(seed)
    r = np.random.default_rng(seed)
    dt, (hq, hk), B = DT[dtype], heads, block
    rot = dim if rot is None else rot
    new = [s[0] for s in seqs]
    length = np.array([a + b for a, b in seqs], np.int64) if lens is None else np.array(lens, np.int64)
    count = -(-length // B)
    pages = int(count.sum()) + 4
    page = r.permutation(pages)[:int(count.sum())].astype(np.int32)
    off = np.concatenate([[0], np.cumsum(count)]).astype(np.int64)
    q_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    T = int(q_off[-1])
    k0 = torch.randn((layers, pages, hk, B, dim), generator=g).to(dt)
    v0 = torch.randn((layers, pages, hk, B, dim), generator=g).to(dt)
    qkv = torch.randn((T, hq + 2 * hk, dim), generator=g).to(dt)
    wq = (1 + 0.3 * torch.randn(dim, generator=g)).to(dt) if norm in ("both", "q") else None
    wk = (1 + 0.3 * torch.randn(dim, generator=g)).to(dt) if norm in ("both", "k") else None
    cos = sin = None
    if rot:
        ang = torch.arange(int(length.max()) + 1)[:, None].double() * 1e4 ** (-torch.arange(0, rot, 2).double() / rot)
        cos, sin = ang.cos().float(), ang.sin().float()
    c = lambda x: None if x is None else x.cuda()  # noqa: E731
    d = c(qkv)
    q, k, v = d[:, :hq], d[:, hq:hq + hk], d[:, hq + hk:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    kp, vp = c(k0), c(v0)
    q_out = q if in_place else torch.full((T, hq, dim), 9.0, dtype=dt, device="cuda")
    e.kv_append(pk.KVPages(kp, vp), layer, (c(torch.from_numpy(off)), c(torch.from_numpy(page)), c(torch.from_numpy(length))),
                c(torch.from_numpy(q_off)), q, k, v, q_out, q_norm=c(wq), k_norm=c(wk), eps=1e-5, cos=c(cos), sin=c(sin),
                interleaved=interleaved)
    e.sync()
    u, tiny = ULP[dtype], 2.0 ** -25 if dtype == "f16" else 0.0
    wkp, wvp = k0.double(), v0.clone()
    ktol = torch.zeros_like(wkp)
    want, qtol = torch.zeros((T, hq, dim), dtype=torch.float64), torch.zeros((T, hq, dim), dtype=torch.float64)
    for s in range(len(seqs)):
        t0, t1 = int(q_off[s]), int(q_off[s + 1])
        for t in range(t0, t1):
            p = int(length[s]) - (t1 - t0) + (t - t0)
            if p < 0:
                continue
            pos = torch.tensor([p])
            y, size = turned(qkv[t:t + 1, :hq], wq, 1e-5, cos, sin, pos, interleaved)
            want[t], qtol[t] = y[0], (u * y.abs() + 2.0 ** -17 * size + tiny)[0]
            y, size = turned(qkv[t:t + 1, hq:hq + hk], wk, 1e-5, cos, sin, pos, interleaved)
            at = int(page[off[s] + p // B])
            wkp[layer, at, :, p % B] = y[0]
            ktol[layer, at, :, p % B] = (u * y.abs() + 2.0 ** -17 * size + tiny)[0]
            wvp[layer, at, :, p % B] = qkv[t, hq + hk:]
    assert bool(((q_out.cpu().double() - want).abs() <= qtol).all()), "q"
    assert bool(((kp.cpu().double() - wkp).abs() <= ktol).all()), "k"
    assert torch.equal(vp.cpu(), wvp), "v"


def _say(*a):
    print("[case]", *a, flush=True)


MIXED = ((1, 0), (1, 15), (5, 14), (33, 0), (1, 200), (17, 100))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_and_sizes(dtype, dim, interleaved):
    _say(dtype, dim, interleaved)
    case(dtype, dim, seqs=MIXED, interleaved=interleaved, seed=dim)
    case(dtype, dim, seqs=MIXED, interleaved=interleaved, rot=32, seed=dim + 1)


@pytest.mark.parametrize("norm", ["both", "q", "k", "none"])
@pytest.mark.parametrize("rot", [0, 16, 48, 112, 128])
def test_norms_and_rotations(norm, rot):
    _say(norm, rot)
    case(norm=norm, rot=rot, seqs=MIXED, seed=rot)
    case(norm=norm, rot=rot, seqs=MIXED, interleaved=True, seed=rot)


@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (7, 1), (14, 2), (33, 3), (64, 8)])
@pytest.mark.parametrize("block", [4, 16, 64])
def test_heads_and_blocks(heads, block):
    _say(heads, block)
    case(heads=heads, block=block, dim=64, seqs=MIXED, seed=heads[0])


def test_in_place_layers_and_rows():
    """Queries rotated where they are, the second of three layers, rows that are tensors of their own."""
    case(in_place=True, layers=3, layer=1, seqs=MIXED)
    case(packed=False, seqs=MIXED)


def test_idle_places():
    """Length 0 or fewer tokens than are new: rows of zeros, and no page written; sequences without new tokens."""
    case(seqs=((1, 0), (1, 0), (0, 9), (4, 0), (0, 0), (2, 7)), lens=[0, 1, 9, 2, 0, 9])
    case(seqs=((1, 0),), lens=[0])


def test_many_tokens():
    case(heads=(4, 1), dim=64, seqs=tuple((1 + i % 40, i % 77) for i in range(150)), seed=4)


def test_small_and_large_values():
    """A row of zeros stays one; rows far from one in size are normed as the others."""
    pk, e = engine(16)
    x = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    x[1] = 1e20
    x[2, :, 0] = 1e-18
    kp, vp = (torch.zeros((1, 2, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i64 = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    q = torch.empty((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    e.kv_append(pk.KVPages(kp, vp), 0, (i64([0, 1]), torch.tensor([1], dtype=torch.int32, device="cuda"), i64([3])),
                i64([0, 3]), x[:, :2], x[:, 2:3], x[:, 3:], q, q_norm=w, k_norm=w, eps=1e-6)
    e.sync()
    assert not bool(q[0].any()) and not bool(kp[0, 1, 0, 0].any())
    # 1e20 squared is past 32 bits: the root's reciprocal is zero
    assert not bool(q[1].isnan().any())
    assert bool(((q[2, :, 0].double() - 1e-15).abs() <= 2.0 ** -7 * 1e-15).all())


def test_malformed_input_is_reported():
    """A page out of range, a position past the rotation's tables or a table too short: the token has a row of zeros, writes
    nothing, and sync reports it; others are as they should be."""
    pk, e = engine(16)
    i64 = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    i32 = lambda v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    x = torch.randn((3, 4, 64), device="cuda").half()
    cos, sin = (torch.randn((40, 32), device="cuda") for _ in range(2))

    def attempt(off=(0, 2, 3), page=(1, 2, 3), length=(20, 3), q_off=(0, 1, 3), rows=40, good=(1, 2)):
        kp, vp = (torch.zeros((1, 5, 1, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2))
        q = torch.full((3, 2, 64), 9.0, dtype=torch.float16, device="cuda")
        e.kv_append(pk.KVPages(kp, vp), 0, (i64(off), i32(page), i64(length)), i64(q_off), x[:, :2], x[:, 2:3], x[:, 3:], q,
                    cos=cos[:rows].contiguous(), sin=sin[:rows].contiguous())
        with pytest.raises(pk.DMError) as err:
            e.sync()
        assert err.value.status == pk.DM_EINVAL
        written = vp[0, :, 0].any(-1).sum().item()
        assert written == len(good)
        for t in range(3):
            if t in good:
                assert bool((vp[0, :, 0] == x[t, 3]).all(-1).any()) and bool((q[t] != 0).any())

    attempt(page=(1, 5, 3))
    attempt(page=(1, -1, 3))
    attempt(rows=19)
    attempt(length=(33, 3))
    attempt(length=(-1, 3))
    attempt(off=(0, 4, 3), good=())
    attempt(q_off=(0, 1, 4), good=(0,))


def test_refusals():
    pk, e = engine(16)
    i64 = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    kv = pk.KVPages(*(torch.zeros((2, 5, 1, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2)))
    tb = (i64([0, 1]), torch.tensor([1], device="cuda", dtype=torch.int32), i64([3]))
    x = torch.zeros((3, 4, 64), dtype=torch.float16, device="cuda")
    q = torch.empty((3, 2, 64), dtype=torch.float16, device="cuda")
    cs = torch.zeros((9, 20), device="cuda")

    def go(layer=0, q_in=x[:, :2], k=x[:, 2:3], out=q, **kw):
        e.kv_append(kv, layer, tb, i64([0, 3]), q_in, k, x[:, 3:], out, **kw)

    go()
    e.sync()
    for kw, what in ((dict(layer=2), "layer"), (dict(cos=cs, sin=cs), "rot_dim"), (dict(eps=-1.0), "eps"),
                     (dict(eps=float("nan")), "eps")):
        with pytest.raises(pk.DMError, match=what):
            go(**kw)
    odd = torch.zeros((3, 260), dtype=torch.float16, device="cuda")
    with pytest.raises(pk.DMError, match="strides"):
        go(q_in=odd[:, :128].unflatten(1, (2, 64))[:, :, :], out=torch.zeros((3, 132), dtype=torch.float16, device="cuda")[
            :, :128].unflatten(1, (2, 64)))
    for kw in (dict(out=q[:2]), dict(k=x[:, 1:3]), dict(q_in=x[:, :2].float()), dict(q_norm=torch.ones(3, device="cuda")),
               dict(q_in=x.transpose(1, 2)[:, :2]), dict(cos=cs)):
        with pytest.raises((ValueError, AttributeError)):
            go(**kw)
    # no token, no sequence: nothing to do
    e.kv_append(kv, 0, (i64([0]), tb[1], i64([3])[:0]), i64([0]), x[:0, :2], x[:0, 2:3], x[:0, 3:], q[:0])
    e.sync()
