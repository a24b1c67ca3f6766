"""What appending does to values that are not finite, and arguments that it refuses."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_append import DT, engine  # noqa: E402


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,rot", [(64, 0), (64, 16), (128, 32), (128, 64), (256, 240)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_elements_past_the_rotation_pass_as_they_are(interleaved, dim, rot, dtype, what):
    """Without a norm they are the input's bits, whatever their neighbours hold."""
    pk, e = engine(16)
    print("[case] past the rotation", interleaved, dim, rot, dtype, what, flush=True)
    T, hq, hk, dt = 21, 5, 3, DT[dtype]
    g = torch.Generator().manual_seed(rot)
    qkv = torch.randn((T, hq + 2 * hk, dim), generator=g).to(dt)
    for t in range(T):
        qkv[t, :, rot + t % (dim - rot)] = what
    qkv = qkv.cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    kp, vp = (torch.zeros((1, 2, hk, 16, dim), dtype=dt, device="cuda") for _ in range(2))
    i64 = dict(dtype=torch.int64, device="cuda")
    tables = (torch.tensor([0, 2], **i64), torch.tensor([1, 0], dtype=torch.int32, device="cuda"), torch.tensor([T], **i64))
    cos = sin = None
    if rot:
        a = torch.arange(T)[:, None] * 100.0 ** -(torch.arange(rot // 2) / rot)
        cos, sin = a.cos().cuda(), a.sin().cuda()
    out = torch.zeros((T, hq, dim), dtype=dt, device="cuda")
    e.kv_append(pk.KVPages(kp, vp), 0, tables, torch.tensor([0, T], **i64), q, k, v, out, cos=cos, sin=sin,
                interleaved=interleaved)
    e.sync()
    got_k = torch.cat([kp[0, 1].transpose(0, 1), kp[0, 0].transpose(0, 1)])[:T]
    for got, given in ((out, q), (got_k, k)):
        assert torch.equal(got[..., rot:].isnan(), given[..., rot:].isnan())
        assert torch.equal(got[..., rot:].nan_to_num(7, 8, 9), given[..., rot:].nan_to_num(7, 8, 9))
        assert bool(got[..., :rot].isfinite().all())


def test_norms_without_weights_are_refused():
    """Weights of no elements are not the absence of a norm."""
    pk, e = engine(16)
    kp, vp = (torch.zeros((1, 1, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i64 = dict(dtype=torch.int64, device="cuda")
    tables = (torch.tensor([0, 1], **i64), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([1], **i64))
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    for name in ("q_norm", "k_norm"):
        for size in (0, 63, 128):
            with pytest.raises(ValueError, match="head_dim"):
                e.kv_append(pk.KVPages(kp, vp), 0, tables, torch.tensor([0, 1], **i64), q, q, q, q,
                            **{name: torch.ones(size, dtype=torch.bfloat16, device="cuda")})
    e.sync()
