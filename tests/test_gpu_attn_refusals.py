"""Batches that attention refuses on the device: reported, and not a row written."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import engine  # noqa: E402


def test_tokens_out_of_order_write_nothing():
    """q_off goes back and forth, so that the sequences together have far more rows than the batch has tokens; the last
    one, in order, is long enough to be cut into parts."""
    pk, e = engine(16)
    n, T, L = 2001, 1280, 8000
    pages = 1 + L // 16
    k = torch.randn((1, pages, 1, 16, 64), device="cuda").bfloat16()
    kv = pk.KVPages(k, torch.randn_like(k))
    q_off = np.array([0, T] * (n // 2) + [T, T + 1])
    assert len(q_off) == n + 1
    off = np.array(list(range(n)) + [n - 1 + L // 16])
    page = np.array([0] * (n - 1) + list(range(1, pages)), np.int32)
    length = np.array([16] * (n - 1) + [L])
    dev = lambda x, t=torch.int64: torch.from_numpy(np.asarray(x)).to(t).cuda()  # noqa: E731
    q = torch.randn((T + 1, 1, 64), device="cuda").bfloat16()
    out, lse = torch.full_like(q, 7), torch.full((T + 1, 1), 7.0, device="cuda")
    tables = (dev(off), dev(page, torch.int32), dev(length))
    print("[case] tokens out of order", flush=True)
    e.attn(e.attn_plan(kv, tables, dev(q_off), T + 1, 1), 0, q, 0.125, out, lse)
    with pytest.raises(pk.DMError) as x:
        e.sync()
    assert x.value.status == pk.DM_EINVAL
    assert bool((out == 7).all()) and bool((lse == 7).all())


@pytest.mark.parametrize("tokens", [-1, 2 ** 31, 2 ** 64])
def test_token_counts_out_of_range_are_refused(tokens):
    pk, e = engine(16)
    k = torch.zeros((1, 1, 1, 16, 64), device="cuda").bfloat16()
    i64 = dict(dtype=torch.int64, device="cuda")
    tables = (torch.tensor([0, 1], **i64), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([1], **i64))
    with pytest.raises(ValueError, match="q_tokens"):
        e.attn_plan(pk.KVPages(k, k.clone()), tables, torch.tensor([0, 1], **i64), tokens, 1)
    e.sync()
