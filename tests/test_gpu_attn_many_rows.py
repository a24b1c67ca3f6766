"""More rows than attention's work area has parts for: neither shared nor cut, and right."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import ULP, engine  # noqa: E402


@pytest.mark.parametrize("n,shares", [(8000, True), (9400, False)])
def test_next_tokens_of_thousands_of_sequences_on_one_prefix(n, shares):
    """64 query heads: twice 9,400 * 64 rows are more than 2^20 and the cut ones, twice 8,000 * 64 fewer."""
    pk, e = engine(16)
    print("[case] many rows", n, flush=True)
    H, G, D, P = 8, 8, 64, 8  # KV heads, query heads of each, pages of the prefix
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn((1, P + n, H, 16, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = (2 * torch.randn((n, H * G, D), generator=g, device="cuda")).bfloat16()
    i64 = dict(dtype=torch.int64, device="cuda")
    s = torch.arange(n, **i64)
    own = 1 + s % 16
    page = torch.cat([torch.arange(P, **i64).expand(n, P), P + s[:, None]], 1).int().reshape(-1).contiguous()
    tables = ((P + 1) * torch.arange(n + 1, **i64), page, 16 * P + own)
    out, lse = torch.empty_like(q), torch.empty((n, H * G), device="cuda")
    kv = pk.KVPages(k, v)
    plan = e.attn_plan(kv, tables, torch.arange(n + 1, **i64), n, H * G, groups=torch.tensor([0, n], **i64))
    e.attn(plan, 0, q, D ** -0.5, out, lse)
    e.sync()
    assert (int(plan.buf[36:40].view(torch.int32)) > 0) == shares  # rows of parts, in the plan's head
    u = ULP["bf16"]
    for h in range(H):
        x = q[:, h * G:(h + 1) * G].double()
        kp, vp = (y[0, :P, h].reshape(-1, D).double() for y in (k, v))
        ko, vo = (y[0, P:, h].double() for y in (k, v))
        sc = torch.cat([x @ kp.T, torch.matmul(x, ko.transpose(1, 2).contiguous())], -1) * D ** -0.5
        hidden = torch.arange(16, device="cuda")[None] >= own[:, None]
        sc[..., 16 * P:].masked_fill_(hidden[:, None], -math.inf)
        w = torch.softmax(sc, -1)
        want = w[..., :16 * P] @ vp + torch.matmul(w[..., 16 * P:], vo)
        mean = w[..., :16 * P] @ vp.abs() + torch.matmul(w[..., 16 * P:], vo.abs())
        tol = u * (want.abs() + mean) * 1.02 + 2.0 ** -20 * mean
        err = (out[:, h * G:(h + 1) * G].double() - want).abs()
        assert bool((err <= tol).all()), (h, float((err / tol).max()))
        far = torch.logsumexp(sc, -1)
        seen = sc.masked_fill(sc == -math.inf, 0).abs().amax(-1)
        assert bool(((lse[:, h * G:(h + 1) * G].double() - far).abs() <= 2.0 ** -18 * (seen + far.abs() + 1)).all())
