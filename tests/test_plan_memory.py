"""The plan of one batch given to attention over another: reported, nothing written, and nothing read outside it."""
import pytest


def test_every_plan_holds_what_is_read_before_its_head_is_known():
    """A call reads the item counts of up to 512 units beside the head: every plan has a head of 64 bytes and room for
    as many, whatever batch it was made for."""
    import paper_2602_06502_amd as pk
    size = pk.load_library().dm_attn_plan_bytes
    for n, groups in ((0, 0), (1, 0), (1, 1), (2, 0), (37, 5), (511, 0), (512, 0), (513, 0), (513, 513), (100_000, 77)):
        units = n + groups
        assert size(n, groups) >= 64 + 4 * max(units, 512) + 64 * units
    assert size(1, 2) == 0 and size(2 ** 31, 0) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,other", [(3, 2), (300, 1), (512, 2), (700, 3)])
def test_plan_of_a_smaller_batch(n, other):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from test_gpu_attn import Batch, engine
    pk, e = engine(16)
    mine = Batch(16, [(1, 20 + i % 50) for i in range(n)], heads=(4, 2), dim=64, seed=20)
    theirs = Batch(16, [(1, 20 + i) for i in range(other)], heads=(4, 2), dim=64, seed=20)
    kv = pk.KVPages(mine.k.cuda(), mine.v.cuda())
    q = mine.qrows.cuda().unflatten(1, (4, 64))
    out = torch.zeros((n, 4, 64), dtype=torch.bfloat16, device="cuda")
    plan = e.attn_plan(kv, mine.tables(), mine.dev(mine.q_off), n, 4)
    short = e.attn_plan(kv, theirs.tables(), theirs.dev(theirs.q_off), other, 4)
    e.sync()
    assert short.buf.numel() == e.lib.dm_attn_plan_bytes(other, 0) < plan.buf.numel()
    own, plan.buf = plan.buf, short.buf
    print("[case] plan of", other, "for", n, flush=True)
    e.attn(plan, 0, q, 0.125, out)
    with pytest.raises(pk.DMError) as x:
        e.sync()
    assert x.value.status == pk.DM_EINVAL and not bool(out.any())
    plan.buf = own
    e.attn(plan, 0, q, 0.125, out)
    e.sync()
    ref, _, tol, _ = mine.reference(0.125)
    assert bool(((out.cpu().double() - ref).abs() <= tol).all())
