"""A captured step, replayed after calls that outgrow the context's work area: equal bits to the eager result."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_attn import Batch  # noqa: E402
from test_gpu_pages import csr, dev, make, plain_fork  # noqa: E402


def test_replays_after_larger_calls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_06502_amd as pk
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    small = Batch(16, [(1, 3000), (1, 40), (2, 900), (1, 5000)], heads=(8, 2), dim=64, seed=3)
    large = Batch(16, [(200, 200), (3000, 3000)], heads=(32, 8), dim=128, seed=4)

    def given(b):
        T = int(b.q_off[-1])
        q = b.qrows.cuda().unflatten(1, (b.hq, b.dim)).contiguous()
        return (pk.KVPages(b.k.cuda(), b.v.cuda()), b.tables(), b.dev(b.q_off), T, b.hq), q, torch.zeros_like(q)

    def call(args, q, out):
        kv, t, q_off, T, hq = args
        e.attn(e.attn_plan(kv, t, q_off, T, hq), 0, q, q.shape[-1] ** -0.5, out)

    # a fork of the large form
    r = np.random.default_rng(9)
    n, pages = 1500, 30_000
    tables, lens, ref = make(r, 16, n, pages - 4000, 12)
    ref = np.concatenate([ref, np.zeros(4000, np.int64)])
    off, page = csr(tables)
    t = (dev(off, np.int64), dev(page, np.int32), dev(lens, np.int64))
    fork = (dev(ref, np.int32), dev(np.arange(n), np.int32), dev(lens, np.int64), dev(np.full(n, 9), np.int64))
    want = plain_fork(16, tables, lens, ref, list(range(n)), lens, [9] * n)
    made = e.alloc_pages_out(pages, n, len(csr(want[0])[1]))

    mine, q, out = given(small)
    more, big_q, big_out = given(large)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call(mine, q, out)
    st.synchronize()
    eager = out.clone()
    print("[case] capture", flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call(mine, q, out)
    for k in range(4):
        print("[case] replay", k, flush=True)
        with torch.cuda.stream(st):
            if k != 2:
                call(more, big_q, big_out)
            if k >= 1:
                e.pages_fork_into(t, *fork, made)
        # what is free by now is taken, and written
        other = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(32)]
        out.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))
        assert all(bool((x == 3).all()) for x in other)
        if k >= 1:
            assert made["page"].tolist() == csr(want[0])[1].tolist()
    e.sync()
    ref_out, _, tol, _ = small.reference()
    assert bool(((eager.cpu().double() - ref_out).abs() <= tol).all())
    e.close()


def test_growth_under_capture_is_refused():
    """The call fails, the capture goes on with what it has and replays."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_06502_amd as pk
    st = torch.cuda.Stream()
    e = pk.DualMap(dict(block=16, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4), stream=st)
    b = Batch(16, [(1, 3000), (2, 900)], heads=(8, 2), dim=64, seed=3)
    q = b.qrows.cuda().unflatten(1, (8, 64)).contiguous()
    out, x = torch.zeros_like(q), torch.zeros(4, device="cuda")
    kv, t, q_off = pk.KVPages(b.k.cuda(), b.v.cuda()), b.tables(), b.dev(b.q_off)
    plan = e.attn_plan(kv, t, q_off, 3, 8)
    e.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        x.add_(1)
        with pytest.raises(pk.DMError, match="capture"):
            e.attn(plan, 0, q, 0.125, out)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert x.tolist() == [k + 1.0] * 4
    e.attn(plan, 0, q, 0.125, out)
    e.sync()
    ref, _, tol, _ = b.reference(0.125)
    assert bool(((out.cpu().double() - ref).abs() <= tol).all())
    e.close()
