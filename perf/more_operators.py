"""Measured cases of differential attention over KV pages and of eviction from them by attention weight.

Differential attention: a pair of query heads reads a pair of KV heads, its two softmax maps are subtracted with a learned
factor and meet the values of both heads side by side.  Eviction: the weight that every cached key has collected, summed
over the queries that saw it; the choice of the tokens that a sequence keeps within a budget; their keys, values and weights
moved to fresh pages.

Sizes are those of the repository's workloads: chat (pages of 16 tokens, histories up to 8,192 tokens, turns of 64 to
512), agent (pages of 32 tokens, system prompts of 2,048 to 8,192 tokens, tails of 128 to 1,024), tiny (256 to 768).
"""
import functools
import math
import random
import zlib

import numpy as np
import torch

DEV = "cuda:0"
own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
GAIN = 0.2  # what a differential layer's normed output is scaled by


def listed():
    return [
        # One conversation's next token in a model of differential layers: the smallest attention call.
        dict(name="diff_one", kind="diff", seqs=1, groups=0, plo=0, phi=0, tlo=256, thi=768, lo=1, hi=1, idle=0, q_heads=16,
             kv_heads=4, dim=64, block=16, norm=True, dtype="bf16"),
        # Next tokens of 64 conversations that share nothing.
        dict(name="diff_chat", kind="diff", seqs=64, groups=0, plo=0, phi=0, tlo=64, thi=8192, lo=1, hi=1, idle=0, q_heads=32,
             kv_heads=8, dim=128, block=16, norm=True, dtype="bf16"),
        # Agent tails behind cached system prompts: a chunk of new tokens each, no norm.
        dict(name="diff_tails", kind="diff", seqs=8, groups=2, plo=2048, phi=8192, tlo=0, thi=0, lo=128, hi=1024, idle=0,
             q_heads=32, kv_heads=8, dim=64, block=32, norm=False, dtype="f16"),
        # Two long prompts with nothing cached: the most work.
        dict(name="diff_prompts", kind="diff", seqs=2, groups=0, plo=0, phi=0, tlo=0, thi=0, lo=7000, hi=8192, idle=0,
             q_heads=32, kv_heads=8, dim=128, block=16, norm=True, dtype="bf16"),
        # The keys' weights after one conversation's next token: the smallest call.
        dict(name="weights_one", kind="weights", seqs=1, groups=0, plo=0, phi=0, tlo=256, thi=768, lo=1, hi=1, idle=0, q_heads=32,
             kv_heads=8, dim=128, block=16, paired=False, last=0, prev=True, dtype="bf16"),
        # After a decode step of 64 conversations, what was collected before carried along.
        dict(name="weights_chat", kind="weights", seqs=64, groups=0, plo=0, phi=0, tlo=64, thi=8192, lo=1, hi=1, idle=0,
             q_heads=32, kv_heads=8, dim=128, block=16, paired=False, last=0, prev=True, dtype="bf16"),
        # After a decode step of 128 agents on 8 system prompts, differential layers.
        dict(name="weights_agent", kind="weights", seqs=128, groups=8, plo=2048, phi=8192, tlo=128, thi=1024, lo=1, hi=1, idle=0,
             q_heads=32, kv_heads=8, dim=64, block=32, paired=True, last=0, prev=True, dtype="f16"),
        # After two long prompts, every query counted: the most work.
        dict(name="weights_prompts", kind="weights", seqs=2, groups=0, plo=0, phi=0, tlo=0, thi=0, lo=7000, hi=8192, idle=0,
             q_heads=32, kv_heads=8, dim=128, block=16, paired=False, last=0, prev=False, dtype="bf16"),
        # Chat histories brought back to some 1,000 tokens, every KV head on its own.
        dict(name="select_chat", kind="select", seqs=16, llo=512, lhi=8192, budget=1024, layers=4, kv_heads=8, share=1, sink=4,
             recent=128, block=16),
        # A few long documents, pairs of heads together.
        dict(name="select_long", kind="select", seqs=4, llo=16_384, lhi=131_072, budget=8192, layers=8, kv_heads=8, share=2,
             sink=4, recent=512, block=32),
        # A small instance's histories moved to their new pages, one of them within its budget.
        dict(name="gather_chat", kind="gather", seqs=4, llo=200, lhi=768, budget=256, layers=2, kv_heads=2, share=1, dim=64,
             block=16, dtype="bf16"),
        # Sixteen long histories, all layers.
        dict(name="gather_pool", kind="gather", seqs=16, llo=2048, lhi=8192, budget=2048, layers=4, kv_heads=8, share=1, dim=128,
             block=16, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["diff", "diff", "diff", "weights", "weights", "weights", "select", "gather"])
    block = rng.choice([4, 8, 16, 16, 32, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    c = dict(kind=kind, block=block)
    if kind in ("select", "gather"):
        kv_heads = rng.choice([1, 2, 4, 6, 8])
        share = rng.choice([s for s in (1, 1, 2, 3, kv_heads) if kv_heads % s == 0])
        top = _log(rng, 24, 65_536 if kind == "select" else 6_000)
        layers, seqs = rng.randrange(1, 5), _log(rng, 1, 32)
        while top * seqs * layers * kv_heads > (3_000_000 if kind == "select" else 1_200_000):
            layers, seqs, top = max(1, layers - 1), max(1, seqs * 3 // 4), max(24, top * 7 // 8)
        c.update(seqs=seqs, llo=rng.choice([1, top // 2]), lhi=top, budget=max(1, int(top * rng.uniform(0.05, 0.9))),
                 layers=layers, kv_heads=kv_heads, share=share)
        if kind == "select":
            c.update(sink=rng.choice([0, 1, 4, 33]), recent=rng.choice([0, 1, 64, 500]))
        else:
            c.update(dim=rng.choice([64, 128, 128, 256]), dtype=dtype)
        return c
    kv_heads = rng.choice([2, 2, 4, 8])
    c.update(kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 2, 3, 4, 7, 8]), idle=0, dtype=dtype)
    if kind == "diff":
        c.update(dim=rng.choice([64, 128]), norm=rng.random() < 0.6)
    else:
        paired = rng.random() < 0.4
        c.update(dim=rng.choice([64, 128] if paired else [64, 128, 128, 256]), paired=paired, last=rng.choice([0, 0, 0, 1, 32]),
                 prev=rng.random() < 0.7)
        if not paired and rng.random() < 0.2:
            c.update(kv_heads=1, q_heads=c["q_heads"] // kv_heads)
    form = rng.choice(["decode", "decode", "drafts", "prompt", "long"])
    if form == "long":
        c.update(seqs=rng.randrange(1, 4), groups=0, plo=0, phi=0, tlo=8192, thi=_log(rng, 16_384, 131_072), lo=1,
                 hi=rng.choice([1, 1, 5]))
    elif form == "prompt":
        hi = _log(rng, 24, 2048)
        c.update(seqs=max(1, min(_log(rng, 1, 64), 6000 // hi)), groups=rng.choice([0, 1, 2]), plo=0, phi=_log(rng, 64, 8192),
                 tlo=0, thi=rng.choice([0, 0, 500]), lo=rng.choice([1, hi // 2]), hi=hi)
    else:
        seqs = _log(rng, 1, 128)
        c.update(seqs=seqs, groups=rng.choice([0, 1, _log(rng, 1, 16)]), plo=0, phi=_log(rng, 64, 8192), tlo=0,
                 thi=_log(rng, 16, 8192 if seqs <= 64 else 1024), lo=1, hi=1 if form == "decode" else rng.randrange(2, 9),
                 idle=rng.choice([0, 0, 1, 3]))
    if c["groups"] == 0:
        c.update(plo=0, phi=0)
    # the plain form's rows of scores and its gathered keys stay below those of the largest listed cases
    while _span(c) * c["seqs"] * max(c["kv_heads"] * c["dim"], c["q_heads"] * c["hi"]) > 2_400_000_000 and c["seqs"] > 1:
        c["seqs"] = max(1, c["seqs"] * 3 // 4)
    return c


def _span(c):
    """Most tokens that a sequence of an attention case can hold, in whole pages."""
    B = c["block"]
    return (-(-c["phi"] // B) + -(-(c["thi"] + c["hi"]) // B)) * B


# ---------------------------------------------------------------------------
# Inputs.  Lengths go by the case, so that sizes do not depend on the seed; their order, every page's place and all values
# go by the seed.
# ---------------------------------------------------------------------------


def _lens(r, n, lo, hi):
    return r.integers(lo, hi + 1, size=n).astype(np.int64)


def _starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)


def _layout(c, seed):
    """Host arrays of a case."""
    r0 = np.random.default_rng(zlib.crc32(repr(sorted((k, v) for k, v in c.items() if k != "name")).encode()))
    r = np.random.default_rng([seed, 78])
    return (_layout_attn if c["kind"] in ("diff", "weights") else _layout_evict)(c, r0, r)


def _layout_attn(c, r0, r):
    B, n, G = c["block"], c["seqs"], c["groups"]
    new = _lens(r0, n, c["lo"], c["hi"])
    tail = _lens(r0, n, c["tlo"], c["thi"]) + new
    order = r.permutation(n)
    new, tail = new[order], tail[order]
    if G:
        G = min(G, n)
        prefix = _lens(r0, G, c["plo"], c["phi"]) // B
        share = 1.0 / np.arange(1, G + 1)  # few prompts have most of the sequences
        group = np.sort(np.concatenate([np.arange(G), r0.choice(G, size=n - G, p=share / share.sum())]))
        grp = np.concatenate([np.searchsorted(group, np.arange(G)), [n]]).astype(np.int64)
        pre = prefix[group]
    else:
        prefix, group, grp, pre = np.zeros(0, np.int64), np.full(n, -1), None, np.zeros(n, np.int64)
    length = pre * B + tail
    pages = -(-tail // B)
    total = int(prefix.sum() + pages.sum())
    ids = r.permutation(total + 3)[:total].astype(np.int32)
    p0, t0 = _starts(prefix), prefix.sum() + _starts(pages)
    rows = []
    for s in range(n):
        if group[s] >= 0:
            rows.append(ids[p0[group[s]]:p0[group[s] + 1]])
        rows.append(ids[t0[s]:t0[s + 1]])
    if c["idle"]:  # places of a fixed batch with no sequence in them: a query and no key
        length[r.permutation(n)[:min(c["idle"], n - 1)]] = 0
    h = dict(off=_starts(pre + pages), page=np.concatenate(rows).astype(np.int32), len=length, n_pages=total + 3,
             q_off=_starts(new), grp=grp)
    if c["kind"] == "weights" and c["prev"]:
        # the last step's tables: the same sequences in another order, without the new tokens
        src = r.permutation(n)
        before = np.empty(n, np.int64)
        before[src] = np.maximum(length - new, 0)
        h.update(src=src.astype(np.int32), keep=np.maximum(length - new, 0), prev_off=_starts(-(-before // B)))
    return h


def _layout_evict(c, r0, r):
    B, n = c["block"], c["seqs"]
    length, budget = _lens(r0, n, c["llo"], c["lhi"]), _lens(r0, n, max(1, c["budget"] // 2), c["budget"])
    length[0] = max(length[0], budget[0] + 1)  # one at the least is past its budget
    room, order = _lens(r0, n, 0, 9), r.permutation(n)
    length, budget, room = length[order], budget[order], room[order]
    past = length > budget
    pages = -(-length // B)
    h = dict(off=_starts(pages), len=length, budget=budget, room=room)
    if c["kind"] == "select":
        h["page"] = r.permutation(int(pages.sum())).astype(np.int32)
        return h
    # the next step's tables: fresh pages for the sequences past their budgets
    to_len = np.where(past, budget, length) + room
    to_pages = -(-to_len // B)
    fresh = np.where(past, to_pages, np.maximum(to_pages - pages, 0))
    total = int(pages.sum() + fresh.sum())
    ids = r.permutation(total + 3)[:total].astype(np.int32)
    a, b = _starts(pages), pages.sum() + _starts(fresh)
    h["page"] = ids[:int(pages.sum())]
    rows = []
    for s in range(n):
        if not past[s]:
            rows.append(ids[a[s]:a[s + 1]])
        rows.append(ids[b[s]:b[s + 1]])
    h.update(to_off=_starts(to_pages), to_page=np.concatenate(rows).astype(np.int32), to_len=to_len, n_pages=total + 3,
             past=past)
    return h


def _randn(g, dtype, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype) if math.prod(shape) < 1 << 28 else \
        torch.empty(*shape, device=DEV, dtype=dtype).normal_(generator=g)


def _collected(g, *shape):
    """Weights that keys may have collected: spread over several powers of ten, some keys never looked at."""
    w = torch.exp(3 * torch.randn(*shape, generator=g, device=DEV) - 6)
    return torch.where(torch.rand(*shape, generator=g, device=DEV) < 0.05, 0.0, w)


@functools.lru_cache(maxsize=None)
def _engine(block):
    """The context that a serving program keeps, one for a page size."""
    from paper_2602_06502_amd import DualMap
    return DualMap(dict(block=block, key_blocks=1, seeds=(1, 2), vnodes=1, max_slots=1, index_log2_slots=4))


def _data(c, h, seed):
    """Tensors of a case from its host arrays."""
    g = torch.Generator(device=DEV).manual_seed(seed * 1000 + 17)
    s = {k: torch.from_numpy(v).to(DEV) for k, v in h.items() if isinstance(v, np.ndarray)}
    H, B = c["kv_heads"], c["block"]
    if c["kind"] in ("select", "gather"):
        s["w"] = _collected(g, c["layers"], H, len(h["page"]) * B)
    if c["kind"] == "select":
        return s
    dt, D = DTYPES[c["dtype"]], c["dim"]
    shape = (c.get("layers", 1), h["n_pages"], H, B, D)
    s["k"], s["v"] = _randn(g, dt, *shape), _randn(g, dt, *shape)
    if c["kind"] == "gather":
        s["kept"] = _some_kept(c, h, s, g)
        return s
    T = int(h["q_off"][-1])
    s["q"] = (2 * _randn(g, torch.float32, T, c["q_heads"], D)).to(dt)
    if c["kind"] == "diff":
        s["lam"] = 0.2 + 0.7 * torch.rand(c["q_heads"] // 2, generator=g, device=DEV)
        s["w"] = (1 + 0.1 * _randn(g, torch.float32, 2 * D)).to(dt) if c["norm"] else None
        return s
    s["lse"] = _far(c, h, s)
    if c["prev"]:
        s["prev"] = _collected(g, H, max(1, int(h["prev_off"][-1]) * B))
    return s


def _some_kept(c, h, s, g):
    """A choice of tokens for every layer and choosing head, in order of position; the list's layout is that of the tables."""
    C, n, top = c["kv_heads"] // c["share"], c["seqs"], int(h["len"].max())
    kept = torch.zeros(c["layers"], C, len(h["page"]) * c["block"], device=DEV, dtype=torch.int32)
    at = torch.arange(top, device=DEV)
    for layer in range(c["layers"]):
        x = torch.rand(C, n, top, generator=g, device=DEV)
        x = torch.where(at < s["len"][:, None], x, 2.0)  # (tokens that there are come first)
        order = torch.argsort(x, -1)
        order = torch.where(at < s["budget"][:, None], order, top)
        order = torch.sort(order, -1).values.int()
        for i in np.flatnonzero(h["past"]):
            a, b = int(h["off"][i]) * c["block"], int(h["budget"][i])
            kept[layer, :, a:a + b] = order[:, i, :b]
    return kept


def _key_heads(c, x):
    """Query heads as [..., KV heads, query heads of each]: in pairs, or one after another."""
    H, r = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    if c["kind"] == "diff" or c["paired"]:
        return x.unflatten(-1, (H // 2, r, 2)).transpose(-1, -2).flatten(-3, -2)
    return x.unflatten(-1, (H, r))


def _far(c, h, s):
    """The log-sum-exp that attention leaves for every query head, -infinity where it sees nothing."""
    out = torch.full(s["q"].shape[:2], -math.inf, device=DEV)
    heads = _key_heads(c, torch.arange(c["q_heads"], device=DEV))  # [H, r]
    for i in range(c["seqs"]):
        t0, t1, L = int(h["q_off"][i]), int(h["q_off"][i + 1]), int(h["len"][i])
        if L <= 0 or t1 == t0:
            continue
        at = s["page"][int(h["off"][i]):int(h["off"][i]) + -(-L // c["block"])].long()
        keys = s["k"][0][at].transpose(0, 1).flatten(1, 2)[:, :L].float()
        seen = L - (t1 - t0) + 1 + torch.arange(t1 - t0, device=DEV)
        later = torch.arange(L, device=DEV) >= seen[:, None]
        for g in range(c["kv_heads"]):
            x = (s["q"][t0:t1, heads[g]].float() @ keys[g].T.contiguous()) * c["dim"] ** -0.5
            out[t0:t1, heads[g]] = torch.logsumexp(x.masked_fill_(later[:, None], -math.inf), -1)
    return out


def prepare(case, seed):
    c, h = case, _layout(case, seed)
    s = _data(c, h, seed)
    s["case"] = c
    B, H = c["block"], c["kv_heads"]
    i32, i64 = dict(device=DEV, dtype=torch.int32), dict(device=DEV, dtype=torch.int64)
    if c["kind"] == "select":
        s["kept"] = torch.zeros(c["layers"], H // c["share"], len(h["page"]) * B, **i32)
        s["keep"], s["grow"] = torch.zeros(c["seqs"], **i64), torch.zeros(c["seqs"], **i64)
    if c["kind"] == "gather":
        s["w_to"] = torch.zeros(c["layers"], H, len(h["to_page"]) * B, device=DEV)
        s["most"] = int(np.where(h["past"], h["budget"], h["len"]).max())
    if c["kind"] in ("diff", "weights"):
        # lengths that the program knows on the host
        s["most_new"] = int((h["q_off"][1:] - h["q_off"][:-1]).max())
        s["most_pages"] = int((h["off"][1:] - h["off"][:-1]).max())
        s.setdefault("grp", None)
    if c["kind"] == "diff":
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:2], device=DEV)
    if c["kind"] == "weights":
        s["w"] = torch.zeros(H, len(h["page"]) * B, device=DEV)
    if own:
        from paper_2602_06502_amd import KVPages
        s["eng"] = e = _engine(B)
        s["tables"] = (s["off"], s["page"], s["len"])
        if "k" in s:
            s["kv"] = KVPages(s["k"], s["v"])
        if c["kind"] in ("diff", "weights"):  # one plan a step, for all layers and for both calls
            plan = e.diff_plan if c["kind"] == "diff" or c["paired"] else e.attn_plan
            s["plan"] = plan(s["kv"], s["tables"], s["q_off"], s["q"].shape[0], c["q_heads"], groups=s["grp"])
    return s


# ---------------------------------------------------------------------------
# One pass: the framework's calls, or the plain form.
# ---------------------------------------------------------------------------


def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _own_diff(s):
    c = s["case"]
    s["eng"].diff_attn(s["plan"], 0, s["q"], c["dim"] ** -0.5, s["lam"], s["out"], s["lse"], norm=s["w"], eps=EPS,
                       gain=GAIN if c["norm"] else 1.0)
    return {"out": s["out"], "lse": s["lse"]}


def _own_weights(s):
    c = s["case"]
    prev = (s["prev"], s["prev_off"], s["src"], s["keep"]) if c["prev"] else None
    s["eng"].attn_weights(s["plan"], 0, s["q"], c["dim"] ** -0.5, s["lse"], s["w"], last=c["last"], prev=prev,
                          decay=0.99 if c["prev"] else 1.0)
    return {"w": s["w"]}


def _own_select(s):
    c = s["case"]
    s["eng"].evict_select(s["tables"], s["w"], s["budget"], s["room"], s["kept"], s["keep"], s["grow"], sink=c["sink"],
                          recent=c["recent"], share=c["share"])
    return {"kept": s["kept"], "keep": s["keep"], "grow": s["grow"]}


def _own_gather(s):
    s["eng"].kv_gather(s["kv"], s["tables"], (s["to_off"], s["to_page"], s["to_len"]), s["budget"], s["kept"], s["w"], s["w_to"])
    return {"k": s["k"], "v": s["v"], "w": s["w_to"]}


def _scores(s):
    """Scores [n, H, new tokens * query heads, keys] with -infinity where a query does not see a key, the token of each
    row's place, and which rows there are."""
    c, T = s["case"], s["q"].shape[0]
    H, D, n = c["kv_heads"], c["dim"], c["seqs"]
    r = c["q_heads"] // H
    count = s["q_off"][1:] - s["q_off"][:-1]
    row = torch.arange(s["most_new"], device=DEV)
    tok = torch.where(row < count[:, None], s["q_off"][:-1, None] + row, T)
    q = _key_heads(c, s["q"][tok.clamp(max=T - 1)].float().transpose(-1, -2))  # [n, rows, D, H, r]
    q = q.permute(0, 3, 1, 4, 2).reshape(n, H, -1, D)
    x = torch.matmul(q, _gathered(s, s["k"]).transpose(-1, -2)) * D ** -0.5
    seen = (s["len"] - count)[:, None] + row + 1
    hidden = torch.arange(x.shape[-1], device=DEV) >= seen[..., None]
    x.masked_fill_(hidden.repeat_interleave(r, dim=1, output_size=seen.shape[1] * r)[:, None], -math.inf)
    return x, tok


def _gathered(s, x):  # [n, H, tokens, D] in 32 bits
    entry = s["off"][:-1, None] + torch.arange(s["most_pages"], device=DEV)
    at = s["page"][entry.clamp(max=s["page"].numel() - 1)].long()
    return x[0][at].permute(0, 2, 1, 3, 4).reshape(at.shape[0], x.shape[2], -1, x.shape[4]).float()


def _plain_diff(s):
    c, T = s["case"], s["q"].shape[0]
    H, D, n, P = c["kv_heads"], c["dim"], c["seqs"], c["q_heads"] // 2
    r = c["q_heads"] // H
    x, tok = _scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = torch.exp_(x.sub_(top))
    total = x.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    v = _gathered(s, s["v"])
    v = torch.cat([v[:, 0::2], v[:, 1::2]], -1)  # [n, H / 2, tokens, 2 D]
    total = torch.where(total == 0, 1.0, total)
    y = [torch.matmul(x[:, m::2], v) / total[:, m::2] for m in (0, 1)]
    y = [z.reshape(n, H // 2, -1, r, 2 * D).permute(0, 2, 1, 3, 4).reshape(n, -1, P, 2 * D) for z in y]
    y = y[0] - s["lam"][:, None] * y[1]
    if s["w"] is not None:
        y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) / (2 * D) + EPS) * s["w"].float() * GAIN
    out = torch.zeros(T + 1, P, 2 * D, device=DEV)
    out[tok] = y
    far = torch.zeros(T + 1, c["q_heads"], device=DEV)
    far[tok] = lse.reshape(n, H // 2, 2, -1, r).permute(0, 3, 1, 4, 2).reshape(n, -1, c["q_heads"])
    s["out"].copy_(out[:T].reshape(s["out"].shape))
    s["lse"].copy_(far[:T])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_weights(s):
    c, T = s["case"], s["q"].shape[0]
    B, H, n = c["block"], c["kv_heads"], c["seqs"]
    x, tok = _scores(s)
    far = _key_heads(c, s["lse"])[tok.clamp(max=T - 1)]  # [n, rows, H, r]
    counted = tok < T
    if c["last"]:
        counted = counted & (tok >= s["q_off"][1:, None] - c["last"])
    far = torch.where(counted[..., None, None] & (far != -math.inf), far, math.inf)
    x = torch.exp_(x.sub_(far.permute(0, 2, 1, 3).reshape(n, H, -1, 1))).sum(2)  # [n, H, keys]
    i = torch.arange(x.shape[-1], device=DEV)
    if c["prev"]:
        at = s["prev_off"][s["src"].long(), None] * B + i
        old = s["prev"][:, at.clamp(max=s["prev"].shape[1] - 1)].transpose(0, 1)
        x = x + torch.where(i < s["keep"][:, None], 1.0, 0.0)[:, None] * (0.99 * old)
    rows = s["w"].shape[1]
    to = torch.where(i < s["len"][:, None], s["off"][:-1, None] * B + i, rows)
    w = torch.cat([s["w"], s["w"][:, :1]], 1)
    w[:, to] = x.transpose(0, 1)
    s["w"].copy_(w[:, :rows])
    return {"w": s["w"]}


def _plain_select(s):
    c, n, B = s["case"], s["case"]["seqs"], s["case"]["block"]
    L, C = s["kept"].shape[:2]
    rows = s["w"].shape[2]
    most = max(c["lhi"], c["budget"] + 1)
    i = torch.arange(most, device=DEV)
    length, budget = s["len"], s["budget"]
    first = budget.clamp(max=c["sink"])
    tail = torch.minimum(budget - first, torch.full_like(budget, c["recent"]))
    must = (i < first[:, None]) | ((i >= (length - tail)[:, None]) & (i < length[:, None]))
    at = (s["off"][:-1, None] * B + i).clamp(max=rows - 1)
    for layer in range(L):
        heads = s["w"][layer].unflatten(0, (C, c["share"]))
        x = heads[:, 0]
        for k in range(1, c["share"]):
            x = x + heads[:, k]
        x = x[:, at]
        x = torch.where(must, math.inf, torch.where(i < length[:, None], x, -1.0))
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices
        order = torch.where(i < budget[:, None], order, most)
        order = torch.sort(order, -1).values.int()  # by position, what is not kept at the end
        here = (i < budget[:, None]) & (length > budget)[:, None]
        out = torch.cat([s["kept"][layer], s["kept"][layer][:, :1]], 1)
        out[:, torch.where(here, s["off"][:-1, None] * B + i, rows)] = order
        s["kept"][layer] = out[:, :rows]
    s["keep"].copy_(torch.where(length > budget, 0, length))
    s["grow"].copy_(s["room"] + torch.where(length > budget, budget, 0))
    return {"kept": s["kept"], "keep": s["keep"], "grow": s["grow"]}


def _plain_gather(s):
    c, B, H = s["case"], s["case"]["block"], s["case"]["kv_heads"]
    past = s["len"] > s["budget"]
    i = torch.arange(s["most"], device=DEV)
    there = i < torch.where(past, s["budget"], s["len"])[:, None]
    rows, to_rows = s["w"].shape[2], s["w_to"].shape[2]
    at = (s["off"][:-1, None] * B + i).clamp(max=rows - 1)
    to = s["to_off"][:-1, None] * B + i
    e = (to // B).clamp(max=s["to_page"].numel() - 1)
    spare = s["k"].shape[1]  # rows that nothing is moved to go past the store
    dst = torch.where(there & past[:, None], s["to_page"][e].long(), spare)
    head = torch.arange(H, device=DEV)[:, None, None]
    for layer in range(c["layers"]):
        kept = s["kept"][layer][:, at].repeat_interleave(c["share"], 0).long()
        kept = torch.where(past[:, None] & there, kept, torch.where(there, i, 0))  # [H, n, rows]
        page = s["page"][s["off"][:-1, None] + kept // B].long()
        for x in (s["k"], s["v"]):
            moved = x[layer][page, head, kept % B]
            y = torch.cat([x[layer], x[layer][:1]])
            y[dst.expand(H, -1, -1), head, (i % B).expand(H, dst.shape[0], -1)] = moved
            x[layer] = y[:spare]
        w = torch.cat([s["w_to"][layer], s["w_to"][layer][:, :1]], 1)
        w[:, torch.where(there, to, to_rows)] = torch.gather(s["w"][layer], 1, (s["off"][:-1, None] * B + kept).flatten(1)
                                                            ).unflatten(1, kept.shape[1:])
        s["w_to"][layer] = w[:, :to_rows]
    return {"k": s["k"], "v": s["v"], "w": s["w_to"]}


_own = {"diff": _own_diff, "weights": _own_weights, "select": _own_select, "gather": _own_gather}
_plain = {"diff": _plain_diff, "weights": _plain_weights, "select": _plain_select, "gather": _plain_gather}


# ---------------------------------------------------------------------------
# What a pass cannot do without.
# ---------------------------------------------------------------------------


def work(case):
    c = case
    h = _layout(c, 0)
    B, H = c["block"], c["kv_heads"]
    if c["kind"] in ("select", "gather"):
        past = h["len"] > h["budget"]
        lists = c["layers"] * H // c["share"] * float(h["budget"][past].sum())
        if c["kind"] == "select":
            return {"bytes": 4.0 * c["layers"] * H * float(h["len"][past].sum()) + 4 * lists + 40.0 * c["seqs"], "flops": 0.0}
        moved = c["layers"] * H * float(h["budget"][past].sum())
        passed = c["layers"] * H * float(h["len"][~past].sum())
        return {"bytes": 2 * 4 * c["dim"] * moved + 8 * (moved + passed) + 4 * lists, "flops": 0.0}
    D, T = c["dim"], int(h["q_off"][-1])
    count = h["q_off"][1:] - h["q_off"][:-1]
    i = np.arange(T) - np.repeat(h["q_off"][:-1], count)
    seen = np.maximum(np.repeat(h["len"] - count, count) + 1 + i, 0)
    used = -(-h["len"] // B)
    pages = np.unique(np.concatenate([h["page"][a:a + u] for a, u in zip(h["off"][:-1], used)])).size
    keys = 2.0 * D * H * B * pages  # bytes of the keys, or values
    rows = T * c["q_heads"]
    if c["kind"] == "diff":
        # a map: a product over D, and one with values of 2 D
        return {"bytes": 2 * keys + rows * (4 * D + 4), "flops": float(6 * D * c["q_heads"] * seen.sum())}
    if c["last"]:
        here = np.repeat(count, count) - i <= c["last"]
        seen, rows = seen[here], int(here.sum()) * c["q_heads"]
    carried = 4.0 * H * float(h["keep"].sum()) if c["prev"] else 0.0
    return {"bytes": keys + rows * (2 * D + 4) + 4.0 * H * float(h["len"].sum()) + carried,
            "flops": float(2 * D * c["q_heads"] * seen.sum())}


# ---------------------------------------------------------------------------
# The operators' definition in 64 bits, one sequence at a time.
# ---------------------------------------------------------------------------


def exact(case, seed):
    c = case
    if c["kind"] == "select" or work(c)["flops"] > 6e12:
        return None
    h = _layout(c, seed)
    s = _data(c, h, seed)
    if c["kind"] == "gather":
        return _moved(c, h, s)
    B, D, H = c["block"], c["dim"], c["kv_heads"]
    r = c["q_heads"] // H
    T = int(h["q_off"][-1])
    diff = c["kind"] == "diff"
    out = torch.zeros(T, c["q_heads"] // 2, 2 * D, device=DEV, dtype=torch.float64)
    lse = torch.full((T, c["q_heads"]), -math.inf, device=DEV, dtype=torch.float64)
    collected = torch.zeros(H, len(h["page"]) * B, device=DEV, dtype=torch.float64)
    for a in range(c["seqs"]):
        t0, t1, L = int(h["q_off"][a]), int(h["q_off"][a + 1]), int(h["len"][a])
        if L <= 0:
            continue
        at = torch.from_numpy(h["page"][h["off"][a]:h["off"][a] + -(-L // B)].astype(np.int64)).to(DEV)
        place = L - (t1 - t0) + torch.arange(t1 - t0, device=DEV)  # positions of the queries
        later = torch.arange(L, device=DEV)[None, :] > place[:, None]
        base = int(h["off"][a]) * B
        for x in range(c["q_heads"]):
            if t1 == t0:
                break
            # the query head's KV head: its own place in its pair, or its group's
            g = 2 * (x // 2 // r) + x % 2 if diff or c["paired"] else x // r
            keys = s["k"][0, at, g].reshape(-1, D)[:L].double()
            z = (s["q"][t0:t1, x].double() @ keys.T) / math.sqrt(D)
            z[later] = -math.inf
            if diff:
                lse[t0:t1, x] = torch.logsumexp(z, 1)
                pair = g // 2
                vals = torch.cat([s["v"][0, at, 2 * pair + m].reshape(-1, D)[:L] for m in (0, 1)], 1).double()
                y = torch.where((place >= 0)[:, None], torch.softmax(z, 1) @ vals, 0.0)
                out[t0:t1, x // 2] += y if x % 2 == 0 else -s["lam"][x // 2].double() * y
            else:
                far = s["lse"][t0:t1, x].double()
                z = torch.where((far > -math.inf)[:, None], torch.exp(z - far[:, None]), 0.0)
                collected[g, base:base + L] += z[max(0, t1 - t0 - c["last"]) if c["last"] else 0:].sum(0)
        if not diff and c["prev"]:
            old, n = int(h["prev_off"][h["src"][a]]) * B, int(h["keep"][a])
            collected[:, base:base + n] += s["prev"][:, old:old + n].double() * 0.99
    if not diff:
        return {"w": collected}
    if s["w"] is not None:
        out = out / torch.sqrt(torch.mean(out ** 2, dim=-1, keepdim=True) + EPS) * s["w"].double() * GAIN
    return {"out": out.reshape(T, c["q_heads"], D), "lse": lse}


def _moved(c, h, s):
    """A store and weights after the move, sequence by sequence."""
    B = c["block"]
    k, v = s["k"].double(), s["v"].double()
    w = torch.zeros(c["layers"], c["kv_heads"], len(h["to_page"]) * B, device=DEV, dtype=torch.float64)
    pages, to_pages = s["page"].long(), s["to_page"].long()
    for a in range(c["seqs"]):
        o0, o1 = int(h["off"][a]), int(h["to_off"][a])
        n = int(h["budget"][a] if h["past"][a] else h["len"][a])
        i = torch.arange(n, device=DEV)
        for layer in range(c["layers"]):
            for g in range(c["kv_heads"]):
                t = s["kept"][layer, g // c["share"], o0 * B:o0 * B + n].long() if h["past"][a] else i
                w[layer, g, o1 * B:o1 * B + n] = s["w"][layer, g, o0 * B + t].double()
                if h["past"][a]:
                    p, p1 = pages[o0 + t // B], to_pages[o1 + i // B]
                    k[layer, p1, g, i % B] = s["k"][layer, p, g, t % B].double()
                    v[layer, p1, g, i % B] = s["v"][layer, p, g, t % B].double()
    return {"k": k, "v": v, "w": w}


if __name__ == "__main__":
    for _case in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(_case, work(_case))
