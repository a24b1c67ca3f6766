#!/usr/bin/env python3
"""Requests routed, then served on one instance: pages, append and attention together.

Two waves of prompts that share templates are routed over four instances
(dm_route_batch); instance 0 and the requests it was given are this GPU.  The
matched blocks of the routing batch are the pages that a request starts from.
Each step is one batch of old sequences with one new token and new ones with
the rest of their prompts:

  pages_fork    the step's tables from the last step's (continued, started from
                a cached prefix, dropped), pages_copy for the pages that several
                go on writing;
  attn_plan     once a step;
  kv_append, attn
                a layer: norm, rotation and page write, then attention in which
                the sequences of a template read its pages once;
  pages_compact when the first wave has gone.

The model is a small decoder of random weights; its products are torch's.
Run: python examples/serve_instance.py
"""
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

BLOCK, VOCAB, LAYERS, HEADS, KV_HEADS, DIM = 16, 4096, 2, 8, 2, 64
WIDTH, PAGES, MAX_POS = HEADS * DIM, 512, 1024


class Decoder:
    """A decoder's weights, and its step over an instance's pages."""

    def __init__(self, device, seed=1):
        import torch
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g) * rows ** -0.5).bfloat16().to(device)

        self.embed = torch.randn(VOCAB, WIDTH, generator=g).bfloat16().to(device)
        self.head = weight(WIDTH, VOCAB)
        self.layers = [dict(qkv=weight(WIDTH, (HEADS + 2 * KV_HEADS) * DIM), o=weight(WIDTH, WIDTH),
                            up=weight(WIDTH, 2 * WIDTH), down=weight(2 * WIDTH, WIDTH),
                            qn=(1 + torch.randn(DIM, generator=g) / 8).bfloat16().to(device),
                            kn=(1 + torch.randn(DIM, generator=g) / 8).bfloat16().to(device))
                       for _ in range(LAYERS)]
        turn = torch.arange(MAX_POS)[:, None] * 10000.0 ** -(torch.arange(DIM // 2) / (DIM // 2))
        self.cos, self.sin = turn.cos().float().to(device), turn.sin().float().to(device)

    def step(self, eng, kv, tables, q_off, tokens, groups=None):
        """Logits of each new token; their keys and values are in the pages afterwards."""
        import torch
        import torch.nn.functional as F
        x = self.embed[tokens]
        T = len(tokens)
        plan = eng.attn_plan(kv, tables, q_off, T, HEADS, groups=groups)
        for i, w in enumerate(self.layers):
            heads = (F.rms_norm(x, (WIDTH,)) @ w["qkv"]).unflatten(1, (HEADS + 2 * KV_HEADS, DIM))
            q, k, v = heads.split((HEADS, KV_HEADS, KV_HEADS), 1)
            eng.kv_append(kv, i, tables, q_off, q, k, v, q, w["qn"], w["kn"], cos=self.cos, sin=self.sin)
            y = torch.empty((T, HEADS, DIM), dtype=x.dtype, device=x.device)
            eng.attn(plan, i, q, DIM ** -0.5, y)
            x = x + y.flatten(1) @ w["o"]
            x = x + F.gelu(F.rms_norm(x, (WIDTH,)) @ w["up"]) @ w["down"]
        return F.rms_norm(x, (WIDTH,)).float() @ self.head.float()


class Instance:
    """One instance's pages, and the sequences that live in them."""

    def __init__(self, eng, model):
        import torch
        import paper_2602_06502_amd as pk
        self.eng, self.model, dev = eng, model, eng.device
        shape = (LAYERS, PAGES, KV_HEADS, BLOCK, DIM)
        self.kv = pk.KVPages(torch.zeros(shape, dtype=torch.bfloat16, device=dev),
                             torch.zeros(shape, dtype=torch.bfloat16, device=dev))
        self.ref = torch.zeros(PAGES, dtype=torch.int32, device=dev)
        self.tables = (torch.zeros(1, dtype=torch.int64, device=dev),
                       torch.zeros(1, dtype=torch.int32, device=dev),
                       torch.zeros(0, dtype=torch.int64, device=dev))
        self.seqs = []  # token lists, in the tables' order

    def step(self, rows):
        """rows: (source sequence, tokens kept, new tokens), those of one prefix
        next to each other.  Returns the logits of each row's last token."""
        import torch
        dev = self.eng.device
        i64 = dict(dtype=torch.int64, device=dev)
        cap = sum((keep + len(new) + BLOCK - 1) // BLOCK for _, keep, new in rows)
        out = self.eng.pages_fork(self.tables, self.ref,
                                  torch.tensor([max(s, 0) for s, _, _ in rows], dtype=torch.int32, device=dev),
                                  torch.tensor([k for _, k, _ in rows], **i64),
                                  torch.tensor([len(new) for _, _, new in rows], **i64), max(cap, 1))
        self.eng.pages_copy(self.kv, out)
        seqs = [(self.seqs[s][:keep] if keep else []) + list(new) for s, keep, new in rows]
        self.tables, self.ref, self.seqs = (out["off"], out["page"], out["len"]), out["ref"], seqs
        q_off = np.cumsum([0] + [len(new) for _, _, new in rows])
        # Runs: neighbours whose sequences begin with the same block.
        runs = [0] + [j for j in range(1, len(seqs)) if seqs[j][:BLOCK] != seqs[j - 1][:BLOCK]] + [len(seqs)]
        new = torch.tensor([t for _, _, n in rows for t in n], **i64)
        y = self.model.step(self.eng, self.kv, self.tables, torch.tensor(q_off, **i64), new,
                            torch.tensor(runs, **i64))
        return y[torch.tensor(q_off[1:] - 1, **i64)]

    def compact(self):
        """The live pages to the front of the store; returns how many there are."""
        out = self.eng.alloc_pages_out(PAGES, 0, self.tables[1].numel())
        self.eng.pages_compact_into(self.tables, self.ref, out)
        self.eng.pages_copy(self.kv, out)
        self.tables, self.ref = (self.tables[0], out["page"], self.tables[2]), out["ref"]
        self.eng.sync()
        return int(out["live"].item())


def main(steps=6, say=print):
    import torch
    import paper_2602_06502_amd as pk
    rng = np.random.default_rng(7)
    eng = pk.DualMap(dict(block=BLOCK, key_blocks=2, seeds=(0x9E3779B97F4A7C15, 0xC2B2AE3D27D4EB4F), vnodes=32,
                          max_slots=4, index_log2_slots=12, ttft_base_us=5000, ttft_per_token_us=20,
                          queue_div=1, slo_us=5_000_000), device="cuda:0")
    eng.build_rings(range(4))
    inst = Instance(eng, Decoder(eng.device))
    templates = [rng.integers(0, VOCAB, int(n)).tolist() for n in rng.integers(3 * BLOCK, 8 * BLOCK, 6)]
    loads = torch.zeros(4, dtype=torch.int64, device=eng.device)
    holder = {}  # block key -> number of the request that holds the block

    def route(clock):
        """A wave of prompts for instance 0: (tokens, matched tokens, block keys)."""
        prompts = [templates[int(t)] + rng.integers(0, VOCAB, int(n)).tolist()
                   for t, n in zip(rng.integers(0, 6, 48), rng.integers(1, 3 * BLOCK, 48))]
        off = np.cumsum([0] + [len(p) for p in prompts])
        d_off = torch.tensor(off, dtype=torch.int64, device=eng.device)
        r = eng.route(torch.tensor(sum(prompts, []), dtype=torch.int32, device=eng.device), d_off, loads,
                      block_keys=True)
        eng.sync()
        eng.kv_save(d_off, r["block_keys"], r["chosen"], clock=clock, cap=1024)
        chosen, cand = r["chosen"].cpu().numpy(), r["cand"].cpu().numpy().reshape(2, -1).T
        match, keys = r["match"].cpu().numpy().reshape(2, -1).T, r["block_keys"].cpu().numpy()
        first = np.cumsum([0] + [len(p) // BLOCK for p in prompts])
        mine = []
        for i in np.flatnonzero(chosen == 0):
            # The last token is computed in any case: its logits are the answer.
            blocks = min(int(match[i][list(cand[i]).index(0)]), (len(prompts[i]) - 1) // BLOCK)
            mine.append((prompts[i], blocks, keys[first[i]:first[i + 1]].tolist()))
        return mine

    live = []  # request numbers, in the tables' order
    told, asked, seen = {}, {}, {}  # request -> tokens answered, prompt, the answers' logits

    def step(new=(), drop=()):
        """One step: live requests go on (dropped ones end), new ones begin."""
        rows = [(j, len(inst.seqs[j]), [told[r][-1]], r) for j, r in enumerate(live) if r not in drop]
        matched = 0
        for prompt, blocks, keys in new:
            r = len(asked)
            asked[r], told[r], seen[r] = prompt, [], []
            while blocks and holder.get(keys[blocks - 1]) not in live:
                blocks -= 1  # the block went with its sequence
            src = live.index(holder[keys[blocks - 1]]) if blocks else -1
            rows.append((src, blocks * BLOCK, prompt[blocks * BLOCK:], r))
            matched += blocks * BLOCK
            for key in keys:
                holder.setdefault(key, r)
        order = sorted(rows, key=lambda x: asked[x[3]][:BLOCK])
        logits = inst.step([x[:3] for x in order])
        live[:] = [x[3] for x in order]
        for r, t, y in zip(live, logits.argmax(1).tolist(), logits):
            told[r].append(t)
            seen[r].append(y)
        return matched

    first = route(1)
    step(first)
    for _ in range(steps):
        step()
    second = route(2)
    matched = step(second)
    say(f"{len(first)} requests, then {len(second)} of which {matched} tokens of "
        f"{sum(len(p) for p, _, _ in second)} were in pages")
    for _ in range(steps):
        step()
    step(drop=range(len(first)))
    before = int((inst.ref > 0).nonzero().max().item()) + 1
    pages = inst.compact()
    say(f"first wave gone: {pages} pages live, the last in place {before - 1} before, {pages - 1} now")
    for _ in range(steps):
        step()
    eng.sync()

    # Every answer again, each request by itself in one pass over fresh pages.
    worst = 0.0
    for r in sorted(asked):
        alone = Instance(eng, inst.model)
        text = asked[r] + told[r][:-1]
        i64 = dict(dtype=torch.int64, device=eng.device)
        n = (len(text) + BLOCK - 1) // BLOCK
        tables = (torch.tensor([0, n], **i64), torch.arange(n, dtype=torch.int32, device=eng.device),
                  torch.tensor([len(text)], **i64))
        y = inst.model.step(eng, alone.kv, tables, torch.tensor([0, len(text)], **i64), torch.tensor(text, **i64))
        y = y[len(asked[r]) - 1:]
        worst = max(worst, float(((torch.stack(seen[r]) - y).abs().amax(1) / y.abs().amax(1)).max()))
    say(f"{len(asked)} requests, {sum(map(len, told.values()))} tokens answered; logits against those of each "
        f"request by itself: largest difference {worst:.4f} of the largest logit")
    eng.sync()
    eng.close()
    return dict(requests=len(asked), matched=matched, pages=pages, before=before, worst=worst)


if __name__ == "__main__":
    main()
