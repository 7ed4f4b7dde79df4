"""The router and one instance's KV blocks together, in small.

Batches of the tiny mixed workload are routed; the requests that land on one instance are prefilled
there from the first token that its cache does not hold: their tokens' keys (rotated to their
positions) and values are appended to 16-token blocks, and they attend over the cached prefix and
themselves.  Some steps of decoding follow.  The model is one attention layer with random weights;
a few results are compared with the same layer on the whole prompt, without a cache.

    python examples/routed_prefill.py
"""

from __future__ import annotations

import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_11152_gb300 import misat  # noqa: E402
from paper_2608_11152_gb300 import workload as wl  # noqa: E402

HIDDEN, HQ, HKV, D, BLOCK = 256, 8, 2, 64, misat.BLOCK_TOKENS


class Layer:
    """Embedding and the projections of one attention layer."""

    def __init__(self, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.embed = torch.randn((wl.VOCAB, HIDDEN), generator=g, device="cuda").bfloat16()
        self.w_qkv = (torch.randn((HIDDEN, (HQ + 2 * HKV) * D), generator=g, device="cuda") / 16).bfloat16()

    def qkv(self, tokens):
        x = self.embed[tokens] @ self.w_qkv
        q, k, v = x.split([HQ * D, HKV * D, HKV * D], dim=1)
        return q.view(-1, HQ, D), k.view(-1, HKV, D), v.view(-1, HKV, D)


class Instance:
    """One instance's blocks: which block holds which key, and the sequences in flight."""

    def __init__(self, layer, n_blocks):
        self.layer = layer
        self.blocks = [torch.zeros((n_blocks, HKV, BLOCK, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.pool = misat.KvPool(*self.blocks, n_q_heads=HQ, rope=misat.Rope(D))
        self.where = {}  # block key -> block
        self.free = list(range(n_blocks - 1, -1, -1))

    def step(self, tables, lens, new):
        """Prefill or decode: `new` holds each sequence's new tokens, lens its tokens with them.
        Returns the new tokens' attention outputs, in the order of the sequences."""
        for table, n in zip(tables, lens):
            while len(table) * BLOCK < n:
                table.append(self.free.pop())
        width = max(len(t) for t in tables)
        table = torch.tensor([t + [-1] * (width - len(t)) for t in tables], dtype=torch.int32, device="cuda")
        off = np.zeros(len(new) + 1, np.int32)
        np.cumsum([len(x) for x in new], out=off[1:])
        batch = self.pool.batch(torch.from_numpy(off).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                table, n_tokens=int(off[-1]), max_q=max(len(x) for x in new))
        q, k, v = self.layer.qkv(torch.from_numpy(np.concatenate(new)).cuda())
        self.q = self.pool.append(batch, k, v, q=q)
        return self.pool.attend(batch, self.q), off


def plain(layer, tokens):
    """The last token's output over the whole prompt, in 32 bits and without a cache."""
    q, k, v = (x.float() for x in layer.qkv(torch.from_numpy(tokens).cuda()))
    i = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    ang = torch.arange(len(tokens), device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-2 * i / D)
    c, s = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def turn(x):
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)

    q, k = turn(q)[-1], turn(k)
    x = torch.einsum("hgd,lhd->hgl", q.view(HKV, HQ // HKV, D), k) / math.sqrt(D)
    return torch.einsum("hgl,lhd->hgd", x.softmax(-1), v).reshape(HQ, D)


def run(instance=0, decode=4, checks=3, inspect=None):
    """Routes the workload's batches; returns counts and the largest difference from plain().  After each step,
    inspect(engine, tables, tokens, new, out) gets the sequences' block tables and tokens, how many of these were
    new, and the outputs of the new ones."""
    sc = wl.config1()
    r = misat.Router(sc.cap_blocks, max_batch=sc.max_batch, max_tokens=sc.max_tokens,
                     protected_frac_q16=sc.protected_frac_q16, mode=sc.mode, hold_delay_q=sc.hold_delay_q,
                     prior_kbar=sc.prior_kbar, prior_T_us=sc.prior_T_us)
    r.set_mixture(sc.rho_ppm)
    r.set_instance_state(sc.backlog_q, sc.tokcost_q, sc.contraction)
    steps = list(sc.warm) + [(sc.batch, None)]
    total = sum(int(b.tok_off[-1]) for b, _ in steps) // BLOCK
    engine = Instance(Layer(), total + len(steps) * sc.max_batch * 2)
    stats = dict(requests=0, tokens=0, hit=0, decoded=0, worst=0.0)
    for b, comp in steps:
        out = r.route(r.device_batch(b))
        inst, hits = out["inst"][:b.n].cpu().numpy(), out["hit_blocks"][:b.n].cpu().numpy()
        keys = r.dump_keys(b.n_tokens // BLOCK + 1)
        r.commit()
        first = np.concatenate(([0], np.cumsum(np.diff(b.tok_off) // BLOCK)))
        mine = [q for q in range(b.n) if inst[q] == instance and b.tok_off[q + 1] > b.tok_off[q]]
        if mine:
            prompts = [b.tokens[b.tok_off[q]:b.tok_off[q + 1]] for q in mine]
            # the last token is computed even where its block is cached: its output is asked for
            held = [min(int(hits[q]), (len(p) - 1) // BLOCK) for q, p in zip(mine, prompts)]
            tables = [[engine.where[int(k)] for k in keys[first[q]:first[q] + h]] for q, h in zip(mine, held)]
            lens = [len(p) for p in prompts]
            o, off = engine.step(tables, lens, [p[h * BLOCK:] for p, h in zip(prompts, held)])
            if inspect:
                inspect(engine, tables, prompts, np.diff(off).tolist(), o)
            for q, t in zip(mine, tables):
                for j, k in enumerate(keys[first[q]:first[q + 1]]):
                    engine.where.setdefault(int(k), t[j])
            for i in sorted(range(len(mine)), key=lambda i: -held[i])[:checks]:
                d = (o[off[i + 1] - 1].float() - plain(engine.layer, prompts[i])).abs().max().item()
                stats["worst"] = max(stats["worst"], d)
            stats["requests"] += len(mine)
            stats["tokens"] += sum(lens)
            stats["hit"] += BLOCK * sum(held)
            # decoding goes on in blocks of its own: the prompt's last block may be another's too
            tails = [list(t) for t in tables]
            for i, t in enumerate(tails):
                if lens[i] % BLOCK:
                    t[-1] = engine.free.pop()
                    for x in engine.blocks:
                        x[t[-1]] = x[tables[i][-1]]
            grown = prompts
            for s in range(decode):
                token = [np.array([(7919 * (s + 1) + 31 * i) % wl.VOCAB], np.int32) for i in range(len(mine))]
                grown = [np.concatenate((p, t)) for p, t in zip(grown, token)]
                o, _ = engine.step(tails, [len(p) for p in grown], token)
                if inspect:
                    inspect(engine, tails, grown, [1] * len(mine), o)
                stats["decoded"] += len(mine)
            if decode:
                d = (o[0].float() - plain(engine.layer, grown[0])).abs().max().item()
                stats["worst"] = max(stats["worst"], d)
            for i, t in enumerate(tails):  # a finished sequence's own blocks are free again
                engine.free.extend(t[lens[i] // BLOCK:])
        if comp is not None:
            r.complete(comp.session, comp.cls, comp.total_blocks, comp.residency_us, comp.done)
    engine.pool.sync()
    r.sync()
    r.close()
    return stats


if __name__ == "__main__":
    s = run()
    print(f"instance 0: {s['requests']} requests, {s['tokens']} prompt tokens, {s['hit']} of them held in its blocks; "
          f"{s['decoded']} tokens decoded; largest difference from the layer without a cache {s['worst']:.4f}")
