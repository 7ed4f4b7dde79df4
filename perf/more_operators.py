"""Operators of an instance's step on its 16-token KV blocks, as cases to be timed: the step's block tables, queries
and keys with a norm for each head, and a tree of drafted tokens.

- tables: each sequence's row of the block table is brought to the length that it has after the step.  Blocks that it
  lacks come from the front of a ring of free blocks, those it no longer needs go to the ring's end; with the offsets,
  lengths, positions and slots of the new tokens.
- norm: root-mean-square norm of each head with a weight (one for all heads, or one for each), then the rotary position,
  in one pass; and the gradients of the input and of the weight.
- append: new tokens' keys (normed, rotated) and values go into the blocks, the queries are normed and rotated in the same
  call; tokens may be nodes of a tree, whose position is their depth's and whose slot is their own.
- tree: depths of the nodes of each sequence's tree from their parents, and a bit for each ancestor of each.
- attend: attention of the nodes over the tokens before the tree and their own ancestors, themselves included.
- keep: the keys and values of the nodes that a check of the drafts accepted move to the slots behind the tokens before.

Lengths follow the repository's workloads: histories up to 32K and 128K tokens, turns of 200 to 2,000 tokens, prompts of
64 to 2,048.  A case fixes its sequence lengths (`lens` seeds them); values, trees and tables come from prepare()'s seed.
"""

import math
import random

import torch

own = False

BLOCK = 16
EPS = 1e-6
ROOT, ABSENT = -1, -2  # parents of a node that follows the tokens before the tree, and of one that is not there
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one decode step of 256 sequences, some of them finished: latency
        dict(name="tables_step_n256", kind="tables", n=256, hist_lo=100, hist_hi=8000, new_lo=1, new_hi=1, spare=24,
             done=20, shared=True, lens=1),
        # a prefill round over many sequences: every token's position and slot
        dict(name="tables_turns_n4096", kind="tables", n=4096, hist_lo=0, hist_hi=30000, new_lo=200, new_hi=2000, spare=0,
             done=100, shared=False, lens=2),
        # queries of prompts of an odd total: part of a head rotated, neighbouring pairs, a weight for each head
        dict(name="norm_prompts_odd_n5003", kind="norm", n=5003, heads=28, d=96, rot=48, half=False, per_head=True,
             offset=0.0, dtype="f16", wtype="f16", backward=False),
        # gradients over a training batch of rollouts: one weight for all heads, kept in 32 bits
        dict(name="norm_backward_n65536", kind="norm", n=65536, heads=32, d=128, rot=128, half=True, per_head=False,
             offset=0.0, dtype="bf16", wtype="f32", backward=True),
        # drafted trees of a serving step: queries, keys and values of 64 sequences' nodes
        dict(name="append_tree_n64", kind="append", n=64, hist_lo=128, hist_hi=4096, new_lo=16, new_hi=32, hq=32, hkv=8,
             d=128, rot=128, half=True, per_head=False, offset=0.0, dtype="bf16", wtype="bf16", tree=True, absent=0,
             lens=3),
        # plan of a serving step's trees: latency
        dict(name="tree_n64", kind="tree", n=64, new_lo=16, new_hi=32, window=0, absent=0, lens=5),
        # wide trees of many sequences, of a fixed shape whose last nodes may be unused, under a sliding window
        dict(name="tree_wide_n1024", kind="tree", n=1024, new_lo=129, new_hi=129, window=7, absent=30, lens=6),
        # a draft check of a nearly idle instance: latency
        dict(name="attend_tree_n4", kind="attend", n=4, hist_lo=17, hist_hi=640, new_lo=12, new_hi=12, hq=32, hkv=8, d=128,
             window=0, absent=0, lse=False, dtype="bf16", lens=7),
        # a draft check of a busy instance: ragged histories, some nodes unused
        dict(name="attend_tree_n96", kind="attend", n=96, hist_lo=512, hist_hi=16000, new_lo=16, new_hi=32, hq=32, hkv=8,
             d=128, window=0, absent=10, lse=False, dtype="bf16", lens=8),
        # a wide tree behind one long session: the one axis to split is the history
        dict(name="attend_tree_long_n1", kind="attend", n=1, hist_lo=130941, hist_hi=130941, new_lo=63, new_hi=63, hq=64,
             hkv=8, d=64, window=0, absent=0, lse=True, dtype="f16", lens=9),
        # accepted paths of a serving step
        dict(name="keep_n64", kind="keep", n=64, hist_lo=128, hist_hi=4096, new_lo=16, new_hi=32, hkv=8, d=128,
             dtype="bf16", lens=10),
        # long accepted paths of many sequences of short histories, small heads
        dict(name="keep_n1024", kind="keep", n=1024, hist_lo=0, hist_hi=300, new_lo=64, new_hi=128, hkv=8, d=64,
             dtype="f16", lens=11),
    ]


_LIMIT = {}


def draw(rng):
    """A case of the same ranges, no costlier than the largest listed one of its kind."""

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if not _LIMIT:
        for c in listed():
            w, m = work(c), _LIMIT.setdefault(c["kind"], {"bytes": 0, "flops": 0})
            for key in m:
                m[key] = max(m[key], w[key])
    kind = rng.choices(["tables", "norm", "append", "tree", "attend", "keep"], [2, 3, 2, 1, 4, 1])[0]
    for _ in range(10000):
        d = rng.choice([64, 64, 128, 128, 128, rng.randrange(16, 129, 8)])
        if kind == "norm":
            d = rng.choice([d, d, 256, rng.randint(1, 120) * 2])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
        dtype = rng.choice(["bf16", "f16"])
        head = dict(d=d, rot=rng.choice([d, d, 2 * rng.randint(1, d // 2)]), half=rng.random() < 0.5,
                    per_head=rng.random() < 0.4, offset=rng.choice([0.0, 0.0, 1.0]))
        hist_hi = rng.choice([0, log_int(1, 32000), log_int(256, 32000)])
        hist = dict(hist_lo=rng.randint(0, hist_hi), hist_hi=hist_hi)
        absent = rng.choice([0, 0, rng.randint(1, 50)])
        lens = rng.randint(100, 1 << 30)
        if kind == "tables":
            new_hi = rng.choice([1, log_int(2, 64), log_int(64, 2048)])
            c = dict(kind=kind, n=log_int(1, 4096), **hist, new_lo=rng.randint(0, new_hi), new_hi=new_hi,
                     spare=rng.choice([0, log_int(1, 200)]), done=rng.choice([0, rng.randint(1, 500)]),
                     shared=rng.random() < 0.5, lens=lens)
        elif kind == "norm":
            dtype = rng.choice(["bf16", "f16", "f32"])
            c = dict(kind=kind, n=log_int(1, 65536), heads=rng.choice([1, 4, 7, 8, 28, 32, 40, 64]), **head, dtype=dtype,
                     wtype=rng.choice([dtype, "f32"]), backward=rng.random() < 0.6)
        elif kind == "append":
            tree = rng.random() < 0.5
            new_hi = log_int(1, 200) if tree else log_int(1, 2048)
            c = dict(kind=kind, n=log_int(1, 256), **hist, new_lo=rng.randint(1, new_hi), new_hi=new_hi, hq=hq, hkv=hkv,
                     **head, dtype=dtype, wtype=rng.choice([dtype, "f32"]), tree=tree, absent=absent if tree else 0,
                     lens=lens)
            c["hist_lo"], c["hist_hi"] = min(c["hist_lo"], 4000), min(c["hist_hi"], 4000)
        elif kind == "tree":
            new_hi = log_int(1, 200)
            c = dict(kind=kind, n=log_int(1, 1024), new_lo=rng.randint(1, new_hi), new_hi=new_hi,
                     window=rng.choice([0, 0, log_int(1, 100)]), absent=absent, lens=lens)
        elif kind == "attend":
            new_hi = log_int(1, 200)
            if rng.random() < 0.3:
                hist = dict(hist_lo=rng.randint(1, 131000), hist_hi=131000)
            c = dict(kind=kind, n=log_int(1, 256), **hist, new_lo=rng.randint(1, new_hi), new_hi=new_hi, hq=hq, hkv=hkv,
                     d=d, window=rng.choice([0, 0, log_int(1, 4096)]), absent=absent, lse=rng.random() < 0.5, dtype=dtype,
                     lens=lens)
            # the plain form takes all sequences at the longest one's length
            longest = max(h + k for h, k in zip(*_lengths(c)))
            if c["n"] * longest * max(2 * hkv * d, hq * c["new_hi"]) > 6 << 30:
                continue
        else:
            new_hi = log_int(1, 200)
            c = dict(kind=kind, n=log_int(1, 1024), **hist, new_lo=rng.randint(1, new_hi), new_hi=new_hi, hkv=hkv, d=d,
                     dtype=dtype, lens=lens)
        if kind in ("append", "keep"):
            old, new = _lengths(c)
            if (sum(old) + sum(new)) * hkv * d > 230 << 20:
                continue
        w = work(c)
        if all(w[key] <= _LIMIT[kind][key] for key in w):
            return c
    raise RuntimeError("no case within the ranges")


def _lengths(case):
    """Tokens held before the step and new tokens, a list of each over the sequences."""
    r = random.Random(case["lens"])
    hist = [r.randint(case.get("hist_lo", 0), case.get("hist_hi", 0)) for _ in range(case["n"])]
    return hist, [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["n"])]


def _rows(case):
    """tables: tokens before and new tokens, blocks in the row, and how many of these first ones are shared."""
    r = random.Random(case["lens"] + 1)
    hist, new = _lengths(case)
    held = [-(-(h + r.randint(0, case["spare"])) // BLOCK) for h in hist]
    shared = [r.randint(0, min(b, 40)) for b in held] if case["shared"] else None
    for i in range(case["n"]):
        if r.randrange(1000) < case["done"]:  # finished: all its own blocks go back
            hist[i] = new[i] = 0
    return hist, new, held, shared


def _present(case):
    """Nodes of each tree that are there: the last ones may not be."""
    r = random.Random(case["lens"] + 2)
    return [n - (r.randint(0, n - 1) if r.randrange(100) < case["absent"] else 0) for n in _lengths(case)[1]]


def _paths(case):
    """keep: nodes accepted of each sequence, and how many of them are in their place already."""
    r = random.Random(case["lens"] + 3)
    count = [r.randint(0, n // 2) for n in _lengths(case)[1]]
    return count, [r.randint(0, min(m, 2)) for m in count]


def work(case):
    kind = case["kind"]
    size = 4 if case.get("dtype") == "f32" else 2
    n = case["n"]
    if kind == "tables":
        hist, new, held, shared = _rows(case)
        need = [-(-(h + k) // BLOCK) for h, k in zip(hist, new)]
        least = [max(a, b) for a, b in zip(need, shared)] if shared else need
        moved = sum(max(a - b, 0) + max(b - c, 0) for a, b, c in zip(need, held, least))
        return {"bytes": 12 * sum(new) + 8 * moved + 4 * n * (6 + case["shared"]), "flops": 0}
    if kind == "norm":
        x = n * case["heads"] * case["d"]
        w = (case["heads"] if case["per_head"] else 1) * case["d"] * (4 if case["wtype"] == "f32" else 2)
        if case["backward"]:
            return {"bytes": 3 * x * size + 4 * n + 2 * w, "flops": 10 * x + 3 * n * case["heads"] * case["rot"]}
        return {"bytes": 2 * x * size + 4 * n + w, "flops": 4 * x + 3 * n * case["heads"] * case["rot"]}
    hist, new = _lengths(case)
    T = sum(new)
    words = -(-max(new) // 32)
    if kind == "tree":
        return {"bytes": 8 * T + 4 * T * words + 4 * n, "flops": 0}
    hkv, d = case["hkv"], case["d"]
    if kind == "keep":
        moved = sum(a - b for a, b in zip(*_paths(case)))
        return {"bytes": 4 * moved * hkv * d * size + 4 * moved + 12 * n, "flops": 0}
    hq = case["hq"]
    if kind == "append":
        w = d * (hq + hkv if case["per_head"] else 2) * (4 if case["wtype"] == "f32" else 2)
        tables = 4 * sum(-(-k // BLOCK) for k in new) + (4 * T if case["tree"] else 0)
        return {"bytes": 2 * T * (hq + 2 * hkv) * d * size + tables + w,
                "flops": T * (hq + hkv) * (4 * d + 3 * case["rot"])}
    pairs = keys = blocks = 0
    win = case["window"]
    for h, k, there in zip(hist, new, _present(case)):
        seen = min(h, win - 1) if win else h  # of a node of depth 0; a deeper one sees at most its depth less
        pairs += there * (max(seen - there, 0) if win else seen) + there
        keys += seen + there
        blocks += -(-(seen + there) // BLOCK)
    out = {"bytes": 2 * T * hq * d * size + 2 * keys * hkv * d * size + 4 * blocks + 4 * T * words,
           "flops": 4 * pairs * hq * d}
    if case["lse"]:
        out["bytes"] += 4 * T * hq
    return out


# ---- inputs ----


def _randn(gen, shape, dtype, std=1.0):
    """Normal values, made in pieces so that no large array of 32-bit values is held."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda") * std)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _weight(gen, case, heads):
    """A trained norm's weight: near one (with the offset), a few elements far from it."""
    shape = (heads, case["d"]) if case["per_head"] else (case["d"],)
    w = 1 - case["offset"] + 0.3 * torch.randn(shape, generator=gen, device="cuda")
    w = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.02, w * 8, w)
    return w.to(DTYPES[case["wtype"]])


def _tables(case, max_pos):
    """cos and sin of every position, [max_pos, rot/2] in 32 bits."""
    rot = case["rot"]
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    ang = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return ang.cos().float(), ang.sin().float()


def _inputs(case, seed):
    """Everything that depends on the case and the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    kind, n = case["kind"], case["n"]
    dt = DTYPES.get(case.get("dtype"))
    if kind == "norm":
        # heads of unlike sizes, as projections give them
        std = torch.exp(0.7 * torch.randn((case["heads"], 1), generator=gen, device="cuda"))
        x = _randn(gen, (n, case["heads"], case["d"]), dt)
        x.mul_(std.to(dt))
        s = dict(x=x, pos=torch.randint(0, 32768, (n,), generator=gen, device="cuda", dtype=torch.int32),
                 w=_weight(gen, case, case["heads"]))
        if case["backward"]:
            s["dy"] = _randn(gen, (n, case["heads"], case["d"]), dt)
        return s
    if kind == "tables":
        hist, new, held, shared = _rows(case)
        need = [-(-(h + k) // BLOCK) for h, k in zip(hist, new)]
        take = sum(max(a - b, 0) for a, b in zip(need, held))
        n_free = take + take // 8 + 100
        n_blocks = sum(held) + n_free
        perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((n, max(need + held) + 3), -1, dtype=torch.int32, device="cuda")
        used = torch.arange(table.shape[1], device="cuda")[None, :] < _ints(held)[:, None]
        table[used] = perm[:sum(held)]
        # a ring that has been in use: its front is anywhere
        head = int(torch.randint(0, n_blocks, (1,), generator=gen, device="cuda"))
        ring = torch.full((n_blocks,), -1, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(n_free, device="cuda")) % n_blocks] = perm[sum(held):]
        return dict(T=sum(new), max_q=max(new), table=table, ring=ring, state=_ints(held + [head, n_free]),
                    new=_ints(new), kv_len=_ints(hist), shared=_ints(shared) if shared else None, n_blocks=n_blocks)
    hist, new = _lengths(case)
    T = sum(new)
    q_off = torch.cat((_ints([0]), _ints(new).cumsum(0, dtype=torch.int32)))
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), _ints(new).long(), output_size=T)
    idx = torch.arange(T, device="cuda") - q_off.long()[seq]  # of a token in its sequence
    s = dict(hist=hist, new=new, T=T, q_off=q_off, seq=seq, idx=idx)
    if "absent" in case:
        # every node hangs on an earlier one or on the tokens before; the last ones may not be there
        parent = (torch.rand(T, generator=gen, device="cuda", dtype=torch.float64) * (idx + 1)).long() - 1
        s["parent"] = torch.where(idx < _ints(_present(case)).long()[seq], parent, ABSENT).to(torch.int32)
    if kind == "tree":
        s["kv_len"] = _ints(new)
        return s
    lens = [h + k for h, k in zip(hist, new)]
    nb = [-(-L // BLOCK) for L in lens]
    n_blocks = sum(nb) + 7
    perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((n, max(nb)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(nb), device="cuda")[None, :] < _ints(nb)[:, None]] = perm[:sum(nb)]
    s.update(table=table, kv_len=_ints(lens), lens=lens)
    hkv, d = case["hkv"], case["d"]
    if kind == "append":
        hq = case["hq"]
        # one fused projection's output: queries, keys and values of a token side by side
        qkv = _randn(gen, (T, (hq + 2 * hkv) * d), dt, 1.5)
        s["q"] = qkv[:, :hq * d].view(T, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(T, hkv, d)
        s["v"] = qkv[:, (hq + hkv) * d:].view(T, hkv, d)
        s["wq"], s["wk"] = _weight(gen, case, hq), _weight(gen, case, hkv)
        s["k_blocks"] = torch.zeros((n_blocks, hkv, BLOCK, d), dtype=dt, device="cuda")
        s["v_blocks"] = torch.zeros((n_blocks, hkv, BLOCK, d), dtype=dt, device="cuda")
        return s
    s["k_blocks"] = _randn(gen, (n_blocks, hkv, BLOCK, d), dt)
    s["v_blocks"] = _randn(gen, (n_blocks, hkv, BLOCK, d), dt)
    if kind == "attend":
        # logits of a standard deviation of two: a few keys stand out of a long history
        s["q"] = _randn(gen, (T, case["hq"], d), dt, 2.0)
        return s
    # keep: accepted nodes in rising order; those that move come from behind all places that are written, so that the same
    # call can be made again
    count, same = _paths(case)
    width = max(count + [1])
    col = torch.arange(width, device="cuda")[None, :]
    m, fix, k = _ints(count).long()[:, None], _ints(same).long()[:, None], _ints(new).long()[:, None]
    nodes = torch.arange(max(new), device="cuda")[None, :]
    chance = torch.rand((n, max(new)), generator=gen, device="cuda").masked_fill_((nodes < m) | (nodes >= k), 2.0)
    order = chance.argsort(1)[:, :width]  # a random choice of the nodes behind the written places
    order = torch.where(col < m - fix, order, 1 << 30).sort(1).values
    path = torch.where(col < fix, col, torch.gather(order, 1, (col - fix).clamp(min=0)))
    s["path"] = torch.where(col < m, path, -1).to(torch.int32).contiguous()
    s["n_keep"] = _ints(count)
    return s


def _ancestors(s, window):
    """[n, N, N]: whether node j of a sequence is node i itself or an ancestor; [n, N] depths, and whether it is there."""
    n, N = len(s["new"]), max(s["new"])
    parent = torch.full((n, N), ABSENT, dtype=torch.int64, device="cuda")
    parent[s["seq"], s["idx"]] = s["parent"].long()
    there = parent != ABSENT
    reach = torch.eye(N, device="cuda") + (parent[..., None] == torch.arange(N, device="cuda")).float()
    for _ in range(max(1, math.ceil(math.log2(N)))):  # steps up to 1, 2, 4, ... generations
        reach = torch.matmul(reach, reach).clamp_(max=1.0)
    up = reach > 0.5
    up &= there[..., None] & there[:, None, :]
    depth = (up.sum(-1) - 1).clamp(min=0)
    if window:
        up &= depth[..., None] - depth[:, None, :] < window
    return up, depth, there


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if own:
        from paper_2608_11152_gb300 import misat

        if kind in ("norm", "append"):
            s["rope"] = misat.Rope(case["rot"], layout=misat.ROPE_HALF if case["half"] else misat.ROPE_INTERLEAVED)
        if kind == "norm":
            s["norm"] = misat.HeadNorm(s["w"], eps=EPS, offset=case["offset"])
            return s
        if kind in ("tables", "tree"):  # the pool's blocks play no part
            s["k_blocks"], s["v_blocks"] = (torch.empty((s.get("n_blocks", sum(s.get("new", ()))), 1, BLOCK, 8),
                                                        dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["pool"] = misat.KvPool(s["k_blocks"], s["v_blocks"], n_q_heads=case.get("hq", case.get("hkv", 1)),
                                 rope=s.get("rope"), max_batch=case["n"])
        if kind == "tables":
            s["tables"] = misat.KvTables(s["pool"], s["table"], s["ring"])
            return s
        table = s["table"] if "table" in s else torch.zeros((case["n"], -(-max(s["new"]) // BLOCK)), dtype=torch.int32,
                                                            device="cuda")
        s["batch"] = s["pool"].batch(s["q_off"], s["kv_len"], table, n_tokens=s["T"], max_q=max(s["new"]))
        if kind == "append":
            s["norms"] = [misat.HeadNorm(w, eps=EPS, offset=case["offset"]) for w in (s["wq"], s["wk"])]
        # a tree's plan serves all layers of a step
        if kind == "attend" or (kind == "append" and case["tree"]):
            s["tree"] = s["pool"].tree(s["batch"], s["parent"], window=case.get("window", 0))
        return s
    if kind == "norm":
        s["cos"], s["sin"] = _tables(case, 32768)
    elif kind == "append":
        s["cos"], s["sin"] = _tables(case, max(s["lens"]))
        s["depth"] = _ancestors(s, 0)[1] if case["tree"] else None
    elif kind == "attend":
        s["up"], s["depth"], s["there"] = _ancestors(s, case["window"])
    return s


# ---- plain forms: elementary operations in 32 bits ----


def _plain_tables(s):
    n, F = s["case"]["n"], s["ring"].shape[0]
    state, table, ring = s["state"].long(), s["table"], s["ring"]
    held, head, count = state[:n], state[n], state[n + 1]
    new, kv_len = s["new"].long(), s["kv_len"].long()
    need = (kv_len + new + BLOCK - 1) // BLOCK
    least = need if s["shared"] is None else torch.maximum(need, s["shared"].long())
    take, give = (need - held).clamp(min=0), (held - least).clamp(min=0)
    take_end, give_end = take.cumsum(0), give.cumsum(0)
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), give)
    j = torch.arange(row.shape[0], device="cuda")
    ring[(head + count + j) % F] = table[row, least[row] + j - (give_end - give)[row]]
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), take)
    j = torch.arange(row.shape[0], device="cuda")
    table[row, held[row] + j - (take_end - take)[row]] = ring[(head + j) % F]
    taken, given = take_end[-1], give_end[-1]
    after = torch.cat((need, ((head + taken) % F)[None], (count - taken + given)[None])).to(torch.int32)
    q_off = torch.cat((new.new_zeros(1), new.cumsum(0)))
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), new, output_size=s["T"])
    pos = kv_len[seq] + torch.arange(s["T"], device="cuda") - q_off[seq]
    slots = table[seq, pos // BLOCK].long() * BLOCK + pos % BLOCK
    return table, ring, after, q_off.to(torch.int32), (kv_len + new).to(torch.int32), pos.to(torch.int32), slots


def _rotate(case, x, cos, sin):
    """x [tokens, heads, d] in 32 bits, cos and sin [tokens, rot/2]."""
    rot = case["rot"]
    c, s = cos[:, None, :], sin[:, None, :]
    y = x.clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if case["half"] else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def _normed(case, x, w):
    """x [tokens, heads, d] in 32 bits; the weight broadcasts over tokens (and heads)."""
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * (w.float() + case["offset"])


def _plain_norm(s):
    case, dt = s["case"], s["x"].dtype
    pos = s["pos"].long()
    cos, sin = s["cos"][pos], s["sin"][pos]
    x = s["x"].float()
    if not case["backward"]:
        return _rotate(case, _normed(case, x, s["w"]), cos, sin).to(dt)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    g = _rotate(case, s["dy"].float(), cos, -sin)
    a = g * (s["w"].float() + case["offset"])
    dx = r * a - x * (r * r * r) * (a * x).mean(-1, keepdim=True)
    dw = (g * x * r).sum(0 if case["per_head"] else (0, 1), dtype=torch.float64)
    return dx.to(dt), dw.to(s["w"].dtype)


def _plain_append(s):
    case, dt = s["case"], s["q"].dtype
    seq, idx = s["seq"], s["idx"]
    slot = s["kv_len"].long()[seq] - (s["q_off"][1:] - s["q_off"][:-1]).long()[seq] + idx
    pos = slot - idx + s["depth"][seq, idx] if case["tree"] else slot
    cos, sin = s["cos"][pos], s["sin"][pos]
    blk = s["table"][seq, slot // BLOCK].long()
    s["k_blocks"][blk, :, slot % BLOCK] = _rotate(case, _normed(case, s["k"].float(), s["wk"]), cos, sin).to(dt)
    s["v_blocks"][blk, :, slot % BLOCK] = s["v"]
    return _rotate(case, _normed(case, s["q"].float(), s["wq"]), cos, sin).to(dt), s["k_blocks"], s["v_blocks"]


def _plain_tree(s):
    up, depth, _ = _ancestors(s, s["case"]["window"])
    words = -(-max(s["new"]) // 32)
    rows = torch.nn.functional.pad(up[s["seq"], s["idx"]], (0, words * 32 - up.shape[-1]))
    bits = (rows.view(-1, words, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    return depth[s["seq"], s["idx"]].to(torch.int32), torch.where(bits >> 31 > 0, bits - (1 << 32), bits).to(torch.int32)


def _plain_attend(s):
    case = s["case"]
    n, hq, hkv, d = case["n"], case["hq"], case["hkv"], case["d"]
    g, N, T = hq // hkv, max(s["new"]), s["T"]
    table = s["table"].long().clamp(min=0)
    L = table.shape[1] * BLOCK
    k = s["k_blocks"][table].transpose(1, 2).reshape(n, hkv, L, d).float()
    v = s["v_blocks"][table].transpose(1, 2).reshape(n, hkv, L, d).float()
    q = torch.zeros((n, N, hq, d), device="cuda")
    q[s["seq"], s["idx"]] = s["q"].float()
    q = q.view(n, N, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * N, d)
    key = torch.arange(L, device="cuda")
    hist = _ints(s["hist"]).long()[:, None, None]
    node = (key - hist).expand(n, N, L)  # of a key in the tree
    see = torch.gather(s["up"], 2, node.clamp(0, N - 1)) & (node >= 0) & (node < N)
    before = key < hist
    if case["window"]:
        before = before & (key > hist + s["depth"][..., None] - case["window"])
    see |= before & s["there"][..., None]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    x.view(n, hkv, g, N, L).masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)  # (a node that is not there)
    x = x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / torch.where(z == 0, 1.0, z)
    o = o.view(n, hkv, g, N, d).permute(0, 3, 1, 2, 4).reshape(n, N, hq, d)
    out = o[s["seq"], s["idx"]].to(s["q"].dtype)
    if not case["lse"]:
        return out
    lse = (m + torch.log(z)).view(n, hkv, g, N).permute(0, 3, 1, 2).reshape(n, N, hq)
    return out, lse[s["seq"], s["idx"]]


def _plain_keep(s):
    hist = s["kv_len"] - (s["q_off"][1:] - s["q_off"][:-1])
    col = torch.arange(s["path"].shape[1], device="cuda")
    row, i = (col < s["n_keep"][:, None]).nonzero(as_tuple=True)
    src, dst = hist.long()[row] + s["path"][row, i], hist.long()[row] + i
    a, b = s["table"][row, src // BLOCK].long(), s["table"][row, dst // BLOCK].long()
    s["k_blocks"][b, :, dst % BLOCK] = s["k_blocks"][a, :, src % BLOCK]
    s["v_blocks"][b, :, dst % BLOCK] = s["v_blocks"][a, :, src % BLOCK]
    return s["k_blocks"], s["v_blocks"], hist + s["n_keep"]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"tables": _plain_tables, "norm": _plain_norm, "append": _plain_append, "tree": _plain_tree,
                "attend": _plain_attend, "keep": _plain_keep}[kind](s)
    if kind == "tables":
        b = s["tables"].step(s["state"], s["new"], s["kv_len"], n_tokens=s["T"], max_q=s["max_q"], shared=s["shared"])
        return s["table"], s["ring"], b.state, b.q_off, b.kv_len, b.positions, b.slots
    if kind == "norm":
        if case["backward"]:
            return s["rope"].norm_backward(s["x"], s["dy"], s["pos"], s["norm"])
        return s["rope"].norm_rotate(s["x"], s["pos"], s["norm"])
    if kind == "append":
        q = s["pool"].append(s["batch"], s["k"], s["v"], q=s["q"], q_norm=s["norms"][0], k_norm=s["norms"][1],
                             tree=s.get("tree"))
        return q, s["k_blocks"], s["v_blocks"]
    if kind == "tree":
        t = s["pool"].tree(s["batch"], s["parent"], window=case["window"])
        return t.depth, t.bits
    if kind == "attend":
        return s["pool"].attend(s["batch"], s["q"], tree=s["tree"], return_lse=case["lse"])
    kv_len = s["pool"].keep(s["batch"], s["path"], s["n_keep"])
    return s["k_blocks"], s["v_blocks"], kv_len


# ---- the definitions in 64 bits ----


def _turns(case, pos):
    """exp(i position frequency) of every pair, [tokens, 1, rot/2]."""
    half = case["rot"] // 2
    freq = torch.tensor([math.exp(-2 * i / case["rot"] * math.log(10000.0)) for i in range(half)], dtype=torch.float64)
    ang = pos.double()[:, None, None] * freq.cuda()
    return torch.polar(torch.ones_like(ang), ang)


def _exact_rotation(case, x, turn):
    """Complex form: the pair (a, b) as a + ib times the turn."""
    half = case["rot"] // 2
    part = x[..., :case["rot"]]
    pairs = torch.stack((part[..., :half], part[..., half:]), -1) if case["half"] else part.unflatten(-1, (half, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    head = torch.cat((z[..., 0], z[..., 1]), -1) if case["half"] else z.flatten(-2)
    return torch.cat((head, x[..., case["rot"]:]), -1)


def _exact_norm(case, x, w):
    length = torch.linalg.vector_norm(x.double(), dim=-1, keepdim=True)
    return x.double() / torch.sqrt(length ** 2 / case["d"] + EPS) * (w.double() + case["offset"])


def _depths(s):
    """Depth of every node by walking up, on the host: [tokens]."""
    out = []
    parent, at = s["parent"].tolist(), 0
    for k in s["new"]:
        mine = []
        for i in range(k):
            p = parent[at + i]
            mine.append(0 if p < 0 else mine[p] + 1)
        out += mine
        at += k
    return torch.tensor(out, device="cuda")


def exact(case, seed):
    kind = case["kind"]
    if kind in ("tables", "tree"):  # whole numbers alone
        return None
    s = _inputs(case, seed)
    if kind == "norm":
        out, grads, step = [], [], max(1, (1 << 26) // (case["heads"] * case["d"]))
        for i in range(0, case["n"], step):  # tokens at a time
            x, turn = s["x"][i:i + step].double(), _turns(case, s["pos"][i:i + step])
            if not case["backward"]:
                out.append(_exact_rotation(case, _exact_norm(case, x, s["w"]), turn))
                continue
            dy, w = s["dy"][i:i + step].double(), s["w"].double() + case["offset"]
            g = _exact_rotation(case, dy, turn.conj())
            norm = torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            unit = x / norm
            grads.append((g * unit).sum(0) if case["per_head"] else (g * unit).sum((0, 1)))
            out.append(((g * w - unit * (g * w * unit).mean(-1, keepdim=True)) / norm))
        return (torch.cat(out), torch.stack(grads).sum(0)) if case["backward"] else torch.cat(out)
    seq = torch.repeat_interleave(torch.arange(case["n"]), torch.tensor(s["new"])).cuda()
    place = torch.cat([torch.arange(h, h + k) for h, k in zip(s["hist"], s["new"])]).cuda()
    hkv, d = case["hkv"], case["d"]
    shape = (s["k_blocks"].shape[0], BLOCK, hkv, d)
    if kind in ("append", "keep"):
        rows = [s[name].double().transpose(1, 2).reshape(-1, hkv, d) for name in ("k_blocks", "v_blocks")]

        def back(flat):
            return flat.view(shape).transpose(1, 2).contiguous()

        def slots(b, p):
            return s["table"][b, torch.div(p, BLOCK, rounding_mode="floor")].long() * BLOCK + p % BLOCK
    if kind == "append":
        pos = torch.tensor(s["hist"]).cuda()[seq] + _depths(s) if case["tree"] else place
        turn, slot = _turns(case, pos), slots(seq, place)
        rows[0][slot] = _exact_rotation(case, _exact_norm(case, s["k"], s["wk"]), turn)
        rows[1][slot] = s["v"].double()
        return _exact_rotation(case, _exact_norm(case, s["q"], s["wq"]), turn), back(rows[0]), back(rows[1])
    if kind == "keep":
        path, count = s["path"].tolist(), s["n_keep"].tolist()
        b = torch.tensor([b for b, m in enumerate(count) for _ in range(m)], dtype=torch.int64).cuda()
        src = torch.tensor([s["hist"][b] + path[b][i] for b, m in enumerate(count) for i in range(m)],
                           dtype=torch.int64).cuda()
        dst = torch.tensor([s["hist"][b] + i for b, m in enumerate(count) for i in range(m)], dtype=torch.int64).cuda()
        for r in rows:
            r[slots(b, dst)] = r[slots(b, src)]
        return back(rows[0]), back(rows[1]), None
    if work(case)["flops"] > 6e12:  # some seconds of 64-bit products
        return None
    hq, win = case["hq"], case["window"]
    g = hq // hkv
    out = torch.zeros((s["T"], hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((s["T"], hq), -math.inf, dtype=torch.float64, device="cuda")
    parent, first = s["parent"].tolist(), 0
    depth = _depths(s)
    for b, (h, n) in enumerate(zip(s["hist"], s["new"])):
        # a node's line of ancestors is its parent's and itself
        line = torch.zeros((n, n), dtype=torch.bool)
        for i in range(n):
            p = parent[first + i]
            if p >= 0:
                line[i] = line[p]
            line[i, i] = p != ABSENT
        line, deep = line.cuda(), depth[first:first + n]
        there = line.diagonal()
        old = there[:, None].expand(n, h)
        if win:
            line = line & (deep[:, None] - deep[None, :] < win)
            old = old & (h + deep[:, None] - torch.arange(h, device="cuda")[None, :] < win)
        seen = torch.cat((old, line), 1)[:, None]
        blocks = s["table"][b, :-(-(h + n) // BLOCK)].long()
        for j in range(hkv):
            k = s["k_blocks"][blocks, j].reshape(-1, d)[:h + n].double()
            v = s["v_blocks"][blocks, j].reshape(-1, d)[:h + n].double()
            rows = max(1, (1 << 28) // (g * (h + n)))  # nodes at a time
            for r in range(0, n, rows):
                m = min(rows, n - r)
                q = s["q"][first + r:first + r + m, j * g:(j + 1) * g].double()
                x = torch.where(seen[r:r + m], (q.reshape(m * g, d) @ k.T).view(m, g, -1) / math.sqrt(d), -math.inf)
                norm = torch.logsumexp(x, -1)
                p = torch.exp(x - torch.where(torch.isinf(norm), 0.0, norm)[..., None])
                out[first + r:first + r + m, j * g:(j + 1) * g] = (p.view(m * g, -1) @ v).view(m, g, d)
                lse[first + r:first + r + m, j * g:(j + 1) * g] = norm
        first += n
    return (out, lse) if case["lse"] else out
