"""Operators beside the router, as cases to be timed: what an inference instance does with the
16-token KV blocks that the router counts.

- rotary: rotary position embedding of queries or keys, and its gradient.  Pairs of the first
  `rot` of `d` elements are turned by position x frequency; pairs are either the two halves of
  that part (i, i + rot/2) or neighbours (2i, 2i + 1).  Frequencies are base^(-2i/rot), plain,
  divided by `factor`, or divided by parts (slow pairs divided, fast pairs kept, with a linear
  ramp in the number of turns over the original length between them).
- append: new tokens' keys (rotated) and values go into a paged cache of blocks
  [block, kv head, 16 tokens, d] through each sequence's block table; the queries are rotated in
  the same call.
- attend: attention of each sequence's new tokens (one, or a chunk) over its cached tokens,
  themselves included: causal, optionally the last `window` keys only, query heads shared over
  kv heads.

Lengths follow the repository's workloads: prompts of 64 to 1,024 and 512 to 2,048 tokens,
agentic histories up to 32K and 128K tokens that grow by 200 to 2,000 tokens a turn.  A case
fixes its sequence lengths (`lens` seeds them); values, positions and block tables come from the
seed of prepare().
"""

import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
BETA_SLOW, BETA_FAST = 1.0, 32.0  # turns over the original length between which frequencies are blended
MAX_POS = 131072
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # queries of one decode step of 64 sequences: latency of a launch
        dict(name="rotary_step_n64", kind="rotary", n=64, heads=32, d=128, rot=128, half=True, scaling="none",
             factor=1.0, max_pos=32768, dtype="bf16", backward=False),
        # prompts of an odd total, half of each head rotated, neighbouring pairs, scaled to a long context
        dict(name="rotary_prompts_odd_n5003", kind="rotary", n=5003, heads=28, d=96, rot=48, half=False,
             scaling="by_parts", factor=8.0, max_pos=131072, dtype="f16", backward=False),
        # gradient of the rotation over a training batch of rollouts
        dict(name="rotary_backward_n65536", kind="rotary", n=65536, heads=32, d=128, rot=128, half=True,
             scaling="linear", factor=4.0, max_pos=32768, dtype="bf16", backward=True),
        # one decode step of 64 sequences: a token each
        dict(name="append_step_n64", kind="append", n=64, hist_lo=128, hist_hi=4096, new_lo=1, new_hi=1, hq=32, hkv=8,
             d=128, rot=128, half=True, scaling="none", factor=1.0, dtype="bf16", lens=1),
        # a batch of short prompts without history: ragged ends, seven queries to a kv head, small heads
        dict(name="append_prompts_n301", kind="append", n=301, hist_lo=0, hist_hi=0, new_lo=64, new_hi=1024, hq=28,
             hkv=4, d=64, rot=32, half=False, scaling="by_parts", factor=4.0, dtype="f16", lens=2),
        # a batch of agentic turns onto their histories
        dict(name="append_turns_n64", kind="append", n=64, hist_lo=1000, hist_hi=4000, new_lo=200, new_hi=2000, hq=32,
             hkv=8, d=128, rot=128, half=True, scaling="none", factor=1.0, dtype="bf16", lens=3),
        # a decode step of a nearly idle instance: latency of the call
        dict(name="attend_step_n4", kind="attend", n=4, hist_lo=17, hist_hi=640, new_lo=1, new_hi=1, hq=32, hkv=8,
             d=128, window=0, lse=False, dtype="bf16", lens=4),
        # a decode step of a busy instance: ragged histories, the cache is read once
        dict(name="attend_step_n256", kind="attend", n=256, hist_lo=512, hist_hi=16000, new_lo=1, new_hi=1, hq=32,
             hkv=8, d=128, window=0, lse=False, dtype="bf16", lens=5),
        # a decode step of one long session: the one axis to split is the history
        dict(name="attend_step_long_n1", kind="attend", n=1, hist_lo=131071, hist_hi=131071, new_lo=1, new_hi=1, hq=64,
             hkv=8, d=128, window=0, lse=True, dtype="f16", lens=6),
        # fresh prompts of odd lengths under a sliding window: small heads, three queries to a kv head
        dict(name="attend_prompts_window_n97", kind="attend", n=97, hist_lo=0, hist_hi=0, new_lo=512, new_hi=2048,
             hq=24, hkv=8, d=64, window=1000, lse=True, dtype="f16", lens=7),
        # agentic turns over cached histories: the ordinary prefill after a prefix hit
        dict(name="attend_turns_n16", kind="attend", n=16, hist_lo=1000, hist_hi=30000, new_lo=200, new_hi=2000, hq=32,
             hkv=8, d=128, window=0, lse=False, dtype="bf16", lens=8),
        # a chunk of a very long session: bound by the matrix products
        dict(name="attend_chunk_long_n1", kind="attend", n=1, hist_lo=129024, hist_hi=129024, new_lo=2048, new_hi=2048,
             hq=32, hkv=8, d=128, window=0, lse=False, dtype="bf16", lens=9),
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
    kind = rng.choices(["rotary", "append", "attend"], [2, 2, 5])[0]
    for _ in range(10000):
        d = rng.choice([64, 64, 128, 128, 128, rng.randrange(16, 129, 8)])
        rot = rng.choice([d, d, 2 * rng.randint(1, d // 2)])
        scaling = rng.choice(["none", "linear", "by_parts"])
        factor = 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 16.0])
        half = rng.random() < 0.5
        if kind == "rotary":
            c = dict(kind=kind, n=log_int(1, 65536), heads=rng.choice([1, 4, 7, 8, 28, 32, 40, 64]), d=d, rot=rot,
                     half=half, scaling=scaling, factor=factor, max_pos=log_int(64, MAX_POS),
                     dtype=rng.choice(["bf16", "f16", "f32"]), backward=rng.random() < 0.5)
        else:
            hkv = rng.choice([1, 2, 4, 8])
            hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
            new_hi = rng.choice([1, log_int(2, 2048), log_int(64, 2048)])
            hist_hi = rng.choice([0, log_int(1, 131000), log_int(256, 131000), log_int(256, 131000)])
            if kind == "append":
                hist_hi = min(hist_hi, 4000)
            c = dict(kind=kind, n=log_int(1, 256), hist_lo=rng.randint(0, hist_hi), hist_hi=hist_hi,
                     new_lo=rng.randint(1, new_hi), new_hi=new_hi, hq=hq, hkv=hkv, d=d,
                     dtype=rng.choice(["bf16", "f16"]), lens=rng.randint(100, 1 << 30))
            if kind == "append":
                c.update(rot=rot, half=half, scaling=scaling, factor=factor)
            else:
                c.update(window=rng.choice([0, 0, log_int(1, 4096)]), lse=rng.random() < 0.5)
            hist, new = _lengths(c)
            tokens = sum(hist) + sum(new)
            if tokens * hkv * d > (230 << 20 if kind == "append" else 2200 << 20):
                continue
        w = work(c)
        if all(w[key] <= _LIMIT[kind][key] for key in w):
            return c
    raise RuntimeError("no case within the ranges")


def _lengths(case):
    """Tokens held before the call and new tokens, a list of each over the sequences."""
    r = random.Random(case["lens"])
    hist = [r.randint(case["hist_lo"], case["hist_hi"]) for _ in range(case["n"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    return hist, new


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rotary":
        x = case["n"] * case["heads"] * case["d"] * size
        return {"bytes": 2 * x + 4 * case["n"], "flops": 3 * case["n"] * case["heads"] * case["rot"]}
    hist, new = _lengths(case)
    T = sum(new)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "append":
        tables = 4 * sum(-(-n // BLOCK) for n in new)
        return {"bytes": 2 * T * (hq + 2 * hkv) * d * size + tables, "flops": 3 * T * (hq + hkv) * case["rot"]}
    pairs = keys = blocks = 0
    win = case["window"]
    for h, n in zip(hist, new):
        L = h + n
        if win:
            a = min(max(win - h, 0), n)  # rows that still see every key
            pairs += a * h + a * (a + 1) // 2 + (n - a) * win
            seen = L - max(0, h - win + 1)
        else:
            pairs += n * h + n * (n + 1) // 2
            seen = L
        keys += seen
        blocks += -(-seen // BLOCK)
    out = {"bytes": 2 * T * hq * d * size + 2 * keys * hkv * d * size + 4 * blocks, "flops": 4 * pairs * hq * d}
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


def _inv_freq(case):
    """Frequencies (radians a position) of the pairs, in 64 bits."""
    rot = case["rot"]
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    elif case["scaling"] == "by_parts":
        turns = _orig_len(case) * f / (2 * math.pi)
        keep = ((turns - BETA_SLOW) / (BETA_FAST - BETA_SLOW)).clamp(0, 1)
        f = f * (keep + (1 - keep) / case["factor"])
    return f


def _orig_len(case):
    return 8192


def _attn_factor(case):
    """Factor on cos and sin that goes with frequencies blended by parts."""
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "by_parts" else 1.0


def _rope(case):
    from paper_2608_11152_gb300 import misat

    scaling = {"none": misat.ROPE_SCALE_NONE, "linear": misat.ROPE_SCALE_LINEAR,
               "by_parts": misat.ROPE_SCALE_BY_PARTS}[case["scaling"]]
    return misat.Rope(case["rot"], base=10000.0, layout=misat.ROPE_HALF if case["half"] else misat.ROPE_INTERLEAVED,
                      scaling=scaling, factor=case["factor"], orig_len=_orig_len(case), beta_slow=BETA_SLOW,
                      beta_fast=BETA_FAST, attn_factor=_attn_factor(case))


def _tables(case, max_pos):
    """cos and sin of every position, [max_pos, rot/2] in 32 bits."""
    ang = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * _inv_freq(case).cuda()
    a = _attn_factor(case)
    return (ang.cos() * a).float(), (ang.sin() * a).float()


def _inputs(case, seed):
    """Everything that depends on the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "rotary":
        x = _randn(gen, (case["n"], case["heads"], case["d"]), dt)
        pos = torch.randint(0, case["max_pos"], (case["n"],), generator=gen, device="cuda", dtype=torch.int32)
        return dict(x=x, pos=pos)
    hist, new = _lengths(case)
    lens = [h + n for h, n in zip(hist, new)]
    nb = [-(-L // BLOCK) for L in lens]
    n_blocks = sum(nb) + 7
    perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["n"], max(nb)), -1, dtype=torch.int32, device="cuda")
    cols = torch.arange(max(nb), device="cuda")
    used = cols[None, :] < torch.tensor(nb, device="cuda")[:, None]
    table[used] = perm[:sum(nb)]
    T = sum(new)
    q_off = np.zeros(case["n"] + 1, np.int32)
    np.cumsum(new, out=q_off[1:])
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    s = dict(hist=hist, new=new, lens=lens, nb=nb, table=table, T=T,
             q_off=torch.from_numpy(q_off).cuda(), kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if case["kind"] == "append":
        # one fused projection's output: queries, keys and values of a token side by side
        qkv = _randn(gen, (T, (hq + 2 * hkv) * d), dt)
        s["q"] = qkv[:, :hq * d].view(T, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(T, hkv, d)
        s["v"] = qkv[:, (hq + hkv) * d:].view(T, hkv, d)
        s["k_blocks"] = torch.zeros((n_blocks, hkv, BLOCK, d), dtype=dt, device="cuda")
        s["v_blocks"] = torch.zeros((n_blocks, hkv, BLOCK, d), dtype=dt, device="cuda")
    else:
        # logits of a standard deviation of two: a few keys stand out of a long history
        s["q"] = _randn(gen, (T, hq, d), dt, 2.0)
        s["k_blocks"] = _randn(gen, (n_blocks, hkv, BLOCK, d), dt)
        s["v_blocks"] = _randn(gen, (n_blocks, hkv, BLOCK, d), dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "rotary":
        if own:
            s["rope"] = _rope(case)
        else:
            s["cos"], s["sin"] = _tables(case, case["max_pos"])
        return s
    if own:
        from paper_2608_11152_gb300 import misat

        s["rope"] = _rope(case) if case["kind"] == "append" else None
        s["pool"] = misat.KvPool(s["k_blocks"], s["v_blocks"], n_q_heads=case["hq"], rope=s["rope"],
                                 max_batch=case["n"])
        s["batch"] = s["pool"].batch(s["q_off"], s["kv_len"], s["table"], n_tokens=s["T"], max_q=max(s["new"]))
    elif case["kind"] == "append":
        s["cos"], s["sin"] = _tables(case, max(s["lens"]))
    return s


# ---- plain forms: elementary operations in 32 bits ----


def _rotate(case, x, cos, sin):
    """x [tokens, heads, d] in 32 bits, cos and sin [tokens, rot/2]."""
    rot = case["rot"]
    c, s = cos[:, None, :], sin[:, None, :]
    y = x.clone()
    if case["half"]:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2] = a * c - b * s
        y[..., rot // 2:rot] = a * s + b * c
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * c - b * s
        y[..., 1:rot:2] = a * s + b * c
    return y


def _plain_rotary(s):
    case = s["case"]
    pos = s["pos"].long()
    sin = s["sin"][pos]
    if case["backward"]:
        sin = -sin
    return _rotate(case, s["x"].float(), s["cos"][pos], sin).to(s["x"].dtype)


def _plain_append(s):
    case = s["case"]
    dt = s["q"].dtype
    i = torch.arange(s["T"], device="cuda")
    q_off = s["q_off"].long()
    b = torch.searchsorted(q_off, i, right=True) - 1
    pos = s["kv_len"].long()[b] - q_off[b + 1] + i
    cos, sin = s["cos"][pos], s["sin"][pos]
    blk = s["table"][b, pos // BLOCK].long()
    s["k_blocks"][blk, :, pos % BLOCK] = _rotate(case, s["k"].float(), cos, sin).to(dt)
    s["v_blocks"][blk, :, pos % BLOCK] = s["v"]
    return _rotate(case, s["q"].float(), cos, sin).to(dt), s["k_blocks"], s["v_blocks"]


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    scale = 1.0 / math.sqrt(d)
    out = torch.empty((s["T"], hq, d), dtype=s["q"].dtype, device="cuda")
    lse = torch.empty((s["T"], hq), dtype=torch.float32, device="cuda") if case["lse"] else None
    t0 = 0
    for b in range(case["n"]):
        n, L = s["new"][b], s["lens"][b]
        blk = s["table"][b, :s["nb"][b]].long()
        q = s["q"][t0:t0 + n].float().view(n, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * n, d)
        pos = torch.arange(L - n, L, device="cuda").repeat(g)
        key = torch.arange(L, device="cuda")
        hide = key[None, :] > pos[:, None]
        if case["window"]:
            hide |= key[None, :] <= pos[:, None] - case["window"]
        k = s["k_blocks"][blk].transpose(0, 1).reshape(hkv, -1, d)[:, :L].float()
        v = s["v_blocks"][blk].transpose(0, 1).reshape(hkv, -1, d)[:, :L].float()
        # a few heads at a time, so that the scores of a long chunk fit
        step = max(1, (1 << 30) // (g * n * L))
        for h in range(0, hkv, step):
            x = torch.matmul(q[h:h + step], k[h:h + step].transpose(1, 2)) * scale
            x.masked_fill_(hide, -math.inf)
            m = x.amax(-1, keepdim=True)
            x = torch.exp(x - m)
            z = x.sum(-1, keepdim=True)
            o = torch.matmul(x, v[h:h + step]) / z
            hs = o.shape[0]
            out[t0:t0 + n].view(n, hkv, g, d)[:, h:h + hs] = o.view(hs, g, n, d).permute(2, 0, 1, 3).to(out.dtype)
            if case["lse"]:
                e = (m + torch.log(z)).view(hs, g, n)
                lse[t0:t0 + n].view(n, hkv, g)[:, h:h + hs] = e.permute(2, 0, 1)
        t0 += n
    return (out, lse) if case["lse"] else out


def run(s):
    case = s["case"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend}[case["kind"]](s)
    if case["kind"] == "rotary":
        return s["rope"].backward(s["x"], s["pos"]) if case["backward"] else s["rope"].rotate(s["x"], s["pos"])
    if case["kind"] == "append":
        q = s["pool"].append(s["batch"], s["k"], s["v"], q=s["q"])
        return q, s["k_blocks"], s["v_blocks"]
    return s["pool"].attend(s["batch"], s["q"], window=case["window"], return_lse=case["lse"])


# ---- the definitions in 64 bits ----


def _exact_rotation(case, x, pos):
    """Complex form: the pair (a, b) as a + ib times exp(i position frequency)."""
    half = case["rot"] // 2
    x = x.double()
    part = x[..., :case["rot"]]
    pairs = torch.stack((part[..., :half], part[..., half:]), -1) if case["half"] else part.unflatten(-1, (half, 2))
    freq = torch.empty(half, dtype=torch.float64)
    for i in range(half):
        f = math.exp(-2 * i / case["rot"] * math.log(10000.0))
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "by_parts":
            turns = f * _orig_len(case) / math.tau
            if turns <= BETA_SLOW:
                f /= case["factor"]
            elif turns < BETA_FAST:
                w = (turns - BETA_SLOW) / (BETA_FAST - BETA_SLOW)
                f = w * f + (1 - w) * f / case["factor"]
        freq[i] = f
    ang = pos.double()[:, None] * freq.cuda()
    if case.get("backward"):
        ang = -ang
    turn = torch.polar(torch.full_like(ang, _attn_factor(case)), ang)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    head = torch.cat((z[..., 0], z[..., 1]), -1) if case["half"] else z.flatten(-2)
    return torch.cat((head, x[..., case["rot"]:]), -1)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotation(case, s["x"], s["pos"])
    if case["kind"] == "append":
        kb, vb = s["k_blocks"].double(), s["v_blocks"].double()
        pos = torch.cat([torch.arange(h, h + n) for h, n in zip(s["hist"], s["new"])]).cuda()
        seq = torch.repeat_interleave(torch.arange(case["n"]), torch.tensor(s["new"])).cuda()
        slot = s["table"][seq, torch.div(pos, BLOCK, rounding_mode="floor")].long() * BLOCK + pos % BLOCK
        flat_k, flat_v = kb.transpose(1, 2).reshape(-1, case["hkv"], case["d"]), vb.transpose(1, 2).reshape(
            -1, case["hkv"], case["d"])
        flat_k[slot] = _exact_rotation(case, s["k"], pos)
        flat_v[slot] = s["v"].double()
        shape = (kb.shape[0], BLOCK, case["hkv"], case["d"])
        return (_exact_rotation(case, s["q"], pos), flat_k.view(shape).transpose(1, 2).contiguous(),
                flat_v.view(shape).transpose(1, 2).contiguous())
    if work(case)["flops"] > 6e12:  # some seconds of 64-bit products
        return None
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    out = torch.zeros((s["T"], hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s["T"], hq), dtype=torch.float64, device="cuda")
    first = 0
    for b in range(case["n"]):
        L, n = s["lens"][b], s["new"][b]
        blocks = s["table"][b, :-(-L // BLOCK)].long()
        for h in range(hkv):
            k = s["k_blocks"][blocks, h].reshape(-1, d)[:L].double()
            v = s["v_blocks"][blocks, h].reshape(-1, d)[:L].double()
            rows = max(1, (1 << 28) // (g * L))  # queries at a time
            for r in range(0, n, rows):
                m = min(rows, n - r)
                where = torch.arange(L - n + r, L - n + r + m, device="cuda")[:, None, None]
                key = torch.arange(L, device="cuda")[None, None, :]
                seen = key <= where
                if case["window"]:
                    seen = seen & (key > where - case["window"])
                q = s["q"][first + r:first + r + m, h * g:(h + 1) * g].double()
                logits = torch.where(seen, (q.reshape(m * g, d) @ k.T).view(m, g, L) / math.sqrt(d), -math.inf)
                norm = torch.logsumexp(logits, -1)
                p = torch.exp(logits - norm[..., None])
                out[first + r:first + r + m, h * g:(h + 1) * g] = (p.view(m * g, L) @ v).view(m, g, d)
                lse[first + r:first + r + m, h * g:(h + 1) * g] = norm
        first += n
    return (out, lse) if case["lse"] else out
