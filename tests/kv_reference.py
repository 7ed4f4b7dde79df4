"""Plain 64-bit definitions of the KV block operators, with the error each result may have.

Tolerances, from the number formats alone (u = half a unit in the last place: 2^-8 for bfloat16,
2^-11 for float16, 2^-24 for 32 bits):
- a rotated element is computed in 32 bits and rounded once: u |y| plus 2^-21 of the pair's size
  (angle to 2^-24 of a quarter turn, sine and cosine to 2 units, two products and a sum);
- attention: each weight is rounded once (u of sum p |v|), the result once (u |o|); products of
  the tensor cores accumulate 16 at a time in 32 bits, at worst truncating (2^-23 each, L / 16 of
  them); a score's error of e changes its weight by e, e = (d + 16) 2^-23 of scale sum |q| |k|;
- the smallest float16 adds 2^-24 wherever a result is rounded to it."""

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24, torch.float32: 1e-37}


def frequencies(rot, base=10000.0, scaling=0, factor=1.0, orig_len=0.0, beta_slow=1.0, beta_fast=32.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == 1:
            f /= factor
        elif scaling == 2:
            g = min(1.0, max(0.0, (orig_len * f / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow)))
            f *= g + (1 - g) / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, pos, freq, half, attn=1.0, backward=False):
    """x [tokens, heads, d]; returns (y, tolerance) in 64 bits."""
    dt = x.dtype
    x = x.detach().double().cpu()
    ang = pos.double().cpu()[:, None] * freq
    c, s = (ang.cos() * attn)[:, None], (ang.sin() * attn * (-1 if backward else 1))[:, None]
    n = len(freq)
    y = x.clone()
    size = torch.zeros_like(x)
    a_i, b_i = (slice(0, n), slice(n, 2 * n)) if half else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., a_i], x[..., b_i]
    y[..., a_i] = a * c - b * s
    y[..., b_i] = a * s + b * c
    size[..., a_i] = size[..., b_i] = (a.abs() + b.abs()) * attn
    return y, U[dt] * (1 + 2.0 ** -20) * y.abs() + 2.0 ** -21 * size + TINY[dt]


def gather(blocks, table_row, length):
    """Rows [length, kv heads, d] of one sequence."""
    if length <= 0:
        return blocks.new_zeros((0, blocks.shape[1], blocks.shape[3]))
    idx = table_row[: -(-length // 16)].long()
    return blocks[idx].permute(0, 2, 1, 3).reshape(-1, blocks.shape[1], blocks.shape[3])[:length]


def attend(q, k_blocks, v_blocks, new, lens, table, scale=None, window=0):
    """Returns out, lse and their tolerances, 64 bits on the CPU's side of the comparison."""
    dt, dev = q.dtype, q.device
    T, hq, d = q.shape
    hkv = k_blocks.shape[1]
    g = hq // hkv
    scale = scale or 1.0 / math.sqrt(d)
    u = U[dt]
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=dev)
    otol = torch.full_like(out, TINY[dt])
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=dev)
    ltol = torch.zeros_like(lse)
    t0 = 0
    for b, (n, L) in enumerate(zip(new, lens)):
        k, v = (gather(x, table[b], L).double() for x in (k_blocks, v_blocks))
        for i in range(0, n, 64):
            m = min(64, n - i)
            pos = torch.arange(L - n + i, L - n + i + m, device=dev)
            key = torch.arange(max(L, 0), device=dev)
            see = key[None] <= pos[:, None]
            if window:
                see &= key[None] > pos[:, None] - window
            qq = q[t0 + i:t0 + i + m].double().view(m, hkv, g, d)
            x = torch.einsum("mhgd,lhd->mhgl", qq, k) * scale
            xa = torch.einsum("mhgd,lhd->mhgl", qq.abs(), k.abs()) * scale
            x = torch.where(see[:, None, None], x, -math.inf)
            xa = torch.where(see[:, None, None], xa, 0.0)
            rows = see.any(-1)
            if not rows.any():
                continue
            z = torch.logsumexp(x, -1)
            p = torch.where(rows[:, None, None, None], torch.exp(x - z[..., None]), 0.0)
            vv = torch.where(torch.isfinite(v), v, 0.0)  # a weight of exactly zero takes nothing
            o = torch.einsum("mhgl,lhd->mhgd", p, vv).reshape(m, hq, d)
            a = torch.einsum("mhgl,lhd->mhgd", p, vv.abs()).reshape(m, hq, d)
            e = (d + 16) * 2.0 ** -23 * xa.amax(-1).reshape(m, hq) + 2.0 ** -20
            out[t0 + i:t0 + i + m] = o
            otol[t0 + i:t0 + i + m] += u * (1 + 2.0 ** -10) * (a + o.abs()) + (
                (L / 16 + 8) * 2.0 ** -23 + 2 * e[..., None]) * a
            lse[t0 + i:t0 + i + m] = torch.where(rows[:, None], z.reshape(m, hq), -math.inf)
            ltol[t0 + i:t0 + i + m] = e + L * 2.0 ** -24 + 2.0 ** -22 * z.reshape(m, hq).abs().nan_to_num(0, 0, 0)
        t0 += n
    return out, otol, lse, ltol


def assert_within(name, got, ref, tol):
    got = got.double().to(ref.device)
    assert got.shape == ref.shape, f"{name}: {tuple(got.shape)} vs {tuple(ref.shape)}"
    bad = ~((got - ref).abs() <= tol) & ~(got == ref)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i].item()} vs "
                             f"{ref[i].item()}, tolerance {tol[i].item()}")
