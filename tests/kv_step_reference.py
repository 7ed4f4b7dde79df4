"""Plain definitions of a step's operators: block tables and trees on lists of numbers, norms and tree attention in 64
bits with the error each result may have.

Tolerances, from the number formats alone (u = half a unit in the last place, as in kv_reference):
- r = 1 / sqrt(mean x^2 + eps): the squares of at most 256 elements are added in 32 bits, at most 32 in a lane and 5
  exchanges between lanes, so their sum is off by 38 2^-24 of itself, r by half that and by the reciprocal root's two units:
  below 1.5 2^-20.  With the products x r w, the weight's offset and the rotation (2^-21 of the pair's size, as in
  kv_reference) a result is off by 2^-18 of its pair's size, and by u |y| of its one rounding.
- the gradient r (a - x r mean(a x r)): a is off by 2^-20 of its pair's size A, the mean by 2^-18 of mean(A |x| r), and r
  as above twice: below 2^-16 r (A + |x| r mean(A |x| r)) in all.
- the weight's gradient: N terms g x r in 32 bits in any order, each off by 2^-18 of G |x| r (G: the pair's size of g), the sum by
  N 2^-24 of the sum of sizes."""

import math

import torch

from tests import kv_reference as ref

BLOCK = 16
U, TINY = {**ref.U, torch.float64: 2.0 ** -53}, {**ref.TINY, torch.float64: 1e-300}
ROOT, ABSENT = -1, -2


# ---- block tables ----


def tables(n, new, kv_len, state, table, ring, shared=None):
    """The step on lists: returns state, q_off, lengths, positions and slots, and changes table and ring."""
    held, head, count = state[:n], state[n], state[n + 1]
    F = len(ring)
    lens = [a + b for a, b in zip(kv_len, new)]
    need = [-(-x // BLOCK) for x in lens]
    taken, given = 0, []
    for b in range(n):
        for c in range(held[b], need[b]):
            table[b][c] = ring[(head + taken) % F]
            taken += 1
        for c in range(max(need[b], shared[b] if shared else 0), held[b]):
            given.append(table[b][c])
    for i, x in enumerate(given):
        ring[(head + count + i) % F] = x
    q_off, positions, slots = [0], [], []
    for b in range(n):
        q_off.append(q_off[-1] + new[b])
        for p in range(kv_len[b], lens[b]):
            positions.append(p)
            slots.append(table[b][p // BLOCK] * BLOCK + p % BLOCK)
    return need + [(head + taken) % F, count - taken + len(given)], q_off, lens, positions, slots


# ---- trees ----


def tree(new, parents, window=0):
    """Depths, and for each node the list of the nodes that it sees (none: not there)."""
    depth, sees, at = [], [], 0
    for n in new:
        lines = []
        for i in range(n):
            p = parents[at + i]
            lines.append(None if p == ABSENT else [i] if p == ROOT else [i] + lines[p])
        for line in lines:
            depth.append(len(line) - 1 if line else 0)
            sees.append((line[:window] if window else line) if line else [])
        at += n
    return depth, sees


def bits(sees, words):
    out = torch.zeros((len(sees), words), dtype=torch.int64)
    for i, line in enumerate(sees):
        for j in line:
            out[i, j // 32] |= 1 << (j % 32)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def attend(q, k_blocks, v_blocks, new, lens, table, depth, sees, window=0, scale=None):
    """As kv_reference.attend, for nodes of trees."""
    dt, dev = q.dtype, q.device
    T, hq, d = q.shape
    hkv = k_blocks.shape[1]
    g = hq // hkv
    scale = scale or 1.0 / math.sqrt(d)
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=dev)
    otol = torch.full_like(out, TINY[dt])
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=dev)
    ltol = torch.zeros_like(lse)
    t0 = 0
    for b, (n, L) in enumerate(zip(new, lens)):
        k, v = (ref.gather(x, table[b], L).double() for x in (k_blocks, v_blocks))
        P = L - n
        see = torch.zeros((n, L), dtype=torch.bool)
        for i in range(n):
            if sees[t0 + i]:
                see[i, max(0, P + depth[t0 + i] - window + 1) if window else 0:P] = True
                see[i, [P + j for j in sees[t0 + i]]] = True
        see = see.to(dev)
        for i in range(0, n, 64):
            m = min(64, n - i)
            ok = see[i:i + m]
            qq = torch.where(ok.any(-1)[:, None, None], q[t0 + i:t0 + i + m].double(), 0.0).view(m, hkv, g, d)
            x = torch.einsum("mhgd,lhd->mhgl", qq, k) * scale
            xa = torch.einsum("mhgd,lhd->mhgl", qq.abs(), k.abs()) * scale
            x = torch.where(ok[:, None, None], x, -math.inf)
            xa = torch.where(ok[:, None, None], xa, 0.0)
            rows = ok.any(-1)
            z = torch.logsumexp(x, -1)
            p = torch.where(rows[:, None, None, None], torch.exp(x - z[..., None]), 0.0)
            o = torch.einsum("mhgl,lhd->mhgd", p, v).reshape(m, hq, d)
            a = torch.einsum("mhgl,lhd->mhgd", p, v.abs()).reshape(m, hq, d)
            e = (d + 16) * 2.0 ** -23 * xa.amax(-1).reshape(m, hq) + 2.0 ** -20
            out[t0 + i:t0 + i + m] = o
            otol[t0 + i:t0 + i + m] += U[dt] * (1 + 2.0 ** -10) * (a + o.abs()) + (
                (L / 16 + 8) * 2.0 ** -23 + 2 * e[..., None]) * a
            lse[t0 + i:t0 + i + m] = z.reshape(m, hq)
            ltol[t0 + i:t0 + i + m] = e + L * 2.0 ** -24 + 2.0 ** -22 * z.reshape(m, hq).abs().nan_to_num(0, 0, 0)
        t0 += n
    return out, otol, lse, ltol


# ---- normed heads ----


def _pairs(n, half):
    return (slice(0, n), slice(n, 2 * n)) if half else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))


def _turned(x, pos, freq, half, attn, back):
    """x turned, and the size of each element's pair (its own size where it is not turned)."""
    n = len(freq)
    ang = pos.double()[:, None] * freq.to(x.device)
    c, s = (ang.cos() * attn)[:, None], (ang.sin() * attn * (-1 if back else 1))[:, None]
    a_i, b_i = _pairs(n, half)
    y, size = x.clone(), x.abs()
    a, b = x[..., a_i], x[..., b_i]
    y[..., a_i], y[..., b_i] = a * c - b * s, a * s + b * c
    size[..., a_i] = size[..., b_i] = (a.abs() + b.abs()) * attn
    return y, size


def norm_rotate(x, pos, freq, half, w, eps=1e-6, offset=0.0, attn=1.0):
    """(y, tolerance) in 64 bits; w None: no norm."""
    dt = x.dtype
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (w.double() + offset)
    y, size = _turned(x, pos, freq, half, attn, False)
    return y, U[dt] * (1 + 2.0 ** -20) * y.abs() + 2.0 ** -18 * size + TINY[dt]


def norm_backward(x, dy, pos, freq, half, w, eps=1e-6, offset=0.0, attn=1.0):
    """(dx, tolerance, dw, tolerance) in 64 bits."""
    dt, wt = x.dtype, w.dtype
    x, dy, w = x.double(), dy.double(), w.double() + offset
    g, G = _turned(dy, pos, freq, half, attn, True)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u = x * r
    a, A = g * w, G * w.abs()
    dx = r * (a - u * (a * u).mean(-1, keepdim=True))
    tol = U[dt] * (1 + 2.0 ** -20) * dx.abs() + 2.0 ** -16 * r * (
        A + u.abs() * (A * u.abs()).mean(-1, keepdim=True)) + TINY[dt]
    over = 0 if w.dim() == 2 else (0, 1)
    N = x.shape[0] * (1 if w.dim() == 2 else x.shape[1])
    dw = (g * u).sum(over)
    wtol = U[wt] * (1 + 2.0 ** -20) * dw.abs() + (2.0 ** -18 + N * 2.0 ** -24) * (G * u.abs()).sum(over) + TINY[wt]
    return dx, tol, dw, wtol
