"""Rotary positions, append to a paged cache, attention over it: against 64-bit definitions."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def misat():
    from paper_2608_11152_gb300 import misat as m

    return m


def rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


class Step:
    """Sequences (new tokens, length after the append) with shuffled blocks; entries of the table
    past a sequence's last block are far outside the pool."""

    def __init__(self, seqs, hkv, d, dtype, seed=1, spare=3, n_blocks=None, kv="random"):
        self.new = [n for n, _ in seqs]
        self.lens = [L for _, L in seqs]
        self.T = sum(self.new)
        nb = [-(-max(L, 0) // 16) for L in self.lens]
        total = sum(nb)
        self.n_blocks = n_blocks or total + spare
        g = torch.Generator().manual_seed(seed)
        ids = torch.randperm(total + spare, generator=g).to(torch.int32) + (self.n_blocks - total - spare)
        self.table = torch.full((len(seqs), max(nb + [1]) + 1), 2 ** 31 - 1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(nb):
            self.table[b, :k] = ids[at:at + k]
            at += k
        self.table = self.table.cuda()
        self.q_off = torch.tensor([0] + torch.tensor(self.new).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        shape = (self.n_blocks, hkv, 16, d)
        if kv == "random":
            self.kb, self.vb = rand(shape, dtype, seed + 1), rand(shape, dtype, seed + 2)
        else:
            self.kb, self.vb = (torch.empty(shape, dtype=dtype, device="cuda") for _ in range(2))

    def poison(self):
        """NaN in every slot that no sequence fills."""
        free = torch.ones((self.n_blocks, 16), dtype=torch.bool)
        for b, L in enumerate(self.lens):
            for i in range(0, L, 16):
                free[int(self.table[b, i // 16]), : min(16, L - i)] = False
        free = free.cuda()
        for x in (self.kb, self.vb):
            x.masked_fill_(free[:, None, :, None], float("nan"))

    def pool(self, hq, **kw):
        return misat().KvPool(self.kb, self.vb, n_q_heads=hq, **kw)

    def batch(self, pool):
        return pool.batch(self.q_off, self.kv_len, self.table, n_tokens=self.T, max_q=max(self.new + [0]))


# ---- rotary ----

ROTARY = [  # heads, d, rot, half
    (1, 2, 2, True), (3, 16, 16, True), (4, 64, 64, True), (4, 64, 64, False), (7, 80, 40, True), (5, 96, 48, False),
    (2, 128, 6, True), (2, 128, 6, False), (3, 13, 10, True), (3, 13, 10, False), (32, 128, 128, True),
    (1, 1024, 1024, True), (40, 256, 64, False),
]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,d,rot,half", ROTARY)
@pytest.mark.parametrize("n", [1, 9, 600])
def test_rotary_layouts(n, heads, d, rot, half, dtype):
    m = misat()
    x = rand((n, heads, d), dtype, n + d)
    g = torch.Generator(device="cuda").manual_seed(n)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[-1] = (1 << 20) - 1
    pos[0] = 0
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    f = ref.frequencies(rot)
    y, tol = ref.rotate(x, pos, f, half)
    ref.assert_within("rotate", rope.rotate(x, pos), y, tol)
    y, tol = ref.rotate(x, pos, f, half, backward=True)
    ref.assert_within("backward", rope.backward(x, pos), y, tol)


@pytest.mark.parametrize("scaling,factor,attn", [(1, 4.0, 1.0), (1, 0.25, 1.0), (2, 8.0, 1.2079), (2, 32.0, 1.0)])
def test_rotary_scaling(scaling, factor, attn):
    m = misat()
    x = rand((257, 8, 128), F32, 3)
    pos = torch.arange(257, device="cuda", dtype=torch.int32) * 4093
    kw = dict(base=500000.0, scaling=scaling, factor=factor, orig_len=8192.0, beta_slow=1.0, beta_fast=4.0)
    rope = m.Rope(128, attn_factor=attn, **kw)
    y, tol = ref.rotate(x, pos, ref.frequencies(128, **kw), True, attn)
    ref.assert_within("rotate", rope.rotate(x, pos), y, tol)


@pytest.mark.parametrize("half", [True, False])
def test_rotary_strides_and_in_place(half):
    m = misat()
    rope = m.Rope(48, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    f = ref.frequencies(48)
    n, heads, d = 37, 5, 64
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 11
    wide = rand((n, heads * d + 200), BF16, 5)
    for x in (wide[:, 8:8 + heads * d].view(n, heads, d),          # aligned rows of a wider tensor
              wide[:, 3:3 + heads * d].view(n, heads, d),          # rows at odd elements
              rand((heads, n, d), BF16, 6).transpose(0, 1),        # heads outermost
              rand((n, heads, d), BF16, 7)[::2][:10],              # every other token
              rand((1, heads, d), BF16, 8).expand(n, heads, d),    # one row read by every token
              rand((n, 1, d), BF16, 9).expand(n, heads, d)):       # one head read as all
        y, tol = ref.rotate(x, pos[:x.shape[0]], f, half)
        ref.assert_within("strided", rope.rotate(x, pos[:x.shape[0]]), y, tol)
    full = rand((n, heads * d + 200), BF16, 10)
    before = full.clone()
    view = full[:, 3:3 + heads * d].view(n, heads, d)
    y, tol = ref.rotate(view, pos, f, half)
    rope.rotate(view, pos, out=view)
    ref.assert_within("in place", view, y, tol)
    assert torch.equal(full[:, :3], before[:, :3]) and torch.equal(full[:, 3 + heads * d:], before[:, 3 + heads * d:])


def test_rotary_gradient_against_differences():
    m = misat()
    kw = dict(scaling=m.ROPE_SCALE_BY_PARTS, factor=4.0, orig_len=2048.0, attn_factor=1.1)
    rope = m.Rope(12, layout=m.ROPE_INTERLEAVED, **kw)
    pos = torch.tensor([0, 1, 77, 100000], device="cuda", dtype=torch.int32)
    x, dy = rand((4, 2, 20), F32, 1), rand((4, 2, 20), F32, 2)
    grad = rope.backward(dy, pos).double()
    for i in range(0, x.numel(), 7):
        e = torch.zeros_like(x).view(-1)
        e[i] = 1.0
        e = e.view_as(x)
        # the map is linear: a difference of any step is exact up to rounding
        diff = (rope.rotate(x + e, pos).double() - rope.rotate(x - e, pos).double()) / 2
        want = (diff * dy.double()).sum()
        # six roundings to 32 bits of values below 8, times |dy| < 4, over the pair
        assert abs(grad.view(-1)[i] - want) < 2 * 4 * 8 * 6 * 2.0 ** -23


def test_rotary_positions_far_out_and_negative():
    m = misat()
    x = rand((6, 2, 64), F32, 1)
    far = [2 ** 31 - 1, -(2 ** 31), -1, 123456789, 1 << 24, (1 << 24) + 1]
    pos = torch.tensor(far, device="cuda", dtype=torch.int32)
    y, tol = ref.rotate(x, pos, ref.frequencies(64), True)
    # the 64-bit angle of the definition itself is only good to 2^31 * 2^-53 radians
    ref.assert_within("rotate", m.Rope(64).rotate(x, pos), y, tol + 2.0 ** -21 * x.double().abs().cpu().amax())


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d,rot,half", [(24, 10, False), (24, 10, True), (72, 34, False), (96, 48, False),
                                        (16, 2, False)])
def test_rotary_copies_the_rest_bit_for_bit(d, rot, half, dtype):
    m = misat()
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED, attn_factor=1.25)
    pos = torch.arange(9, device="cuda", dtype=torch.int32) * 1001
    x = rand((9, 3, d), dtype, 3)
    odd = torch.tensor([float("inf"), -0.0, float("nan"), 1.5, -float("inf"), -1.0, 0.0], dtype=dtype, device="cuda")
    n = 9 * 3 * (d - rot)
    x[..., rot:] = odd[torch.arange(n, device="cuda") % 7].view(9, 3, d - rot)
    bits = torch.int32 if dtype == F32 else torch.int16
    for y in (rope.rotate(x, pos), rope.backward(x, pos)):
        assert torch.equal(y[..., rot:].contiguous().view(bits), x[..., rot:].contiguous().view(bits))
        assert y[..., :rot].isfinite().all()


def test_rotary_empty():
    m = misat()
    rope = m.Rope(16)
    p0 = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert rope.rotate(torch.zeros((0, 4, 16), device="cuda"), p0).shape == (0, 4, 16)


# ---- append ----


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,rot,half", [(4, 4, 64, 64, True), (28, 4, 128, 128, False), (6, 2, 80, 40, True),
                                               (3, 1, 8, 6, True), (8, 8, 24, 10, False), (4, 2, 72, 0, True)])
def test_append(hq, hkv, d, rot, half, dtype):
    m = misat()
    seqs = [(1, 1), (1, 16), (1, 17), (0, 5), (40, 40), (33, 100), (0, 0), (200, 1000), (15, 31)]
    s = Step(seqs, hkv, d, dtype)
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED) if rot else None
    pool = s.pool(hq, rope=rope)
    qkv = rand((s.T, (hq + 2 * hkv) * d), dtype, 4)
    q = qkv[:, :hq * d].view(s.T, hq, d)
    k = qkv[:, hq * d:(hq + hkv) * d].view(s.T, hkv, d)
    v = qkv[:, (hq + hkv) * d:].view(s.T, hkv, d)
    kb0, vb0 = s.kb.clone(), s.vb.clone()
    q_out = pool.append(s.batch(pool), k, v, q=q)
    pool.sync()
    pos = torch.cat([torch.arange(L - n, L) for n, L in seqs])
    f = ref.frequencies(rot) if rot else torch.zeros(0, dtype=torch.float64)
    y, tol = ref.rotate(q, pos, f, half)
    ref.assert_within("q", q_out, y, tol)
    ky, ktol = ref.rotate(k, pos, f, half)
    want_k, want_v, kt = kb0.double().cpu(), vb0.clone(), torch.zeros(kb0.shape, dtype=torch.float64)
    t = 0
    for b, (n, L) in enumerate(seqs):
        for p in range(L - n, L):
            blk = int(s.table[b, p // 16])
            want_k[blk, :, p % 16], kt[blk, :, p % 16] = ky[t], ktol[t]
            want_v[blk, :, p % 16] = v[t]
            t += 1
    ref.assert_within("k", s.kb, want_k, kt)  # tolerance zero in every other slot
    assert torch.equal(s.vb, want_v)
    # without queries; in place; keys and values in other layouts
    s.kb.copy_(kb0)
    s.vb.copy_(vb0)
    pool.append(s.batch(pool), k.transpose(0, 1).contiguous().transpose(0, 1), v.contiguous())
    ref.assert_within("k", s.kb, want_k, kt)
    assert torch.equal(s.vb, want_v)
    pool.append(s.batch(pool), k, v, q=q, q_out=q)
    ref.assert_within("q in place", q, y, tol)


def test_append_malformed_is_a_sticky_error_and_writes_nothing_else():
    m = misat()
    s = Step([(4, 20), (3, 9), (2, 40)], 2, 32, BF16)
    pool = s.pool(2)
    k, v = rand((s.T, 2, 32), BF16, 1), rand((s.T, 2, 32), BF16, 2)
    kb0 = s.kb.clone()
    good = s.table.clone()
    for what in ("block", "negative", "length"):
        s.kb.copy_(kb0)
        s.table.copy_(good)
        s.kv_len.copy_(torch.tensor([20, 9, 40]))
        if what == "block":
            s.table[1, 0] = s.n_blocks
        elif what == "negative":
            s.table[1, 0] = -1
        else:
            s.kv_len[1] = 2
        pool.append(s.batch(pool), k, v)
        with pytest.raises(m.MisatError) as e:
            pool.sync()
        assert e.value.code == m.ERR_INVALID_ARG
        pool.sync()  # cleared
        want = kb0.clone()
        for b, lo, n in ((0, 0, 4), (2, 7, 2)):
            for i in range(n):
                p = s.lens[b] - n + i
                want[int(good[b, p // 16]), :, p % 16] = k[lo + i]
        if what == "length":  # tokens at positions -1, 0, 1: the sequence is skipped whole
            assert torch.equal(s.kb, want)
        else:
            assert torch.equal(s.kb, want)


# ---- attention ----


def check_attend(seqs, hq, hkv, d, dtype, window=0, scale=0.0, std=1.5, poison=True, seed=1):
    s = Step(seqs, hkv, d, dtype, seed=seed)
    q = rand((s.T, hq, d), dtype, seed + 5, std)
    want = ref.attend(q, s.kb, s.vb, s.new, s.lens, s.table, scale or None, window)
    if poison:
        s.poison()
    pool = s.pool(hq, scale=scale)
    batch = s.batch(pool)
    out, lse = pool.attend(batch, q, window=window, return_lse=True)
    pool.sync()
    ref.assert_within("out", out, want[0], want[1])
    ref.assert_within("lse", lse, want[2], want[3])
    again = pool.attend(batch, q, window=window)
    assert torch.equal(again, out)  # the same bits on every call
    return s, q, out


HEADS = [(1, 1, 8), (4, 4, 64), (6, 2, 80), (28, 4, 128), (32, 1, 128), (128, 1, 64), (8, 8, 104), (5, 1, 32)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_attend_single_tokens(hq, hkv, d, dtype):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 3, 700]
    check_attend([(1, L) for L in lens], hq, hkv, d, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_attend_chunks(hq, hkv, d, dtype):
    seqs = [(1, 1), (2, 2), (5, 300), (128, 128), (129, 129), (17, 33), (0, 64), (300, 301), (64, 1025), (1, 513),
            (0, 0), (31, 31)]
    check_attend(seqs, hq, hkv, d, dtype)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 1, 128), (3, 1, 72)])
def test_attend_window(hq, hkv, d, window):
    check_attend([(1, 1), (1, 129), (1, 900), (300, 300), (100, 700), (3, 140), (257, 640)], hq, hkv, d, BF16, window)


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 1, 128)])
def test_attend_rows_without_keys(hq, hkv, d):
    """Positions below zero (more new tokens than the sequence holds) and sequences of length zero."""
    s, q, out = check_attend([(5, 0), (10, 3), (1, 0), (300, 20), (140, 139), (2, 50)], hq, hkv, d, F16)
    assert torch.all(out[:5] == 0) and torch.all(out[5:12] == 0)


@pytest.mark.parametrize("n,hist", [(1, 40000), (2, 20001), (100, 9000), (300, 5000)])
def test_attend_long_histories(n, hist):
    """One or a few rows over a long axis, split between CTAs and joined."""
    check_attend([(n, hist + n)], 8, 2, 128, BF16)
    check_attend([(n, hist + n), (1, 3), (n, hist // 3 + n)], 16, 2, 64, F16)


def test_attend_many_ragged_sequences():
    g = torch.Generator().manual_seed(5)
    seqs = []
    for i in range(700):
        n = 1 if i % 3 else int(torch.randint(0, 40, (1,), generator=g))
        seqs.append((n, n + int(torch.randint(0, 300, (1,), generator=g))))
    check_attend(seqs, 4, 2, 64, BF16, poison=False)


@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 64), (12, 3, 128), (10, 5, 72), (4, 1, 64)])
def test_attend_many_single_tokens(hq, hkv, d, window):
    """Several whole items a processor, two heads at a time; odd numbers of heads, and of blocks."""
    g = torch.Generator().manual_seed(d)
    seqs = [(1, int(torch.randint(1, 600 if i % 7 == 0 else 140, (1,), generator=g))) for i in range(333)]
    check_attend(seqs, hq, hkv, d, BF16, window)
    check_attend([(n + i % 3, L + i % 3) for i, (n, L) in enumerate(seqs)][:200], hq, hkv, d, F16, window)


@pytest.mark.parametrize("hq,hkv,d,window", [(16, 8, 64, 0), (8, 8, 128, 200), (28, 4, 128, 0)])
def test_attend_more_items_than_processors(hq, hkv, d, window):
    """Batches whose items a processor takes several of, in an order that is not theirs."""
    g = torch.Generator().manual_seed(hq)
    seqs = []
    for i in range(60):
        n = [1, 0, 77, 300, 129][i % 5] + int(torch.randint(0, 30, (1,), generator=g)) * (i % 2)
        seqs.append((n, n + int(torch.randint(0, 1500, (1,), generator=g)) * (i % 3)))
    check_attend(seqs, hq, hkv, d, BF16, window)
    check_attend(seqs * 5, hq, hkv, d, F16, window, poison=False)  # 300 sequences


@pytest.mark.parametrize("order", ["rising", "falling", "spikes"])
def test_attend_maxima_that_move(order):
    """Scores whose running maximum moves a little, a lot, or far below what came before."""
    d, hq, L, n = 64, 2, 1500, 150
    s = Step([(n, L)], 1, d, BF16)
    q = torch.zeros((n, hq, d), dtype=BF16, device="cuda")
    q[..., 0] = 8.0
    ramp = torch.arange(L, device="cuda").float()
    x = {"rising": ramp * 0.25, "falling": -ramp * 0.25, "spikes": torch.where(ramp % 211 == 7, ramp, -500.0)}[order]
    k = rand((L, d), BF16, 3, 0.1)
    k[:, 0] = x.to(BF16)
    pos = torch.arange(L, device="cuda")
    s.kb[s.table[0, pos // 16].long(), 0, pos % 16] = k
    s.poison()
    want = ref.attend(q, s.kb.nan_to_num(), s.vb.nan_to_num(), s.new, s.lens, s.table)
    pool = s.pool(hq)
    out, lse = pool.attend(s.batch(pool), q, return_lse=True)
    ref.assert_within("out", out, want[0], want[1])
    ref.assert_within("lse", lse, want[2], want[3])


def test_attend_scale_and_strides():
    hq, hkv, d = 6, 2, 64
    seqs = [(1, 77), (40, 200), (3, 3)]
    check_attend(seqs, hq, hkv, d, BF16, scale=0.5)
    s = Step(seqs, hkv, d, BF16)
    pool = s.pool(hq)
    batch = s.batch(pool)
    q = rand((s.T, hq, d), BF16, 9)
    want = pool.attend(batch, q)
    wide = rand((s.T, hq * d + 37), BF16, 10)
    for view in (wide[:, 16:16 + hq * d].view(s.T, hq, d), wide[:, 5:5 + hq * d].view(s.T, hq, d),
                 rand((hq, s.T, d), BF16, 11).transpose(0, 1)):
        view.copy_(q)
        assert torch.equal(pool.attend(batch, view), want)
        keep = torch.zeros((s.T, hq * d + 37), dtype=BF16, device="cuda")
        res = keep[:, 7:7 + hq * d].view(s.T, hq, d)
        pool.attend(batch, view, out=res)
        assert torch.equal(res, want)
        assert torch.all(keep[:, :7] == 0) and torch.all(keep[:, 7 + hq * d:] == 0)


def test_attend_offsets_beyond_32_bits():
    """The used blocks lie past 2^32 elements of the pool."""
    hkv, d = 8, 128
    n_blocks = (1 << 32) // (hkv * 16 * d) + 300
    s = Step([(1, 700), (20, 900)], hkv, d, BF16, n_blocks=n_blocks, kv="empty")
    small = torch.arange(n_blocks - 200, n_blocks, device="cuda")
    s.kb[small], s.vb[small] = rand((200, hkv, 16, d), BF16, 1), rand((200, hkv, 16, d), BF16, 2)
    assert int(s.table[0, 0]) > n_blocks - 200
    m = misat()
    rope = m.Rope(d)
    pool = s.pool(16, rope=rope)
    batch = s.batch(pool)
    q = rand((s.T, 16, d), BF16, 3)
    k, v = rand((s.T, hkv, d), BF16, 4), rand((s.T, hkv, d), BF16, 5)
    qr = pool.append(batch, k, v, q=q)
    out = pool.attend(batch, qr)
    pool.sync()
    pos = torch.tensor([699] + list(range(880, 900)))
    ky, ktol = ref.rotate(k, pos, ref.frequencies(d), True)
    ref.assert_within("k", ref.gather(s.kb, s.table[1], 900)[880:], ky[1:], ktol[1:])
    tiny = torch.cat([s.table[0, :44], s.table[1, :57]]).long()
    tab = torch.full((2, 57), 0, dtype=torch.int32, device="cuda")
    tab[0, :44], tab[1] = torch.arange(44), torch.arange(44, 101)
    want = ref.attend(qr, s.kb[tiny], s.vb[tiny], s.new, s.lens, tab)
    ref.assert_within("out", out, want[0], want[1])


def test_attend_malformed_is_a_sticky_error():
    m = misat()
    s = Step([(4, 20), (3, 9), (2, 40)], 2, 32, BF16)
    pool = s.pool(2)
    q = rand((s.T, 2, 32), BF16, 1)
    good = pool.attend(s.batch(pool), q)
    table, lens = s.table.clone(), s.kv_len.clone()
    for what in ("block", "negative", "length", "offsets"):
        s.table.copy_(table)
        s.kv_len.copy_(lens)
        off = s.q_off.clone()
        if what == "block":
            s.table[1, 0] = s.n_blocks
        elif what == "negative":
            s.table[1, 0] = -1
        elif what == "length":
            s.kv_len[1] = 16 * s.table.shape[1] + 1
        else:
            s.q_off[1:3] = torch.tensor([1 << 30, 7])
        out = pool.attend(s.batch(pool), q)
        with pytest.raises(m.MisatError) as e:
            pool.sync()
        assert e.value.code == m.ERR_INVALID_ARG
        s.q_off.copy_(off)
        if what != "offsets":
            assert torch.equal(out[:4], good[:4]) and torch.equal(out[7:], good[7:])
        pool.sync()


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("skip", ["front", "back", "all"])
def test_attend_tokens_of_no_sequence_are_a_sticky_error(skip, n):
    m = misat()
    s = Step([(1, 20)] * n, 2, 64, BF16)
    pool = s.pool(4)
    q = rand((n, 4, 64), BF16, 1)
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    if skip == "front":
        off[0] = 1
    elif skip == "back":
        off[n] = n - 1
    else:
        off.zero_()
    lens = torch.full((n,), 21, dtype=torch.int32, device="cuda")
    pool.attend(pool.batch(off, lens, s.table.cuda(), n_tokens=n, max_q=1), q)
    with pytest.raises(m.MisatError) as e:
        pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    pool.sync()


def test_calls_on_other_streams_and_in_a_graph():
    m = misat()
    s = Step([(1, 3000), (40, 200)], 2, 64, BF16)
    pool = s.pool(4, rope=m.Rope(64))
    batch = s.batch(pool)
    q, k, v = rand((s.T, 4, 64), BF16, 1), rand((s.T, 2, 64), BF16, 2), rand((s.T, 2, 64), BF16, 3)
    qr = pool.append(batch, k, v, q=q)
    want = pool.attend(batch, qr)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a = pool.attend(batch, pool.append(batch, k, v, q=q))
        b = pool.attend(batch, qr)
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g_out = pool.attend(batch, pool.append(batch, k, v, q=q))
    s.kb.zero_()
    s.vb.zero_()
    first = pool.attend(batch, pool.append(batch, k, v, q=q))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g_out, first)


def test_empty_batches():
    s = Step([(0, 5), (0, 0)], 2, 64, BF16)
    pool = s.pool(4)
    out = pool.attend(s.batch(pool), torch.empty((0, 4, 64), dtype=BF16, device="cuda"))
    assert out.shape == (0, 4, 64)
    pool.append(s.batch(pool), *(torch.empty((0, 2, 64), dtype=BF16, device="cuda") for _ in range(2)))
    pool.sync()


# ---- refusals ----


def test_refused_arguments():
    m = misat()
    for kw in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=2000), dict(rot_dim=8, layout=2),
               dict(rot_dim=8, base=1.0), dict(rot_dim=8, base=float("nan")), dict(rot_dim=8, scaling=3),
               dict(rot_dim=8, scaling=1, factor=0.0), dict(rot_dim=8, scaling=2, factor=2.0),
               dict(rot_dim=8, scaling=2, factor=2.0, orig_len=10.0, beta_slow=4.0, beta_fast=4.0),
               dict(rot_dim=8, attn_factor=float("inf"))):
        with pytest.raises(m.MisatError) as e:
            m.Rope(**kw)
        assert e.value.code == m.ERR_INVALID_ARG
    rope = m.Rope(16)
    x, pos = rand((4, 2, 16), BF16, 1), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in ((x, pos.long()), (x, pos[:3]), (x.transpose(0, 2), pos), (x.double(), pos), (x.cpu(), pos),
                (x[0], pos)):
        with pytest.raises(ValueError):
            rope.rotate(*bad)
    with pytest.raises(m.MisatError):  # fewer elements than the rotated part
        rope.rotate(rand((4, 2, 8), BF16, 1), pos)
    with pytest.raises(ValueError):
        rope.rotate(x, pos, out=torch.empty_like(x, dtype=F16))

    def blocks(n=4, h=2, d=32, dt=BF16):
        return [torch.zeros((n, h, 16, d), dtype=dt, device="cuda") for _ in range(2)]

    for kw, b in ((dict(n_q_heads=3), blocks()), (dict(n_q_heads=0), blocks()), (dict(n_q_heads=2 * 129), blocks()),
                  (dict(n_q_heads=2), blocks(d=136)), (dict(n_q_heads=2), blocks(d=36)),
                  (dict(n_q_heads=2), blocks(dt=F32)), (dict(n_q_heads=2, scale=-1.0), blocks()),
                  (dict(n_q_heads=2, max_batch=0), blocks()), (dict(n_q_heads=2, rope=m.Rope(64)), blocks())):
        with pytest.raises(m.MisatError) as e:
            m.KvPool(*b, **kw)
        assert e.value.code == m.ERR_INVALID_ARG
    kb, vb = blocks()
    for bad in ((kb, vb[:2]), (kb.transpose(1, 2), vb.transpose(1, 2)), (kb, vb.to(F16)), (kb.cpu(), vb.cpu())):
        with pytest.raises(ValueError):
            m.KvPool(*bad, n_q_heads=2)
    s = Step([(2, 20), (1, 5)], 2, 32, BF16)
    pool = s.pool(4, max_batch=2)
    batch = s.batch(pool)
    q, k = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 1)
    for call in (lambda: pool.attend(batch, q[:2]), lambda: pool.attend(batch, q.to(F16)),
                 lambda: pool.attend(batch, k), lambda: pool.append(batch, k, k[:2]),
                 lambda: pool.append(batch, q, q), lambda: pool.append(batch, k, k, q=k),
                 lambda: pool.batch(s.q_off[:2], s.kv_len, s.table, n_tokens=3, max_q=2),
                 lambda: pool.batch(s.q_off, s.kv_len.long(), s.table, n_tokens=3, max_q=2),
                 lambda: pool.batch(s.q_off, s.kv_len, s.table[0], n_tokens=3, max_q=2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(m.MisatError):
        pool.attend(batch, q, window=-1)
    other = m.KvPool(*blocks(h=1), n_q_heads=4)  # a batch made for other heads
    with pytest.raises(ValueError):
        other.attend(batch, q)
    with pytest.raises(ValueError):
        other.append(batch, k, k)
    small = s.pool(4, max_batch=1)
    with pytest.raises(m.MisatError):
        small.attend(s.batch(small), q)


def test_null_and_misaligned_pointers_are_refused_by_the_library():
    m = misat()
    s = Step([(1, 20)], 2, 32, BF16)
    pool = s.pool(2)
    b = s.batch(pool)
    q = rand((1, 2, 32), BF16, 1)
    p = q.data_ptr()
    st = torch.cuda.current_stream().cuda_stream
    f = m._lib.misat_kv_attend
    assert f(pool._h, b._ref, None, 64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    assert f(pool._h, b._ref, p + 1, 64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    assert f(pool._h, b._ref, p, -64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    assert f(pool._h, b._ref, p, 64, 32, p, 64, 32, p + 2, 0, st) == m.ERR_INVALID_ARG
    assert f(None, b._ref, p, 64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    assert f(pool._h, None, p, 64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    a = m._lib.misat_kv_append
    assert a(pool._h, b._ref, p, 64, 32, None, 64, 32, None, 0, 0, None, 0, 0, st) == m.ERR_INVALID_ARG
    assert a(pool._h, b._ref, p, 64, 32, p, 64, 32, p, 64, 32, None, 0, 0, st) == m.ERR_INVALID_ARG
    assert m._lib.misat_rotary(None, 0, 1, 1, 16, p, 16, 16, p, p, 16, 16, 0, st) == m.ERR_INVALID_ARG
    # results whose heads or tokens would share a place
    assert f(pool._h, b._ref, p, 64, 32, p, 64, 0, None, 0, st) == m.ERR_INVALID_ARG
    rope = m.Rope(16)
    for ts, hs in ((0, 16), (32, 0)):
        assert m._lib.misat_rotary(rope._h, 0, 2, 2, 16, p, 32, 16, s.kv_len.data_ptr(), p, ts, hs, 0, st) == \
            m.ERR_INVALID_ARG
    assert m._lib.misat_kv_create(None, ctypes.byref(ctypes.c_void_p())) == m.ERR_INVALID_ARG
