"""A step's operators where offsets pass 32 bits, and on several streams at once."""

import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as kref  # noqa: E402
from tests import kv_step_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, F32, Step, misat, rand  # noqa: E402
from tests.test_gpu_kv_tree import ints, parents_of  # noqa: E402

pytestmark = pytest.mark.gpu


def test_blocks_beyond_32_bits():
    """Append, attention and kept paths in the last blocks of a pool of more than 2^31 elements."""
    m = misat()
    hkv, d, hq, n_blocks = 8, 128, 16, 140_000
    assert n_blocks * hkv * 16 * d > 2 ** 31
    s = Step([(20, 300), (7, 7), (33, 90)], hkv, d, BF16, n_blocks=n_blocks, kv="empty")
    for x in (s.kb, s.vb):
        x[-64:] = rand((64, hkv, 16, d), BF16, 3)
    pool = s.pool(hq, rope=m.Rope(d))
    batch = s.batch(pool)
    parents = parents_of(s.new, 5)
    tree = pool.tree(batch, ints(parents))
    x = rand((s.T, hq + 2 * hkv, d), BF16, 1)
    w = rand((d,), F32, 2) + 1
    q = pool.append(batch, x[:, hq:hq + hkv], x[:, hq + hkv:], q=x[:, :hq], k_norm=m.HeadNorm(w), tree=tree)
    depth, sees = ref.tree(s.new, parents)
    seq = torch.tensor([b for b, n in enumerate(s.new) for _ in range(n)], device="cuda")
    slot = torch.tensor([L - n + i for n, L in zip(s.new, s.lens) for i in range(n)], device="cuda")
    pos = torch.tensor([L - n for n, L in zip(s.new, s.lens) for i in range(n)], device="cuda") + torch.tensor(depth).cuda()
    f = kref.frequencies(d)
    kref.assert_within("q", q, *ref.norm_rotate(x[:, :hq], pos, f, True, None))
    blk = s.table[seq, slot // 16].long()
    assert int(blk.min()) * hkv * 16 * d > 2 ** 31
    kref.assert_within("k", s.kb[blk, :, slot % 16], *ref.norm_rotate(x[:, hq:hq + hkv], pos, f, True, w))
    assert torch.equal(s.vb[blk, :, slot % 16], x[:, hq + hkv:])
    out = pool.attend(batch, q, tree=tree)
    o, ot, _, _ = ref.attend(q, s.kb, s.vb, s.new, s.lens, s.table, depth, sees)
    kref.assert_within("out", out, o, ot)
    before = s.kb[blk, :, slot % 16].clone()
    pool.keep(batch, ints([[1, 2, 19], [0, 5, 6], [4, 30, 32]]), ints([3, 3, 3]))
    pool.sync()
    after = s.kb[blk, :, slot % 16]
    for first, path in ((0, (1, 2, 19)), (20, (0, 5, 6)), (27, (4, 30, 32))):
        assert torch.equal(after[first:first + 3], before[[first + i for i in path]])


def test_heads_beyond_32_bits():
    m = misat()
    n, heads, d = 150_000, 128, 128
    x = torch.zeros((n, heads, d), dtype=BF16, device="cuda")
    dy = torch.zeros_like(x)
    assert x.numel() > 2 ** 31
    at = [0, 1, n // 2, n - 2, n - 1]
    x[at], dy[at] = rand((5, heads, d), BF16, 1), rand((5, heads, d), BF16, 2)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    w = rand((d,), F32, 3) + 1
    rope, norm, f = m.Rope(d), m.HeadNorm(w), kref.frequencies(d)
    y = rope.norm_rotate(x, pos, norm)
    kref.assert_within("rotate", y[at], *ref.norm_rotate(x[at], pos[at], f, True, w))
    del y
    dx, dw = rope.norm_backward(x, dy, pos, norm, out=dy.clone())
    want = ref.norm_backward(x[at], dy[at], pos[at], f, True, w)
    kref.assert_within("dx", dx[at], *want[:2])
    kref.assert_within("dw", dw, *want[2:])  # (zeros add nothing, in whatever order)


def test_table_rows_beyond_32_bits():
    m = misat()
    n, columns = 5000, 450_000
    table = torch.full((n, columns), -7, dtype=torch.int32, device="cuda")
    assert table.numel() > 2 ** 31
    kb, vb = (torch.zeros((n + 10, 1, 16, 8), dtype=BF16, device="cuda") for _ in range(2))
    pool = m.KvPool(kb, vb, n_q_heads=1)
    free = torch.arange(n + 10, dtype=torch.int32, device="cuda")
    t = m.KvTables(pool, table, free)
    new, zero = torch.ones(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    s = t.step(t.initial(n + 10), new, zero, n_tokens=n, max_q=1)
    pool.sync()
    assert torch.equal(table[:, 0], free[:n]) and (table[:, 1] == -7).all()
    assert torch.equal(s.slots, free[:n].long() * 16) and not s.positions.any()
    last = t.step(s.state, zero, zero, n_tokens=0, max_q=0)
    pool.sync()
    assert last.state[:n].max() == 0 and last.state.tolist()[-1] == n + 10
    assert torch.equal(free.sort().values, torch.arange(n + 10, dtype=torch.int32, device="cuda"))


def test_streams_at_once():
    """Norms on two streams at a time (they share nothing), and a pool's steps that change streams from call to call."""
    m = misat()
    streams = [torch.cuda.Stream() for _ in range(3)]
    x, dy = rand((5000, 8, 64), BF16, 1), rand((5000, 8, 64), BF16, 2)
    pos = torch.arange(5000, dtype=torch.int32, device="cuda")
    rope, norm = m.Rope(64), m.HeadNorm(rand((64,), F32, 3))
    want = rope.norm_backward(x, dy, pos, norm)
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(rope.norm_backward(x, dy, pos, norm))
    torch.cuda.synchronize()
    assert all(torch.equal(a[0], want[0]) and torch.equal(a[1], want[1]) for a in got)
    n = 30
    kb, vb = (torch.zeros((400, 2, 16, 64), dtype=BF16, device="cuda") for _ in range(2))
    pool = m.KvPool(kb, vb, n_q_heads=4)
    t = m.KvTables(pool, torch.zeros((n, 12), dtype=torch.int32, device="cuda"), torch.arange(400, dtype=torch.int32,
                                                                                          device="cuda"))
    state, lens, table, ring = t.initial(400), ints([0] * n), [[0] * 12 for _ in range(n)], list(range(400))
    par, new = ints(parents_of([5] * n, 2)), ints([5] * n)
    path, many = ints([[0, 3]] * n), ints([2] * n)
    q, k = rand((5 * n, 4, 64), BF16, 4), rand((5 * n, 2, 64), BF16, 5)
    torch.cuda.synchronize()
    s, L = state.tolist(), [0] * n
    for i in range(40):  # every call on the next stream, ordered by the pool alone
        with torch.cuda.stream(streams[i % 3]):
            step = t.step(state, new, lens, n_tokens=5 * n, max_q=5, out=state)
        with torch.cuda.stream(streams[(i + 1) % 3]):
            tree = pool.tree(step, par)
        with torch.cuda.stream(streams[(i + 2) % 3]):
            pool.append(step, k, k, tree=tree)
        with torch.cuda.stream(streams[i % 3]):
            out = pool.attend(step, q, tree=tree)
            lens = pool.keep(step, path, many)
        if i % 13 == 12:
            streams[i % 3].synchronize()
            assert torch.isfinite(out).all()
        s, _, _, _, slots = ref.tables(n, [5] * n, L, s, table, ring)
        L = [x + 2 for x in L]
    streams[39 % 3].synchronize()
    assert state.tolist() == s and lens.tolist() == L and step.slots.tolist() == slots
    pool.sync()


def test_a_closed_rotation_is_refused():
    m = misat()
    rope, norm = m.Rope(16), m.HeadNorm(torch.ones(16, device="cuda"))
    x, pos = rand((2, 1, 16), BF16, 1), ints([0, 1])
    rope.norm_rotate(x, pos, norm)
    rope.close()
    with pytest.raises(ValueError):
        rope.norm_rotate(x, pos, norm)
    with pytest.raises(ValueError):
        rope.norm_backward(x, x, pos, norm)
