"""Trees of drafted tokens on KV blocks: their plan, the attention of their nodes, and what is kept of them."""

import math
import random

import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as kref  # noqa: E402
from tests import kv_step_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, F16, Step, misat, rand  # noqa: E402

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def parents_of(new, seed, shape="random", absent=0.0):
    r = random.Random(seed)
    out = []
    for n in new:
        there = n - (r.randint(0, n) if r.random() < absent else 0)
        for i in range(n):
            p = {"random": lambda: r.randint(-1, i - 1), "chain": lambda: i - 1, "roots": lambda: -1,
                 "wide": lambda: max(-1, i // 4 - 1), "late": lambda: -1 if i < n // 2 else r.randint(max(-1, i - 5), i - 1),
                 }[shape]() if i else -1
            out.append(p if i < there else ref.ABSENT)
    return out


# ---- the plan ----


@pytest.mark.parametrize("shape", ["random", "chain", "roots", "wide", "late"])
@pytest.mark.parametrize("window", [0, 1, 3, 33])
@pytest.mark.parametrize("new", [[1], [2, 0, 1], [31, 32, 33, 64, 65], [127, 128, 129, 200], [1024, 1, 1000], [7] * 300])
def test_plan(new, window, shape):
    s = Step([(n, n + 3) for n in new], 1, 8, BF16)
    pool = s.pool(1)
    parents = parents_of(new, len(new) + window, shape, 0.4)
    t = pool.tree(s.batch(pool), ints(parents), window=window)
    pool.sync()
    depth, sees = ref.tree(new, parents, window)
    words = -(-max(new) // 32)
    assert t.depth.tolist() == depth
    assert t.bits.shape == (sum(new), words) and torch.equal(t.bits.cpu(), ref.bits(sees, words))


@pytest.mark.parametrize("bad", [{3: 3}, {3: 5}, {2: -3}, {4: 2 ** 31 - 1}, {4: -2 ** 31}, {1: -2}])
def test_malformed_parents_are_a_sticky_error(bad):
    m = misat()
    s = Step([(4, 9), (6, 6), (5, 40)], 1, 8, BF16)
    pool = s.pool(1)
    parents = [-1, 0, 1, 2] + [-1, 0, 1, 2, 3, 4] + [-1, -1, 0, 1, 2]
    for i, p in bad.items():
        parents[4 + i] = p
    t = pool.tree(s.batch(pool), ints(parents))
    with pytest.raises(m.MisatError) as e:
        pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    first = min(bad)  # it and what hangs on it count as absent
    parents[4 + first:10] = [-2] * (6 - first)
    depth, sees = ref.tree(s.new, parents)
    assert t.depth.tolist() == depth and torch.equal(t.bits.cpu(), ref.bits(sees, 1))
    pool.sync()


def test_malformed_lengths_are_sticky_errors():
    m = misat()
    parents = ints([-1, 0, 1, -1, 0])
    for change in (lambda s: s.kv_len.fill_(1), lambda s: s.q_off.copy_(ints([0, 4, 3, 5])), lambda s: s.q_off.fill_(0),
                   lambda s: s.q_off.copy_(ints([0, 5, 5, 5])), lambda s: s.kv_len.fill_(2 ** 31 - 1),
                   lambda s: s.q_off.copy_(ints([1, 3, 3, 5]))):
        s = Step([(3, 7), (0, 4), (2, 9)], 1, 64, BF16)
        pool = s.pool(1)
        batch = s.batch(pool)
        q = rand((5, 1, 64), BF16, 1)
        good = pool.tree(batch, parents)
        pool.sync()
        change(s)
        path, many = ints([[0], [0], [0]]), ints([1, 0, 1])
        before = s.kb.clone()
        for call in (lambda: pool.tree(batch, parents), lambda: pool.keep(batch, path, many)):
            call()
            if call is not None and s.q_off.tolist() != [1, 3, 3, 5]:
                with pytest.raises(m.MisatError) as e:
                    pool.sync()
                assert e.value.code == m.ERR_INVALID_ARG
        if s.kv_len[0] != 1:  # (kv_len below the new tokens: nodes below position zero)
            pool.attend(batch, q, tree=good)
            with pytest.raises(m.MisatError) as e:
                pool.sync()
            assert e.value.code == m.ERR_INVALID_ARG
        assert torch.equal(s.kb, before)


# ---- attention ----

HEADS = [(4, 4, 64), (8, 1, 128), (6, 2, 72), (28, 4, 64), (32, 2, 128), (128, 1, 64), (3, 1, 8)]


def check(seqs, hq, hkv, d, dtype, shape="random", window=0, absent=0.0, seed=1, std=1.5, scale=None):
    s = Step(seqs, hkv, d, dtype, seed=seed)
    s.poison()
    pool = s.pool(hq, **({"scale": scale} if scale else {}))
    batch = s.batch(pool)
    parents = parents_of(s.new, seed, shape, absent)
    q = rand((s.T, hq, d), dtype, seed + 7, std)
    q[torch.tensor(parents, device="cuda") == ref.ABSENT] = math.nan  # unused rows hold anything
    tree = pool.tree(batch, ints(parents), window=window)
    out, lse = pool.attend(batch, q, return_lse=True, tree=tree)
    pool.sync()
    depth, sees = ref.tree(s.new, parents, window)
    o, ot, l, lt = ref.attend(q, s.kb, s.vb, s.new, s.lens, s.table, depth, sees, window, scale)
    kref.assert_within("out", out, o, ot)
    kref.assert_within("lse", lse, l, lt)
    assert torch.equal(pool.attend(batch, q, tree=tree), out)
    return s, pool, batch, tree, q, out


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("shape", ["random", "wide"])
def test_attend(hq, hkv, d, shape, dtype):
    check([(1, 1), (5, 5), (12, 140), (33, 33), (32, 127), (17, 128 + 17), (3, 700), (64, 300), (0, 9)], hq, hkv, d, dtype,
          shape)


@pytest.mark.parametrize("shape", ["random", "chain", "roots", "late"])
@pytest.mark.parametrize("n,L", [(1, 1), (1, 129), (2, 128), (31, 160), (32, 160), (33, 161), (96, 100), (127, 127), (128, 256),
                                 (129, 130), (130, 500), (255, 400), (257, 257), (600, 640), (1024, 1100)])
def test_attend_tree_sizes(n, L, shape):
    """Trees that begin and end anywhere in a block of keys, and are longer than one."""
    check([(n, L)], 2, 1, 64, BF16, shape)


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 1, 128), (3, 1, 72)])
@pytest.mark.parametrize("window", [1, 2, 5, 16, 100, 129, 1000])
def test_attend_window(hq, hkv, d, window):
    check([(1, 1), (9, 40), (40, 40), (33, 333), (130, 700), (200, 220)], hq, hkv, d, BF16, "late", window)
    check([(9, 40), (65, 1500), (150, 900)], hq, hkv, d, F16, "chain", window)


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("window", [0, 4])
def test_attend_absent_nodes(hq, hkv, d, window):
    check([(8, 8), (16, 40), (40, 41), (12, 4000), (130, 131), (1, 1), (5, 300)], hq, hkv, d, BF16, "random", window, 0.9,
          seed=4)
    check([(16, 30000)], hq, hkv, d, F16, "wide", window, 1.0, seed=2)


@pytest.mark.parametrize("n,hist", [(1, 40000), (60, 40000), (20, 9001), (250, 3000)])
def test_attend_long_histories(n, hist):
    """Items in parts, which the last of several CTAs joins."""
    check([(n, hist + n)], 8, 1, 128, BF16)
    check([(n, hist + n), (3, 50)], 8, 8, 64, F16, "late", 0, 0.5, seed=3)


def test_attend_many_ragged_sequences():
    r = random.Random(4)
    seqs = [(r.choice([0, 1, 4, 16, 33]), 0) for _ in range(300)]
    check([(n, n + r.choice([0, 1, 15, 130, r.randint(0, 900)])) for n, _ in seqs], 4, 1, 64, BF16, "random", 0, 0.2)


@pytest.mark.parametrize("window", [0, 5, 300])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 1, 128), (5, 1, 72)])
def test_a_chain_is_tokens_in_a_row(hq, hkv, d, window):
    """The same products and sums in the same order."""
    s = Step([(1, 9), (20, 20), (130, 400), (7, 3000), (64, 190)], hkv, d, BF16)
    pool = s.pool(hq)
    batch = s.batch(pool)
    q = rand((s.T, hq, d), BF16, 3)
    tree = pool.tree(batch, ints(parents_of(s.new, 0, "chain")), window=window)
    a, la = pool.attend(batch, q, window=window, return_lse=True)
    b, lb = pool.attend(batch, q, return_lse=True, tree=tree)
    pool.sync()
    if window:  # (other blocks are read where the window begins: any node may be a root)
        o, ot, l, lt = kref.attend(q, s.kb, s.vb, s.new, s.lens, s.table, window=window)
        kref.assert_within("out", b, o, ot)
        kref.assert_within("lse", lb, l, lt)
    else:
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_scale_strides_and_in_place():
    hq, hkv, d = 6, 2, 64
    s = Step([(5, 300), (40, 90)], hkv, d, BF16)
    pool = s.pool(hq, scale=0.03)
    batch = s.batch(pool)
    parents = parents_of(s.new, 1)
    tree = pool.tree(batch, ints(parents))
    depth, sees = ref.tree(s.new, parents)
    for pad in (0, 8, 3):
        wide = rand((s.T, hq + 2, d + pad), BF16, 5, 2.0)
        q = wide[:, 1:1 + hq, :d]
        o, ot, l, lt = ref.attend(q, s.kb, s.vb, s.new, s.lens, s.table, depth, sees, 0, 0.03)
        kref.assert_within("out", pool.attend(batch, q, tree=tree), o, ot)
        out = torch.empty((hq, s.T, d + pad), dtype=BF16, device="cuda").transpose(0, 1)[..., :d]
        got, lse = pool.attend(batch, q, out=out, return_lse=True, tree=tree)
        assert got is out
        kref.assert_within("out", out, o, ot)
        kref.assert_within("lse", lse, l, lt)
        assert pool.attend(batch, q, out=q, tree=tree) is q
        kref.assert_within("in place", q, o, ot)


def test_nodes_below_position_zero_see_nothing():
    m = misat()
    s = Step([(6, 6), (4, 30)], 1, 64, BF16)
    pool = s.pool(2)
    batch = s.batch(pool)
    q = rand((10, 2, 64), BF16, 1)
    tree = pool.tree(batch, ints([-1] * 10))
    want = pool.attend(batch, q, tree=tree)
    s.kv_len.copy_(ints([4, 30]))
    out, lse = pool.attend(batch, q, return_lse=True, tree=tree)
    pool.sync()
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()
    # node 2 is at position 0, whose key it sees alone
    assert torch.equal(out[2], s.vb[int(s.table[0, 0]), 0, 0].expand(2, 64)) and torch.equal(out[6:], want[6:])
    assert m.KV_TREE_NODES == 1024


def test_captured_on_another_stream_and_two_graphs_in_turn():
    s = Step([(12, 5000), (12, 40), (12, 900)], 2, 64, BF16)
    pool = s.pool(8)
    batch = s.batch(pool)
    q, par = rand((36, 8, 64), BF16, 1), ints(parents_of(s.new, 3))

    def step():
        tree = pool.tree(batch, par)
        return pool.attend(batch, q, tree=tree), tree.bits

    want = [x.clone() for x in step()]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = step()
        assert torch.equal(got[0], want[0])
    st.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            out = step()
        graphs.append((g, out))
    for seed in (5, 6):
        par.copy_(ints(parents_of(s.new, seed)))
        want = [x.clone() for x in step()]
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    # a plan made on one stream and used on another, and let go of at once
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        tree = pool.tree(batch, par)
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got = pool.attend(batch, q, tree=tree)
        del tree
        junk = [torch.full((36,), -1, dtype=torch.int32, device="cuda") for _ in range(4)]
        st.synchronize()
        assert torch.equal(got, want[0])
        del junk
    pool.sync()


# ---- what is kept ----


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hkv,d", [(1, 8), (8, 128), (3, 72), (40, 64)])
def test_keep(hkv, d, dtype):
    r = random.Random(hkv)
    new = [1, 1, 0, 7, 16, 33, 64, 200, 1024, 5, 40]
    s = Step([(n, n + r.randint(0, 50)) for n in new], hkv, d, dtype)
    s.vb.view(torch.int16)[:] = torch.randint(-2 ** 15, 2 ** 15, s.vb.shape, dtype=torch.int16, device="cuda")  # any bits
    pool = s.pool(hkv)
    paths = []
    for b, n in enumerate(new):
        m = r.randint(0, n) if b not in (1, 8) else n
        paths.append(sorted(r.sample(range(n), m)))
    paths[9] = [1, 2, 3, 4]  # every row is read before the one behind it comes to its place
    width = max(len(p) for p in paths)
    path = ints([p + [-5] * (width - len(p)) for p in paths])
    want = []
    for x in (s.kb, s.vb):
        y = x.clone()
        for b, p in enumerate(paths):
            P = s.lens[b] - new[b]
            for i, j in enumerate(p):
                y[int(s.table[b, (P + i) // 16]), :, (P + i) % 16] = x[int(s.table[b, (P + j) // 16]), :, (P + j) % 16]
        want.append(y)
    got = pool.keep(s.batch(pool), path, ints([len(p) for p in paths]))
    pool.sync()
    assert got.tolist() == [L - n + len(p) for L, n, p in zip(s.lens, new, paths)]
    for x, y in zip((s.kb, s.vb), want):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("bad", [dict(path=[0, 2, 2]), dict(path=[2, 1, 3]), dict(path=[0, 1, 6]), dict(path=[-1, 1, 2]),
                                 dict(many=-1), dict(many=4), dict(many=7), dict(block=-1), dict(block=10 ** 6)])
def test_a_malformed_path_leaves_its_sequence(bad):
    m = misat()
    s = Step([(5, 30), (6, 38), (4, 9)], 2, 16, BF16)
    pool = s.pool(2)
    batch = s.batch(pool)
    good = ints([[1, 2, 4], [1, 3, 5], [0, 1, 3]])
    before = [x.clone() for x in (s.kb, s.vb)]
    row = {b: s.table[b, :3].tolist() for b in range(3)}
    pool.keep(batch, good, ints([3, 0, 2]))
    want = [x.clone() for x in (s.kb, s.vb)]
    for x, y in zip((s.kb, s.vb), before):
        x.copy_(y)
    path, many = good.clone(), ints([3, 3, 2])
    if "path" in bad:
        path[1] = ints(bad["path"])
    if "many" in bad:
        many[1] = bad["many"]
    if "block" in bad:
        s.table[1, 2] = bad["block"]
    got = pool.keep(batch, path, many)
    with pytest.raises(m.MisatError) as e:
        pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    assert got.tolist() == [28, 38, 7]
    assert row[1][0] != row[0][0]
    for x, y in zip((s.kb, s.vb), want):
        assert torch.equal(x, y)


# ---- together ----


def test_a_drafting_step_gives_what_decoding_its_path_gives():
    """Rounds of: blocks, plan, append of normed nodes, attention, acceptance.  After each, the cache and the outputs are those
    of a pool that got the accepted tokens one after the other."""
    m = misat()
    n, nodes, hq, hkv, d, dtype = 5, 11, 8, 2, 64, BF16
    r = random.Random(3)
    rope = m.Rope(d)
    wq, wk = m.HeadNorm(rand((hq, d), BF16, 1) + 1), m.HeadNorm(rand((d,), BF16, 2), offset=1.0)

    def instance(blocks, columns):
        kb, vb = (torch.zeros((blocks, hkv, 16, d), dtype=dtype, device="cuda") for _ in range(2))
        pool = m.KvPool(kb, vb, n_q_heads=hq, rope=rope, max_batch=n)
        t = m.KvTables(pool, torch.zeros((n, columns), dtype=torch.int32, device="cuda"),
                       torch.randperm(blocks, generator=torch.Generator().manual_seed(blocks)).to(torch.int32).cuda())
        return pool, t, t.initial(blocks)

    pool, tables, state = instance(90, 12)
    plain, plain_tables, plain_state = instance(80, 10)
    # prompts
    new = [40, 3, 1, 17, 30]
    T = sum(new)
    x = rand((T, hq + 2 * hkv, d), dtype, 20)
    zero = ints([0] * n)
    lens = zero
    for p, t, s in ((pool, tables, state), (plain, plain_tables, plain_state)):
        batch = t.step(s, ints(new), zero, n_tokens=T, max_q=40, out=s)
        q = p.append(batch, x[:, hq:hq + hkv], x[:, hq + hkv:], q=x[:, :hq], q_norm=wq, k_norm=wk)
        p.attend(batch, q)
    lens = plain_lens = batch.kv_len
    parents = parents_of([nodes] * n, 9, "late")
    for turn in range(6):
        xs = rand((n * nodes, hq + 2 * hkv, d), dtype, 30 + turn)
        batch = tables.step(state, ints([nodes] * n), lens, n_tokens=n * nodes, max_q=nodes, out=state)
        tree = pool.tree(batch, ints(parents))
        q = pool.append(batch, xs[:, hq:hq + hkv], xs[:, hq + hkv:], q=xs[:, :hq], q_norm=wq, k_norm=wk, tree=tree)
        out = pool.attend(batch, q, tree=tree)
        # a path of each tree: from some node up
        _, sees = ref.tree([nodes] * n, parents)
        paths = [sorted(sees[b * nodes + r.randrange(nodes)]) for b in range(n)]
        width = max(map(len, paths))
        lens = pool.keep(batch, ints([p + [0] * (width - len(p)) for p in paths]), ints([len(p) for p in paths]))
        pool.sync()
        for i in range(width):
            go = [i < len(p) for p in paths]
            rows = torch.tensor([b * nodes + paths[b][i] for b in range(n) if go[b]], device="cuda")
            one = plain_tables.step(plain_state, ints([int(g) for g in go]), plain_lens, n_tokens=len(rows), max_q=1,
                                    out=plain_state)
            y = xs[rows]
            q = plain.append(one, y[:, hq:hq + hkv], y[:, hq + hkv:], q=y[:, :hq], q_norm=wq, k_norm=wk)
            want = plain.attend(one, q)
            plain_lens = one.kv_len
            # the same values in another order of sums: the weights' and the result's roundings on both sides, of values
            # of at most 6 (a weighted mean of normal values)
            assert (out[rows].float() - want.float()).abs().max() <= 2 * 2 * 2.0 ** -8 * 6
        plain.sync()
        assert lens.tolist() == plain_lens.tolist()
        for b, L in enumerate(lens.tolist()):
            for a, c in ((pool.k_blocks, plain.k_blocks), (pool.v_blocks, plain.v_blocks)):
                assert torch.equal(kref.gather(a, tables.block_table[b], L), kref.gather(c, plain_tables.block_table[b], L))
    # finished: every block comes back
    tables.step(state, zero, zero, n_tokens=0, max_q=0, out=state)
    pool.sync()
    assert state.tolist()[:n] == [0] * n and state.tolist()[-1] == 90
    held = tables.free.tolist()
    assert sorted(held) == list(range(90))


# ---- refusals ----


def test_refused_arguments():
    m = misat()
    s = Step([(3, 20), (2, 5)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    q, k, par = rand((5, 4, 32), BF16, 1), rand((5, 2, 32), BF16, 2), ints([-1, 0, 0, -1, 0])
    for bad in (par[:4], par.long(), par.cpu(), par[None], [1]):
        with pytest.raises(ValueError):
            pool.tree(batch, bad)
    with pytest.raises(ValueError):
        pool.tree(batch, par, window=1 << 40)
    with pytest.raises(m.MisatError):
        pool.tree(batch, par, window=-1)
    tree = pool.tree(batch, par, window=3)
    with pytest.raises(ValueError, match="window"):
        pool.attend(batch, q, window=4, tree=tree)
    assert torch.equal(pool.attend(batch, q, window=3, tree=tree), pool.attend(batch, q, tree=tree))
    long = pool.batch(s.q_off, s.kv_len, s.table, n_tokens=5, max_q=1025)
    with pytest.raises(m.MisatError):
        pool.tree(long, par)
    with pytest.raises(m.MisatError):
        pool.keep(long, ints([[0], [0]]), ints([0, 0]))
    other = pool.batch(s.q_off, s.kv_len, s.table, n_tokens=5, max_q=4)  # of another shape than the tree's
    for call in (lambda: pool.attend(other, q, tree=tree), lambda: pool.append(other, k, k, tree=tree)):
        with pytest.raises(ValueError, match="tree"):
            call()
    for bad in (q[:4], q.to(F16), k):
        with pytest.raises(ValueError):
            pool.attend(batch, bad, tree=tree)
    with pytest.raises(m.MisatError):
        pool.attend(batch, q, out=q.as_strided(q.shape, (32, 160, 1)), tree=tree)
    path, many = ints([[0, 1], [0, 1]]), ints([1, 1])
    for args in ((path[:1], many), (path.long(), many), (path, many[:1]), (path.t(), many), (path[:, 0], many),
                 (path, many, many.long()), (path, many, many[:1])):
        with pytest.raises(ValueError):
            pool.keep(batch, *args)
    with pytest.raises(m.MisatError):
        pool.keep(batch, path, many, out=s.kv_len)
    pool.sync()
    # by the library
    b, p, st = batch._ref, par.data_ptr(), torch.cuda.current_stream().cuda_stream
    f = m._lib.misat_kv_tree
    bad = m.ERR_INVALID_ARG
    assert f(None, b, p, 0, p, p, 1, st) == bad and f(pool._h, None, p, 0, p, p, 1, st) == bad
    for args in ((None, 0, p, p, 1), (p, 0, None, p, 1), (p, 0, p, None, 1), (p, 0, p, p, 2), (p, 0, p, p, 0), (p, -1, p, p, 1)):
        assert f(pool._h, b, *args, st) == bad
    import ctypes

    a = m._lib.misat_kv_attend_tree
    x = q.data_ptr()
    for kw in (dict(depth=None), dict(bits=None), dict(words=2), dict(window=-1), dict(bits=p + 2)):
        d = m.misat_kv_draft(**{**dict(depth=p, bits=p, words=1, window=0), **kw})
        assert a(pool._h, b, ctypes.byref(d), x, 128, 32, x, 128, 32, None, st) == bad
    assert a(pool._h, b, None, x, 128, 32, x, 128, 32, None, st) == bad
    e = m._lib.misat_kv_keep
    for args in ((None, 2, p, p), (p, -1, p, p), (p, 2, None, p), (p, 2, p, None)):
        assert e(pool._h, b, *args, st) == bad
    assert e(None, b, p, 2, p, p, st) == bad


def test_no_tokens():
    s = Step([(0, 5), (0, 0)], 2, 64, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    tree = pool.tree(batch, ints([]))
    assert tree.depth.shape == (0,) and tree.bits.shape == (0, 0)
    none = torch.empty((0, 4, 64), dtype=BF16, device="cuda")
    assert pool.attend(batch, none, tree=tree).shape == (0, 4, 64)
    assert pool.keep(batch, torch.empty((2, 0), dtype=torch.int32, device="cuda"), ints([0, 0])).tolist() == [5, 0]
    pool.sync()


def test_written_tensors_have_a_new_version():
    s = Step([(3, 20)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    tree = pool.tree(batch, ints([-1, 0, 0]))
    q, k, out = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 2), torch.empty((3, 4, 32), dtype=BF16, device="cuda")
    lens = ints([0])
    for call, tensors in ((lambda: pool.append(batch, k, k, tree=tree), (s.kb, s.vb)),
                          (lambda: pool.append(batch, k, k, q=q, q_out=out, tree=tree), (s.kb, s.vb, out)),
                          (lambda: pool.attend(batch, q, out=out, tree=tree), (out,)),
                          (lambda: pool.keep(batch, ints([[0, 2]]), ints([2]), out=lens), (s.kb, s.vb, lens))):
        before = [t._version for t in tensors]
        call()
        assert all(t._version > v for t, v in zip(tensors, before))
    pool.sync()


def test_objects_of_another_kind_are_refused():
    m = misat()
    s = Step([(3, 20)], 2, 32, BF16)
    rope = m.Rope(32)
    pool = s.pool(4, rope=rope)
    batch = s.batch(pool)
    tree = pool.tree(batch, ints([-1, 0, 0]))
    norm = m.HeadNorm(torch.ones(32, device="cuda"))
    q, k, pos = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 2), ints([0, 1, 2])
    for call in (lambda: pool.attend(tree, q), lambda: pool.attend(batch, q, tree=batch), lambda: pool.attend(pool, q),
                 lambda: pool.append(batch, k, k, k_norm=rope), lambda: pool.append(batch, k, k, tree=norm),
                 lambda: rope.norm_rotate(q, pos, rope), lambda: pool.keep(tree, pos[:, None], pos),
                 lambda: pool.tree(norm, pos)):
        with pytest.raises((ValueError, AttributeError)):
            call()
    pool.sync()


def test_a_captured_step_is_replayed():
    """Blocks, plan, append, attention and what is kept in one graph, whose lengths and tables go on from replay to replay."""
    m = misat()
    n, nodes, hq, hkv, d, dtype = 9, 6, 8, 2, 64, BF16
    rope = m.Rope(d, layout=m.ROPE_INTERLEAVED)
    norm = m.HeadNorm(rand((d,), BF16, 1) + 1)
    x = rand((n * nodes, hq + 2 * hkv, d), dtype, 2)
    par, path, many = ints(parents_of([nodes] * n, 3)), ints([[0, 2, 5]] * n), ints([b % 4 for b in range(n)])
    new = ints([nodes] * n)

    class Side:
        def __init__(self):
            self.kb, self.vb = (torch.zeros((200, hkv, 16, d), dtype=dtype, device="cuda") for _ in range(2))
            self.pool = m.KvPool(self.kb, self.vb, n_q_heads=hq, rope=rope)
            self.tables = m.KvTables(self.pool, torch.zeros((n, 15), dtype=torch.int32, device="cuda"),
                                     torch.arange(200, dtype=torch.int32, device="cuda"))
            self.state, self.lens = self.tables.initial(200), ints(list(range(n)))
            first = self.tables.step(self.state, self.lens, ints([0] * n), n_tokens=n * (n - 1) // 2, max_q=n - 1, out=self.state)
            self.pool.append(first, *(rand((first.n_tokens, hkv, d), dtype, 4) for _ in range(2)))

        def step(self):
            batch = self.tables.step(self.state, new, self.lens, n_tokens=n * nodes, max_q=nodes, out=self.state)
            tree = self.pool.tree(batch, par)
            q = self.pool.append(batch, x[:, hq:hq + hkv], x[:, hq + hkv:], q=x[:, :hq], q_norm=norm, k_norm=norm, tree=tree)
            out, lse = self.pool.attend(batch, q, return_lse=True, tree=tree)
            self.pool.keep(batch, path, many, out=self.lens)
            return out, lse, batch.slots

    eager, graphed = Side(), Side()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        got = graphed.step()
    for turn in range(25):
        want = eager.step()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn
        assert torch.equal(eager.lens, graphed.lens) and torch.equal(eager.state, graphed.state)
        assert torch.equal(eager.tables.block_table, graphed.tables.block_table)
        assert torch.equal(eager.kb, graphed.kb) and torch.equal(eager.vb, graphed.vb)
    eager.pool.sync()
    graphed.pool.sync()
    assert eager.lens.tolist() == [b + 25 * (b % 4) for b in range(n)]


def test_lengths_of_keep_stand_apart():
    """Written by one of several CTAs that read the lengths, the counts and the paths: none of them may be its result."""
    m = misat()
    s = Step([(2, 5), (2, 7), (2, 3)], 2, 64, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    flat = ints([1, 0, 2, 0, 1, 2, 0, 0])
    many, path = flat[:3], flat[3:6].view(3, 1)
    before = s.kb.clone()
    for out in (many, flat[1:4], flat[2:5], path[:, 0], flat[5:8], s.q_off[:3], s.q_off[1:], s.kv_len):
        with pytest.raises(m.MisatError):
            pool.keep(batch, path, many, out=out)
    assert flat.tolist() == [1, 0, 2, 0, 1, 2, 0, 0] and torch.equal(s.kb, before)
    assert s.kv_len.tolist() == [5, 7, 3] and s.q_off.tolist() == [0, 2, 4, 6]
    path = ints([[0], [0], [0]])
    # Lengths behind the counts in one tensor, and in front of them.
    both = ints([0, 0, 0, 1, 0, 1, 0, 0, 0])
    for out in (both[:3], both[6:]):
        assert pool.keep(batch, path, both[3:6], out=out).tolist() == [4, 5, 2]
    pool.sync()
