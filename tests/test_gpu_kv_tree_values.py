"""Trees with nodes that are not there, whose queries, keys and values hold anything, plans of malformed batches, and nodes
beside tokens in a row."""

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


def parents_with_gaps(new, seed, absent):
    """Absent nodes anywhere in a tree, with nodes that are there behind them."""
    r = random.Random(seed)
    out = []
    for n in new:
        there = []
        for i in range(n):
            if r.random() < absent:
                out.append(ref.ABSENT)
            else:
                out.append(r.choice(there + [ref.ROOT]))
                there.append(i)
    return out


def slots_of(s):
    """Block and place of each new token."""
    seq = [b for b, n in enumerate(s.new) for _ in range(n)]
    pos = [L - n + i for n, L in zip(s.new, s.lens) for i in range(n)]
    seq, pos = torch.tensor(seq, device="cuda"), torch.tensor(pos, device="cuda")
    return s.table[seq, pos // 16].long(), pos % 16


def check(seqs, hq, hkv, d, dtype, absent, window=0, seed=1, fill=math.nan):
    """The slots of absent nodes hold `fill`: results are those of the nodes that are there alone."""
    s = Step(seqs, hkv, d, dtype, seed=seed)
    parents = parents_with_gaps(s.new, seed, absent)
    gone = torch.tensor(parents, device="cuda") == ref.ABSENT
    blk, at = slots_of(s)
    clean_k, clean_v = s.kb.clone(), s.vb.clone()
    for x in (clean_k, clean_v):  # (for the reference, in which a product with zero counts)
        x[blk[gone], :, at[gone]] = 0
    for x in (s.kb, s.vb):
        x[blk[gone], :, at[gone]] = fill
    s.poison()
    pool = s.pool(hq)
    batch = s.batch(pool)
    q = rand((s.T, hq, d), dtype, seed + 7, 1.5)
    q[gone] = fill
    tree = pool.tree(batch, ints(parents), window=window)
    out, lse = pool.attend(batch, q, return_lse=True, tree=tree)
    pool.sync()
    depth, sees = ref.tree(s.new, parents, window)
    o, ot, l, lt = ref.attend(q, clean_k, clean_v, s.new, s.lens, s.table, depth, sees, window)
    kref.assert_within("out", out, o, ot)
    kref.assert_within("lse", lse, l, lt)
    assert (out[gone] == 0).all() and (lse[gone] == -math.inf).all()


@pytest.mark.parametrize("fill", [math.nan, math.inf])
@pytest.mark.parametrize("absent", [0.2, 0.9])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 4, 64, BF16), (2, 2, 64, F16), (8, 1, 128, BF16), (28, 4, 64, F16), (6, 2, 72, F16),
                                            (32, 2, 128, BF16), (3, 1, 8, BF16)])
def test_slots_of_absent_nodes_hold_anything(hq, hkv, d, dtype, absent, fill):
    """Trees that begin and end anywhere in a block of keys, one of them behind nothing."""
    check([(1, 1), (5, 5), (12, 140), (33, 33), (32, 128), (17, 128 + 17), (3, 700), (64, 300), (0, 9), (127, 255)], hq, hkv, d,
          dtype, absent, fill=fill)


@pytest.mark.parametrize("hq,hkv,d", [(2, 1, 64), (8, 1, 128), (2, 2, 128)])
@pytest.mark.parametrize("n,L", [(128, 256), (129, 130), (130, 500), (257, 257), (600, 641), (1024, 1100)])
def test_absent_nodes_of_trees_longer_than_a_block(n, L, hq, hkv, d):
    for absent in (0.01, 0.5, 0.99):
        check([(n, L)], hq, hkv, d, BF16, absent, seed=n)


@pytest.mark.parametrize("window", [1, 4, 100])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 1, 128)])
def test_absent_nodes_under_a_window(hq, hkv, d, window):
    check([(8, 8), (16, 40), (40, 41), (130, 700), (1, 1), (5, 300)], hq, hkv, d, BF16, 0.4, window, seed=4)


def test_absent_nodes_behind_long_histories():
    """Items in parts, of which some have none of the tree, and many sequences."""
    check([(20, 30000)], 8, 1, 128, BF16, 0.5)
    check([(250, 3250), (3, 50)], 8, 8, 64, F16, 0.5, seed=3)
    r = random.Random(2)
    seqs = [(r.choice([0, 1, 4, 16, 33]), 0) for _ in range(300)]
    check([(n, n + r.choice([0, 1, 15, 130, r.randint(0, 900)])) for n, _ in seqs], 4, 1, 64, BF16, 0.3)
    check([(n, n + r.choice([0, 1, 15, 130, r.randint(0, 900)])) for n, _ in seqs], 4, 2, 128, F16, 0.3)


@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_padding_rows_of_a_step_of_fixed_shape(d, normed):
    """Append and attention of rows of which the absent ones hold NaN, and of the same with zeros there: the same bits."""
    m = misat()
    s = Step([(12, 40), (12, 12), (12, 300), (12, 139)], 2, d, BF16)
    pool = s.pool(8, rope=m.Rope(d))
    parents = parents_with_gaps(s.new, 5, 0.4)
    gone = torch.tensor(parents, device="cuda") == ref.ABSENT
    norm = m.HeadNorm(rand((d,), BF16, 2) + 1) if normed else None
    batch = s.batch(pool)
    tree = pool.tree(batch, ints(parents))
    x = rand((s.T, 12, d), BF16, 3)
    got = []
    for fill in (0.0, math.nan):
        x[gone] = fill
        q = pool.append(batch, x[:, 8:10], x[:, 10:], q=x[:, :8], q_norm=norm, k_norm=norm, tree=tree)
        got.append(pool.attend(batch, q, tree=tree, return_lse=True))
    pool.sync()
    for a, b in zip(*got):
        assert torch.equal(a, b) and not torch.isnan(a).any()
    assert (got[0][0][gone] == 0).all() and not (got[0][0][~gone] == 0).all()


# ---- the plan of malformed batches ----

BATCHES = {  # q_off, kv_len, and which node of its sequence each token is (None: of none)
    "length below the new tokens": ([0, 3, 3, 5], [2, 4, 9], [None, None, None, 0, 1]),
    "negative length": ([0, 3, 3, 5], [7, 4, -1], [0, 1, 2, None, None]),
    "length past the table": ([0, 3, 3, 5], [7, 4, 2 ** 31 - 1], [0, 1, 2, None, None]),
    "first offset": ([1, 3, 3, 5], [7, 4, 9], [None, 0, 1, 0, 1]),
    "last offset": ([0, 3, 3, 4], [7, 4, 9], [0, 1, 2, 0, None]),
    "no tokens": ([0, 0, 0, 0], [7, 4, 9], [None] * 5),
    "offset past the batch": ([0, 3, 3, 9], [7, 4, 9], [0, 1, 2, None, None]),
    "negative offset": ([-4, 3, 3, 5], [7, 4, 9], [None, None, None, 0, 1]),
    "more than max_q": ([0, 0, 5, 5], [7, 9, 9], [None] * 5),
}


@pytest.mark.parametrize("words", [1, 2])
@pytest.mark.parametrize("what", BATCHES)
def test_plan_of_a_malformed_batch_is_written_whole(what, words):
    """Nodes without a sequence are absent, not what their memory held before."""
    m = misat()
    q_off, kv_len, node = BATCHES[what]
    s = Step([(3, 7), (0, 4), (2, 9)], 1, 64, BF16)
    pool = s.pool(1)
    batch = pool.batch(ints(q_off), ints(kv_len), s.table, n_tokens=5, max_q=4 if words == 1 else 33)
    if what == "more than max_q" and words == 2:
        batch = pool.batch(ints([0, 0, 34, 34]), ints([7, 99, 99]), torch.zeros((3, 9), dtype=torch.int32, device="cuda"),
                           n_tokens=34, max_q=33)
        node = [None] * 34
    T = len(node)
    parents = ints([ref.ROOT] * T)
    depth = torch.full((T,), 77, dtype=torch.int32, device="cuda")
    bits = torch.full((T, words), -1, dtype=torch.int32, device="cuda")
    assert m._lib.misat_kv_tree(pool._h, batch._ref, parents.data_ptr(), 0, depth.data_ptr(), bits.data_ptr(), words,
                                torch.cuda.current_stream().cuda_stream) == 0
    with pytest.raises(m.MisatError) as e:
        pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    assert depth.tolist() == [0] * T
    assert bits.tolist() == [[0 if i is None else 1 << i] + [0] * (words - 1) for i in node]


def test_attention_by_the_plan_of_a_malformed_batch():
    """A sequence that the plan refuses, though the attention takes its length, has no nodes."""
    m = misat()
    s = Step([(3, 7), (0, 4), (2, 9)], 1, 64, BF16)
    pool = s.pool(2)
    batch = s.batch(pool)
    q = rand((5, 2, 64), BF16, 1)
    want = pool.attend(batch, q, tree=pool.tree(batch, ints([-1] * 5)))
    s.kv_len[0] = 2
    junk = [torch.full((10,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    del junk  # (the plan's memory comes from here)
    tree = pool.tree(batch, ints([-1] * 5))
    with pytest.raises(m.MisatError):
        pool.sync()
    out, lse = pool.attend(batch, q, return_lse=True, tree=tree)
    pool.sync()
    assert (out[:3] == 0).all() and (lse[:3] == -math.inf).all() and torch.equal(out[3:], want[3:])


# ---- nodes and tokens in a row ----


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,rot,half", [(4, 2, 64, 64, True), (7, 1, 72, 20, False), (32, 8, 128, 128, True), (3, 3, 24, 6, True),
                                               (2, 1, 64, 64, False)])
@pytest.mark.parametrize("normed", [("k_norm",), ("q_norm",), ("q_norm", "k_norm")])
def test_a_node_is_cached_as_the_token_at_its_position(hq, hkv, d, rot, half, dtype, normed):
    """Any tree's nodes, and each of them appended as a token in a row at the same position, with norms: the same bits."""
    m = misat()
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    norm = m.HeadNorm(rand((d,), dtype, 5) + 1)
    kw = {name: norm for name in normed}
    s = Step([(40, 31040), (300, 7300), (1, 1), (64, 80)], hkv, d, dtype)
    pool = s.pool(hq, rope=rope)
    batch = s.batch(pool)
    r = random.Random(6)
    parents = [r.randint(max(-1, i - 3), i - 1) for n in s.new for i in range(n)]
    x = rand((s.T, hq + 2 * hkv, d), dtype, 3, 2.0)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    got = pool.append(batch, k, v, q=q, tree=pool.tree(batch, ints(parents)), **kw)
    blk, at = slots_of(s)
    cached_k, cached_v = s.kb[blk, :, at], s.vb[blk, :, at]
    depth, _ = ref.tree(s.new, parents)
    first = [L - n for n, L in zip(s.new, s.lens) for _ in range(n)]
    # a sequence for each node, whose one new token is at the node's position
    lens = [p + e + 1 for p, e in zip(first, depth)]
    table = torch.arange(s.T, dtype=torch.int32, device="cuda")[:, None].expand(s.T, max(lens) // 16 + 1).contiguous()
    kb, vb = (torch.zeros((s.T, hkv, 16, d), dtype=dtype, device="cuda") for _ in range(2))
    row = m.KvPool(kb, vb, n_q_heads=hq, rope=rope, max_batch=s.T)
    want = row.append(row.batch(ints(list(range(s.T + 1))), ints(lens), table, n_tokens=s.T, max_q=1), k, v, q=q, **kw)
    pool.sync()
    row.sync()
    t, place = torch.arange(s.T, device="cuda"), ints(lens).long() - 1
    assert torch.equal(got, want)
    assert torch.equal(cached_k, kb[t, :, place % 16]) and torch.equal(cached_v, vb[t, :, place % 16])
