"""Block tables, offsets, positions and slots of a step, from the lengths on the device: against lists of numbers."""

import ctypes
import random

import pytest

torch = pytest.importorskip("torch")

from tests import kv_step_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, misat  # noqa: E402

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Tables:
    """Rows of given blocks over a pool of n_blocks; the rest is in a ring that begins anywhere."""

    def __init__(self, held, columns, n_free, seed=1, places=None, pad=0):
        r = random.Random(seed)
        n = len(held)
        total = sum(held) + n_free
        ids = list(range(total))
        r.shuffle(ids)
        places = places or total or 1
        head = r.randrange(places)
        self.table, at = [], 0
        for h in held:
            self.table.append(ids[at:at + h] + [-7] * (columns - h))
            at += h
        self.ring = [-9] * places
        for i, x in enumerate(ids[at:]):
            self.ring[(head + i) % places] = x
        self.state = list(held) + [head, n_free]
        self.n, self.n_blocks = n, max(total, 1)
        self.kb, self.vb = (torch.zeros((self.n_blocks, 1, 16, 8), dtype=BF16, device="cuda") for _ in range(2))
        self.pool = misat().KvPool(self.kb, self.vb, n_q_heads=1)
        wide = torch.full((n, columns + pad), -7, dtype=torch.int32, device="cuda")
        self.d_table = wide[:, :columns]
        if n and columns:
            self.d_table.copy_(ints(self.table))
        self.d_ring, self.d_state = ints(self.ring), ints(self.state)
        self.tables = misat().KvTables(self.pool, self.d_table, self.d_ring)

    def step(self, new, kv_len, shared=None, state=None, **kw):
        return self.tables.step(self.d_state if state is None else state, ints(new), ints(kv_len), n_tokens=sum(new),
                                max_q=max(new + [0]), shared=None if shared is None else ints(shared), **kw)

    def check(self, new, kv_len, shared=None, **kw):
        got = self.step(new, kv_len, shared, **kw)
        self.pool.sync()
        want = ref.tables(self.n, new, kv_len, self.state, self.table, self.ring, shared)
        for name, g, w in zip(("state", "q_off", "kv_len", "positions", "slots"),
                              (got.state, got.q_off, got.kv_len, got.positions, got.slots), want):
            assert g.tolist() == w, name
        assert self.d_table.tolist() == self.table and self.d_ring.tolist() == self.ring
        return got


def drawn(n, seed, new_hi, hist_hi, spare=40, done=0.1):
    r = random.Random(seed)
    kv, new, held = [], [], []
    for _ in range(n):
        k = r.randint(0, hist_hi)
        h = -(-(k + r.choice([0, 0, r.randint(0, spare)])) // 16)
        held.append(h)
        if r.random() < done:
            k = 0
        kv.append(k)
        new.append(0 if k == 0 and r.random() < 0.5 else r.randint(0, new_hi))
    return new, kv, held


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n,new_hi,hist_hi", [
    (1, 1, 0), (1, 100000, 50), (2, 17, 40), (3, 1, 16), (31, 1, 300), (32, 0, 200), (33, 5, 100), (100, 300, 900),
    (257, 1, 4000), (1000, 3, 90), (1025, 1, 50), (4096, 2, 64), (4097, 40, 33), (9001, 1, 20)])
def test_step(n, new_hi, hist_hi, shared):
    new, kv, held = drawn(n, n + new_hi, new_hi, hist_hi)
    take = sum(max(0, -(-(a + b) // 16) - h) for a, b, h in zip(new, kv, held))
    columns = max([-(-(a + b) // 16) for a, b in zip(new, kv)] + held) + 1
    t = Tables(held, columns, take + 5, seed=n, pad=3)
    r = random.Random(n)
    got = t.check(new, kv, [r.randint(0, h) for h in held] if shared else None)
    # the result serves as a batch of the pool
    if sum(new):
        q = torch.zeros((sum(new), 1, 8), dtype=BF16, device="cuda")
        t.pool.append(got, q, q)
        t.pool.sync()


def test_many_steps_lose_and_double_no_block():
    r = random.Random(5)
    n, columns = 40, 30
    t = Tables([0] * n, columns, 500, places=500)
    state, lens = t.d_state, [0] * n
    for step in range(60):
        for b in range(n):
            if r.random() < 0.1 or lens[b] > 400:
                lens[b] = 0
            elif r.random() < 0.2:
                lens[b] = r.randint(0, lens[b])  # drafts that were not accepted
        new = [r.choice([0, 1, 1, r.randint(2, 60)]) for _ in range(n)]
        got = t.check(new, lens, state=state, out=state if step % 3 else None)
        state = got.state
        t.state = state.tolist()
        lens = got.kv_len.tolist()
        held, head, count = t.state[:n], t.state[n], t.state[n + 1]
        all_blocks = [t.table[b][c] for b in range(n) for c in range(held[b])]
        all_blocks += [t.ring[(head + i) % 500] for i in range(count)]
        assert sorted(all_blocks) == list(range(500))


@pytest.mark.parametrize("n", [0, 1, 50])
def test_steps_without_tokens(n):
    t = Tables([3] * n, 5, 4)
    t.check([0] * n, [0] * n)  # all are given back
    t = Tables([0] * n, 0, 4)  # rows without room
    t.check([0] * n, [0] * n)


def test_exactly_enough_blocks_and_a_full_ring():
    t = Tables([0, 1, 0], 4, 7)
    t.check([33, 40, 16], [0, 8, 0])
    assert t.d_state.tolist()[-1] == 7  # (the state of before is as it was)
    t = Tables([4, 4], 4, 0, places=8)
    t.check([0, 0], [0, 17])


BAD = {
    "blocks": (dict(new=[40, 96], kv=[10, 0]), "OOM"),  # takes 2 + 5 of 3
    "negative new": (dict(new=[5, -1], n_tokens=4, max_q=5), "INVALID_ARG"),
    "negative length": (dict(kv=[-1, 0]), "INVALID_ARG"),
    "length past the row's blocks": (dict(kv=[33, 0]), "INVALID_ARG"),
    "row too short": (dict(new=[1, 100], kv=[0, 0]), "INVALID_ARG"),
    "sum": (dict(n_tokens=7), "INVALID_ARG"),
    "longest": (dict(max_q=3), "INVALID_ARG"),
    "shared past the row's blocks": (dict(shared=[3, 0]), "INVALID_ARG"),
    "negative shared": (dict(shared=[-1, 0]), "INVALID_ARG"),
    "negative held": (dict(state=[-1, 1, 0, 3]), "INVALID_ARG"),
    "held past the row": (dict(state=[2, 7, 0, 3]), "INVALID_ARG"),
    "front": (dict(state=[2, 1, 6, 3]), "INVALID_ARG"),
    "negative front": (dict(state=[2, 1, -1, 3]), "INVALID_ARG"),
    "count": (dict(state=[2, 1, 0, 7]), "INVALID_ARG"),
    "negative count": (dict(state=[2, 1, 0, -1]), "INVALID_ARG"),
    "no room in the ring": (dict(new=[0, 0], kv=[0, 0], state=[2, 1, 0, 4]), "INVALID_ARG"),
    "sums beyond 32 bits": (dict(new=[2 ** 30, 2 ** 30], kv=[0, 0], max_q=2 ** 30, n_tokens=8), "INVALID_ARG"),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", BAD)
def test_a_step_that_cannot_be_made_changes_nothing(what, in_place):
    m = misat()
    case, code = BAD[what]
    t = Tables([2, 1], 6, 3, places=6)
    new, kv = case.get("new", [5, 3]), case.get("kv", [20, 10])
    state = ints(case["state"]) if "state" in case else t.d_state
    before = state.tolist()
    shared = ints(case["shared"]) if "shared" in case else None
    got = t.tables.step(state, ints(new), ints(kv), n_tokens=case.get("n_tokens", sum(new)),
                        max_q=case.get("max_q", max(new)), shared=shared, out=state if in_place else None)
    with pytest.raises(m.MisatError) as e:
        t.pool.sync()
    assert e.value.code == getattr(m, "ERR_" + code)
    assert got.state.tolist() == before and state.tolist() == before
    assert got.q_off.tolist() == [0, 0, 0] and got.kv_len.tolist() == kv
    assert (got.positions == -1).all() and (got.slots == -1).all()
    assert t.d_table.tolist() == t.table and t.d_ring.tolist() == t.ring
    if "state" not in case:
        t.check([5, 3], [20, 10])  # the next one is made


def test_captured_steps_go_on_in_place():
    n = 70
    t = Tables([0] * n, 12, 900)
    new, lens, state = ints([3] * n), torch.zeros(n, dtype=torch.int32, device="cuda"), t.d_state
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t.tables.step(state.clone(), new, lens.clone(), n_tokens=3 * n, max_q=3)  # (loads the kernels)
    s.synchronize()
    t.d_table.copy_(ints(t.table))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        got = t.tables.step(state, new, lens, n_tokens=3 * n, max_q=3, out=state)
        lens.copy_(got.kv_len)
    want = list(t.state)
    for k in range(20):
        g.replay()
        want, q_off, l2, pos, slots = ref.tables(n, [3] * n, [3 * k] * n, want, t.table, t.ring)
        assert state.tolist() == want and lens.tolist() == l2
        assert got.positions.tolist() == pos and got.slots.tolist() == slots
    t.pool.sync()
    assert t.d_table.tolist() == t.table


def test_written_tensors_and_streams():
    t = Tables([1, 1], 6, 9)
    tensors = (t.d_table, t.d_ring, t.d_state)
    before = [x._version for x in tensors]
    t.check([5, 3], [10, 10], out=t.d_state)
    assert all(x._version > b for x, b in zip(tensors, before))
    t.state = t.d_state.tolist()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t.check([5, 3], [15, 13])


def test_refused_arguments():
    m = misat()
    t = Tables([1, 1], 6, 9)
    good = dict(state=t.d_state, new=ints([5, 3]), kv_len=ints([10, 10]), n_tokens=8, max_q=5)
    for kw in (dict(state=t.d_state[:3]), dict(state=t.d_state.long()), dict(new=ints([5, 3]).cpu()),
               dict(new=ints([[5, 3]])), dict(kv_len=ints([10])), dict(shared=ints([0])), dict(out=t.d_state[:2]),
               dict(n_tokens=1 << 40), dict(max_q=1 << 40), dict(new=ints([5, 0, 3, 0])[::2])):
        with pytest.raises(ValueError):
            t.tables.step(**{**good, **kw})
    for kw in (dict(n_tokens=-1), dict(max_q=-1), dict(n_tokens=2 ** 31 - 1)):
        with pytest.raises(m.MisatError) as e:
            t.tables.step(**{**good, **kw})
        assert e.value.code == m.ERR_INVALID_ARG
    for table, ring in ((t.d_table.long(), t.d_ring), (t.d_table[:1], t.d_ring), (t.d_table.t(), t.d_ring),
                        (t.d_table, t.d_ring.float()), (t.d_table, t.d_ring[None])):
        with pytest.raises(ValueError):
            m.KvTables(t.pool, table, ring).step(**good)
    with pytest.raises(m.MisatError):  # a ring without places
        m.KvTables(t.pool, t.d_table, t.d_ring[:0]).step(**good)
    small = m.KvPool(t.kb, t.vb, n_q_heads=1, max_batch=1)
    with pytest.raises(m.MisatError):
        m.KvTables(small, t.d_table, t.d_ring).step(**good)
    # by the library: null pointers, scratch that is too small
    work = torch.empty(1000, dtype=torch.uint8, device="cuda")
    p = work.data_ptr()
    fields = dict(n=2, n_tokens=8, max_q=5, columns=6, table_stride=6, ring_size=9, new_tokens=p, kv_len=p, shared=None,
                  state=p, block_table=p, ring=p, state_out=p, q_off=p, kv_len_out=p, positions=p, slots=p)
    f = m._lib.misat_kv_tables
    for name in ("new_tokens", "kv_len", "state", "block_table", "ring", "state_out", "q_off", "kv_len_out", "positions",
                 "slots"):
        assert f(t.pool._h, ctypes.byref(m.misat_kv_step(**{**fields, name: None})), p, 1000, None) == m.ERR_INVALID_ARG
    for kw in (dict(n=-1), dict(columns=-1), dict(table_stride=5), dict(ring_size=0), dict(n=0)):
        assert f(t.pool._h, ctypes.byref(m.misat_kv_step(**{**fields, **kw})), p, 1000, None) == m.ERR_INVALID_ARG
    s = ctypes.byref(m.misat_kv_step(**fields))
    assert f(None, s, p, 1000, None) == m.ERR_INVALID_ARG
    assert f(t.pool._h, None, p, 1000, None) == m.ERR_INVALID_ARG
    for args in ((None, 1000), (p, 111), (p + 4, 900)):
        assert f(t.pool._h, s, *args, None) == m.ERR_INVALID_ARG


@pytest.mark.parametrize("each", [3, 16, 700, 5000])
def test_many_blocks_given_back_by_a_small_step(each):
    """Of a table with so many places that they are left to a second kernel where they are many."""
    n = 60
    held = [each if b % 3 else 5 for b in range(n)]
    t = Tables(held, 5001, 40, seed=each)
    kv = [0 if b % 3 else 70 for b in range(n)]
    got = t.check([0 if b % 3 else 30 for b in range(n)], kv, [min(7, h) if b % 5 == 0 else 0 for b, h in enumerate(held)])
    t.state = got.state.tolist()
    t.check([1] * n, got.kv_len.tolist(), state=got.state)


@pytest.mark.parametrize("n", [100, 3000, 5000])
@pytest.mark.parametrize("off", [0, 1])
def test_arrays_at_any_boundary_and_lengths_in_place(n, off):
    """By the library: every array of the sequences 4 bytes past a 16-byte boundary, and results over their inputs."""
    m = misat()
    new, kv, held = drawn(n, 7 * n + off, 3, 60)
    t = Tables(held, 10, n + 20, seed=n)
    r = random.Random(n)
    shared = [r.randint(0, h) for h in held]
    want = ref.tables(n, new, kv, t.state, t.table, t.ring, shared)

    def at(values):
        x = ints([0] * off + list(values) + [77])
        return x, x.data_ptr() + 4 * off

    T = sum(new)
    arrays = {k: at(v) for k, v in dict(new_tokens=new, kv_len=kv, shared=shared, state=t.state, q_off=[5] * (n + 1),
                                        positions=[5] * T).items()}
    slots = torch.full((T + 1,), 5, dtype=torch.int64, device="cuda")
    work = torch.empty(24 * n + 64, dtype=torch.uint8, device="cuda")
    p = {k: v[1] for k, v in arrays.items()}
    s = m.misat_kv_step(n=n, n_tokens=T, max_q=max(new), columns=10, table_stride=t.d_table.stride(0), ring_size=len(t.ring),
                        block_table=t.d_table.data_ptr(), ring=t.d_ring.data_ptr(), state_out=p["state"],
                        kv_len_out=p["kv_len"], slots=slots.data_ptr(), **p)
    st = torch.cuda.current_stream().cuda_stream
    assert m._lib.misat_kv_tables(t.pool._h, ctypes.byref(s), work.data_ptr(), work.numel(), st) == 0
    t.pool.sync()
    for name, w in zip(("state", "q_off", "kv_len", "positions"), want):
        assert arrays[name][0].tolist() == [0] * off + w + [77], name
    assert slots.tolist() == want[4] + [5]
    assert t.d_table.tolist() == t.table and t.d_ring.tolist() == t.ring
    assert arrays["new_tokens"][0].tolist()[off:-1] == new and arrays["shared"][0].tolist()[off:-1] == shared
