"""Results of the step's calls that would lie over what the call reads or writes besides: refused before a launch."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests import kv_step_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, Step, misat  # noqa: E402
from tests.test_gpu_kv_tables import Tables, ints  # noqa: E402

pytestmark = pytest.mark.gpu

SEQUENCE_INPUTS = ("new_tokens", "kv_len", "shared", "state")
SEQUENCE_RESULTS = ("state_out", "q_off", "kv_len_out")
WRITTEN = SEQUENCE_RESULTS + ("block_table", "ring", "positions", "slots", "work")


def arrays():
    """Two sequences with 8 new tokens: arrays of a step, of their sizes, in one tensor; and their places in it."""
    size = dict(new_tokens=2, kv_len=2, shared=2, state=4, state_out=4, q_off=3, kv_len_out=2, block_table=7 + 6, ring=9,
                positions=8, slots=16, work=112 // 4)
    at, places = 0, {}
    for name, n in size.items():
        places[name] = at
        at += (n + 7) // 4 * 4  # at least four bytes between them
    return torch.full((at,), 5, dtype=torch.int32, device="cuda"), places, size


def call(t, flat, places):
    m = misat()
    p = {k: flat.data_ptr() + 4 * v for k, v in places.items()}
    work = p.pop("work")
    s = m.misat_kv_step(n=2, n_tokens=8, max_q=5, columns=6, table_stride=7, ring_size=9, **p)
    return m._lib.misat_kv_tables(t.pool._h, ctypes.byref(s), work, 112, torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("name", WRITTEN)
def test_tables_refuse_results_over_other_arrays(name):
    m = misat()
    t = Tables([1, 1], 6, 9)
    flat, places, size = arrays()
    step = 4 if name == "work" else 2 if name == "slots" else 1
    for other in places:
        if other == name:
            continue
        for at in {places[other] - size[name] + step, places[other], places[other] + size[other] - 1}:
            at = at // step * step
            free = name in SEQUENCE_RESULTS and other in SEQUENCE_INPUTS and at == places[other]
            if at < 0 or free or at + size[name] <= places[other] or at >= places[other] + size[other]:
                continue
            assert call(t, flat, {**places, name: at}) == m.ERR_INVALID_ARG, (other, at)
    torch.cuda.synchronize()
    assert (flat == 5).all()


def test_tables_refuse_a_state_in_other_arrays():
    m = misat()
    t = Tables([1, 1], 6, 9)
    flat = ints([9] * 12)
    flat[1:5] = t.d_state
    good = dict(new=ints([5, 3]), kv_len=ints([14, 10]), n_tokens=8, max_q=5)
    for out in (flat[0:4], flat[2:6], t.d_table.view(-1)[:4], t.d_ring[3:7]):
        with pytest.raises(m.MisatError) as e:
            t.tables.step(flat[1:5], out=out, **good)
        assert e.value.code == m.ERR_INVALID_ARG
    t.pool.sync()
    assert t.d_table.tolist() == t.table and t.d_ring.tolist() == t.ring and flat[1:5].tolist() == t.state
    got = t.tables.step(flat[1:5], out=flat[5:9], **good)
    same = t.tables.step(flat[1:5], out=flat[1:5], n_tokens=0, max_q=0, new=ints([0, 0]), kv_len=ints([14, 10]))
    t.pool.sync()
    assert got.state.tolist() != t.state and same.state.tolist() == t.state


@pytest.mark.parametrize("n", [2, 2000, 5000])
def test_results_of_sequences_in_place_of_their_inputs(n):
    """Lengths over the new tokens, the state over itself and the shared blocks that are its first numbers."""
    t = Tables([1] * n, 4, 3 * n)
    new = [b % 30 for b in range(n)]
    kv = [b % 17 for b in range(n)]
    m = misat()
    state, fresh, lens = t.d_state, ints(new), ints(kv)
    T = sum(new)
    q_off, positions = ints([0] * (n + 1)), ints([0] * T)
    slots = torch.zeros(T, dtype=torch.int64, device="cuda")
    work = torch.empty(24 * n + 64, dtype=torch.uint8, device="cuda")
    want = ref.tables(n, new, kv, t.state, t.table, t.ring, [1] * n)
    s = m.misat_kv_step(n=n, n_tokens=T, max_q=max(new), columns=4, table_stride=4, ring_size=len(t.ring),
                        new_tokens=fresh.data_ptr(), kv_len=lens.data_ptr(), shared=state.data_ptr(), state=state.data_ptr(),
                        block_table=t.d_table.data_ptr(), ring=t.d_ring.data_ptr(), state_out=state.data_ptr(),
                        q_off=q_off.data_ptr(), kv_len_out=fresh.data_ptr(), positions=positions.data_ptr(),
                        slots=slots.data_ptr())
    st = torch.cuda.current_stream().cuda_stream
    assert m._lib.misat_kv_tables(t.pool._h, ctypes.byref(s), work.data_ptr(), work.numel(), st) == 0
    t.pool.sync()
    for got, w in zip((state, q_off, fresh, positions, slots), want):
        assert got.tolist() == w
    assert t.d_table.tolist() == t.table and t.d_ring.tolist() == t.ring


def test_lengths_of_keep_are_not_in_the_table():
    m = misat()
    for seqs in ([(2, 5), (2, 20), (2, 3)], [(2, 40)]):
        s = Step(seqs, 2, 64, BF16)
        pool = s.pool(4)
        batch = s.batch(pool)
        n = len(seqs)
        before = s.table.clone()
        path, many = ints([[1]] * n), ints([1] * n)
        for at in range(2):
            with pytest.raises(m.MisatError):
                pool.keep(batch, path, many, out=s.table.view(-1)[at:at + n])
        pool.sync()
        assert torch.equal(s.table, before)


def test_plan_of_a_tree_stands_apart():
    m = misat()
    s = Step([(3, 20), (2, 5)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    flat = ints([-1] * 20)
    p = flat.data_ptr()
    st = torch.cuda.current_stream().cuda_stream
    f = m._lib.misat_kv_tree
    off, lens = s.q_off.data_ptr(), s.kv_len.data_ptr()
    for depth, bits in ((p, p + 40), (p + 16, p + 40), (p + 40, p), (p + 40, p + 16), (p + 40, p + 40), (p + 20, p + 36),
                        (off, p + 40), (p + 40, off - 16), (lens - 4, p + 40), (p + 40, lens + 4)):
        assert f(pool._h, batch._ref, p, 0, depth, bits, 1, st) == m.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (flat == -1).all()
    assert f(pool._h, batch._ref, p, 0, p + 20, p + 40, 1, st) == 0
    pool.sync()
    assert flat[5:15].tolist() == [0] * 5 + [1, 2, 4, 1, 2]
