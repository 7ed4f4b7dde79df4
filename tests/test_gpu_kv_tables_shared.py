"""Shared blocks of a step's tables while sequences finish, wait and come back."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_kv import misat  # noqa: E402
from tests.test_gpu_kv_tables import Tables, ints  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3, 1500, 5000])
def test_a_finished_sequence_keeps_its_shared_number_while_it_waits(n):
    """The same tensor of shared blocks serves the steps after a sequence has finished."""
    m = misat()
    held = [4 if b % 3 else 6 for b in range(n)]
    shared = [2 if b % 3 else 5 for b in range(n)]
    t = Tables(held, 9, 3 * n)
    new, lens = [0 if b % 3 == 0 else 7 for b in range(n)], [0 if b % 3 == 0 else 60 for b in range(n)]
    for _ in range(3):  # in the first one every third finishes, and drops its shared blocks
        got = t.check(new, lens, shared)
        t.d_state, t.state, lens = got.state, got.state.tolist(), got.kv_len.tolist()
    assert t.state[0] == 0 and t.state[1] == 6
    # A row that gets blocks while its number stands: these would never be given back.
    before = t.state
    got = t.step([5] + new[1:], lens, shared)
    with pytest.raises(m.MisatError) as e:
        t.pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    assert got.state.tolist() == before and t.d_table.tolist() == t.table and t.d_ring.tolist() == t.ring
    shared[0] = 0
    got = t.check([5] + new[1:], lens, shared)
    t.d_state, t.state = got.state, got.state.tolist()
    got = t.check([0] * n, [0] * n, shared)
    assert got.state.tolist()[:n] == [0] * n


def test_a_shared_number_below_zero_is_refused_in_a_row_without_blocks():
    m = misat()
    t = Tables([0, 2], 6, 3, places=6)
    t.tables.step(t.d_state, ints([0, 3]), ints([0, 20]), n_tokens=3, max_q=3, shared=ints([-1, 0]))
    with pytest.raises(m.MisatError) as e:
        t.pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG


def test_a_row_shortened_below_its_shared_blocks_is_refused():
    m = misat()
    t = Tables([5, 2], 6, 3)
    got = t.check([0, 3], [20, 20], [4, 0])  # two blocks are left in the first row
    t.d_state, t.state = got.state, got.state.tolist()
    assert t.state[0] == 2
    t.step([1, 1], [20, 23], [4, 0])
    with pytest.raises(m.MisatError) as e:
        t.pool.sync()
    assert e.value.code == m.ERR_INVALID_ARG
    t.check([1, 1], [20, 23], [2, 0])


def test_a_step_serves_the_library_s_calls_as_any_batch():
    m = misat()
    t = Tables([1, 0, 1], 6, 9)
    made = t.step([5, 20, 3], [10, 0, 16])
    plain = t.pool.batch(made.q_off, made.kv_len, t.d_table, n_tokens=28, max_q=20)
    for name in ("n", "n_tokens", "max_q"):
        assert getattr(made, name) == getattr(plain, name)
    for name in ("q_off", "kv_len", "block_table"):
        assert getattr(made, name).data_ptr() == getattr(plain, name).data_ptr()
    x = torch.randn((28, 1, 8), device="cuda").to(t.kb.dtype)
    t.pool.append(plain, x, x)
    want = t.kb.clone()
    t.kb.zero_()
    st = torch.cuda.current_stream().cuda_stream
    assert m._lib.misat_kv_append(t.pool._h, made._ref, x.data_ptr(), 8, 8, x.data_ptr(), 8, 8, None, 0, 0, None, 0, 0, st) == 0
    t.pool.sync()
    assert torch.equal(t.kb, want) and (want != 0).any()
