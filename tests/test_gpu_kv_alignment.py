"""Arrays of the library's KV calls that do not begin at a multiple of their elements: refused before a launch."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_kv import BF16, Step, misat, rand  # noqa: E402

pytestmark = pytest.mark.gpu


def setup():
    s = Step([(3, 20), (2, 5)], 2, 32, BF16)
    m = misat()
    rope = m.Rope(32)
    pool = s.pool(2, rope=rope)
    return m, s, rope, pool, torch.cuda.current_stream().cuda_stream


def test_arrays_of_a_batch():
    m, s, _, pool, st = setup()
    x = rand((5, 2, 32), BF16, 1)
    p = x.data_ptr()
    before = s.kb.clone()
    good = dict(n=2, n_tokens=5, max_q=3, q_off=s.q_off.data_ptr(), kv_len=s.kv_len.data_ptr(), block_table=s.table.data_ptr(),
                table_stride=s.table.shape[1])
    for name in ("q_off", "kv_len", "block_table"):
        b = ctypes.byref(m.misat_kv_batch(**{**good, name: good[name] + 2}))
        assert m._lib.misat_kv_append(pool._h, b, p, 64, 32, p, 64, 32, None, 0, 0, None, 0, 0, st) == m.ERR_INVALID_ARG
        assert m._lib.misat_kv_attend(pool._h, b, p, 64, 32, p, 64, 32, None, 0, st) == m.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(s.kb, before)


def test_arrays_of_a_tree_and_a_path():
    m, s, _, pool, st = setup()
    b = s.batch(pool)._ref
    flat = torch.full((64,), -1, dtype=torch.int32, device="cuda")
    p = flat.data_ptr()
    for i in range(3):
        at = [p, p + 64, p + 128]
        at[i] += 2
        assert m._lib.misat_kv_tree(pool._h, b, at[0], 0, at[1], at[2], 1, st) == m.ERR_INVALID_ARG
        assert m._lib.misat_kv_keep(pool._h, b, at[0], 2, at[1], at[2], st) == m.ERR_INVALID_ARG
    x = rand((5, 2, 32), BF16, 1)
    q = x.data_ptr()
    draft = m.misat_kv_draft(depth=p + 2, bits=p + 64, words=1, window=0)
    assert m._lib.misat_kv_append_norm(pool._h, b, None, None, ctypes.byref(draft), q, 64, 32, q, 64, 32, None, 0, 0, None, 0, 0,
                                       st) == m.ERR_INVALID_ARG
    assert m._lib.misat_kv_attend_tree(pool._h, b, ctypes.byref(draft), q, 64, 32, q, 64, 32, None, st) == m.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (flat == -1).all()


def test_arrays_of_a_step():
    m, s, _, pool, st = setup()
    flat = torch.full((1024,), -1, dtype=torch.int32, device="cuda")
    names = ("new_tokens", "kv_len", "shared", "state", "block_table", "ring", "state_out", "q_off", "kv_len_out", "positions",
             "slots")
    places = {name: flat.data_ptr() + 256 * i for i, name in enumerate(names)}
    work = flat.data_ptr() + 256 * len(names)
    for name in names:
        for off in (2, 4) if name == "slots" else (1, 2):
            step = m.misat_kv_step(n=2, n_tokens=8, max_q=5, columns=6, table_stride=6, ring_size=9,
                                   **{**places, name: places[name] + off})
            assert m._lib.misat_kv_tables(pool._h, ctypes.byref(step), work, 112, st) == m.ERR_INVALID_ARG, name
    torch.cuda.synchronize()
    assert (flat == -1).all()


def test_positions():
    m, _, rope, _, st = setup()
    x = rand((5, 2, 32), BF16, 1)
    out = torch.zeros_like(x)
    pos = torch.zeros(8, dtype=torch.int32, device="cuda")
    w = torch.ones(32, device="cuda")
    dw, work = torch.zeros_like(w), torch.empty(1 << 16, device="cuda")
    norm = ctypes.byref(m.misat_head_norm(w.data_ptr(), 0, m.F32, 1e-6, 0.0))
    p, o, at = x.data_ptr(), out.data_ptr(), pos.data_ptr() + 2
    assert m._lib.misat_rotary(rope._h, m.BF16, 5, 2, 32, p, 64, 32, at, o, 64, 32, 0, st) == m.ERR_INVALID_ARG
    assert m._lib.misat_norm_rotary(rope._h, norm, m.BF16, 5, 2, 32, p, 64, 32, at, o, 64, 32, st) == m.ERR_INVALID_ARG
    assert m._lib.misat_norm_rotary_backward(rope._h, norm, m.BF16, 5, 2, 32, p, 64, 32, p, 64, 32, at, o, 64, 32,
                                             dw.data_ptr(), 32, work.data_ptr(), 1 << 18, st) == m.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 0).all() and (dw == 0).all()
