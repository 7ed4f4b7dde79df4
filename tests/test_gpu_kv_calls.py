"""The KV operators' calls on torch tensors: what they tell torch, and what they refuse."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_kv import BF16, Step, misat, rand  # noqa: E402

pytestmark = pytest.mark.gpu


def test_tensors_that_are_written_have_a_new_version():
    m = misat()
    s = Step([(2, 20), (1, 5)], 2, 32, BF16)
    rope = m.Rope(32)
    pool = s.pool(4, rope=rope)
    batch = s.batch(pool)
    q, k, v = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 2), rand((3, 2, 32), BF16, 3)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")

    def newer(call, *tensors):
        before = [t._version for t in tensors]
        others = [t._version for t in (k, v)]
        call()
        assert all(t._version > b for t, b in zip(tensors, before))
        assert [t._version for t in (k, v)] == others

    out = torch.empty_like(q)
    newer(lambda: rope.rotate(q, pos, out=q), q)
    newer(lambda: rope.backward(q, pos, out=out), out)
    newer(lambda: pool.append(batch, k, v), s.kb, s.vb)
    newer(lambda: pool.append(batch, k, v, q=q, q_out=q), q, s.kb, s.vb)
    newer(lambda: pool.attend(batch, q, out=out), out)
    # a value that a gradient needs and that is then rotated in place is noticed
    x = rand((3, 4, 32), torch.float32, 4).requires_grad_()
    y = x * 1.0
    z = (y * y).sum()
    rope.rotate(y, pos, out=y)
    with pytest.raises(RuntimeError, match="inplace"):
        z.backward()
    # tensors without a version are written as before
    with torch.inference_mode():
        a = rand((3, 4, 32), BF16, 5)
    b = a.clone()
    rope.rotate(a, pos, out=a)
    assert torch.equal(a, rope.rotate(b, pos))
    pool.sync()


def test_a_batch_of_another_device_is_refused():
    m = misat()
    s = Step([(2, 20), (1, 5)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    calls = m._torch_calls()
    other = calls.pool_state(pool._h.value, 1, s.kb, s.vb, 4)  # (looked at, never launched with)
    k = rand((3, 2, 32), BF16, 1)
    with pytest.raises(ValueError, match="^batch: "):
        calls.append(other, batch._state, k, k, None, None)
    with pytest.raises(ValueError, match="^batch: "):
        calls.attend(other, batch._state, k, None, 0, False)


def test_a_rotation_stays_while_a_pool_applies_it():
    m = misat()
    s = Step([(2, 20), (1, 5)], 2, 32, BF16)
    rope = m.Rope(32)
    pools = [s.pool(4, rope=rope) for _ in range(2)]
    q, k = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 2)
    want = pools[0].append(s.batch(pools[0]), k, k, q=q)
    for pool in pools:
        with pytest.raises(m.MisatError) as e:
            rope.close()
        assert e.value.code == m.ERR_STATE
        assert torch.equal(pool.append(s.batch(pool), k, k, q=q), want)
        pool.close()
        pool.close()
    rope.close()
    rope.close()
    with pytest.raises(ValueError, match="rope"):  # not a pool without a rotation
        s.pool(4, rope=rope)
    with pytest.raises(ValueError):
        rope.rotate(q, torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_a_call_that_cannot_be_ordered_behind_the_last_one_is_an_error():
    m = misat()
    s = Step([(1, 3000), (4, 20)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    q = rand((5, 4, 32), BF16, 1)
    out, side = torch.empty_like(q), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = pool.attend(batch, q)
    torch.cuda.synchronize()
    graph, third = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="relaxed"):
        in_graph = pool.attend(batch, q)
        with torch.cuda.stream(third), pytest.raises(m.MisatError) as e:
            pool.attend(batch, q, out=out)
    assert e.value.code == m.ERR_STATE
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(in_graph, want)
    with torch.cuda.stream(third):  # and again once the capture is over
        pool.attend(batch, q, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("odd", [0, 3])
@pytest.mark.parametrize("seqs,hq,hkv,d", [
    ([(1, 40000), (2, 20000)], 8, 2, 128),             # items split between processors
    ([(300, 900), (129, 5000), (1, 7)], 4, 4, 64),     # two tiles of an item
    ([(1, 40 + i) for i in range(333)], 8, 8, 64),     # two heads of an item at a time
    ([(77, 50), (300, 1200)] * 40, 6, 3, 72)])         # many items, rows without keys among them
def test_attend_into_its_queries(seqs, hq, hkv, d, odd):
    s = Step(seqs, hkv, d, BF16)
    pool = s.pool(hq)
    batch = s.batch(pool)
    wide = rand((s.T, hq * d + 8), BF16, 3)
    q = wide[:, odd:odd + hq * d].view(s.T, hq, d)
    keep = wide.clone()
    want, want_lse = pool.attend(batch, q, return_lse=True)
    out, lse = pool.attend(batch, q, out=q, return_lse=True)
    pool.sync()
    assert out is q and torch.equal(q, want) and torch.equal(lse, want_lse)
    assert torch.equal(wide[:, :odd], keep[:, :odd]) and torch.equal(wide[:, odd + hq * d:], keep[:, odd + hq * d:])


def test_results_at_the_address_of_their_input_with_other_strides():
    m = misat()
    x = rand((4096,), BF16, 1)
    y = x.clone()
    rope = m.Rope(32)

    def step(n):
        s = Step([(n, 20)], 2, 32, BF16)
        pool = s.pool(4, rope=rope)
        return pool, s.batch(pool), rand((n, 2, 32), BF16, 2)

    pool, batch, k = step(3)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    a, b, c = (x.as_strided((3, 4, 32), t) for t in ((128, 32, 1), (256, 32, 1), (128, 64, 1)))
    for other in (b, c):
        for call in (lambda: rope.rotate(a, pos, out=other), lambda: pool.append(batch, k, k, q=a, q_out=other),
                     lambda: pool.attend(batch, a, out=other)):
            with pytest.raises(m.MisatError) as e:
                call()
            assert e.value.code == m.ERR_INVALID_ARG
    assert torch.equal(x, y)
    # a single token's stride is not stepped over
    pool, batch, k = step(1)
    one, same = x.as_strided((1, 4, 32), (999, 32, 1)), x.as_strided((1, 4, 32), (128, 32, 1))
    want = rope.rotate(one.clone(), pos[1:2])
    assert torch.equal(rope.rotate(one, pos[1:2], out=same), want)
    want = pool.append(batch, k, k, q=one.clone())
    assert torch.equal(pool.append(batch, k, k, q=one, q_out=same), want)
    want = pool.attend(batch, one.clone())
    assert torch.equal(pool.attend(batch, one, out=same), want)
