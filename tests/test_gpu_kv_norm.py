"""Norm of each head with the rotation behind it, its gradients, and the append that applies it: against 64 bits."""

import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as kref  # noqa: E402
from tests import kv_step_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, F16, F32, Step, misat, rand  # noqa: E402

pytestmark = pytest.mark.gpu

HEADS = [  # heads, d, rot, half
    (1, 2, 2, True), (1, 2, 2, False), (3, 16, 16, True), (4, 64, 64, True), (4, 64, 64, False), (7, 80, 40, True),
    (28, 96, 48, False), (2, 128, 6, True), (2, 128, 6, False), (3, 13, 10, True), (3, 13, 10, False), (32, 128, 128, True),
    (5, 256, 256, True), (5, 256, 256, False), (2, 256, 16, True), (40, 120, 20, False), (70, 250, 250, True),
    (300, 8, 4, False), (1, 128, 128, True)]


def made(n, heads, d, dtype, wdtype, each, seed=0):
    x = rand((n, heads, d), dtype, seed + n + d, 1.7)
    dy = rand((n, heads, d), dtype, seed + n + d + 1)
    w = rand((heads, d) if each else (d,), wdtype, seed + 3) + 0.5
    g = torch.Generator(device="cuda").manual_seed(seed + n)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    return x, dy, w, pos


def within(rope, x, dy, w, pos, freq, half, eps=1e-6, offset=0.0, attn=1.0):
    norm = misat().HeadNorm(w, eps=eps, offset=offset)
    y, tol = ref.norm_rotate(x, pos, freq, half, w, eps, offset, attn)
    kref.assert_within("rotate", rope.norm_rotate(x, pos, norm), y, tol)
    dx, tol, dw, wtol = ref.norm_backward(x, dy, pos, freq, half, w, eps, offset, attn)
    got = rope.norm_backward(x, dy, pos, norm)
    kref.assert_within("dx", got[0], dx, tol)
    assert got[1].shape == w.shape and got[1].dtype == w.dtype
    kref.assert_within("dw", got[1], dw, wtol)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,d,rot,half", HEADS)
@pytest.mark.parametrize("n", [1, 9, 610])
def test_layouts(n, heads, d, rot, half, dtype):
    m = misat()
    each = (n + d) % 2 == 0
    x, dy, w, pos = made(n, heads, d, dtype, F32 if heads % 2 else dtype, each)
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    within(rope, x, dy, w, pos, kref.frequencies(rot), half)


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("n,heads", [(4000, 8), (20011, 5)])
def test_many_tokens(n, heads, each):
    x, dy, w, pos = made(n, heads, 64, F32, F32, each)
    within(misat().Rope(64), x, dy, w, pos, kref.frequencies(64), True, eps=1e-5, offset=1.0)


def test_scaled_rotation_eps_and_offset():
    m = misat()
    x, dy, w, pos = made(77, 6, 64, BF16, F32, True)
    kw = dict(base=500000.0, scaling=2, factor=8.0, orig_len=8192.0, beta_slow=1.0, beta_fast=4.0)
    rope = m.Rope(48, attn_factor=1.25, **kw)
    within(rope, x, dy, w, pos, kref.frequencies(48, **kw), True, eps=0.3, offset=1.0, attn=1.25)


@pytest.mark.parametrize("d,rot", [(64, 64), (60, 20)])
@pytest.mark.parametrize("half", [True, False])
def test_strides_alignment_and_in_place(half, d, rot):
    m = misat()
    heads, n = 5, 33
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    f = kref.frequencies(rot)
    for pad, first in ((8, 0), (8, 1), (3, 0), (0, 0)):
        wide = rand((n, heads * 2, d + pad + first), BF16, 4)
        x, dy = wide[:, :heads, first:first + d], wide[:, heads:, first:first + d]
        table = rand((heads, d + 3), BF16, 5)
        w = table[:, 1:1 + d]
        pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1001
        within(rope, x, dy, w, pos, f, half)
        norm = m.HeadNorm(w)
        dx = rope.norm_backward(x, dy, pos, norm)
        # into given tensors, and over the inputs
        out = torch.empty((heads, n, d), dtype=BF16, device="cuda").transpose(0, 1)
        assert rope.norm_rotate(x, pos, norm, out=out) is out
        kref.assert_within("out", out, *ref.norm_rotate(x, pos, f, half, w))
        x2 = wide.clone()[:, :heads, first:first + d]
        assert rope.norm_rotate(x2, pos, norm, out=x2) is x2
        kref.assert_within("in place", x2, *ref.norm_rotate(x, pos, f, half, w))
        want = ref.norm_backward(x, dy, pos, f, half, w)
        for over in ("x", "grad"):
            copy = wide.clone()
            a, b = copy[:, :heads, first:first + d], copy[:, heads:, first:first + d]
            o = a if over == "x" else b
            got = rope.norm_backward(a, b, pos, norm, out=o)
            assert got[0] is o
            kref.assert_within("dx over " + over, o, *want[:2])
            assert torch.equal(got[1], dx[1])
            rest = b if over == "x" else a
            assert torch.equal(rest, dy if over == "x" else x)


def test_gradients_against_differences():
    """Of the 64-bit definition, at steps of 1e-4: the definition's own gradients, and through them the kernel's."""
    m = misat()
    x, dy, w, pos = (t.double() if t.is_floating_point() else t for t in made(3, 2, 12, F32, F32, True))
    f = kref.frequencies(8)
    loss = lambda x, w: (ref.norm_rotate(x, pos, f, False, w, 1e-3, 1.0)[0] * dy).sum().item()  # noqa: E731
    dx, _, dw, _ = ref.norm_backward(x, dy, pos, f, False, w, 1e-3, 1.0)
    h = 1e-4
    for t, grad, at in ((x, dx, 0), (w, dw, 1)):
        flat = t.view(-1)
        for i in range(0, flat.numel(), 5):
            old = flat[i].item()
            flat[i] = old + h
            up = loss(x, w)
            flat[i] = old - h
            down = loss(x, w)
            flat[i] = old
            # third derivatives times h^2 / 6: heads of size one, r below 2, so below 100 h^2
            assert abs((up - down) / (2 * h) - grad.view(-1)[i].item()) < 1e-6, (at, i)
    rope = m.Rope(8, layout=m.ROPE_INTERLEAVED)
    got = rope.norm_backward(x.float(), dy.float(), pos, m.HeadNorm(w.float(), eps=1e-3, offset=1.0))
    want = ref.norm_backward(x.float(), dy.float(), pos, f, False, w.float(), 1e-3, 1.0)
    kref.assert_within("dx", got[0], *want[:2])
    kref.assert_within("dw", got[1], *want[2:])


def test_zeros_infinities_and_nan_stay_in_their_head():
    m = misat()
    x, dy, w, pos = made(40, 6, 64, BF16, BF16, False)
    rope, norm = m.Rope(32), m.HeadNorm(w)
    clean = rope.norm_rotate(x, pos, norm)
    clean_dx = rope.norm_backward(x, dy, pos, norm)[0]
    bad = x.clone()
    bad[3, 2] = 0.0
    bad[5, 1, 7] = math.inf
    bad[8, 0, 63] = math.nan
    got, (dx, _) = rope.norm_rotate(bad, pos, norm), rope.norm_backward(bad, dy, pos, norm)
    other = torch.ones((40, 6), dtype=torch.bool, device="cuda")
    other[3, 2] = other[5, 1] = other[8, 0] = False
    assert torch.equal(got[other], clean[other]) and torch.equal(dx[other], clean_dx[other])
    assert (got[3, 2] == 0).all()
    # inf / inf for the element and its partner, x / inf = 0 for the others
    nan = torch.isnan(got[5, 1])
    assert nan.nonzero().flatten().tolist() == [7, 23] and (got[5, 1][~nan] == 0).all()
    assert torch.isnan(got[8, 0]).all()


@pytest.mark.parametrize("each", [False, True])
def test_the_same_call_gives_the_same_bits(each):
    m = misat()
    x, dy, w, pos = made(3001, 6, 128, BF16, F32, each)
    rope, norm = m.Rope(128), m.HeadNorm(w)
    first = rope.norm_backward(x, dy, pos, norm)
    for _ in range(5):
        again = rope.norm_backward(x, dy, pos, norm)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_no_tokens_and_no_heads():
    m = misat()
    rope = m.Rope(16)
    for n, h, shape in ((0, 4, (32,)), (0, 4, (4, 32)), (5, 0, (32,)), (5, 0, (0, 32))):
        x = torch.empty((n, h, 32), dtype=BF16, device="cuda")
        pos = torch.zeros(n, dtype=torch.int32, device="cuda")
        w = torch.ones(shape, device="cuda")
        norm = m.HeadNorm(w)
        assert rope.norm_rotate(x, pos, norm).shape == x.shape
        dx, dw = rope.norm_backward(x, x, pos, norm)
        assert dx.shape == x.shape and dw.shape == w.shape and (dw == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,rot,half", [(4, 2, 64, 64, True), (7, 1, 72, 20, False), (32, 8, 128, 128, True),
                                               (3, 3, 24, 0, True)])
@pytest.mark.parametrize("norms", ["both", "q", "k", "none"])
def test_append(hq, hkv, d, rot, half, dtype, norms):
    """With trees (whose positions are depths) and without, into blocks that nothing else of is written."""
    m = misat()
    s = Step([(5, 37), (1, 1), (40, 40), (17, 200), (3, 19)], hkv, d, dtype)
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED) if rot else None
    f = kref.frequencies(rot)
    pool = s.pool(hq, rope=rope)
    batch = s.batch(pool)
    qkv = rand((s.T, hq + 2 * hkv, d), dtype, 9)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    wq, wk = rand((hq, d), F32, 10) + 1, rand((d,), dtype, 11)
    a, b = (wq if norms in ("both", "q") else None), (wk if norms in ("both", "k") else None)
    kw = dict(q_norm=None if a is None else m.HeadNorm(a, eps=1e-4), k_norm=None if b is None else m.HeadNorm(b, offset=1.0))
    g = torch.Generator().manual_seed(3)
    parents = [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for n in s.new for i in range(n)]
    for drafted in (False, True):
        if norms == "none" and not drafted:
            continue
        s.kb.copy_(rand(s.kb.shape, dtype, 1))
        want_k, want_v = s.kb.double(), s.vb.double()
        depth, _ = ref.tree(s.new, parents)
        slot = [L - n + i for n, L in zip(s.new, s.lens) for i in range(n)]
        first = [L - n for n, L in zip(s.new, s.lens) for i in range(n)]
        pos = torch.tensor([p + e for p, e in zip(first, depth)] if drafted else slot, device="cuda")
        tree = pool.tree(batch, torch.tensor(parents, dtype=torch.int32, device="cuda")) if drafted else None
        yk, kt = ref.norm_rotate(k, pos, f, half, b, 1e-6, 1.0)
        tol = torch.zeros_like(want_k)
        seq = [i for i, n in enumerate(s.new) for _ in range(n)]
        for t in range(s.T):
            blk = int(s.table[seq[t], slot[t] // 16])
            want_k[blk, :, slot[t] % 16], tol[blk, :, slot[t] % 16] = yk[t], kt[t]
            want_v[blk, :, slot[t] % 16] = v[t].double()
        got = pool.append(batch, k, v, q=q, tree=tree, **kw)
        pool.sync()
        kref.assert_within("q", got, *ref.norm_rotate(q, pos, f, half, a, 1e-4))
        kref.assert_within("k", s.kb, want_k, tol)
        assert torch.equal(s.vb.double(), want_v)
        s.kb.copy_(rand(s.kb.shape, dtype, 1))
        assert pool.append(batch, k, v, tree=tree, **kw) is None  # without queries
        kref.assert_within("k", s.kb, want_k, tol)
        mine = q.clone()
        assert pool.append(batch, k, v, q=mine, q_out=mine, tree=tree, **kw) is mine
        kref.assert_within("q in place", mine, *ref.norm_rotate(q, pos, f, half, a, 1e-4))


def test_append_of_many_short_sequences():
    """More sequences in a CTA's tokens than a warp looks at at once, empty ones among them."""
    m = misat()
    r = torch.Generator().manual_seed(7)
    new = torch.randint(0, 3, (3000,), generator=r).tolist()
    new[100:400] = [0] * 300
    s = Step([(n, n + int(torch.randint(0, 20, (1,), generator=r))) for n in new], 1, 64, BF16)
    pool = s.pool(2, rope=m.Rope(64))
    x = rand((s.T, 4, 64), BF16, 2)
    one = torch.ones(64, dtype=BF16, device="cuda")
    got = pool.append(s.batch(pool), x[:, 2:3], x[:, 3:], q=x[:, :2], q_norm=m.HeadNorm(one), k_norm=m.HeadNorm(one))
    pool.sync()
    pos = torch.tensor([L - n + i for n, L in zip(s.new, s.lens) for i in range(n)], device="cuda")
    seq = torch.tensor([b for b, n in enumerate(s.new) for _ in range(n)], device="cuda")
    kref.assert_within("q", got, *ref.norm_rotate(x[:, :2], pos, kref.frequencies(64), True, one))
    blk = s.table[seq, pos // 16].long()
    kref.assert_within("k", s.kb[blk, :, pos % 16], *ref.norm_rotate(x[:, 2:3], pos, kref.frequencies(64), True, one))
    assert torch.equal(s.vb[blk, :, pos % 16], x[:, 3:])


def test_append_malformed_is_a_sticky_error_and_writes_nothing_else():
    m = misat()
    s = Step([(4, 20), (3, 9), (2, 40)], 2, 32, BF16)
    pool = s.pool(2)
    norm = m.HeadNorm(torch.ones(32, device="cuda"))
    k, v = rand((s.T, 2, 32), BF16, 1), rand((s.T, 2, 32), BF16, 2)
    kb0, vb0, good = s.kb.clone(), s.vb.clone(), s.table.clone()
    pool.append(s.batch(pool), k, v, k_norm=norm)
    right = s.kb.clone()
    for what in ("block", "negative", "length"):
        s.kb.copy_(kb0)
        s.vb.copy_(vb0)
        s.table.copy_(good)
        s.kv_len.copy_(torch.tensor([20, 9, 40]))
        if what == "length":
            s.kv_len[1] = 2
        else:
            s.table[1, 0] = s.n_blocks if what == "block" else -1
        pool.append(s.batch(pool), k, v, k_norm=norm)
        with pytest.raises(m.MisatError) as e:
            pool.sync()
        assert e.value.code == m.ERR_INVALID_ARG
        want = right.clone()
        blk = int(good[1, 0])
        want[blk] = kb0[blk]
        assert torch.equal(s.kb, want)


def test_captured_and_on_another_stream():
    m = misat()
    x, dy, w, pos = made(300, 4, 64, BF16, F32, False)
    rope, norm = m.Rope(64), m.HeadNorm(w)
    want = (rope.norm_rotate(x, pos, norm), *rope.norm_backward(x, dy, pos, norm))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = (rope.norm_rotate(x, pos, norm), *rope.norm_backward(x, dy, pos, norm))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        got = (rope.norm_rotate(x, pos, norm), *rope.norm_backward(x, dy, pos, norm))
    for scale in (1.0, 2.0):
        x.copy_(x * scale)
        w.add_(0.25)  # the weight is read at every replay
        want = (rope.norm_rotate(x, pos, norm), *rope.norm_backward(x, dy, pos, norm))
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_written_tensors_have_a_new_version():
    m = misat()
    x, dy, w, pos = made(3, 2, 32, BF16, BF16, False)
    rope, norm = m.Rope(32), m.HeadNorm(w)
    a, b = x._version, dy._version
    rope.norm_backward(x, dy, pos, norm, out=dy)
    assert (x._version, dy._version > b) == (a, True)
    rope.norm_rotate(x, pos, norm, out=x)
    assert x._version > a


def test_refused_arguments():
    m = misat()
    rope = m.Rope(16)
    x, dy, w, pos = made(4, 2, 32, BF16, BF16, False)
    for bad in (torch.ones(32), torch.ones((1, 2, 32), device="cuda"), torch.ones(32, device="cuda", dtype=torch.float64), 3):
        with pytest.raises(ValueError):
            m.HeadNorm(bad)
    for weight in (torch.ones(31, device="cuda"), torch.ones((3, 32), device="cuda"), torch.ones(32, device="cuda", dtype=F16),
                   torch.ones(64, device="cuda")[::2], torch.ones((1, 32), device="cuda").expand(2, 32)):
        norm = m.HeadNorm(weight)
        with pytest.raises(ValueError):
            rope.norm_rotate(x, pos, norm)
        with pytest.raises(ValueError):
            rope.norm_backward(x, dy, pos, norm)
    norm = m.HeadNorm(w)
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(offset=math.nan)):
        with pytest.raises(m.MisatError) as e:
            rope.norm_rotate(x, pos, m.HeadNorm(w, **kw))
        assert e.value.code == m.ERR_INVALID_ARG
    for args in ((x, pos.long()), (x, pos[:3]), (x[0], pos), (x.cpu(), pos), (x.double(), pos)):
        with pytest.raises(ValueError):
            rope.norm_rotate(*args, norm)
    with pytest.raises(ValueError):
        rope.norm_backward(x, dy[:3], pos, norm)
    with pytest.raises(ValueError):
        rope.norm_backward(x, dy.float(), pos, norm)
    with pytest.raises(ValueError):
        rope.norm_rotate(x, pos, norm, out=dy.float())
    with pytest.raises(m.MisatError):  # over itself with other strides
        rope.norm_rotate(x, pos, norm, out=x.as_strided(x.shape, (32, 128, 1)))
    long = rand((2, 1, 264), BF16, 1)
    with pytest.raises(m.MisatError):
        rope.norm_rotate(long, pos[:2], m.HeadNorm(torch.ones(264, device="cuda")))
    # gradients' scratch: of a call with so many tokens that it needs some
    T = 4000
    x, dy, w, pos = made(T, 2, 32, BF16, BF16, False)
    n = m.misat_head_norm(w.data_ptr(), 0, m.BF16, 1e-6, 0.0)
    size = ctypes.c_int64()
    assert m._lib.misat_norm_rotary_work(rope._h, ctypes.byref(n), m.BF16, T, 2, 32, ctypes.byref(size)) == 0
    assert size.value > 0
    work, dx, dw = torch.empty(size.value + 16, dtype=torch.uint8, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    st = torch.cuda.current_stream().cuda_stream

    def back(work, size, dw=dw.data_ptr(), norm=n):
        return m._lib.misat_norm_rotary_backward(rope._h, ctypes.byref(norm), m.BF16, T, 2, 32, x.data_ptr(), 64, 32,
                                                 dy.data_ptr(), 64, 32, pos.data_ptr(), dx.data_ptr(), 64, 32, dw, 32, work,
                                                 size, st)

    assert back(work.data_ptr(), size.value) == 0
    assert back(None, size.value) == m.ERR_INVALID_ARG
    assert back(work.data_ptr() + 4, size.value) == m.ERR_INVALID_ARG
    assert back(work.data_ptr(), size.value - 1) == m.ERR_INVALID_ARG
    assert back(work.data_ptr(), size.value, dw=None) == m.ERR_INVALID_ARG
    assert back(work.data_ptr(), size.value, norm=m.misat_head_norm(None, 0, m.BF16, 1e-6, 0.0)) == m.ERR_INVALID_ARG
    assert back(work.data_ptr(), size.value, norm=m.misat_head_norm(w.data_ptr(), 31, m.BF16, 1e-6, 0.0)) == \
        m.ERR_INVALID_ARG
    # append: norms of other heads
    s = Step([(2, 20), (1, 5)], 2, 32, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    q, k = rand((3, 4, 32), BF16, 1), rand((3, 2, 32), BF16, 2)
    each = m.HeadNorm(torch.ones((2, 32), device="cuda"))
    with pytest.raises(ValueError, match="q_norm"):
        pool.append(batch, k, k, q=q, q_norm=each)
    with pytest.raises(ValueError, match="k_norm"):
        pool.append(batch, k, k, q=q, k_norm=m.HeadNorm(torch.ones((4, 32), device="cuda")))
    with pytest.raises(ValueError):
        pool.append(batch, k, k, q=k, k_norm=each)
    pool.sync()


@pytest.mark.parametrize("n", [1, 30, 31, 32, 33, 62, 63])
def test_append_of_tokens_of_no_sequence_is_a_sticky_error(n):
    """Tokens behind the last sequence, or before the first, are in none: nothing of them is written."""
    m = misat()
    s = Step([(1, 3 + b) for b in range(n)], 1, 16, BF16)
    pool = s.pool(1)
    norm = m.HeadNorm(torch.ones(16, device="cuda"))
    x = rand((n + 5, 1, 16), BF16, 1)
    for shift in (0, 5):
        s.kb.zero_()
        batch = pool.batch(s.q_off + shift, s.kv_len, s.table, n_tokens=n + 5, max_q=1)
        q = torch.full_like(x, 7.0)
        pool.append(batch, x, x, q=x, q_out=q, q_norm=norm, k_norm=norm)
        with pytest.raises(m.MisatError) as e:
            pool.sync()
        assert e.value.code == m.ERR_INVALID_ARG
        mine = slice(shift, shift + n)
        rest = torch.ones(n + 5, dtype=torch.bool)
        rest[mine] = False
        assert (q[rest.cuda()] == 7).all() and not (q[mine] == 7).all(-1).any()
        assert int((s.kb != 0).any(-1).sum()) == n


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,d,rot,half", [(9, 154, 106, False), (9, 154, 104, True), (33, 206, 206, False), (5, 252, 56, True),
                                              (64, 36, 36, True), (48, 128, 128, True)])
def test_vectors_of_two_elements(heads, d, rot, half, dtype):
    m = misat()
    x, dy, w, pos = made(333, heads, d, dtype, F32, True)
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    within(rope, x, dy, w, pos, kref.frequencies(rot), half)


@pytest.mark.parametrize("size", [2.0 ** 50, 2.0 ** 20, 2.0 ** -20, 2.0 ** -50])
@pytest.mark.parametrize("half", [True, False])
def test_sizes_of_values(half, size):
    """Squares stay inside 32 bits up to 2^59 an element; small heads are what eps leaves of them."""
    m = misat()
    x, dy, w, pos = made(50, 4, 64, BF16, F32, False)
    within(m.Rope(64, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED), x * size, dy, w, pos, kref.frequencies(64), half)


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("heads,d", [(1, 128), (7, 64), (40, 128), (64, 96), (200, 128), (3, 13)])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 31, 63, 64, 65, 130, 500])
def test_gradients_of_few_tokens(n, heads, d, each):
    """Around the numbers of tokens up to which one cluster of CTAs adds the weight's gradient."""
    m = misat()
    x, dy, w, pos = made(n, heads, d, BF16, F32 if n % 2 else BF16, each)
    rot = d // 4 * 2
    rope = m.Rope(rot, layout=m.ROPE_HALF if n % 3 else m.ROPE_INTERLEAVED)
    within(rope, x, dy, w, pos, kref.frequencies(rot), bool(n % 3))
    norm = m.HeadNorm(w)
    first = rope.norm_backward(x, dy, pos, norm)
    for _ in range(3):
        again = rope.norm_backward(x, dy, pos, norm)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
