"""Attention over a paged cache where the scores or the values are extreme, against the 64-bit definition."""

import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as ref  # noqa: E402
from tests.test_gpu_kv import BF16, F16, Step, rand  # noqa: E402

pytestmark = pytest.mark.gpu

# float16 weights: what one of them may be off by below the range of full precision, as a part of the row's
# largest (half of the smallest step, 2^-24, over the factor 2^11 that the weights carry).
F16_STEP = 2.0 ** -36


def one_head(seqs, hq, d, dtype, k0):
    """A step of one kv head whose scores are the keys' first elements, `k0` of each sequence's positions."""
    s = Step(seqs, 1, d, dtype)
    q = torch.zeros((s.T, hq, d), dtype=dtype, device="cuda")
    q[..., 0] = d ** 0.5
    for b, L in enumerate(s.lens):
        pos = torch.arange(L, device="cuda")
        block = s.table[b, pos // 16].long()
        s.kb[block, 0, pos % 16, 0] = k0(pos).to(dtype)
    return s, q


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("gap", [10.0, 14.0, 17.0, 18.0])
def test_attend_many_small_weights_behind_a_large_one(gap, n, dtype):
    """The first token takes most of the weight and has no value; 131,072 others below it make the result."""
    s, q = one_head([(n, 131073)], 2, 64, dtype, lambda pos: torch.where(pos == 0, gap, 0.0))
    s.kb[..., 1:] = 0
    s.vb.abs_().clamp_(0.25, 1.5)
    s.vb[int(s.table[0, 0]), 0, 0] = 0
    want = ref.attend(q, s.kb, s.vb, s.new, s.lens, s.table)
    pool = s.pool(2)
    out, lse = pool.attend(s.batch(pool), q, return_lse=True)
    pool.sync()
    ref.assert_within("out", out, want[0], want[1] + (131073 * F16_STEP * 1.5 if dtype == F16 else 0.0))
    ref.assert_within("lse", lse, want[2], want[3])


@pytest.mark.parametrize("order", ["rising", "falling", "spikes", "steps"])
def test_attend_maxima_that_move_in_float16(order):
    L, n = 1500, 150

    def k0(pos):
        x = pos.float()
        return {"rising": x * 0.25, "falling": -x * 0.25, "spikes": torch.where(pos % 211 == 7, x, -500.0),
                "steps": (pos // 128) * 2.5}[order]  # a rise of the exponent near the one that moves the reference

    s, q = one_head([(n, L)], 2, 64, F16, k0)
    s.poison()
    want = ref.attend(q, s.kb.nan_to_num(), s.vb.nan_to_num(), s.new, s.lens, s.table)
    pool = s.pool(2)
    out, lse = pool.attend(s.batch(pool), q, return_lse=True)
    pool.sync()
    ref.assert_within("out", out, want[0], want[1] + L * F16_STEP * s.vb.nan_to_num().abs().max().item())
    ref.assert_within("lse", lse, want[2], want[3])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,L", [(1, 30), (3, 300), (1, 5000), (150, 400)])
def test_attend_infinite_and_nan_values_that_are_seen(n, L, dtype):
    """The definition's infinities and NaN: in the rows that see them, and in no other."""
    d, hq = 64, 4
    inf, nan = float("inf"), float("nan")
    s = Step([(n, L), (2, 40)], 1, d, dtype)
    q = rand((s.T, hq, d), dtype, 3)
    pool = s.pool(hq)

    def call(q):
        out, lse = pool.attend(s.batch(pool), q, return_lse=True)
        pool.sync()
        return out, lse

    good, good_lse = call(q)
    # every score of a row is minus infinity: 0 / 0 in each element, and minus infinity as the sum's logarithm
    x = q.clone()
    s.kb[..., 5] = s.kb[..., 5].abs() + 1
    good, good_lse = call(q)
    x[0, 1, 5] = -inf
    out, lse = call(x)
    assert out[0, 1].isnan().all() and lse[0, 1].item() == -inf
    keep = torch.ones((s.T, hq), dtype=torch.bool, device="cuda")
    keep[0, 1] = False
    assert torch.equal(out[keep], good[keep]) and torch.equal(lse[keep], good_lse[keep])
    # a score of plus infinity, and a NaN in a query
    for bad in (inf, nan):
        x = q.clone()
        x[0, 1, 5] = bad
        out, lse = call(x)
        assert out[0, 1].isnan().all() and not lse[0, 1].isfinite()
        assert torch.equal(out[keep], good[keep]) and torch.equal(lse[keep], good_lse[keep])
    # one key that scores minus infinity takes no weight: as if it were not there
    p = L // 2
    at = (int(s.table[0, p // 16]), 0, p % 16)
    kept = s.kb[at].clone()
    x = q.clone()
    x[:n, :, 7] = 1
    s.kb[at][7] = -inf
    out, lse = call(x)
    key = ref.gather(s.kb, s.table[0], L)[:, 0].double()
    val = ref.gather(s.vb, s.table[0], L)[:, 0].double()
    see = torch.arange(L, device="cuda")[None] <= torch.arange(L - n, L, device="cuda")[:, None]
    z = torch.einsum("nhd,ld->nhl", x[:n].double(), key) / d ** 0.5
    z = torch.where(see[:, None], z, -inf).softmax(-1)
    u = ref.U[dtype]
    want = torch.einsum("nhl,ld->nhd", z, val)
    size = torch.einsum("nhl,ld->nhd", z, val.abs())
    xa = torch.einsum("nhd,ld->nhl", x[:n].double().abs(), key.abs().nan_to_num(0, 0, 0)).amax(-1) / d ** 0.5
    tol = u * (1 + 2.0 ** -10) * (size + want.abs()) + (
        (L / 16 + 8) * 2.0 ** -23 + 2 * ((d + 16) * 2.0 ** -23 * xa[..., None] + 2.0 ** -20)) * size + ref.TINY[dtype]
    ref.assert_within("out", out[:n], want, tol + L * F16_STEP * val.abs().max().item())
    s.kb[at] = kept
    # an infinite value that has weight
    kept = s.vb[at].clone()
    s.vb[at][9] = inf
    out, _ = call(q)
    rows = see[:, p]
    assert (out[:n, :, 9][rows] == inf).all()
    other = torch.arange(d, device="cuda") != 9
    assert torch.equal(out[..., other], good[..., other])
    s.vb[at] = kept


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,L", [(1, 700), (20, 700), (1, 9000)])
@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("size", [2.0 ** 5, 2.0 ** 9, 2.0 ** 12])
def test_attend_scores_far_from_zero(size, order, n, L, dtype):
    """Scores up to 2^28, far enough apart that a row is the mean of the values of its highest 128 keys; the exponent
    of a weight is the small difference of two large numbers."""
    d = 64

    def k0(pos):  # whole blocks of one score, a step of the type's last place between them
        step = (pos // 128).double() / (L // 128)
        x = 32768 + (32767.0 if dtype == F16 else 32768.0 - 256) * (step if order == "rising" else 1 - step)
        unit = 32 if dtype == F16 else 256
        return ((x // unit) * unit).float()

    s, q = one_head([(n, L)], 2, d, dtype, k0)
    s.kb[..., 1:] = 0
    q[..., 0] = size * d ** 0.5
    pool = s.pool(2)
    out, lse = pool.attend(s.batch(pool), q, return_lse=True)
    pool.sync()
    x = ref.gather(s.kb, s.table[0], L)[:, 0, 0].double() * size
    v = ref.gather(s.vb, s.table[0], L)[:, 0].double()
    see = torch.arange(L, device="cuda")[None] <= torch.arange(L - n, L, device="cuda")[:, None]
    z = torch.where(see, x[None], -float("inf"))
    p = z.softmax(-1)
    want, size_v = (p @ v)[:, None].expand(n, 2, d), (p @ v.abs())[:, None].expand(n, 2, d)
    u = ref.U[dtype]
    # weights and result rounded once, sums of up to 9,000 terms in 32 bits; a step of scores is 2^10 at least
    tol = u * (1 + 2.0 ** -10) * (size_v + want.abs()) + (L / 16 + 80) * 2.0 ** -23 * size_v + ref.TINY[dtype]
    ref.assert_within("out", out, want, tol)
    top = torch.logsumexp(z, -1)[:, None].expand(n, 2)
    ref.assert_within("lse", lse, top, 2.0 ** -22 * top)
