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
