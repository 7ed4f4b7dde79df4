"""The weight's gradient counts every token and head once: sums of ones, in which one that is missing or doubled shows.

Elements of x are 1 or -1 and positions 0, so a head's mean square is 1 (the product of a sum of d and the rounded 1 / d: to
2^-24), eps = 1e-12 vanishes beside it, r is 1 up to the reciprocal root's two units and that, 2^-21 in all, and a term
g x r is dy x r.  dy is 1 or -1 in about K of the N terms of an element, else 0.  A sum of K terms of size r in 32 bits, in any order,
is off by at most K 2^-24 of K r (adding zero is exact), so dw is off by less than (2^-21 + K 2^-24) K (1 + 2^-20): below 0.2
for K <= 1,700, while a term too few or too many is a whole number."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_kv import BF16, F16, F32, misat  # noqa: E402

pytestmark = pytest.mark.gpu


def check(n, heads, d, rot, half, dtype, each, seed=1):
    m = misat()
    g = torch.Generator(device="cuda").manual_seed(seed + n + d)

    def signs(p=1.0):
        x = torch.randint(0, 2, (n, heads, d), generator=g, device="cuda") * 2 - 1
        return x * (torch.rand((n, heads, d), generator=g, device="cuda") < p)

    terms = n * (1 if each else heads)
    x, dy = signs(), signs(min(1.0, 1400 / terms))
    want = (x * dy).sum(0 if each else (0, 1)).double()
    count = dy.abs().sum(0 if each else (0, 1)).double()
    assert count.max() <= 1700
    rope = m.Rope(rot, layout=m.ROPE_HALF if half else m.ROPE_INTERLEAVED)
    norm = m.HeadNorm(torch.ones((heads, d) if each else (d,), device="cuda"), eps=1e-12)
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    _, dw = rope.norm_backward(x.to(dtype), dy.to(dtype), pos, norm)
    off = (dw.double() - want).abs()
    tol = (2.0 ** -21 + count * 2.0 ** -24) * count * (1 + 2.0 ** -20)
    assert (off <= tol).all(), (off.max().item(), int((off > tol).sum()))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("heads,d,rot,half", [
    (8, 64, 64, True), (5, 64, 32, False), (32, 128, 128, True), (3, 96, 48, False), (40, 128, 64, False), (2, 256, 128, True),
    (7, 60, 60, True), (4, 26, 20, False), (6, 26, 26, True), (1, 13, 10, True), (9, 8, 8, True)])
@pytest.mark.parametrize("n", [610, 4001, 20011])
def test_every_token_counts_once(n, heads, d, rot, half, dtype, each):
    check(n, heads, d, rot, half, dtype, each)


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("heads,d", [(1, 64), (8, 128), (40, 128), (5, 26)])
def test_every_token_of_few_counts_once(heads, d, each):
    """One cluster, and where it changes to two kernels."""
    for n in [*range(1, 70), 96, 127, 128, 129, 191, 192, 193, 255, 256, 257, 383, 385]:
        check(n, heads, d, d - d % 4, True, BF16, each)
