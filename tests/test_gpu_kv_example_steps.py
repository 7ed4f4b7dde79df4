"""examples/routed_prefill.py step by step: the cached keys and values of every sequence, its rotated queries and its
outputs, each against 64 bits within its own rounding."""

import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
U = ref.U[torch.bfloat16]


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_prefill.py")
    spec = importlib.util.spec_from_file_location("routed_prefill", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class Rows:
    """q, k, v of a prompt in 64 bits, rotated, and what they may be off by: the projection is summed in 32 bits
    and rounded to 16 (of both elements of a pair, where it is rotated), the rotation rounds again."""

    def __init__(self, ex, layer, tokens, shift=0):
        x, w = layer.embed[torch.from_numpy(tokens).cuda()].double(), layer.w_qkv.double()
        y = x @ w
        e = U * y.abs() + x.shape[1] * 2.0 ** -23 * (x.abs() @ w.abs())
        n, d = len(tokens), ex.D
        parts = [ex.HQ * d, ex.HKV * d, ex.HKV * d]
        (q, k, v), (eq, ek, ev) = ((t.view(n, -1, d) for t in a.split(parts, 1)) for a in (y, e))
        ang = (torch.arange(n, dtype=torch.float64) + shift)[:, None] * ref.frequencies(d)
        c, s = ang.cos()[:, None].cuda(), ang.sin()[:, None].cuda()

        def turn(a, ea):
            p, r = a[..., :d // 2], a[..., d // 2:]
            out = torch.cat((p * c - r * s, p * s + r * c), -1)
            pair = ea[..., :d // 2] + ea[..., d // 2:] + 2.0 ** -20 * (p.abs() + r.abs())
            return out, torch.cat((pair, pair), -1) + U * out.abs()

        self.q, self.k, self.v = turn(q, eq), turn(k, ek), (v, ev)


def worst(got, want):
    return ((got.double() - want[0]).abs() / want[1]).max().item()


def test_steps_of_the_example_against_64_bits(example):
    ex = example
    seen = dict(steps=0, rows=0)

    def check(engine, tables, tokens, new, out):
        seen["steps"] += 1
        kb, vb = engine.blocks
        lens = [len(t) for t in tokens]
        width = max(len(t) for t in tables)
        table = torch.tensor([t + [-1] * (width - len(t)) for t in tables], dtype=torch.int32, device="cuda")
        at = 0
        for b, L in enumerate(lens):
            r = Rows(ex, engine.layer, tokens[b])
            assert worst(ref.gather(kb, table[b], L), r.k) <= 1
            assert worst(ref.gather(vb, table[b], L), r.v) <= 1
            tail = tuple(t[L - new[b]:] for t in r.q)
            assert worst(engine.q[at:at + new[b]], tail) <= 1
            at += new[b]
            seen["rows"] += L
        o, otol, _, _ = ref.attend(engine.q, kb, vb, new, lens, table)
        assert worst(out, (o, otol)) <= 1
        # the bounds are narrow enough to tell mistakes, on the shortest sequence: the last token's output
        b = int(np.argmin(lens))
        end, L = sum(new[:b + 1]), lens[b]
        assert worst(ref.gather(kb, table[b], L), Rows(ex, engine.layer, tokens[b], shift=1).k) > 1
        q, o, tol = engine.q[end - 1:end], out[end - 1:end].double(), otol[end - 1:end]
        short = ref.attend(q, kb, vb, [1], [L - 1], table[b:b + 1])[0]  # its own key not seen
        late = ref.attend(q, kb, vb, [1], [L - 16], table[b:b + 1, 1:])[0]  # the first block not seen
        assert worst(o, (short, tol)) > 1 and worst(o, (late, tol)) > 1

    stats = ex.run(inspect=check)
    assert seen["steps"] > 5 and seen["rows"] > stats["tokens"]
