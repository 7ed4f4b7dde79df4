"""What the step's calls refuse before they look at a GPU, and the references that the GPU tests compare with."""

import ctypes
import os
import random
import subprocess

import pytest

from paper_2608_11152_gb300 import misat as m

torch = pytest.importorskip("torch")

from tests import kv_step_reference as ref  # noqa: E402

BAD = m.ERR_INVALID_ARG
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_null_handles_are_refused():
    step = m.misat_kv_step(n=1, n_tokens=1, max_q=1, columns=1, table_stride=1, ring_size=1)
    assert m._lib.misat_kv_tables(None, ctypes.byref(step), None, 0, None) == BAD
    norm = m.misat_head_norm(None, 0, m.BF16, 1e-6, 0.0)
    size = ctypes.c_int64()
    assert m._lib.misat_norm_rotary_work(None, ctypes.byref(norm), m.BF16, 1, 1, 8, ctypes.byref(size)) == BAD
    assert m._lib.misat_norm_rotary(None, ctypes.byref(norm), m.BF16, 1, 1, 8, None, 8, 8, None, None, 8, 8, None) == BAD
    assert m._lib.misat_norm_rotary_backward(None, ctypes.byref(norm), m.BF16, 1, 1, 8, None, 8, 8, None, 8, 8, None, None, 8,
                                             8, None, 8, None, 0, None) == BAD
    assert m._lib.misat_kv_tree(None, None, None, 0, None, None, 0, None) == BAD
    assert m._lib.misat_kv_append_norm(None, None, None, None, None, None, 0, 0, None, 0, 0, None, 0, 0, None, 0, 0, None) == BAD
    assert m._lib.misat_kv_attend_tree(None, None, None, None, 0, 0, None, 0, 0, None, None) == BAD
    assert m._lib.misat_kv_keep(None, None, None, 0, None, None, None) == BAD


def test_structures_are_the_header_s(tmp_path):
    """Sizes and offsets of the binding's structures against the compiler's."""
    names = ("misat_kv_step", "misat_head_norm", "misat_kv_draft")
    lines = []
    for n in names:
        lines.append(f'printf("{n} %zu", sizeof({n}));')
        lines += [f'printf(" %zu", offsetof({n}, {f}));' for f, _ in getattr(m, n)._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "misat.h"\nint main(void) {' + "".join(lines) +
                   'printf("%lld %d %d %d\\n", (long long)MISAT_KV_TABLES_WORK(7), MISAT_KV_TREE_NODES, MISAT_KV_ROOT, '
                   "MISAT_KV_ABSENT); return 0;}\n")
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)])
    got = subprocess.check_output([exe], text=True).split("\n")
    for n, line in zip(names, got):
        s = getattr(m, n)
        want = [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
        assert line.split() == [n] + [str(x) for x in want]
    assert got[3].split() == [str(24 * 7 + 64), str(m.KV_TREE_NODES), str(m.KV_ROOT), str(m.KV_ABSENT)]


def test_the_series_of_a_turn_holds_its_bound():
    """sin and cos of up to a quarter half turn, as the normed rotation works them out in 32 bits."""
    import numpy as np

    f = np.float32
    x = np.linspace(-0.25, 0.25, 200001).astype(f)
    y = x * x

    def fma(a, b, c):
        return (np.float64(a) * np.float64(b) + np.float64(c)).astype(f)

    s = fma(y, f(0.0821458866), f(-0.599264529))
    for c in (2.55016404, -5.16771278, -8.74227766e-8):
        s = fma(y, s, f(c))
    s = fma(x, f(3.14159274), x * s)
    c = fma(y, f(-0.0258068913), f(0.235330630))
    for k in (-1.33526277, 4.05871213, -4.93480220, 1.0):
        c = fma(y, c, f(k))
    at = x.astype(np.float64) * np.pi
    # three roundings of at most a value below one, and the terms left out
    assert np.abs(s - np.sin(at)).max() < 1.5 * 2.0 ** -24 and np.abs(c - np.cos(at)).max() < 1.5 * 2.0 ** -24


def test_reference_tables_keep_every_block():
    r = random.Random(1)
    n, blocks = 9, 60
    table, ring = [[-1] * 20 for _ in range(n)], list(range(blocks))
    state, lens = [0] * n + [0, blocks], [0] * n
    for _ in range(200):
        lens = [0 if r.random() < 0.2 else x for x in lens]
        free = state[-1] * 16 - 16 * n
        new = [r.randint(0, max(0, min(40, free // n))) for _ in range(n)]
        state, _, lens, pos, slots = ref.tables(n, new, lens, state, table, ring)
        held = [table[b][c] for b in range(n) for c in range(state[b])]
        held += [ring[(state[n] + i) % blocks] for i in range(state[n + 1])]
        assert sorted(held) == list(range(blocks)) and len(pos) == len(slots) == sum(new)
        assert all(state[b] == -(-lens[b] // 16) for b in range(n))


def test_reference_trees():
    depth, sees = ref.tree([5, 3], [-1, 0, 0, 2, -2, -1, -1, 1], 2)
    assert depth == [0, 1, 1, 2, 0, 0, 0, 1]
    assert sees == [[0], [1, 0], [2, 0], [3, 2], [], [0], [1], [2, 1]]
    assert ref.bits([[0, 31, 32], []], 2).tolist() == [[1 - 2 ** 31, 1], [0, 0]]
