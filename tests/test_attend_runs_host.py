"""The attention's deal of work, compiled for the host: parts that stay inside the buffers while the lengths
change under the call, and parts that cover the batch where they do not."""

import ctypes
import multiprocessing as mp
import os
import random
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2608_11152_gb300", "csrc")


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("runs") / "attend_runs.so")
    subprocess.check_call(["g++", "-O1", "-std=c++20", "-shared", "-fPIC", "-pthread", "-include", "cstring", "-w", "-I",
                           CSRC, "-o", out, os.path.join(HERE, "host", "attend_runs.cpp")])
    return out


def _offsets(new):
    return np.concatenate(([0], np.cumsum(new))).astype(np.int32)


def _deal(lib, x, y, group, hkv, window, grid, switch):
    """x, y: (new tokens, lengths) of the sequences before and after the change."""
    off_x, off_y = _offsets(x[0]), _offsets(y[0])
    len_x, len_y = np.array(x[1], np.int32), np.array(y[1], np.int32)
    p = [a.ctypes.data_as(ctypes.c_void_p) for a in (off_x, off_y, len_x, len_y)]
    seen, error = ctypes.c_int(), ctypes.c_int()
    n = len(x[0])
    tokens, max_q = int(off_x[-1]), int(max(list(x[0]) + list(y[0])))
    stride = int(max(list(x[1]) + list(y[1])) + 15) // 16
    bad = lib.deal(n, *p, tokens, max_q, ctypes.c_int64(stride), group, hkv, window, grid, ctypes.c_int64(switch),
                   ctypes.byref(seen), ctypes.byref(error))
    return bad, seen.value, error.value


def _trials(path, kind, seed, trials, result):
    lib = ctypes.CDLL(path)
    rng = random.Random(seed)
    for _ in range(trials):
        if kind == "columns":  # several items a CTA, chunks among them
            n, new_hi, hist_hi, group, hkv, grid = rng.randint(2, 12), 900, 3000, 4, rng.choice([1, 2, 8]), 3
        elif kind == "natural":  # single tokens
            n, new_hi, hist_hi, group, hkv, grid = rng.randint(2, 40), 1, 2000, 4, rng.choice([2, 3]), 4
        else:  # few items
            n, new_hi, hist_hi, group, hkv, grid = rng.randint(1, 4), 60, 6000, 4, 1, 8
        window = rng.choice([0, 0, 300])

        def lengths():
            new = [rng.randint(0 if new_hi > 1 else 1, new_hi) for _ in range(n)]
            return new, [x + rng.randint(0, hist_hi) for x in new]

        x = lengths()
        y = lengths()
        if rng.random() < 0.5:  # the same tokens, other lengths or an order of their own
            new = list(x[0])
            rng.shuffle(new)
            y = new, [t + rng.randint(0, hist_hi) for t in new]
        if rng.random() < 0.3:
            y = y[0], [-1 if rng.random() < 0.5 else v for v in y[1]]
        reads = (n * 3 * (grid + 1)) * 2
        for switch in [rng.randint(0, reads) for _ in range(3)]:
            bad, _, _ = _deal(lib, x, y, group, hkv, window, grid, switch)
            if bad:
                result.put(f"{bad} parts outside: {kind} {x} -> {y} after {switch} reads, group {group}, {hkv} kv heads, "
                           f"window {window}, {grid} CTAs")
                return
    result.put("")


@pytest.mark.parametrize("kind", ["columns", "natural", "few"])
def test_parts_stay_inside_while_lengths_change(so, kind):
    ctx = mp.get_context("spawn")  # (a division by zero ends the process)
    result = ctx.Queue()
    p = ctx.Process(target=_trials, args=(so, kind, 11, 25, result))
    p.start()
    p.join(240)
    assert p.exitcode == 0, f"ended with {p.exitcode}"
    assert result.get(timeout=5) == ""


@pytest.mark.parametrize("new,lens,group,hkv,grid", [
    ([300, 0, 77, 900], [300, 40, 1000, 2000], 4, 2, 3), ([1] * 20, [17 * i + 1 for i in range(20)], 4, 3, 4),
    ([5, 40], [3000, 40], 4, 1, 8), ([700, 700, 1], [700, 900, 5000], 1, 8, 5)])
def test_steady_lengths_are_dealt_without_an_error(so, new, lens, group, hkv, grid):
    lib = ctypes.CDLL(so)
    bad, seen, error = _deal(lib, (new, lens), (new, lens), group, hkv, 0, grid, 1 << 40)
    assert bad == 0 and error == 0 and seen >= sum(1 for x in new if x) * hkv // 2


@pytest.mark.parametrize("passes", range(18))
def test_query_copies_in_flight_are_waited_for_when_a_wait_runs_out(so, passes):
    lib = ctypes.CDLL(so)
    for kinds in range(81):
        assert lib.queries(passes, kinds) == 0, (passes, kinds)
