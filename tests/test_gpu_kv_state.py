"""What a pool keeps between calls: nothing but its error, and that only until the next sync."""

import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_kv import BF16, Step, misat, rand  # noqa: E402

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plant(tmp_path_factory):
    from paper_2608_11152_gb300 import build

    so = str(tmp_path_factory.mktemp("kv_state") / "kv_state.so")
    subprocess.check_call([build.nvcc(), *build.ARCH, "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart",
                           "shared", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), "-o", so,
                           os.path.join(HERE, "host", "kv_state.cu")])
    f = ctypes.CDLL(so).kv_plant
    f.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32]
    return f


@pytest.mark.parametrize("error", [-1, -7, 0])
def test_arrivals_that_a_call_left_are_gone_after_the_sync(plant, error):
    """A call that gave up inside leaves arrivals of its parts, whatever error was recorded before it."""
    m = misat()
    s = Step([(1, 40000), (3, 20000)], 2, 64, BF16)
    pool = s.pool(4)
    batch = s.batch(pool)
    q = rand((s.T, 4, 64), BF16, 3)
    want = pool.attend(batch, q)
    pool.sync()
    assert plant(pool._h, error, 1000) == 0
    with pytest.raises(m.MisatError) as e:
        pool.sync()
    assert e.value.code == (error or m.ERR_INTERNAL)
    for _ in range(3):
        out = torch.full_like(want, 7.0)
        assert torch.equal(pool.attend(batch, q, out=out), want)
        pool.sync()
