"""How products with a 4-bit head are planned, on the CPU: kd_ops_api.cpp compiled with
launchers that launch nothing (mx4_recorder.cpp)."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2608_03796_amd as kd
from tests.mx4_shapes import FAR, VARIANTS

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2608_03796_amd", "csrc")
FAKE = ctypes.c_void_p(0x10000)  # never dereferenced
FIELDS = ("kind", "nb", "r", "ks", "tok", "splits", "rows", "bytes")
DTYPES = (kd.KD_F32, kd.KD_BF16, kd.KD_MX4)


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libmx4host.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC",
                    os.path.join(CSRC, "kd_ops_api.cpp"), os.path.join(HERE, "mx4_recorder.cpp"),
                    "-o", so], check=True)
    return ctypes.CDLL(so)


def _plan(host, N, D, V, dtype, ld=None):
    v = (ctypes.c_int64 * len(FIELDS))()
    host.rec_plan(*[ctypes.c_int64(x) for x in (N, D, V)], dtype, ctypes.c_int64(ld or D), v)
    return dict(zip(FIELDS, v))


def _head(N, D, V, dtype):
    return kd.KdMx4Head(N, D, V, D, V, dtype, kd.KD_F32, 0)


def _size(host, N, D, V, dtype):
    n = ctypes.c_size_t(0)
    assert host.kd_mx4_logits_workspace_size(ctypes.byref(_head(N, D, V, dtype)), ctypes.byref(n)) == 0
    return n.value


def _logits(host, N, D, V, dtype, n):
    return host.kd_mx4_logits(ctypes.byref(_head(N, D, V, dtype)), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
                              ctypes.c_size_t(n), None)


@pytest.mark.parametrize("D,V,dtype", [
    (4096, 30001, kd.KD_BF16), (8192, 5003, kd.KD_BF16), (8192, 5003, kd.KD_MX4),
    (4096, 30001, kd.KD_F32), (65536, 40, kd.KD_F32), (1824, 1, kd.KD_MX4), (288, 1003, kd.KD_F32),
    (16384, 32768, kd.KD_BF16), (2048, 65536, kd.KD_F32), (4096, 131072, kd.KD_BF16)])
def test_one_workspace_for_every_batch(host, D, V, dtype):
    """A workspace of the size asked for the largest batch does for every smaller one."""
    for N in (1, 5, 63, 64, 65, 200, 2000, 20000):
        size = _size(host, N, D, V, dtype)
        rows = sorted({1, 2, 4, 5, *range(16, N, 16), *range(17, N, 48), N - 1, N} - {0})
        for n in rows:
            if n <= N:
                assert _plan(host, n, D, V, dtype)["bytes"] <= size, (n, N)
                assert _logits(host, n, D, V, dtype, size) == 0, (n, N)


def test_workspace_grows_with_the_rows(host):
    """Seeded sizes: the size asked for never falls as rows are added, and a call refuses
    less than its own rows take."""
    rng = random.Random(5)
    for _ in range(300):
        D, V = 32 * int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 20))
        dtype, last = rng.choice(DTYPES), 0
        for N in sorted(int(2 ** rng.uniform(0, 20)) for _ in range(12)):
            size = _size(host, N, D, V, dtype)
            assert size >= last, (N, D, V, dtype)
            last = size
            n = int(rng.uniform(1, N))
            assert _plan(host, n, D, V, dtype)["bytes"] <= size, (n, N, D, V, dtype)
            assert _logits(host, N, D, V, dtype, _plan(host, N, D, V, dtype)["bytes"] - 1) == 5


NAMES = {"f32": kd.KD_F32, "bf16": kd.KD_BF16, "mx4": kd.KD_MX4}


def _variant(host, N, D, V, dtype):
    p = _plan(host, N, D, V, dtype)
    if p["kind"] == 0:
        return "rows", p["r"], p["ks"]
    if p["kind"] == 1:
        return "wide", p["nb"], p["r"], p["splits"] > 1
    return "tiles", p["tok"], p["splits"] > 1


@pytest.mark.parametrize("name", NAMES)
def test_sizes_take_their_variant(host, name):
    """The sizes that the values are tested at take what they are listed for, and
    nothing that the plan returns is left out (seeded sizes)."""
    for variant, shapes in VARIANTS[name].items():
        for shape in shapes:
            assert _variant(host, *shape, NAMES[name]) == variant, shape
    rng = random.Random(3)
    for _ in range(60000):
        N, D, V = (int(2 ** rng.uniform(0, 13)), 32 * int(2 ** rng.uniform(0, 11)),
                   int(2 ** rng.uniform(0, 20)))
        assert _variant(host, N, D, V, NAMES[name]) in VARIANTS[name], (N, D, V)


def test_far_rows_take_tiles(host):
    for name, *shape in FAR:
        assert _variant(host, *shape, NAMES[name])[0] == "tiles", (name, shape)
