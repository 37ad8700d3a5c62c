"""How the products of the gated block are cut into tiles and parts of K, without a GPU: the header that the library is built
from, in a small C++ library of its own."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64 = ctypes.c_int64


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++") or "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(gxx):
        pytest.skip("no C++ compiler")
    lib = str(tmp_path_factory.mktemp("plan") / "group_plan.so")
    res = subprocess.run([gxx, "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "native", "group_plan.cpp"), "-o", lib],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    so = ctypes.CDLL(lib)
    so.group_plan.argtypes = [ctypes.c_int, i64, i64, i64, i64, ctypes.c_int, ctypes.POINTER(i64)]
    so.group_plan.restype = None
    so.group_parts_bytes.argtypes, so.group_parts_bytes.restype = [i64], i64

    def of(bf16, groups, rows, half, k, most=8):
        out = (i64 * 4)()
        so.group_plan(int(bf16), groups, rows, half, k, most, out)
        return dict(zip(("small", "parts", "m_tiles", "blocks"), out))
    of.bytes = so.group_parts_bytes
    return of


def up(x, y):
    return -(-x // y)


SIZES = sorted({int(1.6 ** i) for i in range(28)} | {63, 64, 65, 255, 256, 257})


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("groups", [1, 2])
def test_every_tile_has_a_workgroup(plan, bf16, groups):
    for rows in SIZES:
        for half in (2, 4, 32, 386, 1024, 1792):
            for k in (4, 64, 640, 5000, 40960):
                p = plan(bf16, groups, rows, half, k)
                tile_m, tile_n = ((64, 64) if p["small"] else (256, 128)) if bf16 else (64, 32)
                tiles = groups * up(rows, tile_m) * up(half, tile_n)
                assert p["m_tiles"] == groups * up(rows, tile_m) and p["blocks"] == up(tiles, 8) * 8 * p["parts"]
                assert 1 <= p["parts"] <= 8 and (bf16 or not p["small"])
                if p["parts"] > 1:
                    part = groups * rows * 2 * half * 4
                    assert p["parts"] * part <= plan.bytes(part) <= 256 << 20 and up(k, 64 if bf16 else 32) >= 8 * p["parts"]
                if p["small"]:
                    here = up(tiles, 8) * p["parts"]
                    assert here <= 3 * 32 and p["small"] == (1 if here <= 2 * 32 else 2)
                assert plan(bf16, groups, rows, half, k, 1)["parts"] == 1


def test_room_for_parts_never_shrinks_with_the_batch(plan):
    sizes = [plan.bytes(n * 4096) for n in SIZES]
    assert sizes == sorted(sizes)


def test_the_gpu_tests_reach_every_form(plan):
    """The sizes that tests/test_gpu_repair_block.py names for it: small tiles, full-sized ones, either in parts."""
    from tests.test_gpu_repair_block import FORMS
    for (n, d, f, dtype), form in FORMS.items():
        p = plan(dtype == "bf16", 1, n, d // 2, 2 * up(f, 64) * 64)     # dX
        assert (("full", "small", "smallest")[p["small"]], p["parts"] > 1) == form, (n, d, f, p)
