"""The rule that cuts linear gradients into workgroups: which shapes of the kernels' tests it sends to the wide tile, and
that the parts it cuts rows into are the ones the workspace has room for."""
import ctypes
import os
import subprocess

import pytest

import paper_2302_05865_amd as fa
from linear_shapes import WIDE_IN_PARTS, WIDE_ONE_PART

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    out = tmp_path_factory.mktemp("plan") / "liblinear_plan.so"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2302_05865_amd", "csrc"),
                           os.path.join(ROOT, "tests", "emul", "linear_plan.cpp"), "-o", str(out)])
    lib = ctypes.CDLL(str(out))

    def run(sizes, features, outputs, dtype):
        splits, tiles = ctypes.c_int(), ctypes.c_int64()
        wide = lib.linear_plan(ctypes.c_int64(sum(sizes)), len(sizes), features, outputs, int(dtype == "bf16"), ctypes.byref(splits),
                               ctypes.byref(tiles))
        return bool(wide), splits.value, tiles.value
    return run


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_wide_tests_are_of_wide_tiles(plan, dtype):
    for shape in WIDE_ONE_PART[dtype]:
        assert plan(*shape, dtype)[:2] == (True, 1), shape
    for shape in WIDE_IN_PARTS[dtype]:
        wide, splits, _ = plan(*shape, dtype)
        assert wide and splits > 1, shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,features,outputs", [([3000], 65, 40), ([0, 0], 70, 50), ([1] * 64, 1, 1), ([256, 128], 1024, 768),
                                                    ([65536], 4096, 4096), ([9000, 1], 33, 257)])
def test_plans_and_workspaces(plan, sizes, features, outputs, dtype):
    wide, splits, tiles = plan(sizes, features, outputs, dtype)
    o, i = {"f32": [(64, 128), (128, 256)], "bf16": [(128, 128), (256, 256)]}[dtype][wide]
    assert tiles == -(-outputs // o) * -(-features // i)
    mean = -(-sum(sizes) // len(sizes))
    assert splits == 1 or splits <= -(-mean // 64)            # a part has a step of 64 rows at least
    need = fa.load_library().fa_linear_grad_workspace((ctypes.c_int64 * len(sizes))(*sizes), len(sizes), features, outputs,
                                                      int(dtype == "bf16"))
    assert need == (0 if splits == 1 else 4 * len(sizes) * splits * (outputs * features + outputs))
