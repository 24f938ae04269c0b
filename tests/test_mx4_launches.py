"""adacc_mx4_*: launch shapes up to the documented sizes, written down instead of launched (tests/csrc/launch_recorder.cpp).  A launch has fewer
than 2^32 threads."""
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, BIG = 1 << 20, 1 << 50

# (function, arguments): rows and columns of blobs up to 2^30
COMPRESS = "adacc_mx4_compress"


def compress(mats, rows, cols, along, across, kind=0):
    return (COMPRESS, [kind, 0, P, mats, rows, cols, cols, rows * cols, None, 0, P if along else None, BIG, P if across else None, BIG, None])


CALLS = {
    "along": compress(1, (1 << 29) + 5, 40, True, False),
    "along, a few bytes a row": compress(1, 1 << 30, 1, True, False),
    "along, rows and columns": compress(1, 1 << 27, 4096, True, False, 2),
    "across, short matrices": compress((1 << 24) + 3, 2, 32, False, True),
    "across, single values": compress(1 << 30, 1, 1, False, True),
    "both": compress(1 << 25, 32, 32, True, True),
    "both, single columns": compress(1 << 26, 5, 1, True, True),
    "small": compress(1, 300, 300, True, True),
    "restoration": ("adacc_mx4_decompress", [P, BIG, 1 << 30, 8, P, 0, 8, None]),
    "small restoration": ("adacc_mx4_decompress", [P, BIG, 100, 100, P, 0, 100, None]),
    "one row": ("adacc_mx4_product", [P, BIG, 1, P, BIG, 1 << 30, 128, None, 0, P, 0, 1 << 30, None]),
    "many groups": ("adacc_mx4_product", [P, BIG, 1 << 18, P, BIG, 1 << 18, 128, P, 4096, P, 0, 1 << 18, None]),
    "few rows of many groups": ("adacc_mx4_product", [P, BIG, 4096 * 31, P, BIG, 1 << 18, 128, P, 4096, P, 0, 1 << 18, None]),
    "linear, many rows": ("adacc_mx4_linear", [0, 0, P, (1 << 29) + 64, 64, P, BIG, 16, 64, None, 0, P, 0, 16, P, BIG, None]),
    "gradient": ("adacc_mx4_gradient", [P, BIG, 1 << 20, P, BIG, 1 << 12, 1 << 20, P, 64, P, 0, 1 << 12, None]),
}

CHILD = """
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
recorder.recorded.restype = ctypes.c_uint64
library = ctypes.CDLL(sys.argv[2])
for name, (function, arguments) in json.load(sys.stdin).items():
    rc = getattr(library, function)(*[ctypes.c_uint64(a or 0) for a in arguments])
    room = (ctypes.c_uint64 * 4000)()
    n = recorder.recorded(room, ctypes.c_uint64(1000))
    print(json.dumps([name, rc, [list(room[4 * i:4 * i + 4]) for i in range(n)]]))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    import paper_2508_00806_amd as adacc
    if shutil.which("g++") is None or not os.path.exists(adacc.LIB_PATH):
        pytest.skip("needs g++ and the built library")
    so = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "csrc", "launch_recorder.cpp"), "-o", so], check=True)
    run = subprocess.run([sys.executable, "-c", CHILD, so, adacc.LIB_PATH], input=json.dumps(CALLS), capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stderr
    return {name: (rc, found) for name, rc, found in map(json.loads, run.stdout.splitlines())}


@pytest.mark.parametrize("name", CALLS)
def test_a_launch_has_fewer_than_2_to_32_threads(launches, name):
    rc, found = launches[name]
    assert rc == 0 and found
    for grid, threads, _, _ in found:
        assert 0 < grid * threads < 1 << 32, (grid, threads)


def workgroups(mats, rows, cols, height, strip):
    return mats * -(-rows // height) * -(-cols // strip)


@pytest.mark.parametrize("name,height,strip,merged", [("along", 32, 512, True), ("along, a few bytes a row", 32, 512, True), ("along, rows and columns", 32, 256, True),
                                                      ("across, short matrices", 128, 256, False), ("across, single values", 128, 256, False),
                                                      ("both", 128, 256, False), ("small", 128, 256, False)])
def test_the_launches_of_a_call_follow_each_other(launches, name, height, strip, merged):
    """Each begins with the workgroup behind the last one of the launch before, and none is left out."""
    _, found = launches[name]
    mats, rows, cols = CALLS[name][1][3:6]
    at = 0
    for grid, _, _, first in found:
        assert first == at
        at += grid
    assert at == (workgroups(1, mats * rows, cols, height, strip) if merged else workgroups(mats, rows, cols, height, strip))


def test_small_calls_take_one_launch(launches):
    assert len(launches["small"][1]) == len(launches["small restoration"][1]) == 1
