"""The 8-bit decode's launch plan (csrc/plan.h), compiled alone on the CPU: pieces
cover every context, partials fit the workspace, limits follow the compute units."""

import ctypes
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_09590_amd", "csrc")

WRAPPER = """
#include "plan.h"
extern "C" int q8(long long segments, int group, long long blocks, int cus, long long slots, int* out) {
  return bros::plan_q8_decode(segments, group, blocks, cus, slots, out, out + 1);
}
extern "C" int by_rows(long long groups, long long blocks, int cus, long long slots, int* out) {
  return bros::plan_q8_prefill_rows(groups, blocks, cus, slots, out, out + 1);
}
extern "C" int waves(long long segments, long long blocks, int cus) { return bros::q8_decode_by_waves(segments, blocks, cus); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan_q8")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text(WRAPPER)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, str(src),
                    "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.q8.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)]

    lib.waves.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int]

    def call(segments, group, blocks, cus=256, slots=1 << 40):
        out = (ctypes.c_int * 2)()
        return tuple(out) if lib.q8(segments, group, blocks, cus, slots, out) else None

    call.waves = lambda segments, blocks, cus=256: bool(lib.waves(segments, blocks, cus))
    lib.by_rows.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)]

    def by_rows(groups, blocks, cus=256, slots=65536):
        out = (ctypes.c_int * 2)()
        return tuple(out) if lib.by_rows(groups, blocks, cus, slots, out) else None

    call.by_rows = by_rows
    return call


def test_pieces_cover_the_context_and_their_partials_fit(plan):
    rng = random.Random(1)
    for _ in range(4000):
        hq, hkv = rng.choice([(32, 8), (64, 8), (8, 1), (16, 8), (8, 8), (3, 3)])
        rows, cus = int(2 ** rng.uniform(0, 24)), rng.choice([32, 64, 96, 256, 304])
        blocks = int(2 ** rng.uniform(0, 27))
        slots = rows * hq + 4096 * min(hq, 8)
        got = plan(rows * hkv, hq // hkv, blocks, cus, slots)
        if got is None:
            continue
        size, n = got
        assert n >= 1 and size * n >= blocks and size * (n - 1) < blocks
        if n > 1:
            assert size % 2 == 0 and rows * hkv * n * (hq // hkv) <= slots


def test_which_calls(plan):
    assert plan(8, 4, 10) == (10, 1)               # one short row: whole
    assert plan(48, 4, 128) == (32, 4)
    assert plan(8, 4, 500) == (16, 32)             # one long row: pieces
    assert plan(16 * 8, 4, 512) == (32, 16)
    assert plan(64 * 8, 4, 512) is None
    assert plan(288 * 8, 8, 1024) is None          # a large batch: the even split
    assert plan(1 << 32, 1, 1) is None
    # on a part of the chip the limits scale
    assert plan(64, 4, 100, cus=32) == (100, 1)
    assert plan(64, 4, 100, cus=256)[1] > 1


def test_which_calls_go_by_waves(plan):
    assert not plan.waves(768, 4) and plan.waves(769, 4) and plan.waves(1024, 16)
    assert not plan.waves(1024, 17) and not plan.waves(1025, 9) and plan.waves(1025, 8) and plan.waves(2048, 24) and not plan.waves(2048, 25)
    assert not plan.waves(1 << 31, 1) and not plan.waves((1 << 32) + 8, 1)      # (a wave's index stays below 2^31)
    assert plan.waves(100, 8, cus=32) and not plan.waves(96, 8, cus=32)


def test_which_chunks_go_by_rows(plan):
    assert plan.by_rows(8, 1) == (1, 1) and plan.by_rows(8, 0) == (1, 1)
    assert plan.by_rows(512, 128) == (128, 1) and plan.by_rows(512, 129) is None
    assert plan.by_rows(768, 96) == (96, 1) and plan.by_rows(513, 97) is None and plan.by_rows(769, 1) is None
    assert plan.by_rows(96, 96, cus=32) == (96, 1) and plan.by_rows(97, 1, cus=32) is None
    # few groups on long contexts: pieces, where the workspace holds their partials
    assert plan.by_rows(24, 250) == (32, 8)
    assert plan.by_rows(24, 250, slots=24 * 8 * 16 - 1) is None
    assert plan.by_rows(24, 120, slots=0) == (120, 1)
    assert plan.by_rows(129, 192) == (192, 1) and plan.by_rows(129, 193) is None and plan.by_rows(128, 200) == (104, 2)
    assert plan.by_rows(24, 2049) is None
    rng = random.Random(2)
    for _ in range(4000):
        groups, blocks, cus = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 27)), rng.choice([32, 96, 256, 304])
        slots = rng.choice([0, 1000, 65536])
        got = plan.by_rows(groups, blocks, cus, slots)
        if got is None:
            continue
        size, n = got
        assert size * n >= blocks and size * (n - 1) < blocks
        assert n == 1 or (size % 8 == 0 and groups * n * 16 <= slots)
