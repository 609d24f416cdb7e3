"""The tiles that attention calls take, as the library plans them on the host (no GPU): the calls of
``attention_paths`` reach what they are meant to reach, and all kinds of tiles between them."""

import ctypes
import os
import subprocess

import pytest

pytest.importorskip("torch")

import paper_2402_15106_amd as dm  # noqa: E402
from paper_2402_15106_amd import _lib, build  # noqa: E402
from tests.attention_paths import PATHS, bounds  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"f32": dm.F32, "bf16": dm.BF16}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "attn_plan")
    subprocess.run([build._hipcc(), "-x", "hip", "--offload-host-only", "-O2", "-std=c++17",
                    os.path.join(ROOT, "tests", "native", "attn_plan.cpp"), "-o", exe], check=True, capture_output=True, timeout=120)

    def run(calls):
        text = "".join("%d %d %d %d %d %r %d %d %d\n" % c for c in calls)
        return subprocess.run([exe], input=text, check=True, capture_output=True, text=True, timeout=10).stdout.split("\n")[:-1]
    return run


def call_of(dtype, hd, dim, cap, Hk, G, what, room, *_):
    qb, kb = bounds(what)
    return Hk * G, Hk, hd, TYPES[dtype], dim, cap, qb[-1] + room, kb[-1] + room, len(qb) - 1


def test_calls_take_the_plans_that_they_are_meant_for(plan):
    got = plan([call_of(*p) for p in PATHS])
    assert len(got) == len(PATHS)
    assert [(p, g) for p, g in zip(PATHS, got) if p[-1] != g] == []


def test_every_kind_of_tile_is_among_them():
    """Tiles of 128 rows, whole and cut, for each type and width in each pass (bfloat16: for each way of scoring), heads that
    share their keys among them, rows two by two, and both kinds of tiles in one backward pass."""
    seen = set()
    for dtype, hd, dim, cap, Hk, G, what, room, p in PATHS:
        width = 32 if hd <= 32 else 64 if hd <= 64 else 128
        scores = "any" if dtype == "f32" else (cap > 0, dim if cap == 0 and dim == 0 else (dim > 0) + (dim > 2))
        tiles = p.split()
        seen |= {(dtype, width, i, t[0], int(t[1:]) > 1, scores) for i, t in enumerate(tiles[:3])}
        seen |= {(dtype, width, "shared", i, t[0], int(t[1:]) > 1) for i, t in enumerate(tiles[:3]) if G > 1}
        seen |= {(dtype, width, "pairs", int(tiles[2][1:]) > 1)} if tiles[3] == "1" else set()
        seen |= {(dtype, "both", tiles[1][0] + tiles[2][0])}
    for width in (32, 64, 128):
        for cut in (False, True):
            for i in range(3):
                for scores in ((False, 0), (True, 0), (False, 1), (False, 2), (True, 2)):
                    assert ("bf16", width, i, "W", cut, scores) in seen, (width, cut, i, scores)
                assert ("bf16", width, "shared", i, "W", cut) in seen
                assert ("f32", width, i, "W", cut, "any") in seen, (width, cut, i)
            assert ("bf16", width, "pairs", cut) in seen
    assert {("bf16", "both", "FW"), ("f32", "both", "FW"), ("f32", "both", "WF")} <= seen


def test_plans_agree_with_the_scratch_of_the_library(plan):
    """The same code as the library's: the parts of a plan are what its scratch has room for."""
    lib = dm.load_library()
    for p, g in zip(PATHS, plan([call_of(*p) for p in PATHS])):
        H, Hk, hd, dtype, dim, cap, nq, nk, S = call_of(*p)
        f, b = ctypes.c_size_t(), ctypes.c_size_t()
        # bounds are read on the device only: any address will do here
        st = lib.dsmp_attention_workspace(dm.attention_desc(H, Hk, hd, dtype, dim=dim, cap=cap), _lib.CSegments(nq, S, 64),
                                          _lib.CSegments(nk, S, 64), ctypes.byref(f), ctypes.byref(b))
        assert st == dm.OK
        sf, sq, sk = (int(t[1:]) for t in g.split()[:3])
        assert f.value == (0 if sf == 1 else sf * nq * H * (hd + 2) * 4), (p, g)
        parts = [nq * H * 4] * 2 + [sq * nq * H * hd * 4 if sq > 1 else 0] + [sk * nk * Hk * hd * 4 if sk > 1 else 0] * 2
        assert sum(parts) <= b.value <= sum(parts) + 5 * 256, (p, g)
