"""Which kernel attention with masked and reshaped scores gets, on a machine without a GPU (scored_plan_probe.hip)."""
import os
import subprocess

import pytest

from paper_2603_08026_amd import binding, build
from tests import scored_shapes as S


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """shapes -> their plans"""
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    exe = str(tmp_path_factory.mktemp("scored") / "probe")
    d, so = os.path.split(binding.LIB_PATH)
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-O1", "-rdynamic", os.path.join(build.TESTS, "scored_plan_probe.hip"), "-o", exe, "-L" + d, "-l:" + so,
                        "-Wl,-rpath," + d], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(shapes):
        calls = [" ".join(str(int(x)) for x in (s.t == "bf16", s.H, s.Hkv, s.dh, s.pages, s.lists, s.lengths, s.B, s.L, s.cap, 1 if s.pages else s.B, s.room, 0))
                 for s in shapes]
        r = subprocess.run([exe], input="\n".join(calls) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        got = [[int(x) for x in line.split(" ")] for line in r.stdout.splitlines()]
        assert len(got) == len(calls)
        return got
    return run


def held(s, plan):
    bq, splits, fused, once, launch = plan[:5]
    assert (bq, splits > 1, bool(once)) == (s.bq, s.split, s.once), (s, plan)
    assert s.merge == ("" if splits == 1 else "launch" if launch else "last") and (splits == 1 or launch != fused), (s, plan)


def test_shapes_of_the_gpu_tests(plans):
    """Every call of the tests on the GPU gets the kernel that it is there for."""
    for s, plan in zip(S.ALL, plans(S.ALL)):
        held(s, plan)


def test_plans_fit_their_scratch(plans):
    """Partial rows fit the context's scratch, splits the merge's lanes, tiles of split keys the counters, rows the words of a launch's merge: also for lists
    of more rows than the context was made for."""
    shapes = []
    for t in ("bf16", "f32"):
        for H, Hkv, dh in ((2, 1, 64), (8, 2, 64), (28, 4, 128), (32, 32, 128), (64, 1, 128)):
            for pages, room in ((True, 1), (True, 64), (True, 4096), (False, 0)):
                for B in (1, 3, 64, 65, 300):
                    for L in (16, 1600, 40000):
                        if not pages and (L > 1600 or B * L * H * dh > 2 ** 27):
                            continue
                        for cap in sorted({1, B, 8 * B, 9 * B, 100 * B, 5000}):
                            if pages or cap <= B * L:
                                shapes.append(S.Shape(t, H, Hkv, dh, pages, True, pages or B % 2 == 1, B, L, cap, room or L, 0, False, "", False))
    kinds = set()
    for s, plan in zip(shapes, plans(shapes)):
        bq, splits, fused, once, launch, tiles, target, elems, rows, counters = plan
        assert 1 <= splits <= 128, (s, plan)
        if splits > 1:
            assert splits * s.cap * s.H * s.dh <= elems, (s, plan)
            assert 0 < target <= 1024, (s, plan)
            assert bool(launch) != bool(fused), (s, plan)
            assert not fused or tiles <= counters, (s, plan)
            assert not launch or s.cap <= rows, (s, plan)
        kinds.add((s.t, bq, "" if splits == 1 else "launch" if launch else "last"))
    assert kinds == {("f32", 2, ""), ("f32", 2, "last"), ("f32", 32, ""), ("f32", 32, "last"), *(("bf16", n, m) for n in (32, 128) for m in ("", "last", "launch"))}
