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
