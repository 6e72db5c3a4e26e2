"""Entry points of requests over pages and of masked scores on a machine without a GPU (pages_probe.hip): what they refuse before anything is
launched, which attention kernel a call gets, and the rotation's turns."""
import math
import os
import subprocess
from decimal import Decimal, getcontext

import pytest

from paper_2603_08026_amd import binding, build


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    exe = str(tmp_path_factory.mktemp("pages") / "probe")
    d, so = os.path.split(binding.LIB_PATH)
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-O1", "-rdynamic", os.path.join(build.TESTS, "pages_probe.hip"), "-o", exe, "-L" + d, "-l:" + so,
                        "-Wl,-rpath," + d], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(*args):
        r = subprocess.run([exe, *(str(a) for a in args)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return r.stdout.splitlines()
    return run


def test_refusals(probe):
    """Every call has the code that its name says (none: 0), and one that is refused launches nothing."""
    launched, calls = 0, 0
    for line in probe("refuse"):
        words = line.split(" ")
        if not words[-1].lstrip("-").isdigit():  # a kernel: of the call whose line comes next
            launched += 1
            continue
        want = int(words[-2]) if len(words) > 2 and words[-2].lstrip("-").isdigit() else 0
        assert int(words[-1]) == want, line
        assert launched == 0 or want == 0, line
        assert launched or want or words[0] == "nothing", line
        launched, calls = 0, calls + 1
    assert calls > 60


@pytest.mark.parametrize("theta,dh", [(10000.0, 128), (500000.0, 64), (0.25, 64)])
def test_turns(probe, theta, dh):
    """theta^(-2p/dh) / 2 pi modulo 1, in 2^-64: off by the roundings of a 64-bit mantissa (the power's, the quotient's) times the whole turns."""
    getcontext().prec = 50
    pi = Decimal("3.14159265358979323846264338327950288419716939937510")
    for p, line in enumerate(probe("turns", theta, dh)):
        whole = (Decimal(theta).ln() * Decimal(-2 * p) / Decimal(dh)).exp() / (2 * pi)
        want = (whole % 1) * 2 ** 64
        off = abs(Decimal(int(line)) - want)
        assert min(off, 2 ** 64 - off) <= 8 * math.ceil(whole), (p, line, want)


# bf16, heads, KV heads, head_dim, over pages, sequences, keys at most, rows -> packed rows of a workgroup, whether keys are split
@pytest.mark.parametrize("t,H,Hkv,dh,pages,B,L,rows,bq,split", [
    (1, 32, 32, 128, 1, 1, 4096, 1, 128, True), (1, 28, 4, 128, 1, 32, 32768, 32, 128, True), (1, 32, 32, 128, 1, 16, 1280, 512, 128, False),
    (1, 28, 4, 128, 1, 4, 8192, 8192, 128, False), (1, 32, 32, 128, 0, 16, 1280, 2048, 128, False), (1, 8, 2, 64, 0, 2, 200, 2, 32, False),
    (0, 4, 4, 64, 1, 1, 4096, 1, 2, True), (0, 4, 4, 64, 0, 2, 1000, 800, 32, False)])
def test_plans(probe, t, H, Hkv, dh, pages, B, L, rows, bq, split):
    """Few rows of long sequences split their keys, many do not, and no plan has more splits than its scratch or 128."""
    got = [int(x) for x in probe("plan", t, H, Hkv, dh, pages, B, L, rows)[0].split(" ")]
    assert got[0] == bq and (got[1] > 1) == split and got[1] <= 128
