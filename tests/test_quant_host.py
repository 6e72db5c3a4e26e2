"""Entry points of normalised heads and of the 8-bit cache on a machine without a GPU (quant_probe.hip): what they refuse before anything is launched."""
import os
import subprocess

import pytest

from paper_2603_08026_amd import binding, build


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    exe = str(tmp_path_factory.mktemp("quant") / "probe")
    d, so = os.path.split(binding.LIB_PATH)
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-O1", "-rdynamic", os.path.join(build.TESTS, "quant_probe.hip"), "-o", exe, "-L" + d, "-l:" + so,
                        "-Wl,-rpath," + d], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(case, t, hidden, H, Hkv, dh, B, L, max_rows, cap):
        args = [str(a) for a in (case, int(t == "bf16"), hidden, H, Hkv, dh, B, L, max_rows, cap)]
        r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return r.stdout.splitlines()
    return run


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("case,weights", [("refresh", "wq wk wv bq bk bv g_attn"), ("step", "wq wk wv bq bk bv g_attn wo w_gate w_up w_down g_ffn")])
def test_misaligned_weights_are_refused(probe, case, weights, t):
    """Kernels read 16 bytes of a matrix, bias or gain at a time."""
    lines, launched = probe(case, t, 256, 4, 2, 64, 2, 100, 200, 30), []
    at = {}
    for line in lines:
        name, *rc = line.split(" ")
        if name in ("none", *weights.split()):
            at[name] = int(rc[0])
            launched.append(name)
        else:  # a kernel: of the call whose line comes next
            assert not launched, line
    assert at == dict({n: -1 for n in weights.split()}, none=0)


def test_all_tokens_need_no_room_in_the_context(probe):
    """Where a call keeps nothing of a row, no list means all tokens whatever the context's lists hold."""
    lines = [x.split(" ") for x in probe("all rows", "bf16", 256, 4, 2, 128, 2, 200, 3, 3)]
    assert [x for x in lines if len(x) == 2] == [["attention", "0"], ["write", "0"], ["read", "0"]]
