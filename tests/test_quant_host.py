"""Entry points of normalised heads and of the 8-bit cache on a machine without a GPU (quant_probe.hip): what they refuse before anything is launched, the scratch that a
context has for them, and how attention over the cache is planned."""
import os
import subprocess

import pytest

from paper_2603_08026_amd import binding, build
from tests.test_gpu_quant_refresh import B as BATCH, L as LENGTH, PLANS
from tests.test_gpu_quant_splits import SPLIT


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


@pytest.mark.parametrize("t,hidden,H,Hkv,dh", [("bf16", 4096, 32, 32, 128), ("bf16", 3584, 28, 4, 128), ("bf16", 512, 8, 2, 64), ("f32", 256, 4, 4, 64)])
@pytest.mark.parametrize("max_rows", [1, 3, 8, 32, 106, 2048])
def test_scratch_of_a_context(probe, t, hidden, H, Hkv, dh, max_rows):
    """Partial results of attention over codes take the scratch that the GEMMs ask for, or 512 workgroups of 32 rows (heads of 128: 8 MiB) if that is more."""
    gemms, quant = (int(n) for n in probe("scratch", t, hidden, H, Hkv, dh, 4, 1024, max_rows, max_rows)[0].split(" "))
    assert gemms <= quant <= max(gemms, 512 * 32 * dh)
    if max_rows * H * dh * 16 >= 512 * 32 * dh:
        assert quant == gemms


# type, heads, KV heads, head_dim, sequences, keys, rows of a list -> rows in a tile, splits, keys of a split: as with scratch without end
@pytest.mark.parametrize("t,H,Hkv,dh,B,L,rows,bq,splits,chunk", [
    ("bf16", 2, 1, 128, 1, 32768, 1, 32, 37, 896), ("bf16", 28, 4, 128, 1, 32768, 1, 32, 37, 896), ("bf16", 32, 32, 128, 1, 32768, 1, 32, 8, 4096),
    ("bf16", 32, 32, 128, 8, 32768, 8, 32, 1, 32768), ("bf16", 28, 4, 128, 8, 4096, 32, 32, 7, 640), ("bf16", 8, 2, 64, 1, 32768, 2, 32, 32, 1024),
    ("f32", 4, 4, 64, 1, 32768, 1, 1, 27, 1216), ("f32", 32, 32, 128, 1, 32768, 3, 1, 5, 6560)])
def test_plans_of_few_rows(probe, t, H, Hkv, dh, B, L, rows, bq, splits, chunk):
    assert probe("plan", t, 256, H, Hkv, dh, B, L, rows, rows) == ["%d %d %d" % (bq, splits, chunk)]


# what the GPU tests of merged splits say that their cases run
@pytest.mark.parametrize("t,H,Hkv,dh,B,L,rows,splits,chunk", SPLIT)
def test_splits_of_the_merged_cases(probe, t, H, Hkv, dh, B, L, rows, splits, chunk):
    bq, *got = probe("plan", t, 256, H, Hkv, dh, B, L, rows * B, rows * B)[0].split(" ")
    assert [int(n) for n in got] == [splits, chunk] and int(bq) == (32 if t == "bf16" else 1)
    assert splits > 8  # (the merge reads eight at a time)


# ... and those of projections that the device plans
@pytest.mark.parametrize("hidden,H,Hkv,dh,count,splits,tiled,tail", PLANS)
def test_plans_of_the_refreshed_rows(probe, hidden, H, Hkv, dh, count, splits, tiled, tail):
    assert probe("q|k|v", "bf16", hidden, H, Hkv, dh, BATCH, LENGTH, 0, count) == ["%d %d %d" % (splits, tiled, tail)]
