"""The launches that attention over the block-scaled FP8 KV cache plans, from the library's own host code (kvb_plan_check.cpp):
that the GPU tests' cases take the tiles and runs which they are there for, and that runs and tiles fit."""
import os
import shutil
import subprocess

import pytest

import test_gpu_kvb
import test_gpu_kvb_range

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    rocm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    if cxx is None or not os.path.isdir(os.path.join(rocm, "hip")):
        pytest.skip("g++ or the HIP headers are missing")
    out = str(tmp_path_factory.mktemp("plan") / "check")
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-isystem", rocm,
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_20537_amd", "csrc"),
                    os.path.join(ROOT, "tests", "kvb_plan_check.cpp"), "-o", out], check=True)

    def run(n, T, hkv, G, d, copies=1, n_sel=0):
        """{tile: [(runs, blocks of a run) of its sequences]}"""
        seqs = [str(x) for _ in range(copies) for pair in zip(n, T) for x in pair]
        lines = subprocess.run([out, str(hkv * G), str(hkv), str(d), str(n_sel), *seqs], check=True, capture_output=True, text=True, timeout=60).stdout
        launches = [line.split() for line in lines.splitlines()]
        return {int(x[0]): [tuple(map(int, s.split(",")[1:])) for s in x[1:]] for x in launches}

    return run


def cases(test, names):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_cases_of_many_rows_take_tiles_of_128(plan, d):
    cut = whole = 0
    for n, T, hkv, G, copies in cases(test_gpu_kvb.test_attend_many_rows, "n, T, hkv, G, copies"):
        got = plan(n, T, hkv, G, d, copies)
        # of 64 channels tiles of 16 are the faster where few rows meet many blocks
        assert (128 in got) == (not (d == 64 and n[0] in (1999, 3500))), (n, T, got)
        cut += any(runs > 1 for runs, _ in got.get(128, []))
        whole += any(runs == 1 for runs, _ in got.get(128, []))
    assert cut >= 2 and whole >= 8
    for n, T, copies in cases(test_gpu_kvb.test_nan_and_infinities_stay_where_they_are_seen, "n, T, copies"):
        assert copies == 1 or 128 in plan([n], [T], 1, 3, d, copies)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_cases_of_the_range_tests(plan, d):
    for i, (n, T, G, copies) in enumerate(test_gpu_kvb_range.NARROW + test_gpu_kvb_range.WIDE):
        got = plan([n], [T], 1, G, d, copies)
        assert list(got) == [16 if i < 2 else 128] and all((runs > 1) == (i % 2 == 1) for runs, _ in got[16 if i < 2 else 128]), (n, T, got)
    n, T, G, copies = test_gpu_kvb_range.LONG
    assert plan([n], [T], 1, G, d, copies) == {128: [(1, -(-n // 64))] * copies}


@pytest.mark.parametrize("d", [64, 128, 256])
def test_runs_cover_the_blocks(plan, d):
    """Every run has blocks, no list's run more than a wave has lanes, and all together those of the sequence."""
    for n in (1, 64, 65, 513, 1000, 4097, 16385, 131072, 1 << 20):
        for T, G in ((1, 1), (1, 8), (5, 3), (129, 1), (161, 8), (4000, 4)):
            if T > n:
                continue
            for n_sel in (0, 1, 64, 65, 1000):
                got = plan([n, n], [T, 1], 2, G, d, n_sel=n_sel)
                blocks = n_sel or -(-n // 64)
                assert sorted(got) in ([16], [16, 128]) and sum(map(len, got.values())) == 2
                for runs, per in [x for seqs in got.values() for x in seqs]:
                    assert (runs - 1) * per < blocks <= runs * per and (not n_sel or per <= 64)
