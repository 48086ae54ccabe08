"""The sizes the GPU tests give the experts' products reach every kernel that
the rules choose between: a rule that moves must take its test cases along."""
import os
import shutil
import subprocess

import pytest

from tests.block_kernels import CASES

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1710_02368_amd", "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """kernels(cases) -> (forward, input gradient, weight gradient) of each."""
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("rules") / "experts_rules_main")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-I", INCLUDE,
                    os.path.join(HERE, "host_wave", "experts_rules_main.cpp"), "-o", exe], check=True)

    def ask(cases):
        lines = "".join(f"{int(d == 'bf16')} {r} {len(c)} {i} {o}\n" for d, r, c, i, o in cases)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout
        return [line.split("|") for line in out.splitlines()]

    return ask


BF16 = {"128x128 direct", "128x128 staged", "128x128 tiny", "256x256 direct"}
FP32 = {f"{t} {way}" for t in ("128x128", "64x64", "64x32") for way in ("staged", "tiny")}
WANT = {("bf16", 0): BF16 | {"few 16x16 staged", "few 32x32 staged"}, ("bf16", 1): BF16,
        ("bf16", 2): BF16 | {f"128x128 {way} parts" for way in ("direct", "staged", "tiny")},
        ("fp32", 0): FP32 | {"few 16x16 staged", "few 32x32 staged"}, ("fp32", 1): FP32,
        ("fp32", 2): FP32 | {f"64x64 {way} parts" for way in ("staged", "tiny")}}


def test_the_cases_reach_every_kernel(kernels):
    got = {k: set() for k in WANT}
    for case, names in zip(CASES, kernels(CASES)):
        for prod, name in enumerate(names):
            got[case[0], prod].add(name)
    for k in WANT:
        assert got[k] == WANT[k], (k, "not reached:", WANT[k] - got[k], "not expected:", got[k] - WANT[k])


def test_no_size_takes_another_kernel(kernels):
    """Over a grid of sizes nothing is chosen but the kernels above."""
    cases = [(d, r, [0] * e, i, o) for d in ("bf16", "fp32") for r in (1, 16, 100, 600, 3000, 20000, 300000)
             for e in (1, 3, 8, 64, 130, 1024) for i in (1, 3, 5, 64, 260, 1001, 4096, 30000)
             for o in (1, 3, 7, 72, 519, 2048, 9000)]
    for case, names in zip(cases, kernels(cases)):
        for prod, name in enumerate(names):
            assert name in WANT[case[0], prod], (case[0], case[1], len(case[2]), *case[3:], name)
