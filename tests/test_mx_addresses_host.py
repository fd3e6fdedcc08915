"""The 4-bit product stays within its arguments and within the workspace that it asks
for: built for the CPU, its kernels run with pages that fault around each of them
(tests/cpu_build/mx_addresses.cpp).  A read past a workspace cannot be seen in the
results, as what it reads is thrown away."""
import os
import re
import subprocess

import pytest

from paper_2304_13724_amd import build as hip_build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cpu_build")
F32, BF16, MX4 = 0, 1, 4


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("mx")
    with open(os.path.join(hip_build.PKG, "csrc", "bgmf_mx.hip")) as f:
        text = re.sub(r"asm volatile\([^;]*\);", ";", f.read())
    text = text.replace("../../include/bgmf.h", "bgmf.h")
    kernels, out = str(where / "kernels.inc"), str(where / "mx_addresses")
    with open(kernels, "w") as f:
        f.write(text)
    clang = os.path.join(os.path.dirname(os.path.dirname(hip_build.HIPCC)), "llvm", "bin", "clang++")
    res = subprocess.run(
        [clang, "-O2", "-std=c++17", "-w", "-I", HERE, "-I", os.path.join(hip_build.PKG, "csrc"),
         "-I", os.path.join(hip_build.ROOT, "include"), f'-DKERNELS="{kernels}"',
         os.path.join(HERE, "mx_addresses.cpp"), "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return out


def check(program, cases):
    lines = "".join(" ".join(map(str, c)) + "\n" for c in cases)
    res = subprocess.run([program], input=lines, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.count("in bounds") == len(cases), \
        (res.stdout.splitlines()[-1:], res.returncode, res.stderr[-500:])


# tiles of 64 users (the second number of items: and 128 items), one step of up to two
# blocks: rows that end at each of the workspace's multiples of 256 and before it, where
# the last tile has nothing behind it
EDGES = [33, 64, 192, 193, 256, 449, 512, 705, 768, 1024]


@pytest.mark.parametrize("k", [20, 64])
@pytest.mark.parametrize("type_", [F32, MX4])
def test_tiles_of_64_users(program, type_, k):
    check(program, [(type_, rows, items, k, BF16) for rows in EDGES
                    for items in (1_000, 128 * (254 // ((rows + 127) // 128)))])


@pytest.mark.parametrize("type_", [F32, BF16, MX4])
def test_all_kinds_of_tiles(program, type_):
    check(program, [
        (type_, 1, 1, 1, F32), (type_, 1, 5000, 64, F32), (type_, 32, 127, 200, BF16),
        (type_, 17, 333, 2500, F32), (type_, 40, 100, 96, F32), (type_, 100, 30, 3000, BF16),
        (type_, 37, 10_003, 200, BF16), (type_, 200, 300, 128, F32), (type_, 250, 301, 129, F32),
        (type_, 250, 16_400, 100, BF16), (type_, 700, 5_600, 64, BF16),
        (type_, 769, 4_700, 33, F32), (type_, 257, 16_385, 2_100, BF16)])
