"""What the compiler makes of the sweep's hand-over of a column slice: every
store of a progress word comes after a wait for the wave's earlier stores.
Without that wait the word can be visible before the slice is, and the next
holder may read the slice as it was.  Compiles bgmf_sgd.hip for gfx950 (no GPU
needed) and reads the assembly.
"""
import os
import re
import subprocess

import pytest

from paper_2304_13724_amd import build as hip_build

SRC = os.path.join(hip_build.PKG, "csrc", "bgmf_sgd.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: instructions in the order of the assembly}"""
    out = str(tmp_path_factory.mktemp("sgd") / "sgd.s")
    flags = [f for f in hip_build.FLAGS if f not in ("-shared",) and not f.startswith("-W")]
    res = subprocess.run(
        [hip_build.HIPCC, *flags, "-I", os.path.join(hip_build.ROOT, "include"),
         "--cuda-device-only", "-S", SRC, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    found, body = {}, None
    with open(out) as f:
        for line in f:
            m = re.match(r"(_Z\S*k_sgd_\S*):", line)
            if m:
                body = found[m.group(1)] = []
            elif line.startswith(".Lfunc_end"):
                body = None
            elif body is not None:
                text = line.split(";")[0].strip()
                if text and not text.startswith("."):
                    body.append(text)
                elif text.startswith(".LBB"):
                    body.append(text)
    return found


def waits_for_stores(body, at):
    """Whether a wait for all vector memory precedes instruction ``at`` with no
    vector memory instruction, branch or label in between."""
    for text in reversed(body[:at]):
        if re.match(r"s_waitcnt\b.*\bvmcnt\(0\)", text):
            return True
        if re.match(r"(buffer|global|flat|scratch)_|s_cbranch|s_branch|\.LBB", text):
            return False
    return False


def test_progress_follows_the_slice(kernels):
    assert len(kernels) == 30  # five widths, masked or not: V in LDS, and in memory in two ways
    for name, body in kernels.items():
        words = [i for i, text in enumerate(body)
                 if re.match(r"global_store_dwordx2 .*\bsc1\b", text)]
        assert words, name  # the progress words are the kernels' only 8-byte device-scope stores
        for i in words:
            assert waits_for_stores(body, i), (name, body[max(0, i - 12):i + 1])


def test_the_check_itself():
    store, word = "buffer_store_dword v1, v2, s[0:3], 0 offen sc1", "global_store_dwordx2 v1, v[2:3], s[0:1] sc1"
    assert waits_for_stores([store, "s_waitcnt vmcnt(0) lgkmcnt(0)", "v_mov_b32 v1, 0", word], 3)
    assert not waits_for_stores([store, "s_waitcnt lgkmcnt(0)", word], 2)
    assert not waits_for_stores(["s_waitcnt vmcnt(0)", store, word], 2)
