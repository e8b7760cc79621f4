"""What the compiler made of the kernels between hidden states and token ids: none may need scratch memory (the selection of the
best tokens once did, for a few bytes, and took half as long again), and the tiles of bpe_linear must fit a compute unit as often
as the estimate that chooses them says.  Device-only compilations to assembly; no GPU."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import CSRC, ROOT, _usage


@pytest.fixture(scope="module")
def usage(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    from paper_2603_02597_amd.build import FLAGS
    found = {}
    for name in ("bpe_linear", "bpe_grammar", "bpe_logits"):
        out = str(tmp_path_factory.mktemp("isa") / (name + ".s"))
        flags = [f for f in FLAGS if f not in ("-shared", "-fPIC")]
        r = subprocess.run([hipcc, *flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only",
                            "-Rpass-analysis=kernel-resource-usage", os.path.join(CSRC, name + ".hip"), "-o", out],
                           capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-3000:]
        assert "loop not unrolled" not in r.stderr, name
        found.update(_usage(r.stderr))
    return found


def test_no_kernel_needs_scratch_memory(usage):
    assert len(usage) >= 30, sorted(usage)
    for k, u in usage.items():
        assert u.get("ScratchSize", 0) == 0 and u.get("VGPRs Spill", 0) == 0, (k, u)


def test_tiles_fit_as_often_as_the_estimate_says(usage):
    text = open(os.path.join(CSRC, "bpe_linear.hip")).read()
    tiles = re.findall(r"\{(\d+), (\d+), (\d+), [\d.]+, [\d.]+, \d+\}", text)
    assert len(tiles) == 6
    for bm, bn, resident in tiles:
        kernels = [u for k, u in usage.items() if f"linear_block_kernel" in k and f"Li{bm}ELi{bn}E" in k and "Lb1E" in k]
        assert len(kernels) == 2
        for u in kernels:
            waves = 512 // (-(-(u["VGPRs"] + u.get("AGPRs", 0)) // 8) * 8)           # per SIMD; a workgroup is one wavefront on each
            assert min(waves, 160 * 1024 // u["LDS Size"]) >= int(resident), (bm, bn, u)


def test_selection_and_adjusting_fill_a_compute_unit(usage):
    """Four workgroups of 256 threads for the selection, two of 1,024 for the adjusting of logits with lists."""
    for k, u in usage.items():
        if "top_part_kernel" in k:
            assert u["VGPRs"] <= 128 and 160 * 1024 // u["LDS Size"] >= 4, (k, u)
        if "adjust_kernel" in k:
            assert u["VGPRs"] <= 64 and (u.get("LDS Size", 0) == 0 or 160 * 1024 // u["LDS Size"] >= 2), (k, u)
