"""Compile-time guard for the kernels of tables held in 4 bits and of draws: none keeps registers in scratch memory, and every width and
type has its instantiation.  Uses hipcc's resource-usage remarks; no GPU needed."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not available")
@pytest.mark.parametrize("name,kernels", (
    ("mar_mxfp", {"k_quantise": 3, "k_mxfp_rows": 3}),
    # seven widths; four types of queries, two heights of a wave's rows
    ("mar_mxfp_scores", {"k_mxfp_pack": 7 * 4, "k_mxfp_few": 7 * 4 * 2, "k_mxfp_scores": 7 * 3 * 2}),
    ("mar_sample", {"k_draw_small": 3 * 2, "k_draw_scan": 3, "k_draw_hist": 3, "k_draw_range": 1, "k_draw_weigh": 3, "k_draw_rows": 3, "k_draw_slowly": 3})))
def test_no_scratch_memory(name, kernels, tmp_path):
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(ROOT, "paper_2101_08358_amd", "csrc", name + ".hip"), "-o", str(tmp_path / "x.o")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    seen = dict.fromkeys(kernels, 0)
    for b in re.split(r"remark: Function Name: ", r.stderr)[1:]:
        function = b.split()[0]
        length, rest = re.match(r"_Z(\d+)(.*)", function).groups()
        seen[rest[:int(length)]] += 1
        assert int(re.search(r"ScratchSize \[bytes/lane\]: (\d+)", b).group(1)) == 0, function
        # the draws' small kernel without filters: two workgroups of 1,024 threads a CU
        if "k_draw_small" in function and "Lb0E" in function:
            assert int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", b).group(1)) == 8, function
    assert seen == kernels, seen
