"""Compile-time guard for the kernels of the operators on whole tables: none keeps registers in scratch memory, and every width has
its instantiation in every way that rows come.  Uses hipcc's resource-usage remarks; no GPU needed."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not available")
@pytest.mark.parametrize("name,kernels", (
    # three types; seven widths from images and from rows, six for few queries
    ("mar_softmax", {"k_softmax": 3 * 20, "k_softmax_pack": 3 * 7, "k_answer": 3 * 4}),
    ("mar_softmax_loss", {"k_softmax": 3 * 7 * 2, "k_loss_rows": 3 * 2, "k_loss_table": 3}),
    ("mar_dropout", {"k_dropout": 3})))
def test_no_scratch_memory(name, kernels, tmp_path):
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(ROOT, "paper_2101_08358_amd", "csrc", name + ".hip"), "-o", str(tmp_path / "x.o")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    seen = dict.fromkeys(kernels, 0)
    for b in re.split(r"remark: Function Name: ", r.stderr)[1:]:
        function = b.split()[0]
        kind = re.match(r"_Z\d+(k_[a-z_]+)I", function).group(1)
        seen[kind] += 1
        assert int(re.search(r"ScratchSize \[bytes/lane\]: (\d+)", b).group(1)) == 0, function
    assert seen == kernels, seen
