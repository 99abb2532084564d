"""The rules by which the operators on whole tables divide work into launches of fewer than 2^32 threads, called through the library's
own functions up to the largest problems that it takes.  No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2101_08358_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not available")


def _run(tmp_path, body):
    """Compiles a main() around `body` against the library's headers and library, runs it and returns what it prints."""
    src, exe, lib = tmp_path / "rules.hip", tmp_path / "rules", os.path.dirname(CSRC)
    src.write_text('#include <stdio.h>\n#include "mar_softmax_dev.h"\nint main() {\n' + body + "\nreturn 0;\n}\n")
    if not os.path.exists(os.path.join(lib, "libmarius_hip.so")):
        from paper_2101_08358_amd import build
        build.build()
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe), "-L", lib,
                        "-lmarius_hip", "-Wl,-rpath," + lib], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.split()


def test_every_launch_holds_fewer_than_2_32_threads(tmp_path):
    """Contraction passes of every type and width: parts are only taken as one launch can hold; the joining kernels as well."""
    out = _run(tmp_path, """
  long taken = 0, bad = 0;
  for (int64_t rows : {(int64_t)1, (int64_t)65536, (int64_t)16777216, (int64_t)33554560, MAR_SOFTMAX_MAX_ROWS - 255, MAR_SOFTMAX_MAX_ROWS})
    for (int64_t queries : {(int64_t)33, (int64_t)513, (int64_t)65537, (int64_t)16777216, (int64_t)33554560, (int64_t)MAR_SOFTMAX_MAX_QUERIES})
      for (int dtype = 0; dtype < 3; ++dtype) for (int dim : {1, 32, 50, 100, 128, 192, 256, 400}) for (int pass = 0; pass < 3; ++pass) {
        const int64_t n_x = pass == 2 ? rows : queries, n_y = pass == 2 ? queries : rows;
        const SmPlan p = sm_plan(dtype, dim, pass, SM_IMAGES, n_x, n_y, 1);
        const int64_t units = (int64_t)p.stripes * p.parts;
        ++taken;
        if ((units + 7) / 8 * 8 * 256 >= 1ll << 32 || units > INT32_MAX || (int64_t)p.parts * p.tps < p.ntiles) ++bad;
        if (pass == 1 && sm_loss_waves(p.parts, n_x) * 64 * n_x >= 1ll << 32) ++bad;
      }
  printf("%ld %ld", taken, bad);""")
    assert int(out[0]) > 2000 and out[1] == "0", out


def test_launches_cover_every_workgroup_once(tmp_path):
    """The layout of both matrices of the largest problem, and sums of parts of tables of 400 columns, take several launches."""
    out = _run(tmp_path, """
  long bad = 0, most = 0;
  for (int64_t blocks : {(int64_t)0, (int64_t)1, sm_most_blocks(256), sm_most_blocks(256) + 1, sm_tiles(MAR_SOFTMAX_MAX_ROWS) + sm_tiles(513),
                         sm_tiles(MAR_SOFTMAX_MAX_ROWS) + sm_tiles(MAR_SOFTMAX_MAX_QUERIES), (MAR_SOFTMAX_MAX_ROWS * 100 + 255) / 256}) {
    int64_t at = 0;
    long launches = 0;
    sm_launches(blocks, 256, [&](int64_t first, unsigned n) {
      if (first != at || n == 0 || (int64_t)n * 256 >= 1ll << 32) ++bad;
      at = first + n; ++launches;
    });
    if (at != blocks) ++bad;
    if (launches > most) most = launches;
  }
  printf("%ld %ld", bad, most);""")
    assert out[0] == "0" and int(out[1]) > 1, out
