"""The rules by which scores of 4-bit tables and draws divide their work, called through the library's own functions up to the largest
problems that it takes: every launch below 2^32 threads, all rows and queries covered, sums within their types.  No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2101_08358_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not available")


def _run(tmp_path, header, body):
    src, exe = tmp_path / "rules.hip", tmp_path / "rules"
    src.write_text('#include <stdio.h>\n#include "%s"\nint main() {\n%s\nreturn 0;\n}\n' % (header, body))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.split()


def test_scores(tmp_path):
    out = _run(tmp_path, "mar_mxfp.h", """
  long taken = 0, bad = 0;
  for (int64_t rows : {(int64_t)1, (int64_t)31, (int64_t)1000, (int64_t)65536, (int64_t)65537, (int64_t)1048576, (int64_t)40000000, MAR_SOFTMAX_MAX_ROWS - 1, MAR_SOFTMAX_MAX_ROWS})
    for (int queries : {1, 31, 32, 33, 64, 224, 225, 1000, 4096, 100000, 10000000, MAR_SOFTMAX_MAX_QUERIES}) for (int dim : {1, 64, 65, 192, 193, 256, 257, 400})
    for (int dtype : {MAR_DTYPE_FP32, MAR_DTYPE_FP16, MAR_DTYPE_MXFP4}) {
      mar_mxfp p = {};
      p.dtype = dtype;
      p.num_rows = rows; p.num_queries = queries; p.dim = dim;
      const MxPlan r = mx_plan(&p);
      const int64_t tiles = mx_tiles(queries), threads = (int64_t)r.grid * (r.few ? 256 : 512);
      ++taken;
      if (threads >= 1ll << 32 || r.grid < 1 || r.few != (queries <= 32)) ++bad;
      if (r.few) { if ((int64_t)r.stripes * 32 * r.rt < rows || r.grid > (r.stripes + 3) / 4) ++bad; continue; }
      if ((int64_t)r.stripes * r.parts != r.grid || (int64_t)r.stripes * 256 * r.rt < rows || (int64_t)r.parts * r.tiles_part < tiles) ++bad;
      if ((int64_t)(r.parts - 1) * r.tiles_part >= tiles) ++bad;       // no part without tiles
      if ((int64_t)r.stripes * 256 * r.rt > INT32_MAX || tiles * ((dim + 63) / 64) * 256 >= 1ll << 32) ++bad;
    }
  printf("%ld %ld", taken, bad);""")
    assert int(out[0]) == 9 * 12 * 8 * 3 and out[1] == "0", out


def test_draws(tmp_path):
    out = _run(tmp_path, "mar_sample_dev.h", """
  long taken = 0, bad = 0;
  for (int64_t rows : {(int64_t)DRAW_SMALL + 1, (int64_t)20000, (int64_t)131072, (int64_t)1000003, (int64_t)50000000, MAR_SOFTMAX_MAX_ROWS - 2047, MAR_SOFTMAX_MAX_ROWS})
    for (int queries : {1, 2, 7, 64, 100, 1000, 2047, 2048, 2049, 100000, MAR_SOFTMAX_MAX_QUERIES}) for (int top_k : {0, 512, 513, 2000000}) {
      mar_sampling p = {};
      p.num_rows = rows; p.num_queries = queries; p.top_k = top_k;
      const DrawLayout L = draw_layout(&p);
      ++taken;
      if (L.chunks < 1 || L.chunks > 256 || (int64_t)L.chunks * L.chunk_rows < rows || (int64_t)(L.chunks - 1) * L.chunk_rows >= rows) ++bad;
      if (L.chunk_rows % 2048 || L.chunk_rows > 1 << 21 || L.hist_bits < 10 || (int64_t)L.chunk_rows << L.hist_bits >= 1ll << 32) ++bad;
      if (L.blocks < 1 || L.blocks > L.chunk_rows / 2048 || L.groups != L.chunks * L.blocks * (256 / L.merge)) ++bad;
      if (L.merge < 1 || L.merge & (L.merge - 1) || L.merge > 16 || (L.groups < 4096 && L.merge > 1)) ++bad;
      if (L.list < 1000 || (L.list > DRAW_LIST && L.list > rows / 32) || (int64_t)L.segments * DRAW_SEGMENT < rows || L.mass_pitch % 16 || L.mass_pitch < L.segments) ++bad;
      if (L.bytes % 256 || L.mass + (size_t)queries * L.mass_pitch * 8 > L.bytes) ++bad;
      int64_t at = 0;
      sm_launches((int64_t)queries * L.chunks, 256, [&](int64_t first, unsigned n) { if (first != at || (int64_t)n * 256 >= 1ll << 32) ++bad; at = first + n; });
      if (at != (int64_t)queries * L.chunks) ++bad;
    }
  for (int64_t rows : {(int64_t)1, (int64_t)DRAW_SMALL}) { mar_sampling p = {}; p.num_rows = rows; p.num_queries = 9; if (draw_layout(&p).bytes != 256) ++bad; }
  printf("%ld %ld", taken, bad);""")
    assert int(out[0]) == 77 * 4 and out[1] == "0", out
