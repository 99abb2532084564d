"""How draws with top-k divide their rows into groups: enough of them for a top-k of up to 2,048 wherever the rows allow it, whatever the number
of queries, so that no call leaves the way by groups' maxima without need.  No GPU needed."""
import pytest

from test_launch_rules_mxfp import _run, pytestmark  # noqa: F401  (skipped without hipcc)


def test_groups_for_every_top_k(tmp_path):
    out = _run(tmp_path, "mar_sample_dev.h", """
  long taken = 0, bad = 0, slow = 0;
  for (int64_t rows : {(int64_t)16385, (int64_t)17000, (int64_t)20000, (int64_t)30000, (int64_t)50000, (int64_t)60000, (int64_t)100000, (int64_t)140000, (int64_t)1000003, (int64_t)20000000})
    for (int queries : {1, 2, 7, 64, 100, 300, 500, 700, 1000, 2048, 5000}) for (int top_k : {1, 50, 512, 513, 600, 800, 1000, 1152, 1500, 1900, 2047, 2048}) {
      mar_sampling p = {};
      p.num_rows = rows; p.num_queries = queries; p.top_k = top_k;
      const DrawLayout L = draw_layout(&p);
      ++taken;
      const int64_t wanted = 2 * top_k < rows / 8 ? 2 * top_k : rows / 8;      // a group has eight rows at least
      if (L.groups < wanted) ++bad;
      if (!draw_picks(top_k, L.groups)) ++slow;
      if (L.blocks > L.chunk_rows / 2048 || (int64_t)L.groups != (int64_t)L.chunks * L.blocks * (256 / L.merge)) ++bad;
    }
  printf("%ld %ld %ld", taken, bad, slow);""")
    assert int(out[0]) == 10 * 11 * 12 and out[1] == "0" and out[2] == "0", out


def test_a_top_k_of_each_query_alone(tmp_path):
    """The problem's top_k is 0 where the queries have their own: groups by the default serve the largest."""
    out = _run(tmp_path, "mar_sample_dev.h", """
  long bad = 0;
  for (int64_t rows : {(int64_t)16385, (int64_t)20000, (int64_t)50000, (int64_t)131072, (int64_t)1000003, (int64_t)20000000})
    for (int queries : {1, 64, 300, 1000, 2048, 5000}) {
      mar_sampling p = {};
      p.num_rows = rows; p.num_queries = queries;
      if (!draw_picks(2048, draw_layout(&p).groups)) ++bad;
    }
  if (draw_picks(0, 1 << 20) || draw_picks(2049, 1 << 20) || draw_picks(100, 99)) ++bad;
  printf("%ld", bad);""")
    assert out[0] == "0", out
