"""Room for the rows of top-p's border: a workgroup's list at least, however few rows there are.  No GPU needed."""
from test_launch_rules_mxfp import _run, pytestmark  # noqa: F401  (skipped without hipcc)


def test_list_of_a_border(tmp_path):
    out = _run(tmp_path, "mar_sample_dev.h", """
  long bad = 0;
  for (int64_t rows : {(int64_t)16385, (int64_t)17000, (int64_t)40000, (int64_t)100000, (int64_t)131072, (int64_t)262143, (int64_t)262144, (int64_t)1000003, MAR_SOFTMAX_MAX_ROWS})
    for (int queries : {1, 1000, 100000}) {
      mar_sampling p = {};
      p.num_rows = rows; p.num_queries = queries;
      const DrawLayout L = draw_layout(&p);
      if (L.list < DRAW_LIST || L.list < rows / 32 || (L.list > DRAW_LIST && L.list > rows / 32)) ++bad;
      if (L.lists + (size_t)queries * L.list * 8 > L.mass) ++bad;
    }
  printf("%ld", bad);""")
    assert out[0] == "0", out


def test_workspace_of_a_batch(tmp_path):
    """Histograms and lists take turns in the same memory: no more than the larger of them beside sums, maxima and a few words a query."""
    out = _run(tmp_path, "mar_sample_dev.h", """
  long bad = 0;
  for (int64_t rows : {(int64_t)16385, (int64_t)100000, (int64_t)1000003, (int64_t)50000000})
    for (int64_t queries : {1, 100, 1000}) {
      mar_sampling p = {};
      p.num_rows = rows; p.num_queries = (int)queries;
      const DrawLayout L = draw_layout(&p);
      const size_t hists = queries * L.chunks * DRAW_BINS * 4, lists = queries * L.list * 8;
      const size_t others = queries * (L.chunks * (sizeof(DrawChunk) + 20) + L.groups * 4 + sizeof(DrawRange) + 8 + L.mass_pitch * 8) + 10 * 256;
      if (L.bytes > (hists > lists ? hists : lists) + others) ++bad;
    }
  printf("%ld", bad);""")
    assert out[0] == "0", out
