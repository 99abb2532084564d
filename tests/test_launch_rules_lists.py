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
