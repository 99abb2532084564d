"""Refusals of the operators on tables held in 4 bits and of draws: codes and texts, before anything touches the GPU.  No compute calls."""
import ctypes

import pytest

import paper_2101_08358_amd as mar

FAKE = 0x10000                                               # a non-null, aligned address that is never dereferenced
NAN, INF = float("nan"), float("inf")


def refused(call, code):
    with pytest.raises(mar.MarError) as e:
        call()
    assert e.value.code == code and mar.mar_last_error() != ""


def test_struct_layouts_match_header():
    assert ctypes.sizeof(mar.MarMxfp) == 72
    assert mar.MarMxfp.score_stride.offset == 40 and mar.MarMxfp.num_queries.offset == 48 and mar.MarMxfp.scale.offset == 64
    assert ctypes.sizeof(mar.MarSampling) == 48
    assert mar.MarSampling.num_queries.offset == 16 and mar.MarSampling.temperature.offset == 32 and mar.MarSampling.reserved.offset == 44


@pytest.mark.parametrize("bad,code", ((dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(rows=-1), -2), (dict(rows=1 << 31), -2), (dict(dim=0), -2),
                                      (dict(dim=(1 << 24) + 1, xs=1 << 25, cs=1 << 25, ss=1 << 25), -2), (dict(xs=49), -1), (dict(xs=(1 << 40) + 1), -1), (dict(cs=31), -1),
                                      (dict(cs=16), -1), (dict(cs=40), -1), (dict(cs=1 << 41), -1), (dict(ss=1), -1), (dict(ss=1 << 41), -1), (dict(x=None), -1), (dict(c=None), -1),
                                      (dict(s=None), -1), (dict(x=FAKE + 2), -1), (dict(x=FAKE + 1, dtype=1), -1), (dict(c=FAKE + 8), -1)))
def test_quantise_arguments(bad, code):
    a = dict(x=FAKE, xs=50, rows=10, dim=50, dtype=0, c=FAKE, cs=32, s=FAKE + 1, ss=2)
    a.update(bad)
    refused(lambda: mar.mar_mxfp_quantise(a["x"], a["xs"], a["rows"], a["dim"], a["dtype"], a["c"], a["cs"], a["s"], a["ss"], 0), code)


@pytest.mark.parametrize("bad,code", ((dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(rows=-1), -2), (dict(rows=1 << 31), -2), (dict(n=-1), -2), (dict(n=1 << 31), -2),
                                      (dict(dim=0), -2), (dict(dim=(1 << 24) + 1, os=1 << 25, cs=1 << 25, ss=1 << 25), -2), (dict(os=49), -1), (dict(os=(1 << 40) + 1), -1),
                                      (dict(cs=24), -1), (dict(cs=40), -1), (dict(ss=1), -1), (dict(out=None), -1), (dict(c=None), -1), (dict(s=None), -1), (dict(out=FAKE + 2), -1),
                                      (dict(out=FAKE + 1, dtype=2), -1), (dict(c=FAKE + 8), -1), (dict(ids=FAKE + 2), -1)))
def test_rows_arguments(bad, code):
    a = dict(c=FAKE, cs=32, s=FAKE + 1, ss=2, rows=10, dim=50, ids=FAKE, n=5, dtype=0, out=FAKE, os=50)
    a.update(bad)
    refused(lambda: mar.mar_mxfp_rows(a["c"], a["cs"], a["s"], a["ss"], a["rows"], a["dim"], a["ids"], a["n"], a["dtype"], a["out"], a["os"], 0), code)


def _scores_problem(**kw):
    base = dict(num_rows=1000, codes_stride=32, scales_stride=2, query_stride=50, query_scales_stride=0, score_stride=1000, num_queries=10, dim=50, dtype=0, score_dtype=0,
                scale=1.0, reserved=0)
    base.update(kw)
    return mar.MarMxfp(**base)


@pytest.mark.parametrize("bad,code", ((dict(dtype=4), -1), (dict(dtype=-1), -1), (dict(score_dtype=3), -1), (dict(score_dtype=-1), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
                                      (dict(scale=NAN), -1), (dict(scale=INF), -1), (dict(num_rows=0), -2), (dict(num_rows=0x1fffff01, score_stride=1 << 31), -2),
                                      (dict(num_queries=-1), -2), (dict(num_queries=0x3ffff01), -2), (dict(dim=0), -2), (dict(dim=401, codes_stride=512, scales_stride=16, query_stride=500), -2),
                                      (dict(codes_stride=16), -1), (dict(codes_stride=40), -1), (dict(scales_stride=1), -1), (dict(query_stride=49), -1), (dict(query_stride=1 << 41), -1),
                                      (dict(score_stride=999), -1), (dict(score_stride=1 << 41), -1), (dict(reserved=1), -1),
                                      (dict(dtype=3, query_stride=50, query_scales_stride=2), -1), (dict(dtype=3, query_stride=32, query_scales_stride=1), -1)))
def test_score_problems_are_checked_everywhere(bad, code):
    p = _scores_problem(**bad)
    refused(lambda: mar.mar_mxfp_scores_workspace_bytes(p), code)
    refused(lambda: mar.mar_mxfp_scores(p, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0), code)


@pytest.mark.parametrize("bad,code", ((dict(q=None), -1), (dict(c=None), -1), (dict(s=None), -1), (dict(out=None), -1), (dict(q=FAKE + 2), -1), (dict(c=FAKE + 8), -1),
                                      (dict(out=FAKE + 2), -1), (dict(ws=None), -1), (dict(ws=FAKE + 128), -1), (dict(n=100), -3),
                                      (dict(p=_scores_problem(dtype=3, query_stride=32, query_scales_stride=2), qs=None), -1),
                                      (dict(p=_scores_problem(dtype=3, query_stride=32, query_scales_stride=2), q=FAKE + 8), -1),
                                      (dict(p=_scores_problem(score_dtype=1), out=FAKE + 1), -1)))
def test_scores_arguments(bad, code):
    a = dict(p=_scores_problem(), q=FAKE, qs=FAKE, c=FAKE, s=FAKE + 1, out=FAKE, ws=FAKE, n=1 << 40)
    a.update(bad)
    refused(lambda: mar.mar_mxfp_scores(a["p"], a["q"], a["qs"], a["c"], a["s"], a["out"], a["ws"], a["n"], 0), code)


def _sampling(**kw):
    base = dict(num_rows=1000, score_stride=1000, num_queries=10, num_draws=1, dtype=0, top_k=0, temperature=1.0, top_p=1.0, min_p=0.0, reserved=0)
    base.update(kw)
    return mar.MarSampling(**base)


@pytest.mark.parametrize("bad,code", ((dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(temperature=-0.1), -1), (dict(temperature=NAN), -1), (dict(top_k=-1), -1), (dict(top_p=-0.1), -1),
                                      (dict(top_p=1.1), -1), (dict(top_p=NAN), -1), (dict(min_p=-0.1), -1), (dict(min_p=1.1), -1), (dict(min_p=NAN), -1), (dict(reserved=1), -1),
                                      (dict(num_rows=0), -2), (dict(num_rows=0x1fffff01, score_stride=1 << 31), -2), (dict(num_queries=-1), -2), (dict(num_queries=0x3ffff01), -2),
                                      (dict(num_draws=0), -2), (dict(num_draws=65537), -2), (dict(score_stride=999), -1), (dict(score_stride=1 << 41), -1)))
def test_draw_problems_are_checked_everywhere(bad, code):
    p = _sampling(**bad)
    refused(lambda: mar.mar_sample_rows_workspace_bytes(p), code)
    refused(lambda: mar.mar_sample_rows(p, FAKE, None, 0, None, None, None, None, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 50, 0), code)


@pytest.mark.parametrize("bad,code", ((dict(s=None), -1), (dict(u=None), -1), (dict(ids=None), -1), (dict(s=FAKE + 2), -1), (dict(u=FAKE + 2), -1), (dict(ids=FAKE + 1), -1),
                                      (dict(lp=FAKE + 2), -1), (dict(kept=FAKE + 3), -1), (dict(t=FAKE + 2), -1), (dict(k=FAKE + 2), -1), (dict(tp=FAKE + 1), -1), (dict(mp=FAKE + 2), -1),
                                      (dict(allowed=FAKE, stride=31), -1), (dict(allowed=FAKE, stride=-1), -1), (dict(allowed=FAKE + 2, stride=32), -1), (dict(ws=None), -1),
                                      (dict(ws=FAKE + 16), -1), (dict(n=0), -3)))
def test_draw_arguments(bad, code):
    a = dict(s=FAKE, allowed=None, stride=0, t=FAKE, k=FAKE, tp=FAKE, mp=FAKE, u=FAKE, ids=FAKE, lp=FAKE, kept=FAKE, ws=FAKE, n=1 << 40)
    a.update(bad)
    refused(lambda: mar.mar_sample_rows(_sampling(), a["s"], a["allowed"], a["stride"], a["t"], a["k"], a["tp"], a["mp"], a["u"], a["ids"], a["lp"], a["kept"], a["ws"], a["n"], 0), code)


def test_no_problem_and_workspaces():
    lib, n = mar.load_library(), ctypes.c_size_t(0)
    assert lib.mar_mxfp_scores_workspace_bytes(None, ctypes.byref(n)) == -1 and lib.mar_sample_rows_workspace_bytes(None, ctypes.byref(n)) == -1
    assert lib.mar_mxfp_scores_workspace_bytes(ctypes.byref(_scores_problem()), None) == -1
    assert lib.mar_sample_rows_workspace_bytes(ctypes.byref(_sampling()), None) == -1
    for q in (0, 1, 33, 1000):
        for dtype, stride in ((0, 50), (1, 50), (3, 32)):
            small, big = (mar.mar_mxfp_scores_workspace_bytes(_scores_problem(num_queries=t, dtype=dtype, query_stride=stride, query_scales_stride=2)) for t in (q, q + 64))
            assert 0 < small < big and small % 256 == 0 and big % 256 == 0
        small, big = (mar.mar_sample_rows_workspace_bytes(_sampling(num_queries=q, num_rows=v, score_stride=v)) for v in (10, 1_000_000))
        assert 0 < small <= big and small % 256 == 0 and big % 256 == 0
