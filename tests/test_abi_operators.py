"""Refusals of the operators on whole tables: codes and texts, before anything touches the GPU.  No compute calls."""
import ctypes

import pytest

import paper_2101_08358_amd as mar

FAKE = 0x10000                                               # a non-null, aligned address that is never dereferenced


def _problem(**kw):
    base = dict(num_rows=1000, row_stride=50, query_stride=50, num_queries=10, dim=50, dtype=0, scale=1.0)
    base.update(kw)
    return mar.MarSoftmax(**base)


def test_struct_layout_matches_header():
    assert ctypes.sizeof(mar.MarSoftmax) == 40
    assert mar.MarSoftmax.num_queries.offset == 24 and mar.MarSoftmax.scale.offset == 36


BAD_PROBLEMS = ((dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
                (dict(scale=float("inf")), -1), (dict(num_rows=0), -2), (dict(num_rows=1 << 31), -2), (dict(num_queries=-1), -2), (dict(dim=0), -2),
                (dict(dim=401, row_stride=500, query_stride=500), -2), (dict(row_stride=49), -1), (dict(query_stride=49), -1),
                (dict(row_stride=1 << 31), -1), (dict(num_queries=0x7fffff01), -2),
                (dict(num_rows=0x1fffff01), -2), (dict(num_queries=0x3ffff01), -2))


@pytest.mark.parametrize("bad,code", BAD_PROBLEMS)
def test_problems_are_checked_everywhere(bad, code):
    p = _problem(**bad)
    calls = (lambda: mar.mar_log_probs_workspace_bytes(p, 5), lambda: mar.mar_softmax_loss_workspace_bytes(p),
             lambda: mar.mar_log_probs(p, FAKE, FAKE, FAKE, None, 0, 0, FAKE, None, None, None, FAKE, 1 << 40, 0),
             lambda: mar.mar_softmax_loss(p, FAKE, FAKE, FAKE, None, FAKE, None, None, 0, None, 0, FAKE, 1 << 40, 0))
    for call in calls:
        with pytest.raises(mar.MarError) as e:
            call()
        assert e.value.code == code and mar.mar_last_error() != ""


def test_workspace_grows_with_the_problem():
    for dtype in (0, 1, 2):
        small, big = (mar.mar_softmax_loss_workspace_bytes(_problem(num_rows=v, num_queries=t, dtype=dtype)) for v, t in ((100, 10), (100_000, 1000)))
        assert 0 < small < big and small % 256 == 0 and big % 256 == 0
        a, b = (mar.mar_log_probs_workspace_bytes(_problem(num_rows=100_000, num_queries=500, dtype=dtype), k) for k in (0, 10))
        assert 0 < a < b and b % 256 == 0
        assert mar.mar_log_probs_workspace_bytes(_problem(num_queries=0, dtype=dtype), 0) > 0


def _log_probs(**kw):
    a = dict(p=_problem(), q=FAKE, w=FAKE, targets=FAKE, allowed=None, stride=0, top=2, lp=FAKE, en=FAKE, ids=FAKE, tp=FAKE, ws=FAKE, n=1 << 40)
    a.update(kw)
    mar.mar_log_probs(a["p"], a["q"], a["w"], a["targets"], a["allowed"], a["stride"], a["top"], a["lp"], a["en"], a["ids"], a["tp"], a["ws"], a["n"], 0)


@pytest.mark.parametrize("bad,code", ((dict(q=None), -1), (dict(w=None), -1), (dict(targets=None), -1), (dict(top=-1), -2), (dict(top=33), -2), (dict(ids=None), -1),
                                      (dict(tp=None), -1), (dict(q=FAKE + 2), -1), (dict(w=FAKE + 1), -1), (dict(lp=FAKE + 2), -1), (dict(ids=FAKE + 1), -1),
                                      (dict(allowed=FAKE, stride=31), -1), (dict(allowed=FAKE, stride=-1), -1), (dict(allowed=FAKE + 2, stride=32), -1),
                                      (dict(ws=None), -1), (dict(ws=FAKE + 16), -1), (dict(n=0), -3)))
def test_log_probs_arguments(bad, code):
    with pytest.raises(mar.MarError) as e:
        _log_probs(**bad)
    assert e.value.code == code and mar.mar_last_error() != ""


def _loss(**kw):
    a = dict(p=_problem(), q=FAKE, w=FAKE, targets=FAKE, weights=None, loss=FAKE, lse=FAKE, gq=FAKE, gqs=50, gw=FAKE, gws=50, ws=FAKE, n=1 << 40)
    a.update(kw)
    mar.mar_softmax_loss(a["p"], a["q"], a["w"], a["targets"], a["weights"], a["loss"], a["lse"], a["gq"], a["gqs"], a["gw"], a["gws"], a["ws"], a["n"], 0)


@pytest.mark.parametrize("bad,code", ((dict(q=None), -1), (dict(w=None), -1), (dict(targets=None), -1), (dict(q=FAKE + 2), -1), (dict(gq=FAKE + 2), -1), (dict(gw=FAKE + 1), -1),
                                      (dict(gqs=49), -1), (dict(gws=0), -1), (dict(weights=FAKE + 1), -1), (dict(loss=FAKE + 2), -1), (dict(ws=None), -1),
                                      (dict(ws=FAKE + 128), -1), (dict(n=100), -3)))
def test_softmax_loss_arguments(bad, code):
    with pytest.raises(mar.MarError) as e:
        _loss(**bad)
    assert e.value.code == code and mar.mar_last_error() != ""


@pytest.mark.parametrize("bad,code", ((dict(dtype=3), -1), (dict(p=1.0), -1), (dict(p=-0.1), -1), (dict(p=float("nan")), -1), (dict(p=0.99999999), -1), (dict(p=0.999999), -2),
                                      (dict(rows=-1), -2), (dict(rows=1 << 31), -2), (dict(dim=0), -2), (dict(xs=49), -1), (dict(os=49), -1), (dict(step=1 << 62), -2),
                                      (dict(x=None), -1), (dict(out=None), -1), (dict(x=FAKE + 2), -1), (dict(out=FAKE + 1, dtype=1), -1),
                                      (dict(rows=0x7fffffff, dim=1 << 20, xs=1 << 20, os=1 << 20), -2)))
def test_dropout_arguments(bad, code):
    a = dict(x=FAKE, xs=50, rows=10, dim=50, dtype=0, p=0.5, seed=1, step=2, out=FAKE, os=50)
    a.update(bad)
    with pytest.raises(mar.MarError) as e:
        mar.mar_dropout(a["x"], a["xs"], a["rows"], a["dim"], a["dtype"], a["p"], a["seed"], a["step"], a["out"], a["os"], 0)
    assert e.value.code == code and mar.mar_last_error() != ""
