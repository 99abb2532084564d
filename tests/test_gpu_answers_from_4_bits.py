"""The operators on tables held in 4 bits together, as they serve: a table is quantised once; heads are fetched by id, queries formed, scored
against the whole table, and answers drawn; in graphs, on other streams, and beside the operators on whole tables."""
import numpy as np
import pytest
import torch

import mxfp_util as mu
import paper_2101_08358_amd as mar

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Server:
    """A DistMult model whose node table is held in 4 bits; all buffers are the caller's."""

    def __init__(self, V, d, Q, n, four=False, seed=1, top_k=50, top_p=0.9, score=torch.float32):
        g = torch.Generator().manual_seed(seed)
        self.V, self.d, self.Q, self.n, self.four = V, d, Q, n, four
        nb = mu.blocks_of(d)
        byte = dict(dtype=torch.uint8, device=DEV)
        self.table = (torch.randn((V, d), generator=g) * 0.5).to(DEV)
        self.rels = torch.randn((7, d), generator=g).to(DEV)
        self.codes, self.scales = torch.zeros((V, 16 * nb), **byte), torch.zeros((V, nb), **byte)
        mar.mar_mxfp_quantise(self.table, d, V, d, mar.DTYPE_FP32, self.codes, 16 * nb, self.scales, nb)
        self.heads = torch.randint(0, V, (Q,), generator=g, dtype=torch.int32).to(DEV)
        self.rel = torch.randint(0, 7, (Q,), generator=g).to(DEV)
        self.u = torch.rand((Q, n), generator=g).to(DEV)
        self.rows, self.q = torch.zeros((Q, d), device=DEV), torch.zeros((Q, d), device=DEV)
        self.q_codes, self.q_scales = torch.zeros((Q, 16 * nb), **byte), torch.zeros((Q, nb), **byte)
        self.scores = torch.zeros((Q, V), dtype=score, device=DEV)
        self.ids, self.log_probs = torch.zeros((Q, n), dtype=torch.int32, device=DEV), torch.zeros((Q, n), device=DEV)
        self.kept = torch.zeros(Q, dtype=torch.int32, device=DEV)
        types = {torch.float32: mar.DTYPE_FP32, torch.bfloat16: mar.DTYPE_BF16}
        self.p = mar.MarMxfp(V, 16 * nb, nb, 16 * nb if four else d, nb if four else 0, V, Q, d, mar.DTYPE_MXFP4 if four else mar.DTYPE_FP32, types[score], 1.0, 0)
        self.s = mar.MarSampling(V, V, Q, n, types[score], top_k, 0.8, top_p, 0.0, 0)
        self.ws = torch.full((mar.mar_mxfp_scores_workspace_bytes(self.p) + 256,), 0x5A, **byte)
        self.ds = torch.full((mar.mar_sample_rows_workspace_bytes(self.s) + 256,), 0x5A, **byte)
        self.par = (0.8, top_k, top_p, 0.0)

    def call(self):
        nb = mu.blocks_of(self.d)
        mar.mar_mxfp_rows(self.codes, 16 * nb, self.scales, nb, self.V, self.d, self.heads, self.Q, mar.DTYPE_FP32, self.rows, self.d)
        torch.mul(self.rows, self.rels[self.rel], out=self.q)
        q, qs = self.q, None
        if self.four:
            mar.mar_mxfp_quantise(self.q, self.d, self.Q, self.d, mar.DTYPE_FP32, self.q_codes, 16 * nb, self.q_scales, nb)
            q, qs = self.q_codes, self.q_scales
        mar.mar_mxfp_scores(self.p, q, qs, self.codes, self.scales, self.scores, self.ws, self.ws.numel() - 256)
        mar.mar_sample_rows(self.s, self.scores, None, 0, None, None, None, None, self.u, self.ids, self.log_probs, self.kept, self.ds, self.ds.numel() - 256)

    def outputs(self):
        return self.rows, self.scores, self.ids, self.log_probs, self.kept

    def check(self):
        codes, scales = mu.quantise(self.table.double().cpu().numpy())
        assert np.array_equal(self.codes.cpu().numpy(), codes) and np.array_equal(self.scales.cpu().numpy(), scales)
        w = mu.values(codes, scales, self.d)
        assert np.array_equal(self.rows.double().cpu().numpy(), w[self.heads.cpu().numpy()])
        q = self.q.double().cpu().numpy()
        if self.four:
            q = mu.values(*mu.quantise(q), self.d)
        eps = torch.finfo(self.scores.dtype).eps / 2
        want, bound = mu.score_bound(q, w, "mxfp4" if self.four else "fp32", 1.0, eps)
        got = self.scores.double().cpu().numpy()
        assert (np.abs(got - want) <= bound).all()
        for i in range(self.Q):                              # of the scores as they are
            ids, lp, kept = mu.draws(got[i], None, float(np.float32(self.par[0])), self.par[1], float(np.float32(self.par[2])), self.par[3], self.u[i].double().cpu().numpy())
            assert self.kept[i].item() == kept and np.array_equal(self.ids[i].cpu().numpy(), ids)
            assert (np.abs(self.log_probs[i].double().cpu().numpy() - lp) <= np.abs(lp) * 2.0 ** -24 + 2.0 ** -40).all()
        assert (self.ws[-256:] == 0x5A).all() and (self.ds[-256:] == 0x5A).all()       # nothing beyond what was asked for


CASES = (dict(V=3000, d=50, Q=5, n=9), dict(V=20_001, d=100, Q=70, n=2), dict(V=5001, d=400, Q=40, n=3, four=True, top_k=0), dict(V=33_333, d=75, Q=1, n=20, top_k=0, top_p=0.95),
         dict(V=40_000, d=128, Q=33, n=1, four=True, score=torch.bfloat16), dict(V=18_000, d=200, Q=64, n=4, top_k=0, score=torch.bfloat16))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%dx%d" % (c["Q"], c["V"], c["d"]))
def test_serving(case):
    s = Server(**case)
    s.call()
    torch.cuda.synchronize()
    s.check()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%dx%d" % (c["Q"], c["V"], c["d"]))
def test_captured_and_replayed(case):
    """Replays with eager work and other inputs between them give what eager calls give."""
    s = Server(**case)
    s.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    for turn in range(4):
        g = torch.Generator().manual_seed(100 + turn)
        s.heads.copy_(torch.randint(0, s.V, (s.Q,), generator=g, dtype=torch.int32))
        s.u.copy_(torch.rand((s.Q, s.n), generator=g))
        s.call()
        torch.cuda.synchronize()
        want = [t.clone() for t in s.outputs()]
        for t in s.outputs():
            t.zero_()
        s.ws.fill_(0xFF)
        s.ds[:-256].fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(s.outputs(), want))


def test_two_streams_at_once():
    """Two models served on streams of their own, with workspaces of their own, give what each gives alone."""
    a, b = Server(30_000, 100, 64, 3, seed=2), Server(17_000, 75, 20, 5, seed=3, top_k=0)
    for s in (a, b):
        s.call()
    torch.cuda.synchronize()
    want = [[t.clone() for t in s.outputs()] for s in (a, b)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for s in (a, b):
            for t in s.outputs():
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for s, stream in zip((a, b), streams):
                with torch.cuda.stream(stream):
                    s.call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for s, w in zip((a, b), want) for x, y in zip(s.outputs(), w))


def test_beside_log_probabilities():
    """Greedy draws from scores are the most probable rows that mar_log_probs names on the values the codes stand for."""
    s = Server(8000, 96, 30, 1, top_k=1)
    s.call()
    w = torch.from_numpy(mu.values(s.codes.cpu().numpy(), s.scales.cpu().numpy(), 96)).float().to(DEV)
    p = mar.MarSoftmax(8000, 96, 96, 30, 96, mar.DTYPE_FP32, 1.0)
    ws = torch.empty(mar.mar_log_probs_workspace_bytes(p, 1), dtype=torch.uint8, device=DEV)
    ids, lp = torch.zeros((30, 1), dtype=torch.int32, device=DEV), torch.zeros((30, 1), device=DEV)
    mar.mar_log_probs(p, s.q, w, None, None, 0, 1, None, None, ids, lp, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(ids, s.ids) and (s.kept == 1).all() and (s.log_probs == 0).all()
