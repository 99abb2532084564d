"""Measured calls of the operators on tables held in 4 bits: rows to microscaled 4-bit floats and back, scores of queries against
such a table, and rows drawn from scores.

Four kinds of case:

* ``quantise``: rows to codes and block scales, and the values they stand for (what a user looks at before a table is replaced).
* ``rows``: given rows of such a table, as the heads of queries are fetched.
* ``scores``: queries against every row of such a table.
* ``sample``: rows drawn by their scores with temperature, top-k, top-p and min-p from given random numbers.

Embeddings are drawn as they are in the middle of training (a few tenths), scores as products of such rows, ids follow a power law as
in the benchmark's graphs, table sizes are the benchmark's (the large ones cut) or generic.

Microscaled 4-bit floats: 32 columns of a row share a scale 2^e, e = floor(log2 of the largest magnitude) - 2, held as the byte
e + 127; a column is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it (ties to the even code, at most 6) with a sign bit, the even
column of a byte in its low four bits.  Rows are whole blocks: zeros fill the last one.

Where ``own`` is false ``run`` computes the operators in their plain form, from elementary operations in 32 bits (weights of draws, whose
sums decide at borders, in 64).
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EMB_STD = 0.3
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
PLAIN_VALUES = 1 << 28       # values that the plain forms of the table operators hold at a time
PLAIN_DRAWS = 1 << 26        # scores that the plain form of the draws sorts at a time


def _quantise(name, dtype, rows, dim):
    return {"name": name, "kind": "quantise", "dtype": dtype, "rows": rows, "dim": dim}


def _rows(name, dtype, ids, rows, dim):
    return {"name": name, "kind": "rows", "dtype": dtype, "ids": ids, "rows": rows, "dim": dim}


def _scores(name, dtype, out, queries, rows, dim, scale=1.0):
    """dtype: the queries', "mxfp4" for queries that are brought to 4 bits in the same pass; out: the scores'."""
    return {"name": name, "kind": "scores", "dtype": dtype, "out": out, "queries": queries, "rows": rows, "dim": dim, "scale": scale}


def _sample(name, dtype, queries, rows, draws=1, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, known_out=False, spread=2.5):
    """mixed: every query has parameters of its own; known_out: 16 known answers a query are not drawn; spread: of the scores."""
    return {"name": name, "kind": "sample", "dtype": dtype, "queries": queries, "rows": rows, "draws": draws, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed, "known_out": known_out, "spread": spread}


def listed():
    return [
        # the benchmark's smallest table (10,000 nodes of 50 floats): latency of two calls
        _quantise("quantise_tiny", "fp32", 10_000, 50),
        # a cut of the benchmark's widest table, the last block of a row half full
        _quantise("quantise_wide", "fp32", 1_000_003, 400),
        # the heads of a batch of the smallest graph: latency
        _rows("rows_tiny", "fp32", 1_000, 10_000, 50),
        # the heads of the largest batch from a table of 400 columns, in 16 bits
        _rows("rows_wide", "bf16", 100_000, 2_000_000, 400),
        # one query against a small knowledge graph's nodes, 75 columns: latency
        _scores("scores_one_small", "fp16", "fp32", 1, 14_951, 75),
        # one query against millions of rows: the table is read once
        _scores("scores_one_large", "bf16", "fp32", 1, 4_000_000, 100),
        # a batch in the framework's own type, odd sizes, a temperature
        _scores("scores_ragged", "fp32", "fp32", 999, 120_007, 390, scale=1.25),
        # the largest: queries in 4 bits as well, a vocabulary-sized table, scores in 16 bits
        _scores("scores_wide", "mxfp4", "bf16", 4_096, 131_072, 400),
        # one answer drawn from a small knowledge graph's nodes: latency
        _sample("draw_one_small", "fp32", 1, 14_951, temperature=0.8, top_k=50, top_p=0.95),
        # a served batch, every request with parameters of its own
        _sample("draw_served", "fp32", 64, 131_072, mixed=True),
        # the nucleus of flat distributions over a large table: no top-k to cut them short
        _sample("draw_nucleus", "bf16", 100, 1_000_003, temperature=0.9, top_p=0.9),
        # hard negatives of a batch: 100 draws a query, the known answers left out
        _sample("draw_negatives", "fp32", 1_000, 14_951, draws=100, temperature=1.3, known_out=True),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    kind = rng.choice(("quantise", "rows", "scores", "scores", "sample", "sample"))
    dtype = rng.choice(("fp32", "bf16", "fp16"))
    dim = log_uniform(16, 400)
    if kind == "quantise":
        case = _quantise("", dtype, log_uniform(1_000, 400_000_000 // dim), dim)
    elif kind == "rows":
        case = _rows("", dtype, log_uniform(1, 100_000), log_uniform(1_000, 2_000_000), dim)
    elif kind == "scores":
        queries = log_uniform(1, 4_096)
        rows = log_uniform(1_000, min(4_000_000, 500_000_000 // queries))
        case = _scores("", rng.choice((dtype, dtype, dtype, "mxfp4")), rng.choice(("fp32", "bf16", "fp16")), queries, rows, dim,
                       round(rng.uniform(0.5, 1.5), 2))
    else:
        queries = log_uniform(1, 1_000)
        rows = log_uniform(1_000, min(1_000_000, 100_000_000 // queries))
        case = _sample("", dtype, queries, rows, rng.choice((1, 1, log_uniform(1, 200))), round(rng.uniform(0.3, 1.5), 2),
                       rng.choice((0, 0, log_uniform(1, 2_000))), rng.choice((1.0, round(rng.uniform(0.3, 0.99), 3))),
                       rng.choice((0.0, round(rng.uniform(0.0, 0.2), 3))), rng.random() < 0.3, rng.random() < 0.3, round(rng.uniform(1.0, 4.0), 2))
    del case["name"]
    return case


def _power_law(g, n, rows):
    """Ids with P(id) ~ (id + 1)^-1.2 by the inverse of the continuous law's distribution."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    x = (1.0 - u * (1.0 - (rows + 1.0) ** -0.2)) ** -5.0
    return (x.long() - 1).clamp_(0, rows - 1).to(torch.int32)


def _embeddings(g, rows, dim, dtype):
    return (torch.randn((rows, dim), generator=g, device="cuda") * EMB_STD).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = dict(case)
    kind = case["kind"]
    if kind == "sample":
        Q, V = case["queries"], case["rows"]
        st["scores"] = (torch.randn((Q, V), generator=g, device="cuda") * case["spread"]).to(DTYPES[case["dtype"]])
        st["uniforms"] = torch.rand((Q, case["draws"]), generator=g, device="cuda")
        st["allowed"] = None
        if case["known_out"]:
            allowed = torch.full((Q, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
            known = _power_law(g, Q * 16, V).view(Q, 16).long()
            for j in range(16):
                word = known[:, j:j + 1] // 32
                allowed.scatter_(1, word, allowed.gather(1, word) & ~(1 << (known[:, j:j + 1] % 32)).to(torch.int32))
            st["allowed"] = allowed

        def pick(values, dtype):
            at = torch.randint(0, len(values), (Q,), generator=g, device="cuda")
            return torch.tensor(values, dtype=dtype, device="cuda")[at]
        st["per_query"] = (None,) * 4
        if case["mixed"]:
            st["per_query"] = (pick((0.0, 0.6, 0.8, 1.0, 1.2), torch.float32), pick((0, 0, 1, 20, 50, 1000), torch.int32),
                               pick((1.0, 1.0, 0.5, 0.9, 0.95), torch.float32), pick((0.0, 0.0, 0.05, 0.1), torch.float32))
    else:
        dim = case["dim"]
        if kind == "quantise":
            st["x"] = _embeddings(g, case["rows"], dim, DTYPES[case["dtype"]])
        else:
            st["codes"], st["scales"] = _plain_quantise(_embeddings(g, case["rows"], dim, torch.float32))
        if kind == "rows":
            st["ids"] = _power_law(g, case["ids"], case["rows"])
        if kind == "scores":
            st["q"] = _embeddings(g, case["queries"], dim, DTYPES.get(case["dtype"], torch.bfloat16))
    if own:
        _prepare_own(st)
    return st


# ------------------------------------------------------------------------------------------ the framework's operators -----
def _prepare_own(st):
    import paper_2101_08358_amd as mar
    types = {"fp32": mar.DTYPE_FP32, "bf16": mar.DTYPE_BF16, "fp16": mar.DTYPE_FP16, "mxfp4": mar.DTYPE_MXFP4}
    st["type"] = types[st["dtype"]]
    byte, f32, i32 = (dict(dtype=t, device="cuda") for t in (torch.uint8, torch.float32, torch.int32))
    if st["kind"] == "sample":
        Q, V, n = st["queries"], st["rows"], st["draws"]
        st["problem"] = mar.MarSampling(V, V, Q, n, st["type"], st["top_k"], st["temperature"], st["top_p"], st["min_p"], 0)
        st.update(ids=torch.empty((Q, n), **i32), log_probs=torch.empty((Q, n), **f32), kept=torch.empty(Q, **i32))
        st["workspace"] = torch.empty(mar.mar_sample_rows_workspace_bytes(st["problem"]), **byte)
        return
    dim, blocks = st["dim"], (st["dim"] + 31) // 32
    if st["kind"] == "quantise":
        st.update(codes=torch.empty((st["rows"], 16 * blocks), **byte), scales=torch.empty((st["rows"], blocks), **byte))
        st["out"] = torch.empty((st["rows"], dim), dtype=torch.bfloat16, device="cuda")
    elif st["kind"] == "rows":
        st["out"] = torch.empty((st["ids"].numel(), dim), dtype=DTYPES[st["dtype"]], device="cuda")
    else:
        Q, V = st["queries"], st["rows"]
        four = st["dtype"] == "mxfp4"
        if four:
            st.update(q_codes=torch.empty((Q, 16 * blocks), **byte), q_scales=torch.empty((Q, blocks), **byte))
        st["problem"] = mar.MarMxfp(V, 16 * blocks, blocks, 16 * blocks if four else dim, blocks if four else 0, V, Q, dim, st["type"],
                                    types[st["out"]], st["scale"], 0)
        st["result"] = torch.empty((Q, V), dtype=DTYPES[st["out"]], device="cuda")
        st["workspace"] = torch.empty(mar.mar_mxfp_scores_workspace_bytes(st["problem"]), **byte)


def _run_own(st):
    import paper_2101_08358_amd as mar
    kind = st["kind"]
    if kind == "sample":
        allowed, ws = st["allowed"], st["workspace"]
        mar.mar_sample_rows(st["problem"], st["scores"], allowed, allowed.shape[1] if allowed is not None else 0, *st["per_query"], st["uniforms"],
                            st["ids"], st["log_probs"], st["kept"], ws, ws.numel())
        return st["ids"], st["log_probs"], st["kept"]
    dim, blocks = st["dim"], (st["dim"] + 31) // 32
    if kind == "quantise":
        n = st["rows"]
        mar.mar_mxfp_quantise(st["x"], dim, n, dim, st["type"], st["codes"], 16 * blocks, st["scales"], blocks)
        mar.mar_mxfp_rows(st["codes"], 16 * blocks, st["scales"], blocks, n, dim, None, n, mar.DTYPE_BF16, st["out"], dim)
        return st["out"], st["scales"]
    if kind == "rows":
        mar.mar_mxfp_rows(st["codes"], 16 * blocks, st["scales"], blocks, st["rows"], dim, st["ids"], st["ids"].numel(), st["type"], st["out"], dim)
        return st["out"]
    q, q_scales, ws = st["q"], None, st["workspace"]
    if st["dtype"] == "mxfp4":
        mar.mar_mxfp_quantise(q, dim, q.shape[0], dim, mar.DTYPE_BF16, st["q_codes"], 16 * blocks, st["q_scales"], blocks)
        q, q_scales = st["q_codes"], st["q_scales"]
    mar.mar_mxfp_scores(st["problem"], q, q_scales, st["codes"], st["scales"], st["result"], ws, ws.numel())
    return st["result"]


# ---------------------------------------------------------------------------------------------------- the plain forms -----
def _plain_quantise(x):
    rows, dim = x.shape
    blocks = (dim + 31) // 32
    codes = torch.empty((rows, 16 * blocks), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, blocks), dtype=torch.uint8, device="cuda")
    step = max(1, PLAIN_VALUES // (32 * blocks))
    for i in range(0, rows, step):
        v = torch.nn.functional.pad(x[i:i + step].float(), (0, 32 * blocks - dim)).view(-1, blocks, 32)
        largest = v.abs().amax(2)
        e = (torch.frexp(largest).exponent - 3).clamp(min=-127)
        e = torch.where(largest > 0, e, torch.full_like(e, -127))
        v = torch.ldexp(v, -e[:, :, None])
        a = v.abs()
        code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * torch.signbit(v)
        code = code.view(-1, 16 * blocks, 2)
        codes[i:i + step] = code[:, :, 0] + 16 * code[:, :, 1]
        scales[i:i + step] = (e + 127).to(torch.uint8)
    return codes, scales


def _plain_values(codes, scales, dim):
    """The values in 32 bits."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
    pair = torch.stack((level[(codes & 15).int()], level[(codes >> 4).int()]), dim=2)
    v = torch.ldexp(pair.view(codes.shape[0], -1, 32), scales.int()[:, :, None] - 127)
    return v.view(codes.shape[0], -1)[:, :dim]


def _run_plain_quantise(st):
    codes, scales = _plain_quantise(st["x"])
    out = torch.empty((st["rows"], st["dim"]), dtype=torch.bfloat16, device="cuda")
    step = max(1, PLAIN_VALUES // (16 * codes.shape[1]))
    for i in range(0, st["rows"], step):
        out[i:i + step] = _plain_values(codes[i:i + step], scales[i:i + step], st["dim"])
    return out, scales


def _run_plain_rows(st):
    ids = st["ids"].long()
    return _plain_values(st["codes"][ids], st["scales"][ids], st["dim"]).to(DTYPES[st["dtype"]])


def _run_plain_scores(st):
    q, dim = st["q"].float(), st["dim"]
    if st["dtype"] == "mxfp4":
        q = _plain_values(*_plain_quantise(q), dim)
    out = torch.empty((q.shape[0], st["rows"]), dtype=DTYPES[st["out"]], device="cuda")
    step = max(1, min(PLAIN_VALUES // (2 * dim), PLAIN_VALUES // q.shape[0]))
    for i in range(0, st["rows"], step):
        w = _plain_values(st["codes"][i:i + step], st["scales"][i:i + step], dim)
        out[:, i:i + step] = (q @ w.T) * st["scale"]
    return out


def _parameters(st):
    """Temperature, top-k, top-p and min-p of every query as columns in 64 bits; greedy queries as top-k 1 at temperature 1."""
    Q = st["queries"]
    given = (st["temperature"], st["top_k"], st["top_p"], st["min_p"])
    temperature, top_k, top_p, min_p = (torch.full((Q, 1), float(torch.tensor(one, dtype=torch.float32)), dtype=torch.float64, device="cuda")
                                        if each is None else each.double()[:, None] for one, each in zip(given, st["per_query"]))
    greedy = temperature == 0
    top_k = torch.where(greedy, torch.ones_like(top_k), torch.where(top_k == 0, torch.full_like(top_k, st["rows"]), top_k))
    top_p = torch.where(top_p >= 1, torch.full_like(top_p, math.inf), top_p)
    return torch.where(greedy, torch.ones_like(temperature), temperature), top_k, top_p, min_p


def _run_plain_sample(st):
    V = st["rows"]
    parameters = _parameters(st)
    step = max(1, PLAIN_DRAWS // V)
    outs = []
    for i in range(0, st["queries"], step):
        part = slice(i, i + step)
        temperature, top_k, top_p, min_p = (a[part] for a in parameters)
        s = st["scores"][part].float()
        if st["allowed"] is not None:
            bits = (st["allowed"][part][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
            s = torch.where(bits.view(s.shape[0], -1)[:, :V].bool(), s, torch.full_like(s, -math.inf))
        s, order = s.sort(dim=1, descending=True, stable=True)
        z = (s.double() - s[:, :1].double()) / temperature
        w = torch.exp(z)
        rank = torch.arange(V, device="cuda")
        w = torch.where(rank < top_k, w, torch.zeros_like(w))
        mass = w.cumsum(1)
        kept = (rank < top_k) & (s > -math.inf) & (mass - w < top_p * mass[:, -1:]) & (w >= min_p)
        w = torch.where(kept, w, torch.zeros_like(w))
        del mass, s
        w = torch.zeros_like(w).scatter_(1, order, w)
        mass = w.cumsum(1)
        total = mass[:, -1:].contiguous()
        ids = torch.searchsorted(mass, st["uniforms"][part].double() * total, right=True).clamp_(max=V - 1)
        outs.append((ids.to(torch.int32), torch.log(w.gather(1, ids) / total).float(), kept.sum(1).to(torch.int32)))
    return tuple(torch.cat(parts) for parts in zip(*outs))


def run(state):
    if own:
        return _run_own(state)
    return {"quantise": _run_plain_quantise, "rows": _run_plain_rows, "scores": _run_plain_scores, "sample": _run_plain_sample}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------- in 64 bits, by definition -----
def _exact_block(v):
    """Blocks [.., 32] in 64 bits: exponents and the nearest representable values, found by trying all of them."""
    largest = v.abs().amax(-1, keepdim=True)
    e = torch.where(largest > 0, torch.floor(torch.log2(largest)), torch.full_like(largest, -125.0))
    e = torch.where(torch.exp2(e) > largest, e - 1, torch.where(torch.exp2(e + 1) <= largest, e + 1, e)) - 2
    e = torch.where(largest > 0, e, torch.full_like(e, -127.0)).clamp(-127, 127)
    unit = torch.exp2(e)
    best, off = torch.zeros_like(v), v.abs()
    for code, level in enumerate(LEVELS[1:], 1):
        now = (v.abs() - level * unit).abs()
        better = (now < off) | ((now == off) & (code % 2 == 0))
        best, off = torch.where(better, level * unit, best), torch.where(better, now, off)
    return e, torch.copysign(best, v)


def _exact_values(codes, scales, dim):
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    out = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    for half in range(2):
        code = (codes.long() // 16 ** half) % 16
        out[:, half::2] = level[code % 8] * (1 - 2 * (code // 8))
    return (out * torch.exp2(scales.double() - 127).repeat_interleave(32, 1))[:, :dim]


def _exact_sample(st):
    ids, log_probs, counts = [], [], []
    temperature, top_k, top_p, min_p = _parameters(st)
    for i in range(st["queries"]):
        s = st["scores"][i].double() / temperature[i]
        rows = torch.arange(s.numel(), device="cuda")
        if st["allowed"] is not None:
            rows = rows[((st["allowed"][i].long()[rows // 32] >> (rows % 32)) & 1) == 1]
        # ties go to the lowest id: a stable order of ids that ascend
        rows = rows[torch.argsort(-st["scores"][i].double()[rows], stable=True)][:int(top_k[i])]
        p = torch.exp(s[rows] - s[rows[0]])
        p = p / p.sum()
        reached = torch.cumsum(p, 0) >= top_p[i]             # a row stays while those before it have not reached top_p
        stay = torch.cat((torch.ones(1, dtype=torch.bool, device="cuda"), ~reached[:-1])) & (p >= min_p[i] * p[0])
        rows, p = rows[stay], p[stay] / p[stay].sum()
        rows, order = torch.sort(rows)
        p = p[order]
        u = st["uniforms"][i].double()
        at = torch.searchsorted(torch.cumsum(p, 0), u, right=True).clamp(max=rows.numel() - 1)
        ids.append(rows[at].to(torch.int32))
        log_probs.append(torch.log(p[at]))
        counts.append(rows.numel())
    return torch.stack(ids), torch.stack(log_probs), torch.tensor(counts, dtype=torch.int32, device="cuda")


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(st)
    dim = case["dim"]
    blocks = (dim + 31) // 32
    if case["kind"] == "rows":
        return _exact_values(st["codes"][st["ids"].long()], st["scales"][st["ids"].long()], dim)
    if case["kind"] == "quantise":
        values = torch.empty((case["rows"], dim), dtype=torch.float64, device="cuda")
        scales = torch.empty((case["rows"], blocks), dtype=torch.uint8, device="cuda")
        for i in range(0, case["rows"], 1 << 18):
            x = st["x"][i:i + (1 << 18)].double()
            x = torch.cat((x, x.new_zeros((x.shape[0], 32 * blocks - dim))), 1)
            e, v = _exact_block(x.view(-1, blocks, 32))
            values[i:i + (1 << 18)] = v.reshape(x.shape[0], -1)[:, :dim]
            scales[i:i + (1 << 18)] = (e[:, :, 0] + 127).to(torch.uint8)
        return values, scales
    q = st["q"].double()
    if case["dtype"] == "mxfp4":
        x = torch.cat((q, q.new_zeros((q.shape[0], 32 * blocks - dim))), 1)
        q = _exact_block(x.view(-1, blocks, 32))[1].reshape(q.shape[0], -1)[:, :dim].contiguous()
    out = torch.empty((case["queries"], case["rows"]), dtype=torch.float64, device="cuda")
    for i in range(0, case["rows"], 1 << 18):
        out[:, i:i + (1 << 18)] = torch.matmul(q, _exact_values(st["codes"][i:i + (1 << 18)], st["scales"][i:i + (1 << 18)], dim).t())
    return out.mul_(case["scale"])


def work(case):
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if case["kind"] == "sample":
        Q, V, n = case["queries"], case["rows"], case["draws"]
        mask = Q * ((V + 31) // 32) * 4 if case["known_out"] else 0
        return {"bytes": Q * V * size[case["dtype"]] + mask + Q * n * 12 + Q * 4 * (5 if case["mixed"] else 1), "flops": Q * V}
    dim = case["dim"]
    packed = 17 * ((dim + 31) // 32)
    if case["kind"] == "quantise":
        n = case["rows"] * dim
        return {"bytes": n * size[case["dtype"]] + 2 * case["rows"] * packed + 2 * n, "flops": 2 * n}
    if case["kind"] == "rows":
        n = case["ids"]
        return {"bytes": n * 4 + min(n, case["rows"]) * packed + n * dim * size[case["dtype"]], "flops": n * dim}
    T, V = case["queries"], case["rows"]
    queries = T * dim * size.get(case["dtype"], 2)
    return {"bytes": queries + V * packed + T * V * size[case["out"]], "flops": 2 * T * V * dim}
