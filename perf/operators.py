"""Measured calls of the operators on whole tables: dropout of queries, log probabilities of answers, and the softmax
loss over all rows with its gradients.

Three kinds of case:

* ``dropout``: one application to a block of rows (the backward pass is the same call on the gradient's rows).
* ``log_probs``: queries against every row of a table: log probability of each query's answer, entropy of its
  distribution, the most probable rows.
* ``loss``: a training call: loss and log-sum-exp of every query, gradients of queries and table.

Embeddings are drawn as they are in the middle of training (a few tenths), answers follow a power law as in the
benchmark's graphs, table sizes are the benchmark's (the large ones cut) or generic.

Where ``own`` is false ``run`` computes the operators in their plain form, from elementary operations in 32 bits.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EMB_STD = 0.3
PLAIN_LOGITS = 1 << 28       # scores that the plain forms hold at a time


def _dropout(name, dtype, rows, dim, p, backward=False):
    return {"name": name, "kind": "dropout", "dtype": dtype, "rows": rows, "dim": dim, "p": p, "backward": backward}


def _log_probs(name, dtype, queries, rows, dim, top, mask="", scale=1.0):
    """mask: "" none, "known" all rows but 16 known answers a query, "half" half of the rows."""
    return {"name": name, "kind": "log_probs", "dtype": dtype, "queries": queries, "rows": rows, "dim": dim, "top": top, "mask": mask,
            "scale": scale}


def _loss(name, dtype, queries, rows, dim, weighted=False, scale=1.0):
    """weighted: a weight for every query, some queries without an answer."""
    return {"name": name, "kind": "loss", "dtype": dtype, "queries": queries, "rows": rows, "dim": dim, "weighted": weighted, "scale": scale}


def listed():
    return [
        # a batch of the benchmark's smallest graph (1,000 edges, 50 floats): latency
        _dropout("dropout_tiny", "fp32", 1_000, 50, 0.2),
        # the benchmark's largest batch: 100,000 queries of 400 floats
        _dropout("dropout_wide", "fp32", 100_000, 400, 0.1),
        # the gradient of hidden states in 16 bits, generic sizes, the last row block short
        _dropout("dropout_bf16_backward", "bf16", 16_001, 4_096, 0.1, backward=True),
        # one query answered from a small knowledge graph (15k nodes): latency
        _log_probs("answer_one_small", "fp32", 1, 14_951, 100, 10),
        # one query against millions of rows in 16 bits: the table is read once
        _log_probs("answer_one_large", "bf16", 1, 4_000_000, 100, 10),
        # a batch of a small knowledge graph's test edges, the known answers taken out
        _log_probs("answers_known_out", "fp32", 1_000, 14_951, 100, 10, mask="known"),
        # odd sizes, half of the rows allowed, a temperature
        _log_probs("answers_ragged", "fp16", 333, 120_007, 75, 5, mask="half", scale=1.25),
        # a large batch against a vocabulary-sized table, 400 columns
        _log_probs("answers_wide", "bf16", 4_096, 131_072, 400, 16),
        # the benchmark's smallest graph: 1,000 queries against its 10,000 nodes
        _loss("loss_tiny", "fp32", 1_000, 10_000, 50),
        # a small knowledge graph's batch (10,000 queries) against all its nodes, the framework's own type
        _loss("loss_kg_small", "fp32", 10_000, 14_951, 100),
        # odd sizes, queries without an answer, weights of either sign
        _loss("loss_ragged", "fp16", 777, 33_333, 75, weighted=True),
        # the largest: 8,192 queries, 65,536 rows, 400 columns in 16 bits
        _loss("loss_wide", "bf16", 8_192, 65_536, 400),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    dtype = rng.choice(("fp32", "bf16", "fp16"))
    kind = rng.choice(("dropout", "log_probs", "loss"))
    if kind == "dropout":
        dim = log_uniform(16, 4_096)
        rows = log_uniform(200, min(100_000, 40_000_000 // dim))
        case = _dropout("", dtype, rows, dim, round(rng.uniform(0.02, 0.6), 3), rng.random() < 0.5)
    elif kind == "log_probs":
        queries, dim = log_uniform(1, 4_096), log_uniform(16, 400)
        rows = log_uniform(1_000, min(2_000_000, 400_000_000 // queries))
        case = _log_probs("", dtype, queries, rows, dim, rng.choice((1, 3, 5, 10, 16, 32)), rng.choice(("", "", "known", "half")),
                          round(rng.uniform(0.5, 1.5), 2))
    else:
        queries, dim = log_uniform(50, 10_000), log_uniform(16, 400)
        rows = log_uniform(1_000, min(200_000, 400_000_000 // queries))
        case = _loss("", dtype, queries, rows, dim, rng.random() < 0.5, round(rng.uniform(0.5, 1.5), 2))
    del case["name"]
    return case


def _answers(g, n, rows):
    """Ids with P(id) ~ (id + 1)^-1.2 by the inverse of the continuous law's distribution."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    x = (1.0 - u * (1.0 - (rows + 1.0) ** -0.2)) ** -5.0
    return (x.long() - 1).clamp_(0, rows - 1).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, dim = DTYPES[case["dtype"]], case["dim"]

    def rows_of(n):
        return (torch.randn((n, dim), generator=g, device="cuda") * EMB_STD).to(dt)
    st = dict(case)
    if case["kind"] == "dropout":
        st.update(x=rows_of(case["rows"]), seed=seed * 7919 + 13, step=seed % 1000 + 1)
        if own:
            st["out"] = torch.empty_like(st["x"])
        return st
    T, V = case["queries"], case["rows"]
    st.update(q=rows_of(T), w=rows_of(V), targets=_answers(g, T, V))
    if case["kind"] == "log_probs":
        st["allowed"] = None
        if case["mask"]:
            words = (V + 31) // 32
            if case["mask"] == "half":
                allowed = torch.randint(-(1 << 31), 1 << 31, (T, words), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
            else:
                allowed = torch.full((T, words), -1, dtype=torch.int32, device="cuda")
                known = _answers(g, T * 16, V).view(T, 16).long()
                for j in range(16):
                    word = known[:, j:j + 1] // 32
                    allowed.scatter_(1, word, allowed.gather(1, word) & ~(1 << (known[:, j:j + 1] % 32)).to(torch.int32))
            t = st["targets"].long()[:, None]
            allowed.scatter_(1, t // 32, allowed.gather(1, t // 32) | (1 << (t % 32)).to(torch.int32))
            st["allowed"] = allowed
    else:
        st["weights"] = None
        if case["weighted"]:
            st["weights"] = torch.rand(T, generator=g, device="cuda") * 2.0 - 0.5
            st["targets"][torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    if own:
        import paper_2101_08358_amd as mar
        dtype = {"fp32": mar.DTYPE_FP32, "bf16": mar.DTYPE_BF16, "fp16": mar.DTYPE_FP16}[case["dtype"]]
        st["problem"] = mar.MarSoftmax(V, dim, dim, T, dim, dtype, case["scale"])
        f32 = dict(dtype=torch.float32, device="cuda")
        if case["kind"] == "log_probs":
            nbytes = mar.mar_log_probs_workspace_bytes(st["problem"], case["top"])
            st.update(log_probs=torch.empty(T, **f32), entropy=torch.empty(T, **f32), top_log_probs=torch.empty((T, case["top"]), **f32),
                      top_ids=torch.empty((T, case["top"]), dtype=torch.int32, device="cuda"))
        else:
            nbytes = mar.mar_softmax_loss_workspace_bytes(st["problem"])
            st.update(loss=torch.empty(T, **f32), lse=torch.empty(T, **f32), grad_q=torch.empty_like(st["q"]), grad_w=torch.empty_like(st["w"]))
        st["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------------ the framework's operators -----
def _run_own(st):
    import paper_2101_08358_amd as mar
    if st["kind"] == "dropout":
        dtype = {"fp32": mar.DTYPE_FP32, "bf16": mar.DTYPE_BF16, "fp16": mar.DTYPE_FP16}[st["dtype"]]
        mar.mar_dropout(st["x"], st["dim"], st["rows"], st["dim"], dtype, st["p"], st["seed"], st["step"], st["out"], st["dim"])
        return st["out"]
    ws = st["workspace"]
    if st["kind"] == "log_probs":
        stride = st["allowed"].shape[1] if st["allowed"] is not None else 0
        mar.mar_log_probs(st["problem"], st["q"], st["w"], st["targets"], st["allowed"], stride, st["top"], st["log_probs"], st["entropy"],
                          st["top_ids"], st["top_log_probs"], ws, ws.numel())
        return st["log_probs"], st["entropy"], st["top_ids"], st["top_log_probs"]
    mar.mar_softmax_loss(st["problem"], st["q"], st["w"], st["targets"], st["weights"], st["loss"], st["lse"], st["grad_q"], st["dim"],
                         st["grad_w"], st["dim"], ws, ws.numel())
    return st["loss"], st["lse"], st["grad_q"], st["grad_w"]


# ---------------------------------------------------------------------------------------------------- the plain forms -----
def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 on int64 tensors that hold 32-bit words."""
    m32 = 0xFFFFFFFF
    k0, k1 = seed & m32, (seed >> 32) & m32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & m32) ^ c1 ^ k0, p1 & m32, ((p0 >> 32) & m32) ^ c3 ^ k1, p0 & m32
        k0, k1 = (k0 + 0x9E3779B9) & m32, (k1 + 0xBB67AE85) & m32
    return c0, c1, c2, c3


def _plain_dropout(st):
    rows, dim = st["rows"], st["dim"]
    groups = (dim + 7) // 8
    r = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c = torch.arange(groups, device="cuda")[None, :].expand(rows, groups)
    n = torch.full_like(c, st["step"] & 0xFFFFFFFF)
    words = _philox(r, c, n, torch.full_like(c, 0xC0000000 | (st["step"] >> 32)), st["seed"])
    u = torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], dim=2).view(rows, groups * 8)[:, :dim]
    threshold = int(math.floor(st["p"] * 65536 + 0.5))
    x = st["x"].float() * (65536.0 / (65536 - threshold))
    return torch.where(u >= threshold, x, torch.zeros_like(x)).to(st["x"].dtype)


def _allowed_rows(words, V):
    bits = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return bits.view(words.shape[0], -1)[:, :V].bool()


def _plain_log_probs(st):
    q, w, V, k = st["q"].float(), st["w"].float(), st["rows"], st["top"]
    outs = []
    for i in range(0, q.shape[0], max(1, PLAIN_LOGITS // V)):
        part = slice(i, i + max(1, PLAIN_LOGITS // V))
        s = (q[part] @ w.T) * st["scale"]
        if st["allowed"] is not None:
            s = torch.where(_allowed_rows(st["allowed"][part], V), s, torch.full_like(s, -math.inf))
        m = s.amax(1, keepdim=True)
        z = s - m
        e = torch.exp(z)
        total = e.sum(1)
        lse = torch.log(total)
        entropy = lse - (e * torch.where(e > 0, z, torch.zeros_like(z))).sum(1) / total
        log_prob = z.gather(1, st["targets"][part].long()[:, None])[:, 0] - lse
        # the order of the most probable rows: values next to one another are told apart in 64 bits
        ids = torch.topk(s, min(k + 8, V), dim=1).indices.sort(1).values
        exact = (q[part].double()[:, None, :] * w[ids].double()).sum(2) * float(st["scale"])
        exact = torch.where(torch.isfinite(s.gather(1, ids)), exact, torch.full_like(exact, -math.inf))
        exact, order = exact.sort(dim=1, descending=True, stable=True)
        ids = ids.gather(1, order)[:, :k]
        outs.append((log_prob, entropy, ids.to(torch.int32), (exact[:, :k] - (m + lse[:, None]).double()).float()))
    return tuple(torch.cat(parts) for parts in zip(*outs))


def _plain_loss(st):
    q, w, V = st["q"].float(), st["w"].float(), st["rows"]
    losses, lses, gq, gw = [], [], [], torch.zeros_like(w)
    for i in range(0, q.shape[0], max(1, PLAIN_LOGITS // V)):
        part = slice(i, i + max(1, PLAIN_LOGITS // V))
        t = st["targets"][part].long()[:, None]
        has = t >= 0
        s = (q[part] @ w.T) * st["scale"]
        m = s.amax(1, keepdim=True)
        lse = m + torch.log(torch.exp(s - m).sum(1, keepdim=True))
        losses.append(torch.where(has, lse - s.gather(1, t.clamp(min=0)), torch.zeros_like(lse))[:, 0])
        lses.append(lse[:, 0])
        u = has.float() * st["scale"]
        if st["weights"] is not None:
            u = u * st["weights"][part][:, None]
            losses[-1] = losses[-1] * st["weights"][part]
        p = torch.exp(s - lse)
        p.scatter_add_(1, t.clamp(min=0), torch.full_like(lse, -1.0))
        p = p * u
        gq.append(p @ w)
        gw += p.T @ q[part]
    return torch.cat(losses), torch.cat(lses), torch.cat(gq).to(st["q"].dtype), gw.to(st["w"].dtype)


def run(state):
    if own:
        return _run_own(state)
    return {"dropout": _plain_dropout, "log_probs": _plain_log_probs, "loss": _plain_loss}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------- in 64 bits, by definition -----
def _mul32(a, m):
    """High and low 32 bits of a (tensor of 32-bit words) times m, in 16-bit limbs."""
    a0, a1, m0, m1 = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    low, mid, mid2, high = a0 * m0, a1 * m0, a0 * m1, a1 * m1
    carry = (low >> 16) + (mid & 0xFFFF) + (mid2 & 0xFFFF)
    return high + (mid >> 16) + (mid2 >> 16) + (carry >> 16), ((carry & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_dropout(case, x, seed, step):
    rows, dim = x.shape
    out = torch.empty((rows, dim), dtype=torch.float64, device="cuda")
    threshold = int(math.floor(case["p"] * 65536 + 0.5))
    keep = 1.0 - threshold / 65536.0
    for g in range((dim + 7) // 8):
        ctr = [torch.arange(rows, device="cuda"), torch.full((rows,), g, device="cuda"), torch.full((rows,), step & 0xFFFFFFFF, device="cuda"),
               torch.full((rows,), 0xC0000000 + (step >> 32), device="cuda")]
        key = [seed % (1 << 32), (seed >> 32) % (1 << 32)]
        for _ in range(10):
            h0, l0 = _mul32(ctr[0], 0xD2511F53)
            h1, l1 = _mul32(ctr[2], 0xCD9E8D57)
            ctr = [h1 ^ ctr[1] ^ key[0], l1, h0 ^ ctr[3] ^ key[1], l0]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        for e in range(min(8, dim - 8 * g)):
            u = (ctr[e // 2] >> (16 * (e % 2))) % 65536
            out[:, 8 * g + e] = (u >= threshold).double() * x[:, 8 * g + e].double() / keep
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "dropout":
        return _exact_dropout(case, st["x"], st["seed"], st["step"])
    q, w = st["q"].double(), st["w"].double()
    T, V = q.shape[0], w.shape[0]
    step = max(1, (1 << 27) // V)
    if case["kind"] == "log_probs":
        k, rows = case["top"], []
        for i in range(0, T, step):
            s = torch.matmul(q[i:i + step], w.t()).mul_(case["scale"])
            if st["allowed"] is not None:
                words = st["allowed"][i:i + step].long()
                col = torch.arange(V, device="cuda")
                s.masked_fill_(((words[:, col // 32] >> (col % 32)) & 1) == 0, -math.inf)
            logp = s - torch.logsumexp(s, 1, keepdim=True)
            entropy = -(logp.exp() * logp.masked_fill(logp == -math.inf, 0.0)).sum(1)
            best, ids = torch.topk(logp, min(k + 4, V), dim=1)
            ids, order = ids.sort(1)
            best, order = best.gather(1, order).sort(dim=1, descending=True, stable=True)
            ids = ids.gather(1, order)
            rows.append((logp.gather(1, st["targets"][i:i + step].long().unsqueeze(1)).squeeze(1), entropy, ids[:, :k].to(torch.int32), best[:, :k]))
        return tuple(torch.cat(parts) for parts in zip(*rows))
    scale = case["scale"]
    gw, rows = torch.zeros_like(w), []
    for i in range(0, T, step):
        t = st["targets"][i:i + step].long()
        s = torch.matmul(q[i:i + step], w.t()).mul_(scale)
        lse = torch.logsumexp(s, 1)
        u = torch.ones_like(lse) if st["weights"] is None else st["weights"][i:i + step].double()
        u = torch.where(t < 0, torch.zeros_like(u), u)
        at = torch.arange(t.numel(), device="cuda")
        loss = u * (lse - s[at, t.clamp(min=0)])
        d = torch.exp(s - lse[:, None])
        d[at, t.clamp(min=0)] -= 1.0
        d *= (u * scale)[:, None]
        rows.append((loss, lse, torch.matmul(d, w)))
        gw += torch.matmul(d.t().contiguous(), q[i:i + step])
    loss, lse, gq = (torch.cat(parts) for parts in zip(*rows))
    return loss, lse, gq, gw


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "dropout":
        n = case["rows"] * case["dim"]
        return {"bytes": 2 * n * e, "flops": n}
    T, V, d = case["queries"], case["rows"], case["dim"]
    if case["kind"] == "log_probs":
        mask = T * ((V + 31) // 32) * 4 if case["mask"] else 0
        return {"bytes": (T + V) * d * e + mask + T * 4 + T * (8 + 8 * case["top"]), "flops": 2 * T * V * d}
    return {"bytes": 2 * (T + V) * d * e + T * 4 * (2 if case["weighted"] else 1) + 8 * T, "flops": 6 * T * V * d}
