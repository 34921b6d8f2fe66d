"""What the training and serving operators around the graph layers are timed on: dropout, attention over a pattern with capped and biased
scores, log probabilities of labels.  `own` chooses who computes them: False, plain torch operations; True, this library.

Sizes are those of the benchmark, of perf/cases.py and of the tests (a mini-batch of 1,024 seeds with 47 classes, 100,000 nodes of about 20
entries, 233,000 nodes with 602 features and 41 classes, 2.45 M nodes) or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _drop(name, dtype, rows, cols, p, add=False):
    c = {"op": "dropout", "type": dtype, "rows": rows, "cols": cols, "p": p, "add": add}
    return dict(c, name=name) if name else c


def _logp(name, dtype, rows, classes, top=0, train=False, labelled=1.0, entropy_grad=False):
    c = {"op": "logprobs", "type": dtype, "rows": rows, "classes": classes, "top": top, "train": train, "labelled": labelled, "entropy_grad": entropy_grad}
    return dict(c, name=name) if name else c


def _attn(name, dtype, graph, nodes, links, heads, kv_heads, d, dv, train=False, cap=0.0, buckets=0, p=0.0):
    """graph: er / rmat = `links` distinct undirected links, mirrored, plus self loops; docs = `nodes` small graphs of 10 to `links` nodes, every node
    attending to all of its own graph; block = `nodes` destinations with `links` sampled sources each and themselves."""
    c = {"op": "attention", "type": dtype, "graph": graph, "nodes": nodes, "links": links, "heads": heads, "kv_heads": kv_heads, "d": d, "dv": dv,
         "train": train, "cap": cap, "buckets": buckets, "p": p}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the features of a mini-batch's seeds: the smallest call
        _drop("drop_seeds", "f32", 1024, 100, 0.5),
        # the input features of the benchmark's graph, ragged rows of 602
        _drop("drop_features", "f32", 233_000, 602, 0.5),
        # hidden states of the 2.45 M-node graph in half the bits, added to the residual stream
        _drop("drop_residual_bf16", "bf16", 2_450_000, 256, 0.1, add=True),
        # the loss of a sampled mini-batch
        _logp("logp_seeds_train", "f32", 1024, 47, train=True),
        # full-graph training: 41 classes, two thirds of the nodes labelled, an entropy term in the loss
        _logp("logp_nodes_train", "f32", 233_000, 41, train=True, labelled=0.66, entropy_grad=True),
        # ranking every entity for many queries at once
        _logp("logp_rank_bf16", "bf16", 4096, 100_003, top=10),
        # the same for two queries: few rows, a long axis
        _logp("logp_rank_two", "f32", 2, 250_000, top=5),
        # training over a large class set
        _logp("logp_wide_train_f16", "f16", 16_384, 50_021, train=True),
        # one attention layer on a 10,000-node graph: latency
        _attn("attn_er10k", "f32", "er", 10_000, 50_000, 4, 4, 16, 16),
        # a training step on 100,000 nodes: capped scores, 16 distance buckets, dropped weights
        _attn("attn_rmat100k_train", "f32", "rmat", 100_000, 1_000_000, 4, 4, 32, 32, train=True, cap=20.0, buckets=16, p=0.1),
        # training on batches of small graphs with a bias by distance, the last bucket masked
        _attn("attn_docs_train_bf16", "bf16", "docs", 8192, 60, 8, 8, 16, 16, train=True, buckets=32, p=0.1),
        # inference on a power-law graph of 90 entries per row, four query heads to a key head
        _attn("attn_rmat233k_bf16", "bf16", "rmat", 233_000, 10_000_000, 8, 2, 64, 64, cap=30.0),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("dropout", "logprobs", "logprobs", "attention", "attention", "attention"))
    dtype = rng.choice(("f32", "f32", "bf16", "f16"))
    if op == "dropout":
        cols = _logint(rng, 8, 2048)
        rows = _logint(rng, 256, max(512, min(2_450_000, 400_000_000 // cols)))
        return _drop(None, dtype, rows, cols, rng.choice((0.1, 0.25, 0.5, 0.6)), rng.random() < 0.4)
    if op == "logprobs":
        classes = _logint(rng, 2, 250_000)
        rows = _logint(rng, 1, max(2, min(2_450_000, 400_000_000 // classes)))
        train = rng.random() < 0.5
        top = 0 if train else rng.choice((0, 1, 5, 10, 16))
        return _logp(None, dtype, rows, classes, min(top, classes), train, rng.choice((1.0, 0.5)), train and rng.random() < 0.5)
    graph = rng.choice(("er", "rmat", "docs", "block"))
    kv = rng.choice((1, 2, 3, 4, 8))
    heads = kv * rng.choice((1, 1, 1, 2, 4)) if kv <= 4 else kv
    d = rng.choice((8, 16, 20, 25, 32, 48, 64, 96, 128))
    dv = d if rng.random() < 0.75 else rng.choice((8, 24, 33, 64))
    train = rng.random() < 0.6
    budget = (1.5e9 if train else 4e9) / (heads * max(d, dv))
    if graph == "docs":
        links = _logint(rng, 12, 200)
        nodes = _logint(rng, 16, max(32, min(8192, budget / (0.4 * links * links))))
    else:
        nodes = _logint(rng, 500, 400_000)
        degree = _logint(rng, 2, max(3, min(300, nodes // 20, budget / nodes)))
        links = degree if graph == "block" else max(1, nodes * degree // 2)
    return _attn(None, dtype, graph, nodes, links, heads, kv, d, dv, train, rng.choice((0.0, 0.0, 20.0, 30.0)), rng.choice((0, 0, 8, 32)),
                 rng.choice((0.0, 0.1, 0.5)) if train else 0.0)


# ------------------------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * (int(seed) + 1))
    return g


def _rmat_keys(g, n, m):
    u = torch.zeros(m, dtype=torch.int64, device=DEV)
    v = torch.zeros(m, dtype=torch.int64, device=DEV)
    for _ in range(max(1, math.ceil(math.log2(n)))):
        x = torch.rand(m, generator=g, device=DEV)
        u.mul_(2).add_(x >= 0.76)
        v.mul_(2).add_(((x >= 0.57) & (x < 0.76)) | (x >= 0.95))
    ok = (u < n) & (v < n) & (u != v)
    u, v = u[ok], v[ok]
    return torch.minimum(u, v) * n + torch.maximum(u, v)


def _er_keys(g, n, m):
    u = torch.randint(0, n, (m,), generator=g, device=DEV)
    v = torch.randint(0, n, (m,), generator=g, device=DEV)
    u, v = u[u != v], v[u != v]
    return torch.minimum(u, v) * n + torch.maximum(u, v)


def _doc_sizes(case):
    span = case["links"] - 10 + 1
    return [10 + (i * 7919) % span for i in range(case["nodes"])]


def _entries(g, case):
    """(n_rows, n_cols, sorted row * n_cols + col)"""
    n, links = case["nodes"], case["links"]
    if case["graph"] == "docs":
        size = torch.tensor(_doc_sizes(case), dtype=torch.int64, device=DEV)
        n = int(size.sum())
        of_row = torch.repeat_interleave(torch.arange(size.numel(), device=DEV), size)
        start = torch.cumsum(size, 0) - size
        per_row = size[of_row]
        row = torch.repeat_interleave(torch.arange(n, device=DEV), per_row)
        first = torch.cumsum(per_row, 0) - per_row
        col = torch.arange(row.numel(), device=DEV) - first[row] + start[of_row][row]
        return n, n, row * n + col
    if case["graph"] == "block":
        n_cols = 4 * n
        row = torch.arange(n, device=DEV)
        col = torch.randint(0, n_cols, (n, links), generator=g, device=DEV)
        return n, n_cols, torch.unique(torch.cat([(row[:, None] * n_cols + col).reshape(-1), row * n_cols + row]))
    keys, m = torch.empty(0, dtype=torch.int64, device=DEV), int(links * 1.35) + 64
    for _ in range(40):
        keys = torch.unique(torch.cat([keys, (_rmat_keys if case["graph"] == "rmat" else _er_keys)(g, n, m)]))
        if keys.numel() >= links:
            break
        m = 2 * (links - keys.numel()) + links // 16 + 64
    keys = keys[torch.randperm(keys.numel(), generator=g, device=DEV)[:links]]
    u = torch.div(keys, n, rounding_mode="floor")
    v = keys - u * n
    i = torch.arange(n, device=DEV)
    return n, n, torch.sort(torch.cat([keys, v * n + u, i * (n + 1)]))[0]


def _normal(g, dtype, *shape, std=1.0):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def prepare(case, seed):
    g, dtype = _gen(seed), TYPES[case["type"]]
    s = {"case": case, "drop_seed": 0x9D2C_5680_0000_0001 + 977 * int(seed), "offset": 3 + int(seed)}
    if own:
        from paper_2306_15155_amd import Context, csr_struct
        s["ctx"] = Context(0)
    if case["op"] == "dropout":
        s["X"] = _normal(g, dtype, case["rows"], case["cols"])
        s["add"] = _normal(g, dtype, case["rows"], case["cols"]) if case["add"] else None
        return s
    if case["op"] == "logprobs":
        n, c = case["rows"], case["classes"]
        s["Z"] = _normal(g, dtype, n, c, std=2.0)
        s["labels"] = torch.randint(0, c, (n,), generator=g, device=DEV).to(torch.int32)
        if case["labelled"] < 1.0:
            s["labels"][torch.rand(n, generator=g, device=DEV) >= case["labelled"]] = -1
        # the gradient of the summed negative log likelihood, and of an entropy bonus
        s["g_logp"] = torch.full((n,), -1.0, device=DEV) if case["train"] else None
        s["g_entropy"] = torch.full((n,), -0.05, device=DEV) if case["entropy_grad"] else None
        return s
    n_rows, n_cols, keys = _entries(g, case)
    row = torch.div(keys, n_cols, rounding_mode="floor")
    col = keys - row * n_cols
    heads, kv, d, dv = case["heads"], case["kv_heads"], case["d"], case["dv"]
    ptr = torch.zeros(n_rows + 1, dtype=torch.int64, device=DEV)
    ptr[1:] = torch.cumsum(torch.bincount(row, minlength=n_rows), 0)
    s.update(n_rows=n_rows, n_cols=n_cols, row_ptr=ptr.to(torch.int32), col_idx=col.to(torch.int32), scale=1.0 / math.sqrt(d))
    s["Q"], s["K"], s["V"] = _normal(g, dtype, n_rows, heads * d), _normal(g, dtype, n_cols, kv * d), _normal(g, dtype, n_cols, kv * dv)
    s["buckets"] = s["bias"] = None
    if case["buckets"]:
        # a self edge is in bucket 0, the others spread with a preference for near ones; the last bucket of a batch of graphs is masked
        nb = case["buckets"]
        far = (torch.rand(col.numel(), generator=g, device=DEV).square() * (nb - 1)).to(torch.int64) + 1
        s["buckets"] = torch.where(row == col, torch.zeros_like(far), far.clamp(max=nb - 1)).to(torch.uint8)
        s["bias"] = _normal(g, torch.float32, heads, nb, std=0.5)
        if case["graph"] == "docs":
            s["bias"][:, nb - 1] = -math.inf
    if case["train"]:
        s["dY"] = _normal(g, dtype, n_rows, heads * dv)
        order = torch.argsort(col * n_rows + row)      # entries by column: the transposed pattern
        t_ptr = torch.zeros(n_cols + 1, dtype=torch.int64, device=DEV)
        t_ptr[1:] = torch.cumsum(torch.bincount(col, minlength=n_cols), 0)
        t_pos = torch.empty_like(order)
        t_pos[order] = torch.arange(order.numel(), device=DEV)
        s.update(t_order=order.to(torch.int32), t_ptr=t_ptr.to(torch.int32), t_col=row[order].to(torch.int32), t_pos=t_pos.to(torch.int32))
    if own:
        s["A"] = csr_struct(n_rows, n_cols, s["row_ptr"], s["col_idx"])
        if case["train"]:
            s["At"] = csr_struct(n_cols, n_rows, s["t_ptr"], s["t_col"])
    return s


# ----------------------------------------------------------------------------------------------------------------- plain forms

_M32 = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32 with seven rounds (Salmon et al. 2011): four 32-bit words (as int64) per counter."""
    k0, k1 = seed & _M32, (seed >> 32) & _M32
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57       # wraps modulo 2^64, which keeps both halves
        c0, c1, c2, c3 = ((b >> 32) & _M32) ^ c1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ c3 ^ k1, a & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return c0, c1, c2, c3


def _threshold(p):
    return min(_M32, int(round(p * 4294967296.0)))


def _plain_dropout(s):
    case, X = s["case"], s["X"]
    n, c = X.shape
    quads = (c + 3) // 4
    q = torch.arange(quads, device=DEV)[None, :].expand(n, quads).reshape(-1)
    r = torch.arange(n, device=DEV)[:, None].expand(n, quads).reshape(-1)
    zero = torch.zeros((), dtype=torch.int64, device=DEV)
    words = _philox(q, r, zero, zero + s["offset"], s["drop_seed"])
    t = _threshold(case["p"])
    keep = torch.stack([w >= t for w in words], 1).reshape(n, quads * 4)[:, :c]
    y = torch.where(keep, X.float() * (1.0 / (1.0 - case["p"])), 0.0)
    if s["add"] is not None:
        y = y + s["add"].float()
    return {"Y": y.to(X.dtype)}


def _plain_logprobs(s):
    case, z = s["case"], s["Z"].float()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    l = e.sum(1, keepdim=True)
    lse = m + torch.log(l)
    stats = torch.cat([m, torch.log(l)], 1)
    entropy = (torch.log(l) - (e * (z - m)).sum(1, keepdim=True) / l)[:, 0]
    has = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long()[:, None]
    out = {"stats": stats, "logp": torch.where(has, (torch.gather(z, 1, at) - lse)[:, 0], 0.0), "entropy": entropy}
    if case["top"]:
        v, i = torch.sort(z, dim=1, descending=True, stable=True)     # equal values: the lowest class first
        out["top_idx"], out["top_logp"] = i[:, : case["top"]].to(torch.int32), v[:, : case["top"]] - lse
    if case["train"]:
        p = e / l
        gl = torch.where(has, s["g_logp"], 0.0)[:, None]
        dz = -gl * p
        dz.scatter_add_(1, at, gl)
        if s["g_entropy"] is not None:
            dz -= s["g_entropy"][:, None] * p * (z - lse + entropy[:, None])
        out["dZ"] = dz.to(s["Z"].dtype)
    return out


def _keep(s, row, col, h):
    t = _threshold(s["case"]["p"])
    zero = torch.zeros((), dtype=torch.int64, device=DEV)
    return _philox(col, row, zero + (0x80000000 | (h >> 2)), zero + s["offset"], s["drop_seed"])[h & 3] >= t


def _plain_attention(s):
    case = s["case"]
    heads, kv, d, dv, cap, p = case["heads"], case["kv_heads"], case["d"], case["dv"], case["cap"], case["p"]
    n_rows, n_cols, dtype = s["n_rows"], s["n_cols"], s["Q"].dtype
    ptr = s["row_ptr"].long()
    col = s["col_idx"].long()
    row = torch.repeat_interleave(torch.arange(n_rows, device=DEV), ptr[1:] - ptr[:-1])
    bucket = None if s["buckets"] is None else s["buckets"].long()
    by_row = lambda x, how="sum", start=0.0: torch.segment_reduce(x, how, offsets=ptr, axis=0, initial=start)  # noqa: E731
    Y = torch.empty(n_rows, heads * dv, device=DEV)
    stats = torch.empty(n_rows, heads, 2, device=DEV)
    train = case["train"]
    if train:
        order, t_ptr = s["t_order"].long(), s["t_ptr"].long()
        by_col = lambda x: torch.segment_reduce(x[order], "sum", offsets=t_ptr, axis=0, initial=0.0)  # noqa: E731
        dQ, dK, dV = torch.empty(n_rows, heads * d, device=DEV), torch.zeros(n_cols, kv * d, device=DEV), torch.zeros(n_cols, kv * dv, device=DEV)
        dbias = None if bucket is None else torch.zeros(heads, case["buckets"], device=DEV)
    for h in range(heads):
        g = h * kv // heads
        q, k, v = (s[x][:, i * w:(i + 1) * w].float() for x, i, w in (("Q", h, d), ("K", g, d), ("V", g, dv)))
        x = (q[row] * k[col]).sum(1) * s["scale"]
        slope = 1.0
        if cap > 0.0:
            th = torch.tanh(x / cap)
            x, slope = cap * th, 1.0 - th * th
        if bucket is not None:
            x = x + s["bias"][h][bucket]
        m = by_row(x, "max", -math.inf)
        e = torch.exp(x - m[row])
        l = by_row(e)
        stats[:, h, 0], stats[:, h, 1] = m, torch.log(l)
        alpha = e / l[row]
        keep = (_keep(s, row, col, h).float() / (1.0 - p)) if p > 0.0 else None
        w = alpha if keep is None else alpha * keep
        y = by_row(w[:, None] * v[col])
        Y[:, h * dv:(h + 1) * dv] = y
        if train:
            dy = s["dY"][:, h * dv:(h + 1) * dv].float()
            dyr = dy[row]
            dp = (dyr * v[col]).sum(1)
            if keep is not None:
                dp = dp * keep
            dt = alpha * (dp - (dy * y).sum(1)[row])
            dV[:, g * dv:(g + 1) * dv] += by_col(w[:, None] * dyr)
            del dyr
            if bucket is not None:
                dbias[h] = torch.stack([torch.where(bucket == b, dt, 0.0).sum() for b in range(case["buckets"])])
            ds = (dt * slope * s["scale"])[:, None]
            dQ[:, h * d:(h + 1) * d] = by_row(ds * k[col])
            dK[:, g * d:(g + 1) * d] += by_col(ds * q[row])
    out = {"Y": Y.to(dtype), "stats": stats}
    if train:
        out.update(dQ=dQ.to(dtype), dK=dK.to(dtype), dV=dV.to(dtype))
        if dbias is not None:
            out["dbias"] = dbias
    return out


# ------------------------------------------------------------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if not own:
        return {"dropout": _plain_dropout, "logprobs": _plain_logprobs, "attention": _plain_attention}[case["op"]](s)
    ctx = s["ctx"]
    if case["op"] == "dropout":
        return {"Y": ctx.dropout(s["X"], case["p"], s["drop_seed"], s["offset"], add=s["add"])}
    if case["op"] == "logprobs":
        r = ctx.logprobs(s["Z"], s["labels"], top=case["top"])
        out = {"stats": r.stats, "logp": r.logp, "entropy": r.entropy}
        if case["top"]:
            out["top_idx"], out["top_logp"] = r.top_idx, r.top_logp
        if case["train"]:
            out["dZ"] = ctx.logprobs_backward(s["Z"], s["labels"], r.stats, g_logp=s["g_logp"], entropy=r.entropy, g_entropy=s["g_entropy"])
        return out
    opts = dict(n_kv_heads=case["kv_heads"], scale=s["scale"], cap=case["cap"], buckets=s["buckets"], bias=s["bias"], p=case["p"], seed=s["drop_seed"],
                offset=s["offset"])
    Y, stats = ctx.attention(s["A"], s["Q"], s["K"], s["V"], case["heads"], **opts)
    out = {"Y": Y, "stats": stats}
    if case["train"]:
        dQ, dK, dV, dbias = ctx.attention_backward(s["A"], s["At"], s["t_pos"], s["Q"], s["K"], s["V"], case["heads"], Y, stats, s["dY"], **opts)
        out.update(dQ=dQ, dK=dK, dV=dV)
        if dbias is not None:
            out["dbias"] = dbias
    return out


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits

def _words64(c0, c1, c2, c3, seed):
    """The generator again, its products from 16-bit halves."""
    def mul(x, m):
        lo, hi = x & 0xFFFF, x >> 16
        ml, mh = m & 0xFFFF, m >> 16
        mid = hi * ml + (lo * ml >> 16)
        mid2 = lo * mh + (mid & 0xFFFF)
        return (hi * mh + (mid >> 16) + (mid2 >> 16)) & _M32, ((mid2 & 0xFFFF) << 16) | (lo * ml & 0xFFFF)

    k = [seed & _M32, seed >> 32 & _M32]
    for _ in range(7):
        h0, l0 = mul(c0, 0xD2511F53)
        h1, l1 = mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k[0], l1, h0 ^ c3 ^ k[1], l0
        k = [(k[0] + 0x9E3779B9) & _M32, (k[1] + 0xBB67AE85) & _M32]
    return [c0, c1, c2, c3]


def _exact_dropout(s):
    case, X = s["case"], s["X"]
    n, c = X.shape
    t, Y = round(case["p"] * 2 ** 32), torch.empty(n, c, dtype=torch.float64, device=DEV)
    per = max(1, 40_000_000 // c)
    for lo in range(0, n, per):
        x = X[lo:lo + per].double()
        r = torch.arange(lo, lo + x.size(0), device=DEV)[:, None]
        q = torch.arange((c + 3) // 4, device=DEV)[None, :]
        for j, w in enumerate(_words64(q, r, 0 * q, 0 * q + s["offset"], s["drop_seed"])):
            part = x[:, j::4]
            part *= (w[:, : part.size(1)] >= t).double() / (1.0 - case["p"])
        Y[lo:lo + per] = x if s["add"] is None else x + s["add"][lo:lo + per].double()
    return {"Y": Y}


def _exact_logprobs(s):
    case, parts = s["case"], {}
    n, c = s["Z"].shape
    per = max(1, 100_000_000 // c)
    for lo in range(0, n, per):
        z = s["Z"][lo:lo + per].double()
        lab = s["labels"][lo:lo + per].long()
        lp = z - torch.logsumexp(z, 1, keepdim=True)
        p = lp.exp()
        i = torch.arange(z.size(0), device=DEV)
        has = (lab >= 0).double()
        ent = -(p * lp).sum(1)
        top = z.amax(1)
        got = {"stats": torch.stack([top, (z - lp)[:, 0] - top], 1), "logp": lp[i, lab.clamp(min=0)] * has, "entropy": ent}
        if case["top"]:
            # order by value, then by class from the lowest: one whole number for both
            bits = s["Z"][lo:lo + per].float().view(torch.int32).long()
            bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
            key = bits * 2 ** 20 - torch.arange(c, device=DEV)
            got["top_idx"] = torch.topk(key, case["top"], dim=1, sorted=True)[1].to(torch.int32)
            got["top_logp"] = torch.gather(lp, 1, got["top_idx"].long())
        if case["train"]:
            gl = s["g_logp"][lo:lo + per].double() * has
            dz = -p * gl[:, None]
            dz[i, lab.clamp(min=0)] += gl
            if s["g_entropy"] is not None:
                dz -= s["g_entropy"][lo:lo + per].double()[:, None] * p * (lp + ent[:, None])
            got["dZ"] = dz
        for k, v in got.items():
            parts.setdefault(k, []).append(v)
    return {k: torch.cat(v) for k, v in parts.items()}


def _exact_attention(s):
    """Entries taken in pieces; sums over rows and columns by indexed addition."""
    case = s["case"]
    heads, kv, d, dv, p = case["heads"], case["kv_heads"], case["d"], case["dv"], case["p"]
    n_rows, n_cols, nnz = s["n_rows"], s["n_cols"], s["col_idx"].numel()
    if nnz * heads * max(d, dv) > 12_000_000_000:
        return None
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    Y, stats = new(n_rows, heads, dv), new(n_rows, heads, 2)
    dQ, dK, dV, dbias = new(n_rows, heads, d), new(n_cols, kv, d), new(n_cols, kv, dv), new(heads, max(1, case["buckets"]))
    row = torch.searchsorted(s["row_ptr"].long(), torch.arange(nnz, device=DEV), right=True) - 1
    col = s["col_idx"].long()
    step = max(1, 200_000_000 // max(d, dv))
    for h in range(heads):
        g = h // (heads // kv)
        q = s["Q"].view(n_rows, heads, d)[:, h].double()
        k, v = s["K"].view(n_cols, kv, d)[:, g].double(), s["V"].view(n_cols, kv, dv)[:, g].double()
        raw = torch.cat([torch.einsum("ed,ed->e", q[row[a:a + step]], k[col[a:a + step]]) for a in range(0, nnz, step)]) * s["scale"]
        x = case["cap"] * torch.tanh(raw / case["cap"]) if case["cap"] > 0.0 else raw
        inner = 1.0 - (x / case["cap"]) ** 2 if case["cap"] > 0.0 else torch.ones_like(raw)
        if s["bias"] is not None:
            x = x + s["bias"][h].double()[s["buckets"].long()]
        top = torch.full((n_rows,), -math.inf, dtype=torch.float64, device=DEV).scatter_reduce_(0, row, x, "amax")
        z = new(n_rows).index_add_(0, row, torch.exp(x - top[row]))
        stats[:, h] = torch.stack([top, torch.log(z)], 1)
        a = torch.exp(x - stats[:, h].sum(1)[row])
        kept = torch.ones_like(a)
        if p > 0.0:
            zero = torch.zeros_like(row)
            kept = (_words64(col, row, zero + (2 ** 31 + h // 4), zero + s["offset"], s["drop_seed"])[h % 4] >= round(p * 2 ** 32)).double() / (1.0 - p)
        for b in range(0, nnz, step):
            e = slice(b, b + step)
            Y[:, h].index_add_(0, row[e], (a[e] * kept[e])[:, None] * v[col[e]])
        if not case["train"]:
            continue
        dy = s["dY"].view(n_rows, heads, dv)[:, h].double()
        da = torch.cat([torch.einsum("ed,ed->e", dy[row[b:b + step]], v[col[b:b + step]]) for b in range(0, nnz, step)]) * kept
        dt = a * (da - new(n_rows).index_add_(0, row, a * da)[row])
        if s["bias"] is not None:
            dbias[h].index_add_(0, s["buckets"].long(), dt)
        ds = dt * inner * s["scale"]
        for b in range(0, nnz, step):
            e = slice(b, b + step)
            dQ[:, h].index_add_(0, row[e], ds[e, None] * k[col[e]])
            dK[:, g].index_add_(0, col[e], ds[e, None] * q[row[e]])
            dV[:, g].index_add_(0, col[e], (a[e] * kept[e])[:, None] * dy[row[e]])
    out = {"Y": Y.flatten(1), "stats": stats}
    if case["train"]:
        out.update(dQ=dQ.flatten(1), dK=dK.flatten(1), dV=dV.flatten(1))
        if s["bias"] is not None:
            out["dbias"] = dbias
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "logprobs": _exact_logprobs, "attention": _exact_attention}[case["op"]](s)


# ---------------------------------------------------------------------------------------------------------------------------- work

def work(case):
    """Every input read once, every output written once; the products of attention (its backward forms the scores and the products with dY
    again), a few operations an element for the others."""
    b = torch.finfo(TYPES[case["type"]]).bits // 8
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * b * (3.0 if case["add"] else 2.0), "flops": 2.0 * n}
    if case["op"] == "logprobs":
        n = case["rows"] * case["classes"]
        rows = case["rows"] * (16.0 + 8.0 * case["top"])
        return {"bytes": n * b * (3.0 if case["train"] else 1.0) + rows * (2.0 if case["train"] else 1.0), "flops": n * (8.0 if case["train"] else 4.0)}
    if case["graph"] == "docs":
        sizes = _doc_sizes(case)
        n_rows = n_cols = sum(sizes)
        nnz = sum(x * x for x in sizes)
    elif case["graph"] == "block":
        n_rows, n_cols, nnz = case["nodes"], 4 * case["nodes"], case["nodes"] * (case["links"] + 1)
    else:
        n_rows = n_cols = case["nodes"]
        nnz = 2 * case["links"] + case["nodes"]
    heads, kv, d, dv = case["heads"], case["kv_heads"], case["d"], case["dv"]
    q, k, v, y = n_rows * heads * d, n_cols * kv * d, n_cols * kv * dv, n_rows * heads * dv
    pattern = nnz * (5.0 if case["buckets"] else 4.0) + 4.0 * n_rows
    total, flops = b * (q + k + v + y) + pattern + 4.0 * n_rows * heads, 2.0 * nnz * heads * (d + dv)
    if case["train"]:
        total += b * (2 * q + 2 * k + 2 * v + 2 * y) + pattern + 4.0 * (nnz + n_cols) + 4.0 * n_rows * heads
        flops += 2.0 * nnz * heads * (3 * d + 2 * dv)
    return {"bytes": total, "flops": flops}
