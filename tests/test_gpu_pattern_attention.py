"""Attention over a pattern and its gradients on the GPU against the definition in 64 bits: head layouts and widths, types, rows from no entry to
thousands, masks, strides, dropped weights, capture."""
import math

import numpy as np
import pytest
import torch

import operators_ref as ref
from operators_ref import HALF, TINY, TYPES, U, within
from paper_2306_15155_amd import Context, SenseiError, csr_struct

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def pattern(kind, seed):
    rng = np.random.default_rng(seed)
    if kind == "random":          # rows of 0 to 12 entries
        return ref.Pattern(90, 130, [rng.choice(130, rng.integers(0, 13), replace=False) for _ in range(90)])
    if kind == "hub":             # one row and one column of nearly everything, the rest short
        n = 700
        return ref.Pattern(n, n, [np.arange(n - 3) if i == 350 else np.append(rng.choice(n, 2, replace=False), 11) for i in range(n)])
    if kind == "sparse":          # runs of empty rows and columns, entries at both ends
        return ref.Pattern(3000, 2500, [[0] if i == 0 else [7, 2499] if i in (1, 900, 901, 2999) else [] for i in range(3000)])
    if kind == "lead":            # empty rows first and last
        return ref.Pattern(600, 40, [rng.choice(40, 9, replace=False) if 200 <= i < 300 else [] for i in range(600)])
    if kind == "one":
        return ref.Pattern(1, 1, [[0]])
    if kind == "row":             # a single row of many entries
        return ref.Pattern(1, 5000, [np.arange(5000)])
    if kind == "column":          # many rows of one entry, the same
        return ref.Pattern(3000, 2, [[1]] * 3000)
    if kind == "empty":
        return ref.Pattern(50, 60, [[]] * 50)
    if kind == "docs":            # batched graphs
        size = rng.integers(1, 30, 20)
        first = np.cumsum(size) - size
        return ref.Pattern(int(size.sum()), int(size.sum()), [np.arange(f, f + s) for f, s in zip(first, size) for _ in range(s)])
    raise ValueError(kind)


def wide(x, dtype, extra, lead=0):
    buf = torch.full((x.shape[0], x.shape[1] + extra + lead), float("nan"), dtype=TYPES[dtype], device=DEV)
    v = buf[:, lead: lead + x.shape[1]]
    v.copy_(x)
    return v


class Inputs:
    def __init__(self, P, heads, kv, d, dv, dtype="f32", buckets=0, seed=0, extra=(0, 0, 0, 0)):
        g = torch.Generator().manual_seed(seed)
        make = lambda n, w: torch.randn(n, w, generator=g).to(TYPES[dtype])  # noqa: E731
        self.P, self.heads, self.kv, self.dtype = P, heads, kv, dtype
        self.host = [make(P.n_rows, heads * d), make(P.n_cols, kv * d), make(P.n_cols, kv * dv), make(P.n_rows, heads * dv)]
        self.dev = [wide(t, dtype, e, e % 3) for t, e in zip(self.host, extra)]
        up = lambda a: torch.from_numpy(a.astype(np.int32)).to(DEV)  # noqa: E731
        self.A = csr_struct(P.n_rows, P.n_cols, up(P.row_ptr), up(P.col))
        self.At = csr_struct(P.n_cols, P.n_rows, up(P.t_ptr), up(P.t_col))
        self.t_pos = up(P.t_pos) if P.nnz else torch.zeros(1, dtype=torch.int32, device=DEV)
        self.bucket = self.bias = None
        if buckets:
            self.bucket = torch.randint(0, buckets, (P.nnz,), generator=g).to(torch.uint8)
            self.bias = torch.randn(heads, buckets, generator=g)

    def check(self, ctx, grad=True, **kw):
        want = self.want(grad, **kw)
        got = self.got(ctx, grad, **kw)
        e = want["err"]
        within(got["Y"], want["Y"], e["Y"], "Y")
        within(got["stats"], want["stats"], e["stats"], "stats")
        if grad:
            for k in ("dQ", "dK", "dV") + (("dbias",) if self.bias is not None else ()):
                within(got[k], want[k], e[k], k)
        return got

    def want(self, grad=True, **kw):
        q, k, v, dy = (t.double().numpy() for t in self.host)
        kw = dict(kw)
        scale = kw.pop("scale", None) or (q.shape[1] // self.heads) ** -0.5
        return ref.attention(self.P, q, k, v, self.heads, self.kv, np.float32(scale).astype(np.float64), bucket=None if self.bucket is None else self.bucket.numpy(),
                             bias=None if self.bias is None else self.bias.double().numpy(), dY=dy if grad else None, half=HALF[self.dtype] * 1.01 + U,
                             tiny=TINY[self.dtype], **kw)

    def got(self, ctx, grad=True, **kw):
        Q, K, V, dY = self.dev
        kw = dict(kw, n_kv_heads=self.kv, buckets=None if self.bucket is None else self.bucket.to(DEV), bias=None if self.bias is None else self.bias.to(DEV))
        Y, stats = ctx.attention(self.A, Q, K, V, self.heads, **kw)
        out = {"Y": Y, "stats": stats}
        if grad:
            out["dQ"], out["dK"], out["dV"], out["dbias"] = ctx.attention_backward(self.A, self.At, self.t_pos if self.bucket is not None else None, Q, K, V, self.heads, Y,
                                                                                   stats, dY, **kw)
        return out


KINDS = ["random", "hub", "sparse", "lead", "one", "row", "column", "empty", "docs"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_patterns(ctx, kind, dtype):
    Inputs(pattern(kind, 1), 3, 3, 12, 12, dtype, seed=2).check(ctx)


@pytest.mark.parametrize("kind", ["random", "hub", "sparse", "row", "docs"])
def test_everything_at_once(ctx, kind):
    x = Inputs(pattern(kind, 3), 4, 2, 20, 9, "f32", buckets=7, seed=4, extra=(3, 1, 2, 5))
    x.bias[1, 2] = x.bias[3, 0] = -np.inf
    x.check(ctx, cap=1.5, p=0.3, seed=0xABCDEF0123456789, offset=3, scale=0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,dv", [(1, 1), (3, 5), (4, 4), (8, 8), (15, 16), (17, 2), (25, 25), (32, 32), (33, 64), (64, 64), (65, 7), (100, 128), (128, 128), (129, 130),
                                  (256, 256), (7, 255)])
def test_head_widths(ctx, d, dv, dtype):
    Inputs(pattern("random", d), 2, 2, d, dv, dtype, buckets=3, seed=d, extra=(1, 2, 0, 1)).check(ctx, p=0.2, cap=4.0)


@pytest.mark.parametrize("heads,kv,d", [(1, 1, 16), (2, 1, 64), (4, 1, 32), (8, 2, 16), (6, 3, 24), (5, 5, 8), (12, 4, 40), (16, 16, 4), (9, 1, 130), (17, 17, 33), (64, 8, 8)])
def test_head_layouts(ctx, heads, kv, d):
    Inputs(pattern("random", heads), heads, kv, d, d, "f32", buckets=2, seed=heads).check(ctx, p=0.5, seed=5)
    Inputs(pattern("hub", heads), heads, kv, d, d, "f16", seed=heads).check(ctx, cap=3.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,kv,d,dv,buckets", [(4, 2, 96, 96, 5), (8, 2, 128, 40, 0), (6, 1, 72, 200, 3), (16, 1, 8, 8, 32), (64, 8, 8, 16, 64), (32, 2, 20, 33, 32), (4, 4, 5, 9, 128)])
def test_shared_heads_and_bias_tables(ctx, heads, kv, d, dv, buckets, dtype):
    """two query heads a lane (wide heads that share a key head), tables of the bias' gradient that ask for more lanes a head or smaller workgroups, masked buckets"""
    x = Inputs(pattern("random", d), heads, kv, d, dv, dtype, buckets=buckets, seed=d, extra=(0, 8, 0, 3))
    if buckets:
        x.bias[1:, 1] = -np.inf
    x.check(ctx, cap=6.0, p=0.3, seed=11)


@pytest.mark.parametrize("n,ld", [(270, 4_200_000), (250, 4_000_000)])
def test_rows_far_apart(ctx, n, ld):
    """leading dimensions past 2^24 bytes and offsets past 2^32 in every matrix of the backward; the same just below both"""
    rng = np.random.default_rng(1)
    P = ref.Pattern(n, n, [np.append(rng.choice(n, 6, replace=False), n - 1) for _ in range(n)])
    x = Inputs(P, 2, 1, 16, 16, "f32", seed=3)
    for k in range(4):
        buf = torch.empty(n * ld, device=DEV)
        v = buf.view(n, ld)[:, 7: 7 + x.host[k].shape[1]]
        v.copy_(x.host[k])
        x.dev[k] = v
    x.check(ctx, p=0.2)
    x.dev = None


def test_many_columns(ctx):
    """column numbers past 2^24"""
    m = 2 ** 24 + 100
    rng = np.random.default_rng(2)
    P = ref.Pattern(30, m, [np.unique(np.concatenate([rng.integers(0, m, 20), [m - 1 - i]])) for i in range(30)])
    x = Inputs(P, 1, 1, 4, 4, "f32", seed=5)
    want, got = x.want(grad=False), x.got(ctx, grad=True)
    for k in ("Y", "stats"):
        within(got[k], want[k], want["err"][k], k)
    hit = torch.zeros(m, dtype=torch.bool, device=DEV)
    hit[torch.from_numpy(P.col).to(DEV)] = True
    assert torch.all(got["dK"][~hit] == 0) and torch.all(got["dV"][~hit] == 0) and torch.all(got["dV"][hit].abs().sum(1) > 0)


def test_calls_on_two_streams_at_once(ctx):
    x, y = Inputs(pattern("hub", 5), 4, 2, 16, 16, "f32", buckets=5, seed=6), Inputs(pattern("hub", 6), 4, 2, 16, 16, "f32", buckets=5, seed=7)
    want = [v.got(ctx, p=0.4, seed=1) for v in (x, y)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(5):
        for k, v in enumerate((x, y)):
            with torch.cuda.stream(streams[k]):
                got[k] = v.got(ctx, p=0.4, seed=1)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(want[k][n], got[k][n]) for n in want[k])


def test_masked_entries_have_no_share(ctx):
    """bias of -inf hides infinities and NaN in keys and values, also where it leaves a row nothing; the type's lowest value does not"""
    P = pattern("random", 9)
    x = Inputs(P, 2, 2, 16, 16, "f32", buckets=4, seed=1)
    x.bias[:, 1] = -np.inf
    bad = P.n_cols // 2
    x.bucket[torch.from_numpy(P.col == bad)] = 1
    x.bucket[torch.from_numpy(P.row == 5)] = 1
    x.host[1][bad], x.host[2][bad] = np.nan, np.inf
    for t, v in zip(x.dev, x.host):
        t.copy_(v)
    got = x.got(ctx, p=0.25)
    x.host[1][bad] = x.host[2][bad] = 0.0            # the definition leaves them out: any number will do
    want = x.want(p=0.25)
    for k in ("Y", "stats", "dQ", "dK", "dV", "dbias"):
        within(got[k], want[k], want["err"][k], k)
    assert torch.all(got["Y"][5] == 0) and torch.all(torch.isneginf(got["stats"][5])) and torch.all(got["dQ"][5] == 0) and torch.all(got["dK"][bad] == 0)
    low = Inputs(P, 2, 2, 16, 16, "f32", buckets=1, seed=1)
    low.bias[:] = torch.finfo(torch.float32).min
    got = low.got(ctx)                               # every score is that number: uniform weights
    deg = np.bincount(P.row, minlength=P.n_rows)
    v = low.host[2].double().numpy()
    mean = np.stack([v[P.col[P.row == i]].mean(0) if deg[i] else np.zeros(32) for i in range(P.n_rows)])
    within(got["Y"], mean, 2 * U * (deg[:, None] + 20) * 5.0, "uniform rows")
    assert torch.all(torch.isfinite(got["dK"]))


def test_buckets_past_the_table_count_as_its_last(ctx):
    x = Inputs(pattern("random", 2), 2, 1, 8, 8, "f32", buckets=3, seed=3)
    x.bucket[::5] = 200
    x.check(ctx)


def test_nan_stays_in_its_rows(ctx):
    P = pattern("random", 4)
    x = Inputs(P, 2, 2, 8, 8, seed=2)
    j = int(P.col[0])
    clean = x.got(ctx, grad=False)["Y"]
    x.dev[2][j, 3] = float("nan")
    Y = x.got(ctx, grad=False)["Y"]
    rows = torch.zeros(P.n_rows, dtype=torch.bool)
    rows[torch.from_numpy(P.row[P.col == j])] = True
    assert torch.equal(torch.isnan(Y[:, 3]).cpu(), rows) and torch.equal(Y[~rows.to(DEV)], clean[~rows.to(DEV)])
    assert not torch.isnan(Y[:, :3]).any() and not torch.isnan(Y[:, 4:]).any()


def test_results_repeat_and_masks_follow_offsets(ctx):
    x = Inputs(pattern("hub", 5), 4, 2, 16, 16, "f32", buckets=5, seed=6)
    a, b = x.got(ctx, p=0.4, seed=1, offset=9), x.got(ctx, p=0.4, seed=1, offset=9)
    assert all(torch.equal(a[k], b[k]) for k in a)
    step = torch.full((1,), 4, dtype=torch.int32, device=DEV)
    c = x.got(ctx, p=0.4, seed=1, offset=5, offset_dev=step)
    assert all(torch.equal(a[k], c[k]) for k in a)
    assert not torch.equal(a["Y"], x.got(ctx, p=0.4, seed=1, offset=8)["Y"])


def test_larger_patterns(ctx):
    """enough entries for every chunk length, rows longer than several chunks"""
    for n, deg, heads, kv, d in ((20_000, 30, 8, 4, 8), (3000, 700, 2, 2, 16), (200, 5000, 1, 1, 32)):
        rng = np.random.default_rng(n)
        m = max(n, 2 * deg)
        P = ref.Pattern(n, m, list(np.sort(rng.integers(0, m, (n, deg)), axis=1)))
        Inputs(P, heads, kv, d, d, "f32", seed=n).check(ctx, grad=n < 10_000)


def test_wrong_arguments_raise(ctx):
    x = Inputs(pattern("random", 1), 2, 2, 8, 8, buckets=3)
    Q, K, V, dY = x.dev
    b, t = x.bucket.to(DEV), x.bias.to(DEV)
    for bad in (lambda: ctx.attention(x.A, Q.double(), K, V, 2), lambda: ctx.attention(x.A, Q.cpu(), K, V, 2), lambda: ctx.attention(x.A, Q, K, V, 2, buckets=b),
                lambda: ctx.attention(x.A, Q, K, V, 2, buckets=b[:-1], bias=t), lambda: ctx.attention(x.A, Q, K, V, 2, buckets=b, bias=t[:1]),
                lambda: ctx.attention(x.A, Q, K, V, 2, buckets=b.int(), bias=t), lambda: ctx.attention(x.A, Q, K, V, 2, buckets=b, bias=t.half())):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: ctx.attention(x.A, Q, K, V, 3), lambda: ctx.attention(x.A, Q, K[:-1], V, 2), lambda: ctx.attention(x.A, Q, K.half(), V, 2),
                lambda: ctx.attention(x.A, Q, K, V, 2, p=1.0), lambda: ctx.attention(x.A, Q, K, V, 2, cap=-1.0), lambda: ctx.attention(x.A, Q, K, V, 2, n_kv_heads=4)):
        with pytest.raises(SenseiError):
            bad()
    Y, stats = ctx.attention(x.A, Q, K, V, 2, buckets=b, bias=t)
    with pytest.raises(SenseiError):
        ctx.attention_backward(x.A, x.At, None, Q, K, V, 2, Y, stats, dY, buckets=b, bias=t)
    assert ctx.attention_backward(x.A, x.At, x.t_pos, Q, K, V, 2, Y, stats, dY, buckets=b, bias=t, want_dbias=False)[3] is None


def test_training_step_of_all_of_them(ctx):
    """Dropout, projections, attention, a product, the loss and their backward passes as one training step, against automatic differentiation in 64
    bits; then the same step captured and replayed with new masks."""
    n, f, heads, d, classes = 400, 24, 4, 8, 11
    rng = np.random.default_rng(8)
    P = ref.Pattern(n, n, [np.append(rng.choice(n, 9, replace=False), i) for i in range(n)])
    x = Inputs(P, heads, 2, d, d, buckets=4, seed=1)
    g = torch.Generator().manual_seed(2)
    X, Wq, Wk, Wv, Wo = (torch.randn(s, generator=g) * w for s, w in (((n, f), 1.0), ((f, heads * d), 0.2), ((f, 2 * d), 0.2), ((f, 2 * d), 0.2), ((heads * d, classes), 0.2)))
    labels = torch.randint(0, classes, (n,), generator=g).to(torch.int32)
    bucket, bias = x.bucket.to(DEV), x.bias.to(DEV)
    Xd, Wqd, Wkd, Wvd, Wod, lab = (t.to(DEV) for t in (X, Wq, Wk, Wv, Wo, labels))
    WoT = Wod.t().contiguous()
    gl = torch.full((n,), -1.0 / n, device=DEV)

    def step(offset, dev=None):
        H = ctx.dropout(Xd, 0.25, 77, offset, offset_dev=dev)
        Q, K, V = ctx.gemm(H, Wqd), ctx.gemm(H, Wkd), ctx.gemm(H, Wvd)
        opt = dict(n_kv_heads=2, cap=5.0, buckets=bucket, bias=bias, p=0.2, seed=78, offset=offset, offset_dev=dev)
        Y, stats = ctx.attention(x.A, Q, K, V, heads, **opt)
        Z = ctx.gemm(Y, Wod)
        r = ctx.logprobs(Z, lab)
        dZ = ctx.logprobs_backward(Z, lab, r.stats, g_logp=gl)
        dY = ctx.gemm(dZ, WoT)
        dQ, dK, dV, dbias = ctx.attention_backward(x.A, x.At, x.t_pos, Q, K, V, heads, Y, stats, dY, **opt)
        return [r.logp, dZ, dQ, dK, dV, dbias, ctx.dropout(ctx.gemm(dQ, Wqd.t().contiguous()), 0.25, 77, offset, offset_dev=dev)]

    got = step(6)
    # the same step in 64 bits, differentiated by torch
    keep = torch.from_numpy(ref.keep_elements(n, f, 0.25, 77, 6))
    H = torch.where(keep, X.double() / 0.75, 0.0)
    Q, K, V = (H @ w.double() for w in (Wq, Wk, Wv))
    b = x.bias.double()
    for t in (Q, K, V, b):
        t.requires_grad_()
    row, col = torch.from_numpy(P.row), torch.from_numpy(P.col)
    ys = []
    for h in range(heads):
        k = h // 2
        s = 5.0 * torch.tanh((Q[row, h * d:h * d + d] * K[col, k * d:k * d + d]).sum(1) * d ** -0.5 / 5.0) + b[h][x.bucket.long()]
        e = torch.exp(s)
        a = e / torch.zeros(n, dtype=torch.float64).index_add(0, row, e)[row]
        w = a * torch.from_numpy(ref.keep_entries(P.row, P.col, h, 0.2, 78, 6)) / 0.8
        ys.append(torch.zeros(n, d, dtype=torch.float64).index_add(0, row, w[:, None] * V[col, k * d:k * d + d]))
    Z = torch.cat(ys, 1) @ Wo.double()
    Z.retain_grad()
    logp = torch.log_softmax(Z, 1)[torch.arange(n), labels.long()]
    (-logp.mean()).backward()
    want = [logp.detach(), Z.grad, Q.grad, K.grad, V.grad, b.grad, torch.where(keep, (Q.grad @ Wq.double().t()) / 0.75, 0.0)]
    # every stage adds at most a few hundred roundings of its largest value (sums of 24 to 32 products, of ten entries, the products' operands): 2^-24 * 512
    for u, v in zip(got, want):
        within(u, v.numpy(), 512 * U * float(v.abs().max()), "training step")

    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = step(20, word)
    torch.cuda.synchronize()
    for k in range(4):
        word.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, step(20 + k)):
            assert torch.equal(u, v)


@pytest.mark.parametrize("d", [16, 25])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_infinite_keys(ctx, dtype, d):
    """rows that do not attend to an infinite key keep theirs; where vectors are whole pieces a score of -inf has no share, one of +inf makes NaN"""
    P = pattern("random", 4)
    x = Inputs(P, 2, 2, d, d, dtype, seed=7)
    j = int(P.col[0])
    rows = torch.zeros(P.n_rows, dtype=torch.bool)
    rows[torch.from_numpy(P.row[P.col == j])] = True
    rows = rows.to(DEV)
    x.dev[0].abs_().add_(1)                       # products with a key of one sign have that sign
    x.dev[1][j] = -60000.0
    low = x.got(ctx, grad=False)["Y"]
    for key in (-math.inf, math.inf):
        x.dev[1][j] = key
        Y = x.got(ctx, grad=False)["Y"]
        assert torch.equal(Y[~rows], low[~rows])
        if key > 0:
            assert torch.isnan(Y[rows]).all()
        elif d == 16:
            several = rows & torch.from_numpy(np.diff(P.row_ptr) > 1).to(DEV)
            assert several.any() and torch.equal(Y[several], low[several])
