"""Dropout and log probabilities on the GPU against their definitions in 64 bits: types, odd sizes, leading dimensions, rows without classes, ties,
in place, captured and replayed."""
import numpy as np
import pytest
import torch

import operators_ref as ref
from operators_ref import HALF, TINY, TYPES, U, within
from paper_2306_15155_amd import Context, SenseiError, binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def normal(seed, dtype, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TYPES[dtype])


def strided(t, extra, lead=0):
    """the same values with a longer leading dimension, from an element further on"""
    buf = torch.full((t.shape[0], t.shape[1] + extra + lead), float("nan"), dtype=t.dtype, device=DEV)
    v = buf[:, lead: lead + t.shape[1]]
    v.copy_(t.to(DEV))
    return v, buf


# ------------------------------------------------------------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,extra,lead", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 8, 3, 1), (64, 100, 0, 0), (33, 129, 5, 3), (1000, 41, 0, 0), (2, 5000, 1, 1)])
def test_dropout(ctx, dtype, rows, cols, extra, lead):
    x, add = normal(1, dtype, rows, cols), normal(2, dtype, rows, cols)
    X, _ = strided(x, extra, lead)
    R, _ = strided(add, extra + 2, 0)
    for p, a, A in ((0.5, None, None), (0.1, add, R), (0.0, add, R)):
        want, err = ref.dropout(x, p, 0x1234567890ABCDEF, 17, a)
        Y, buf = strided(torch.zeros(rows, cols, dtype=TYPES[dtype]), extra, lead)
        got = ctx.dropout(X, p, 0x1234567890ABCDEF, 17, add=A, out=Y)
        within(got, want, err + HALF[dtype] * np.abs(want) * 1.01 + TINY[dtype], "dropout")
        untouched = torch.ones_like(buf, dtype=torch.bool)
        untouched[:, lead: lead + cols] = False
        assert torch.isnan(buf[untouched]).all()


def test_dropout_masks(ctx):
    x = torch.ones(300, 90, device=DEV)
    a = ctx.dropout(x, 0.4, 5, 1)
    assert torch.equal(a, ctx.dropout(x, 0.4, 5, 1)) and not torch.equal(a, ctx.dropout(x, 0.4, 5, 2)) and not torch.equal(a, ctx.dropout(x, 0.4, 6, 1))
    step = torch.ones(1, dtype=torch.int32, device=DEV)
    assert torch.equal(a, ctx.dropout(x, 0.4, 5, 0, offset_dev=step)) and torch.equal(a, ctx.dropout(x, 0.4, 5, 2, offset_dev=-step))
    # dropped elements are 0 whatever was there, kept ones pass; in place; the mask is the same for every type
    x[:] = float("inf")
    assert torch.equal(ctx.dropout(x, 0.4, 5, 1, out=x), torch.where(a > 0, float("inf"), 0.0))
    h = ctx.dropout(torch.ones(300, 90, device=DEV, dtype=torch.bfloat16), 0.4, 5, 1)
    assert torch.equal(h > 0, a > 0)
    r = torch.ones(300, 90, device=DEV)
    assert torch.equal(ctx.dropout(torch.ones_like(r), 0.4, 5, 1, add=r, out=r), a + 1)


def test_dropout_many_units(ctx):
    """sizes past the switch to several units a lane, one unit short of whole workgroups; a mask over rows that no launch grid would count alone"""
    for rows, cols, dtype in ((70_001, 131, "bf16"), (16_411, 513, "f32")):
        x = torch.ones(rows, cols, dtype=TYPES[dtype], device=DEV)
        got = (ctx.dropout(x, 0.25, 3, 9) != 0).cpu().numpy()
        assert np.array_equal(got, ref.keep_elements(rows, cols, 0.25, 3, 9))


# -------------------------------------------------------------------------------------------------------------- log probabilities

def check_logprobs(ctx, z, Z, labels, top, dtype, grad=True):
    n, c = z.shape
    lab = None if labels is None else torch.from_numpy(labels.astype(np.int32)).to(DEV)
    r = ref.logprobs(z, labels if labels is not None else np.full(n, -1), top)
    got = ctx.logprobs(Z, lab, top=top)
    el = ref.logs_bound(r, c)
    within(got.stats, np.stack([r["m"], r["logs"]], 1), np.stack([0 * el, el], 1), "stats")
    fin = np.where(np.isfinite(r["logp"]), np.abs(r["logp"]), 0)
    if labels is not None:
        within(got.logp, r["logp"], el + 2 * U * (fin + np.abs(np.where(np.isfinite(r["logs"]), r["logs"], 0))), "logp")
    spread = np.where(np.isfinite(r["d"]), np.abs(r["d"]) * r["p"], 0.0).sum(1)
    ee = el + 4 * U * (ref.sum_depth(c) + 8) * (spread + 1) + 4 * U * np.abs(r["entropy"])
    within(got.entropy, r["entropy"], ee, "entropy")
    if top:
        assert np.array_equal(got.top_idx.cpu().numpy(), r["top_idx"])
        tl = np.take_along_axis(r["lp"], r["top_idx"], 1)
        within(got.top_logp, tl, el[:, None] + 2 * U * (np.abs(np.where(np.isfinite(tl), tl, 0)) + 8), "top_logp")
    if not grad:
        return
    rng = np.random.default_rng(3)
    g, h = rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)
    lab = torch.full((n,), -1, dtype=torch.int32, device=DEV) if lab is None else lab
    dZ = ctx.logprobs_backward(Z, lab, got.stats, g_logp=torch.from_numpy(g).to(DEV), entropy=got.entropy, g_entropy=torch.from_numpy(h).to(DEV))
    want = ref.logprobs_grad(r, labels if labels is not None else np.full(n, -1), g.astype(np.float64), h.astype(np.float64))
    alp = np.where(r["p"] > 0, np.abs(np.where(np.isfinite(r["lp"]), r["lp"], 0)), 0)
    ep = r["p"] * (el[:, None] + 4 * U * (alp + np.abs(np.where(np.isfinite(r["logs"]), r["logs"], 0))[:, None] + 2)) + 2.0 ** -126
    err = ep * (np.abs(g)[:, None] + np.abs(h)[:, None] * (alp + np.abs(r["entropy"])[:, None] + 1)) + r["p"] * np.abs(h)[:, None] * (ee + el)[:, None]
    within(dZ, want, err + 4 * U * (np.abs(want) + np.abs(g)[:, None] * (r["p"] + np.abs(want > 0))) + HALF[dtype] * np.abs(want) * 1.01 + TINY[dtype], "dZ")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,classes,top", [(1, 1, 1), (5, 2, 2), (7, 3, 0), (300, 41, 5), (33, 47, 47), (1000, 8, 1), (64, 64, 64), (3, 65, 7), (17, 300, 10),
                                              (9, 2047, 20), (4, 4099, 64), (600, 5001, 3), (70, 127, 12), (70, 129, 12), (41, 511, 9), (41, 513, 9), (11, 1025, 33)])
def test_logprobs(ctx, dtype, rows, classes, top):
    z = normal(rows + classes, dtype, rows, classes, std=2.0)
    rng = np.random.default_rng(classes)
    labels = rng.integers(-1, classes + 1, rows)                # one below and one above the classes: no label
    Z, _ = strided(z, (rows * 7) % 5, rows % 3)
    check_logprobs(ctx, z, Z, labels, top, dtype)


@pytest.mark.parametrize("dtype,rows,classes,top", [("f32", 1, 20_000, 8), ("bf16", 2, 70_003, 64), ("f16", 3, 300_007, 5), ("f32", 100, 33_000, 1), ("f32", 1, 1_000_001, 0),
                                                    ("bf16", 513, 16_400, 4)])
def test_logprobs_of_long_rows(ctx, dtype, rows, classes, top):
    z = normal(classes, dtype, rows, classes, std=2.0)
    Z, _ = strided(z, 1, 1)
    check_logprobs(ctx, z, Z, np.arange(rows) * 7919 % classes, top, dtype, grad=rows * classes < 3_000_000)


@pytest.mark.parametrize("rows,classes", [(4, 50), (3, 700), (5, 9000), (2, 40_000)])
def test_logprobs_of_masked_rows(ctx, rows, classes):
    """classes at -inf, a row of nothing else, a row of the type's lowest value, one class left, logits far from zero, many equal ones"""
    z = normal(8, "f32", rows, classes, std=3.0)
    z[0, ::2] = -np.inf
    z[0, 1] = torch.finfo(torch.float32).min
    z[1] = -np.inf
    labels = np.full(rows, 1)
    check_logprobs(ctx, z, z.to(DEV), labels, 6, "f32")
    z[0] = torch.finfo(torch.float32).min
    z[1, classes - 1] = 3.0
    labels[0], labels[1] = 5, classes - 1
    check_logprobs(ctx, z, z.to(DEV), labels, 6, "f32")
    z[0] = 1.5                                            # ties: the lowest classes first
    z[0, 17] = -0.0
    z[0, 20:40] = 2.0
    z[1] = torch.arange(classes) * 0.0
    z[1, 3] = -0.0
    check_logprobs(ctx, z, z.to(DEV), labels, 30, "f32")
    z = z * 0.01 + 12_345.0
    check_logprobs(ctx, z, z.to(DEV), labels, 3, "f32")


def test_logprobs_where_one_lane_holds_all_the_highest(ctx):
    """the highest classes a stride apart, so that they fall to one lane and its list runs out again and again"""
    for classes, stride in ((9000, 1024), (600, 256), (60, 16), (40_000, 1024)):
        z = normal(4, "f32", 2, classes, std=0.1)
        z[:, ::stride] += torch.arange(z[:, ::stride].shape[1]).flip(0) + 10.0
        check_logprobs(ctx, z, z.to(DEV), np.array([0, 1]), min(24, classes), "f32", grad=False)
        z[:, :8] = z[:, :8].sort(descending=True)[0] + 100.0
        check_logprobs(ctx, z, z.to(DEV), np.array([0, 1]), 12, "f32", grad=False)


def test_logprobs_not_finite(ctx):
    for classes in (5, 400, 30_000):
        z = torch.zeros(3, classes)
        z[0, 2], z[1, 3] = float("nan"), float("inf")
        r = ctx.logprobs(z.to(DEV), torch.tensor([1, 3, 2], dtype=torch.int32, device=DEV), top=2)
        assert torch.isnan(r.logp[:2]).all() and torch.isnan(r.entropy[:2]).all() and torch.isnan(r.top_logp[:2]).all()
        assert r.top_idx.tolist() == [[2, 0], [3, 0], [0, 1]] and torch.isfinite(r.logp[2])


def test_logprobs_backward_in_place_and_parts(ctx):
    z = normal(2, "f32", 50, 333)
    lab = torch.arange(50, dtype=torch.int32, device=DEV)
    Z, g = z.to(DEV), torch.randn(50, device=DEV)
    r = ctx.logprobs(Z, lab)
    only_g = ctx.logprobs_backward(Z, lab, r.stats, g_logp=g)
    only_h = ctx.logprobs_backward(Z, lab, r.stats, entropy=r.entropy, g_entropy=g)
    both = ctx.logprobs_backward(Z, lab, r.stats, g_logp=g, entropy=r.entropy, g_entropy=g)
    # each term rounds by itself: three roundings of values of at most |g| (2 + log 333)
    assert torch.all((both - only_g - only_h).abs() <= 4 * U * g.abs()[:, None] * 8)
    assert torch.all(ctx.logprobs_backward(Z, lab, r.stats) == 0)
    same = ctx.logprobs_backward(Z, lab, r.stats, g_logp=g, out=Z)
    assert same.data_ptr() == Z.data_ptr() and torch.equal(same, only_g)


def test_wrong_arguments_raise(ctx):
    Z = torch.zeros(4, 5, device=DEV)
    lab = torch.zeros(4, dtype=torch.int32, device=DEV)
    with pytest.raises(SenseiError):
        ctx.logprobs(Z, lab, top=6)
    for bad in (lambda: ctx.logprobs(Z, lab[:3]), lambda: ctx.logprobs(Z, lab.long()), lambda: ctx.logprobs(Z.double(), lab), lambda: ctx.logprobs(Z.t(), lab),
                lambda: ctx.logprobs(Z.cpu(), lab), lambda: ctx.dropout(Z.t(), 0.5, 1), lambda: ctx.dropout(Z.cpu(), 0.5, 1)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(SenseiError):
        ctx.dropout(Z, 1.0, 1)
    with pytest.raises(SenseiError):
        ctx.dropout(Z, 0.5, 1, add=Z.bfloat16())
    assert ctx.dropout(Z[:0], 0.5, 1).shape == (0, 5) and ctx.logprobs(Z[:0], lab[:0], top=2).top_idx.shape == (0, 2)


def test_offsets_past_32_bits(ctx):
    ld = 600_000_000
    buf = torch.empty(3 * ld, dtype=torch.float16, device=DEV)
    Z = buf.view(3, ld)[:, 11: 11 + 5000]
    z = normal(9, "f16", 3, 5000)
    Z.copy_(z)
    check_logprobs(ctx, z, Z, np.array([5, 4999, -1]), 4, "f16")
    want, err = ref.dropout(z, 0.3, 8, 2)
    within(ctx.dropout(Z, 0.3, 8, 2, out=Z), want, err + HALF["f16"] * np.abs(want) * 1.01 + TINY["f16"], "dropout")


def test_captured_and_replayed(ctx):
    """dropout and a long-row loss in one graph: every replay draws the mask that the device word says and matches the eager calls, which have workspaces
    of their own"""
    X, lab = normal(3, "f32", 2, 60_000).to(DEV), torch.tensor([5, 50_000], dtype=torch.int32, device=DEV)
    step, g = torch.zeros(1, dtype=torch.int32, device=DEV), torch.ones(2, device=DEV)

    def run(offset, dev=None):
        Y = ctx.dropout(X, 0.3, 42, offset, offset_dev=dev)
        r = ctx.logprobs(Y, lab, top=4)
        return (Y, r.stats, r.logp, r.entropy, r.top_idx, ctx.logprobs_backward(Y, lab, r.stats, g_logp=g))

    run(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = run(10, step)
    torch.cuda.synchronize()
    for k in range(4):
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, run(10 + k)):
            assert torch.equal(a, b)


def test_another_stream(ctx):
    X = normal(3, "bf16", 500, 77).to(DEV)
    want = ctx.dropout(X, 0.2, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = ctx.dropout(X, 0.2, 1)
    s.synchronize()
    assert torch.equal(got, want)
    assert binding.lib().sensei_status_string(0) == b"ok"
