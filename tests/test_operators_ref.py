"""The 64-bit definitions that the GPU tests of dropout, attention and log probabilities compare with: gradients against differences, the generator
against itself in plain integers, the mask's independence of order.  And the refusals of the entry points, which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import operators_ref as ref
from paper_2306_15155_amd import binding


def test_generator_in_plain_integers():
    def words(c, seed):
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(7):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        return c
    rng = np.random.default_rng(1)
    c = rng.integers(0, 2 ** 32, (4, 50), dtype=np.uint64)
    got = ref.philox(*c, 0xFEDCBA9876543210)
    assert [[int(x) for x in got[:, i]] for i in range(50)] == [words([int(x) for x in c[:, i]], 0xFEDCBA9876543210) for i in range(50)]
    # words are spread evenly: the share below p 2^32 of 160,000 of them stays within five standard deviations
    kept = ref.keep_elements(400, 400, 0.3, 7, 11).mean()
    assert abs(kept - 0.7) < 5 * np.sqrt(0.21 / 160_000)


def _differences(f, x, n, rng, step=1e-6):
    at = [tuple(rng.integers(0, s) for s in x.shape) for _ in range(n)]
    out = []
    for i in at:
        old = x[i]
        x[i] = old + step
        hi = f()
        x[i] = old - step
        lo = f()
        x[i] = old
        out.append((hi - lo) / (2 * step))
    return at, np.array(out)


@pytest.mark.parametrize("cap,buckets,p,heads,kv", [(0.0, 0, 0.0, 2, 2), (2.5, 5, 0.3, 4, 2), (3.0, 4, 0.0, 3, 1), (0.0, 3, 0.5, 2, 1)])
def test_attention_gradients_against_differences(cap, buckets, p, heads, kv):
    rng = np.random.default_rng(5)
    n, m, d, dv = 9, 12, 5, 4
    P = ref.Pattern(n, m, [rng.choice(m, rng.integers(0, m), replace=False) for _ in range(n)])
    Q, K, V, dY = (rng.normal(size=s) for s in ((n, heads * d), (m, kv * d), (m, kv * dv), (n, heads * dv)))
    bucket = rng.integers(0, buckets, P.nnz) if buckets else None
    bias = rng.normal(size=(heads, buckets)) if buckets else None
    if buckets:
        bias[0, 0] = -np.inf
    args = dict(cap=cap, bucket=bucket, bias=bias, p=p, seed=99, offset=4)
    g = ref.attention(P, Q, K, V, heads, kv, 0.6, dY=dY, **args)
    loss = lambda: float((ref.attention(P, Q, K, V, heads, kv, 0.6, **args)["Y"] * dY).sum())  # noqa: E731
    # central differences of a smooth function: step^2 of its third derivative and 1e-16 / step of rounding, both below 1e-8 of these values
    for x, name in ((Q, "dQ"), (K, "dK"), (V, "dV")) + (((bias, "dbias"),) if buckets else ()):
        at, num = _differences(loss, x, 25, rng)
        ana = np.array([g[name][i] for i in at])
        fin = np.array([np.isfinite(x[i]) for i in at])
        assert np.allclose(ana[fin], num[fin], rtol=1e-6, atol=2e-8), name
        assert np.all(ana[~fin] == 0.0)


def test_logprobs_gradients_against_differences():
    rng = np.random.default_rng(6)
    z = rng.normal(size=(6, 9))
    z[2, 3] = -np.inf
    labels, g, h = np.array([1, -1, 4, 8, 9, 0]), rng.normal(size=6), rng.normal(size=6)

    def loss():
        r = ref.logprobs(torch.from_numpy(z), labels)
        return float((r["logp"] * g).sum() + (r["entropy"] * h).sum())

    ana = ref.logprobs_grad(ref.logprobs(torch.from_numpy(z), labels), labels, g, h)
    at, num = _differences(loss, z, 54, rng)
    fin = np.array([np.isfinite(z[i]) for i in at])
    assert np.allclose(np.array([ana[i] for i in at])[fin], num[fin], rtol=1e-6, atol=2e-8)
    assert ana[2, 3] == 0.0


def test_weights_mask_does_not_depend_on_the_order_of_the_entries():
    row, col = np.array([3, 0, 7]), np.array([5, 5, 1])
    for h in (0, 5):
        a, b = ref.keep_entries(row, col, h, 0.5, 3, 1), ref.keep_entries(row[::-1], col[::-1], h, 0.5, 3, 1)
        assert np.array_equal(a, b[::-1])


# ---- refusals: the checks stand before anything is launched, the context is not looked into

CTX = ctypes.create_string_buffer(4096)
A = binding.CsrStruct(100, 120, 1000, 0x1000, 0x2000, None)
AT = binding.CsrStruct(120, 100, 1000, 0x3000, 0x4000, None)


def mat(ptr, rows, cols, ld=None, type=0):
    return binding.TMatStruct(ptr, rows, cols, cols if ld is None else ld, type)


def opts(**kw):
    o = dict(n_heads=4, n_kv_heads=2, scale=0.25, cap=0.0, bucket=None, bias=None, n_buckets=0, p=0.0, seed=1, offset=0, offset_dev=None)
    o.update(kw)
    return binding.AttentionOpts(*o.values())


def test_dropout_refuses():
    L = binding.lib()
    call = lambda X, add=None, p=0.5, Y=0x900000, ldy=64, ctx=CTX: L.sensei_dropout(ctx, X, None if add is None else ctypes.byref(add), p, 1, 0, None, Y, ldy, None)  # noqa: E731
    X = mat(0x100000, 100, 64)
    assert call(X, ctx=None) == 1
    assert call(X, p=1.0) == 1 and call(X, p=-0.1) == 1 and call(X, p=float("nan")) == 1
    assert call(X, ldy=63) == 1 and call(X, Y=None) == 1
    assert call(mat(0x100000, 100, 64, type=3)) == 1 and call(mat(0x100000, 100, 64, ld=60)) == 1 and call(mat(None, 100, 64)) == 1
    assert call(mat(0x100002, 100, 64)) == 1 and call(X, Y=0x900002) == 1          # not an element's address
    assert call(X, Y=0x100000, ldy=70) == 1                                          # in place with another leading dimension
    assert call(X, Y=0x100100) == 1                                                  # overlapping
    assert call(X, add=mat(0x200000, 100, 65)) == 1 and call(X, add=mat(0x200000, 100, 64, type=1)) == 1 and call(X, add=mat(0x900100, 100, 64)) == 1
    assert call(mat(0x100000, 2 ** 32, 64)) == 1
    assert call(mat(0x100000, 0, 64)) == 0 and call(mat(None, 5, 0), ldy=0) == 0


def test_logprobs_refuses():
    L = binding.lib()
    n = ctypes.c_size_t()
    assert L.sensei_logprobs_workspace(10, 0, 0, 0, ctypes.byref(n)) == 1 and L.sensei_logprobs_workspace(10, 5, 6, 0, ctypes.byref(n)) == 1
    assert L.sensei_logprobs_workspace(10, 100, 65, 0, ctypes.byref(n)) == 1 and L.sensei_logprobs_workspace(10, 100, 5, 3, ctypes.byref(n)) == 1
    assert L.sensei_logprobs_workspace(1000, 47, 5, 0, ctypes.byref(n)) == 0 and n.value == 0
    assert L.sensei_logprobs_workspace(2, 250_000, 5, 0, ctypes.byref(n)) == 0 and n.value > 0
    ok = dict(Z=mat(0x100000, 10, 50), labels=0x10000, top=3, stats=0x20000, logp=0x30000, ent=0x40000, idx=0x50000, tlp=0x60000, ws=None, n=0, ctx=CTX)

    def call(**kw):
        a = dict(ok, **kw)
        return L.sensei_logprobs(a["ctx"], a["Z"], a["labels"], a["top"], a["stats"], a["logp"], a["ent"], a["idx"], a["tlp"], a["ws"], a["n"], None)

    assert call(ctx=None) == 1 and call(labels=None) == 1 and call(top=51) == 1 and call(top=-1) == 1 and call(idx=None) == 1 and call(tlp=None) == 1
    assert call(stats=0x20004) == 1 and call(logp=0x100004) == 1 and call(ent=0x30000) == 1 and call(Z=mat(0x100000, 10, 0)) == 1
    assert call(Z=mat(0x10000000, 2, 250_000), top=0) == 1                           # no workspace where one is needed
    assert call(Z=mat(0x10000000, 2, 250_000), top=0, ws=0x90000000, n=8) == 3
    assert call(Z=mat(0x100000, 0, 50)) == 0
    B = dict(Z=mat(0x100000, 10, 50), labels=0x10000, stats=0x20000, g=0x30000, ent=0x40000, h=0x50000, dZ=0x200000, ld=50, ctx=CTX)

    def back(**kw):
        a = dict(B, **kw)
        return L.sensei_logprobs_backward(a["ctx"], a["Z"], a["labels"], a["stats"], a["g"], a["ent"], a["h"], a["dZ"], a["ld"], None)

    assert back(ctx=None) == 1 and back(labels=None) == 1 and back(stats=None) == 1 and back(ent=None) == 1 and back(dZ=None) == 1 and back(ld=49) == 1
    assert back(dZ=0x100000, ld=51) == 1 and back(dZ=0x100010) == 1 and back(dZ=0x30000 - 100) == 1
    assert back(Z=mat(0x100000, 0, 50)) == 0


def test_attention_refuses():
    L = binding.lib()
    n = ctypes.c_size_t()
    q = lambda o, d=16, dv=16, type=0, a=A: L.sensei_attention_workspace(ctypes.byref(a), ctypes.byref(o), d, dv, type, ctypes.byref(n))  # noqa: E731
    assert q(opts()) == 0 and n.value > 0
    for bad in (dict(n_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(n_heads=514), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=1e-45), dict(scale=float("nan")),
                dict(n_buckets=129), dict(n_buckets=-1), dict(n_heads=32, n_buckets=33), dict(p=1.0), dict(p=-1e-9), dict(p=float("nan"))):
        assert q(opts(**bad)) == 1, bad
    assert q(opts(), d=0) == 1 and q(opts(), d=257) == 1 and q(opts(), dv=0) == 1 and q(opts(), type=3) == 1 and q(opts(), a=binding.CsrStruct(-1, 5, 0, 0x1000)) == 1
    base = dict(A=A, Q=mat(0x1000000, 100, 64), K=mat(0x2000000, 120, 32), V=mat(0x3000000, 120, 48), o=opts(), Y=0x4000000, ldy=96, stats=0x5000000, ws=0x60000000,
                n=1 << 30, ctx=CTX)

    def call(**kw):
        a = dict(base, **kw)
        return L.sensei_attention(a["ctx"], ctypes.byref(a["A"]), a["Q"], a["K"], a["V"], ctypes.byref(a["o"]), a["Y"], a["ldy"], a["stats"], a["ws"], a["n"], None)

    assert call(ctx=None) == 1 and call(Y=None) == 1 and call(stats=None) == 1 and call(ws=None) == 1 and call(ws=0x60000080) == 1 and call(n=256) == 3
    assert call(ldy=95) == 1 and call(stats=0x5000004) == 1 and call(Y=0x1000100) == 1 and call(Y=0x60000100) == 1 and call(stats=0x4000100) == 1
    assert call(Q=mat(0x1000000, 99, 64)) == 1 and call(K=mat(0x2000000, 100, 32)) == 1 and call(V=mat(0x3000000, 100, 48)) == 1
    assert call(Q=mat(0x1000000, 100, 66)) == 1 and call(K=mat(0x2000000, 120, 30)) == 1 and call(V=mat(0x3000000, 120, 47)) == 1
    assert call(K=mat(0x2000000, 120, 32, type=1)) == 1 and call(Q=mat(0x1000000, 100, 64, ld=63)) == 1
    assert call(o=opts(n_buckets=4)) == 1 and call(o=opts(n_buckets=4, bias=0x7000)) == 1 and call(o=opts(n_heads=0)) == 1
    assert call(A=binding.CsrStruct(0, 120, 0, 0x1000, None), Q=mat(None, 0, 64)) == 0
    back = dict(base, At=AT, t_pos=0x8000, Y=mat(0x4000000, 100, 96), dY=mat(0x7000000, 100, 96), dQ=0x10000000, dK=0x11000000, dV=0x12000000, ld=(64, 32, 48), dbias=None)

    def grad(**kw):
        a = dict(back, **kw)
        return L.sensei_attention_backward(a["ctx"], ctypes.byref(a["A"]), ctypes.byref(a["At"]), a["t_pos"], a["Q"], a["K"], a["V"], ctypes.byref(a["o"]), a["Y"], a["stats"],
                                           a["dY"], a["dQ"], a["ld"][0], a["dK"], a["ld"][1], a["dV"], a["ld"][2], a["dbias"], a["ws"], a["n"], None)

    assert grad(n=256) == 3
    assert grad(ctx=None) == 1 and grad(At=A) == 1 and grad(dQ=None) == 1 and grad(dK=None) == 1 and grad(dV=None) == 1 and grad(stats=None) == 1 and grad(ws=None) == 1
    assert grad(Y=mat(0x4000000, 100, 95)) == 1 and grad(dY=mat(0x7000000, 99, 96)) == 1 and grad(dY=mat(0x7000000, 100, 96, type=2)) == 1
    assert grad(ld=(63, 32, 48)) == 1 and grad(ld=(64, 31, 48)) == 1 and grad(ld=(64, 32, 47)) == 1
    assert grad(dK=0x10000100) == 1 and grad(dQ=0x7000000) == 1 and grad(dV=0x60000100) == 1 and grad(dQ=0x10000002) == 1
    assert grad(o=opts(n_buckets=4, bias=0x9000, bucket=0xA000), t_pos=None) == 1
    assert grad(o=opts(n_buckets=4, bias=0x9000, bucket=0xA000), dbias=0x9000) == 1
