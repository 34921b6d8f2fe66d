"""Dropout, attention over a pattern and log probabilities in 64 bits on the CPU, written from their definitions, with a bound on the rounding
error of the fp32 (and 16-bit) computation element by element."""
import numpy as np
import torch

U = 2.0 ** -24                                   # half a step of fp32, relative
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}     # what a store under the normal range may lose


# ---- the generator, in Python's integers turned into arrays of 64 bits

def philox(c0, c1, c2, c3, seed):
    c0, c1, c2, c3 = (np.asarray(c, dtype=np.uint64) for c in np.broadcast_arrays(c0, c1, c2, c3))
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    lo, hi = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(7):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)     # both factors below 2^32
        c0, c1, c2, c3 = (b >> hi) ^ c1 ^ np.uint64(k0), b & lo, (a >> hi) ^ c3 ^ np.uint64(k1), a & lo
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([c0, c1, c2, c3])


def keep_elements(rows, cols, p, seed, offset):
    q = np.arange((cols + 3) // 4)
    w = philox(q[None, :], np.arange(rows)[:, None], 0, offset, seed)                 # 4, rows, quads
    return np.moveaxis(w, 0, 2).reshape(rows, -1)[:, :cols] >= np.uint64(round(p * 2 ** 32))


def keep_entries(row, col, h, p, seed, offset):
    return philox(col, row, 2 ** 31 + h // 4, offset, seed)[h % 4] >= np.uint64(round(p * 2 ** 32))


def dropout(X, p, seed, offset=0, add=None):
    """float64 result and its bound in units that the caller's type adds its own rounding to"""
    x = X.double().numpy()
    y = np.where(keep_elements(*x.shape, p, seed, offset), x / (1.0 - p), 0.0)
    err = 3 * U * np.abs(y)                                # the factor's rounding and the product's
    if add is not None:
        y = y + add.double().numpy()
        err = err + U * np.abs(y)
    return y, err


# ---- log probabilities

def logprobs(Z, labels, top=0):
    z = Z.double().numpy()
    n, c = z.shape
    m = z.max(1)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(np.isneginf(z), -np.inf, z - np.where(np.isneginf(m), 0.0, m)[:, None])
        e = np.exp(d)
        s = e.sum(1)
        logs = np.log(s)
        lp = d - logs[:, None]
        p = np.where(s[:, None] > 0, e / np.where(s > 0, s, 1.0)[:, None], 0.0)
        ent = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
    lp = np.where(s[:, None] > 0, lp, -np.inf)
    has = (labels >= 0) & (labels < c)
    logp = np.where(has, lp[np.arange(n), np.where(has, labels, 0)], 0.0)
    order = np.lexsort((np.broadcast_to(np.arange(c), z.shape), -z), axis=1)[:, :top] if top else None
    return {"m": m, "logs": logs, "lp": lp, "p": p, "entropy": ent, "logp": logp, "top_idx": order, "d": d}


def sum_depth(classes):
    """Additions behind one another in a row's sum: the classes of a lane (at least four lanes a row), then joins of lanes and workgroups."""
    return min(classes, 40 + classes // 256 * 2 if classes > 2048 else 40 + classes // 4) + 16


def logs_bound(r, classes):
    """of log s: every addition and every raise of the maximum rounds, exp carries its argument's rounding"""
    spread = np.where(np.isfinite(r["d"]), np.abs(r["d"]) * r["p"], 0.0).sum(1)
    return 4 * U * sum_depth(classes) + 2 * U * np.abs(np.where(np.isfinite(r["logs"]), r["logs"], 0)) + 4 * U * (spread + 1)


def logprobs_grad(r, labels, g_logp=None, g_entropy=None):
    p, n = r["p"], r["p"].shape[0]
    dz = np.zeros_like(p)
    if g_logp is not None:
        has = (labels >= 0) & (labels < p.shape[1])
        g = np.where(has, g_logp, 0.0)
        dz -= p * g[:, None]
        dz[np.arange(n), np.where(has, labels, 0)] += g
    if g_entropy is not None:
        dz -= np.where(p > 0, p * (np.where(p > 0, r["lp"], 0.0) + r["entropy"][:, None]), 0.0) * g_entropy[:, None]
    return dz


# ---- attention over a pattern

class Pattern:
    def __init__(self, n_rows, n_cols, lists):
        """lists: the columns of every row"""
        self.n_rows, self.n_cols = n_rows, n_cols
        lists = [np.unique(np.asarray(x, dtype=np.int64)) for x in lists]
        self.row = np.repeat(np.arange(n_rows), [len(x) for x in lists])
        self.col = np.concatenate(lists) if lists and sum(map(len, lists)) else np.zeros(0, dtype=np.int64)
        self.nnz = self.col.size
        self.row_ptr = np.concatenate([[0], np.cumsum(np.bincount(self.row, minlength=n_rows))])
        order = np.lexsort((self.row, self.col))
        self.t_ptr = np.concatenate([[0], np.cumsum(np.bincount(self.col, minlength=n_cols))])
        self.t_col = self.row[order]
        self.t_pos = np.empty(self.nnz, dtype=np.int64)
        self.t_pos[order] = np.arange(self.nnz)


def _add_at(n, index, x):
    out = np.zeros((n,) + x.shape[1:])
    np.add.at(out, index, x)
    return out


def attention(P, Q, K, V, heads, kv, scale, cap=0.0, bucket=None, bias=None, p=0.0, seed=0, offset=0, dY=None, half=U, tiny=0.0):
    """float64 numpy operands.  A dict of the outputs, and under "err" the bound of each: U a rounding of fp32, `half` the last one to the type."""
    d, dv, ratio = Q.shape[1] // heads, V.shape[1] // kv, heads // kv
    row, col, n, m_cols = P.row, P.col, P.n_rows, P.n_cols
    Y, stats, dQ, dK, dV = np.zeros((n, heads * dv)), np.zeros((n, heads, 2)), np.zeros(Q.shape), np.zeros(K.shape), np.zeros(V.shape)
    eY, es, eQ, eK, eV = np.zeros(Y.shape), np.zeros(stats.shape), np.zeros(Q.shape), np.zeros(K.shape), np.zeros(V.shape)
    dbias, eb = (np.zeros(bias.shape), np.zeros(bias.shape)) if bias is not None else (None, None)
    deg, tdeg = np.bincount(row, minlength=n), np.bincount(col, minlength=m_cols)
    for h in range(heads):
        g = h // ratio
        hs, gs, hv, gv = slice(h * d, h * d + d), slice(g * d, g * d + d), slice(h * dv, h * dv + dv), slice(g * dv, g * dv + dv)
        q, k, v = Q[row, hs], K[col, gs], V[col, gv]
        b = bias[h][np.minimum(bucket, bias.shape[1] - 1)] if bias is not None else np.zeros(P.nnz)
        use = ~np.isneginf(b)
        q, k, v, b = q * use[:, None], np.where(use[:, None], k, 0.0), np.where(use[:, None], v, 0.0), np.where(use, b, 0.0)
        x = (q * k).sum(1) * scale
        ex = (d + 3) * U * (np.abs(q) * np.abs(k)).sum(1) * abs(scale)
        slope, eslope = np.ones(P.nnz), np.zeros(P.nnz)
        if cap > 0:
            th = np.tanh(x / cap)
            slope = 1 - th * th
            x = cap * th
            eslope = 2 * np.abs(th) * slope * ex / cap + 8 * U
            ex = ex * slope + 8 * U * np.abs(x)           # a tanh of relative accuracy, times the cap
        x = x + b
        ex = ex + 2 * U * np.abs(x)
        top = np.full(n, -np.inf)
        np.maximum.at(top, row, np.where(use, x, -np.inf))
        base = np.where(np.isneginf(top), 0.0, top)
        e = np.where(use, np.exp(x - base[row]), 0.0)
        l = _add_at(n, row, e)
        with np.errstate(divide="ignore"):
            stats[:, h, 0], stats[:, h, 1] = top, np.log(l)
        lsafe = np.where(l > 0, l, 1.0)
        alpha = e / lsafe[row]
        exm = np.zeros(n)
        np.maximum.at(exm, row, ex)
        far = _add_at(n, row, alpha * np.abs(x - base[row]))
        el = 2 * exm + 4 * U * (deg + 16) + 2 * U * np.abs(np.log(lsafe)) + 4 * U * far       # of log l
        es[:, h, 0], es[:, h, 1] = exm + U * np.abs(base), el
        ep = alpha * (ex + exm[row] + el[row] + 4 * U * (np.abs(x - base[row]) + 2))
        keep = keep_entries(row, col, h, p, seed, offset) / (1.0 - p) if p > 0 else np.ones(P.nnz)
        w, ew = alpha * keep, ep * keep + 4 * U * alpha * keep
        Y[:, hv] = _add_at(n, row, w[:, None] * v)
        ay = _add_at(n, row, w[:, None] * np.abs(v))
        eY[:, hv] = _add_at(n, row, ew[:, None] * np.abs(v)) + 2 * U * (deg[:, None] + 16) * ay + half * np.abs(Y[:, hv]) + tiny
        if dY is None:
            continue
        dy, y = dY[:, hv], Y[:, hv]
        dyr = dy[row]
        dp, edp = (dyr * v).sum(1) * keep, (dv + 4) * U * (np.abs(dyr) * np.abs(v)).sum(1) * keep
        D, eD = (dy * y).sum(1), (dv + 4) * U * (np.abs(dy) * np.abs(y)).sum(1) + (np.abs(dy) * eY[:, hv]).sum(1)
        dt = alpha * (dp - D[row])
        edt = ep * (np.abs(dp - D[row]) + edp + eD[row]) + alpha * (edp + eD[row]) + 4 * U * alpha * (np.abs(dp) + np.abs(D[row]))
        ds, eds = dt * slope * scale, abs(scale) * (edt * slope + np.abs(dt) * eslope + edt * eslope) + 4 * U * np.abs(dt * slope * scale)
        ads = np.abs(ds) + eds
        dQ[:, hs] = _add_at(n, row, ds[:, None] * k)
        eQ[:, hs] = _add_at(n, row, eds[:, None] * np.abs(k)) + 2 * U * (deg[:, None] + 16) * _add_at(n, row, ads[:, None] * np.abs(k))
        dK[:, gs] += _add_at(m_cols, col, ds[:, None] * q)
        eK[:, gs] += _add_at(m_cols, col, eds[:, None] * np.abs(q)) + 2 * U * (ratio * tdeg[:, None] + 16) * _add_at(m_cols, col, ads[:, None] * np.abs(q))
        dV[:, gv] += _add_at(m_cols, col, w[:, None] * dyr)
        eV[:, gv] += _add_at(m_cols, col, ew[:, None] * np.abs(dyr)) + 2 * U * (ratio * tdeg[:, None] + 16) * _add_at(m_cols, col, w[:, None] * np.abs(dyr))
        if bias is not None:
            nb, bin_ = bias.shape[1], np.minimum(bucket, bias.shape[1] - 1)
            dbias[h] = np.bincount(bin_, weights=np.where(use, dt, 0.0), minlength=nb)
            count = np.bincount(bin_, minlength=nb)
            eb[h] = np.bincount(bin_, weights=edt, minlength=nb) + 2 * U * np.minimum(count + 16, 1024) * np.bincount(bin_, weights=np.abs(dt) + edt, minlength=nb)
    out = {"Y": Y, "stats": stats, "err": {"Y": eY, "stats": es}}
    if dY is not None:
        out.update(dQ=dQ, dK=dK, dV=dV, dbias=dbias)
        out["err"].update(dQ=eQ + half * np.abs(dQ) + tiny, dK=eK + half * np.abs(dK) + tiny, dV=eV + half * np.abs(dV) + tiny, dbias=eb)
    return out


def within(got, want, err, what):
    """|got - want| <= err everywhere, infinities and NaN in the same places"""
    got = got.detach().double().cpu().numpy() if isinstance(got, torch.Tensor) else np.asarray(got, dtype=np.float64)
    want, err = np.asarray(want, dtype=np.float64), np.broadcast_to(np.asarray(err, dtype=np.float64), np.shape(want))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), f"{what}: infinities or NaN differ"
    diff = np.abs(got[~odd] - want[~odd])
    assert np.all(np.isfinite(got[~odd])), f"{what}: not finite"
    bound = err[~odd] + 1e-300
    assert diff.size == 0 or np.all(diff <= bound), f"{what}: {np.max(diff / bound):.3g} times the bound, at {np.argmax(diff / bound)}"
