"""CPU oracle for the layers of a transformer over the rows of a sparse tensor: layer normalisation, attention with a
sliding window and first rows that stay visible, its single-token step over a ring cache, and distillation from a
teacher's top logits.

TEST INFRASTRUCTURE ONLY, like the rest of `oracle/`: plain numpy in float64, each function is the definition written
out, row by row where that is clearest.  Pinned against torch's autograd and against differences in
tests/test_token_oracle.py.  Beside a result stands, where rounding matters, a bound of its error: `u` is half a step of
the type that probabilities, their gradients and results are rounded to (relative to the value), `g` the relative error of
a 32-bit sum of products and an exponential.
"""
from __future__ import annotations

import numpy as np


# ---- layer normalisation ---------------------------------------------------------------------------------------
def layer_norm_fwd(x, gamma, beta, eps):
    """Returns (y, mean, rstd): every row by itself, biased variance."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64), mean, rstd


def layer_norm_bwd(x, dy, gamma, mean, rstd):
    """Returns (dx, dgamma, dbeta) from the forward pass's mean and rstd."""
    x, dy, mean, rstd = (np.asarray(t, np.float64) for t in (x, dy, mean, rstd))
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * np.asarray(gamma, np.float64)
    dx = rstd[:, None] * (g - g.mean(axis=1)[:, None] - xhat * (g * xhat).mean(axis=1)[:, None])
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)


# ---- windowed attention ----------------------------------------------------------------------------------------
def visible(a, b, left, right, sinks):
    """[a][b]: query i stands at position i + b - a and sees key j."""
    p = np.arange(a)[:, None] + (b - a)
    j = np.arange(b)[None, :]
    return (j <= p + right) & ((j >= p - left) | (j < sinks))


def _each(q_starts, k_starts, heads, kv_heads):
    for c in range(len(q_starts) - 1):
        for h in range(heads):
            yield slice(q_starts[c], q_starts[c + 1]), slice(k_starts[c], k_starts[c + 1]), h, h // (heads // kv_heads)


def _scores(q, k, seen, scale):
    with np.errstate(invalid="ignore", over="ignore"):
        return np.where(seen, (q @ k.T) * scale, -np.inf)


def _times(p, rows, seen):
    """p @ rows over the seen pairs only: what is not seen adds nothing, whatever it holds."""
    fine = np.isfinite(rows)
    out = np.where(seen, p, 0.0) @ np.where(fine, rows, 0.0)
    for j in np.flatnonzero(~fine.all(axis=1)):
        with np.errstate(invalid="ignore"):
            out[seen[:, j]] += p[seen[:, j], j, None] * np.where(fine[j], 0.0, rows[j])
    return out


def window_attn_fwd(q, k, v, q_starts, k_starts, left, right, sinks, scale, u=0.0, g=0.0):
    """q [n_q][h][d], k / v [n_k][kv][d] -> (o, lse, bound of |o|'s error).  Rows that see nothing: 0, -inf."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n_q, heads, _ = q.shape
    o, lse, bound = np.zeros_like(q), np.full((n_q, heads), -np.inf), np.zeros_like(q)
    for qs, ks, h, kh in _each(q_starts, k_starts, heads, k.shape[1]):
        a, b = qs.stop - qs.start, ks.stop - ks.start
        if a <= 0 or b <= 0:
            continue
        seen = visible(a, b, left, right, sinks)
        some = seen.any(axis=1)
        s = _scores(q[qs, h], k[ks, kh], seen, scale)
        top = np.where(some, s.max(axis=1), 0.0)
        with np.errstate(invalid="ignore"):
            e = np.exp(s - top[:, None])
        total = e.sum(axis=1)
        p = e / np.where(some, total, 1.0)[:, None]
        o[qs, h] = _times(p, v[ks, kh], seen)
        with np.errstate(divide="ignore"):
            lse[qs, h] = np.where(some, top + np.log(total), -np.inf)
        with np.errstate(invalid="ignore"):
            mag = _times(p, np.abs(v[ks, kh]), seen)
            bound[qs, h] = (u + g) * mag + u * np.abs(o[qs, h])
    return o, lse, bound


def window_attn_bwd(q, k, v, o, do, lse, q_starts, k_starts, left, right, sinks, scale, u=0.0, g=0.0):
    """Gradients of sum(o * do) from the forward pass's o and lse: ((dq, dk, dv), bounds of their errors)."""
    q, k, v, o, do, lse = (np.asarray(t, np.float64) for t in (q, k, v, o, do, lse))
    out = [np.zeros_like(t) for t in (q, k, v)]
    err = [np.zeros_like(t) for t in (q, k, v)]
    for qs, ks, h, kh in _each(q_starts, k_starts, q.shape[1], k.shape[1]):
        a, b = qs.stop - qs.start, ks.stop - ks.start
        if a <= 0 or b <= 0:
            continue
        seen = visible(a, b, left, right, sinks)
        Q, K, V, D = q[qs, h], k[ks, kh], v[ks, kh], do[qs, h]
        s = _scores(Q, K, seen, scale)
        with np.errstate(invalid="ignore"):
            p = np.where(seen, np.exp(np.where(seen, s, 0.0) - np.where(seen.any(axis=1), lse[qs, h], 0.0)[:, None]), 0.0)
            delta = (D * o[qs, h]).sum(axis=1)[:, None]
            ds = np.where(seen, p * (D @ V.T - delta), 0.0)
            wide = np.where(seen, p * (np.abs(D) @ np.abs(V).T + np.abs(D * o[qs, h]).sum(axis=1)[:, None]), 0.0)
        # delta's own error: that of the rounded o that it may be taken from (window_attn_fwd's bound)
        with np.errstate(invalid="ignore"):
            mag = _times(p, np.abs(V), seen)
            e_delta = u * (np.abs(D) * (np.abs(o[qs, h]) + mag)).sum(axis=1)[:, None]
            e_ds = u * np.abs(ds) + g * wide + np.where(seen, p * e_delta, 0.0)
        out[0][qs, h] += scale * _times(ds, K, seen)
        out[1][ks, kh] += scale * _times(ds.T, Q, seen.T)
        out[2][ks, kh] += _times(p.T, D, seen.T)
        with np.errstate(invalid="ignore"):
            err[0][qs, h] += abs(scale) * (_times(e_ds, np.abs(K), seen) + g * _times(np.abs(ds), np.abs(K), seen))
            err[1][ks, kh] += abs(scale) * (_times(e_ds.T, np.abs(Q), seen.T) + g * _times(np.abs(ds).T, np.abs(Q), seen.T))
            err[2][ks, kh] += (u + g) * _times(p.T, np.abs(D), seen.T)
    return out, [e + u * np.abs(t) for e, t in zip(err, out)]


def step_slot(j, sinks, cap):
    return j if j < sinks else sinks + (j - sinks) % (cap - sinks)


def window_attn_step(q, k_new, v_new, k_cache, v_cache, lens, left, sinks, scale, u=0.0, g=0.0):
    """Writes the new rows into the caches (in place); returns (o, bound of its error)."""
    batch, heads, _ = q.shape
    kv, cap = k_cache.shape[2], k_cache.shape[1]
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(batch):
        p = int(lens[b])
        if p < 0:
            continue
        k_cache[b, step_slot(p, sinks, cap)], v_cache[b, step_slot(p, sinks, cap)] = k_new[b], v_new[b]
        low = max(p - left, p + 1 - (cap - sinks), 0)
        at = [step_slot(j, sinks, cap) for j in range(min(sinks, p + 1, low))] + [step_slot(j, sinks, cap) for j in range(low, p + 1)]
        K, V = np.asarray(k_cache[b, at], np.float64), np.asarray(v_cache[b, at], np.float64)
        for h in range(heads):
            s = K[:, h // (heads // kv)] @ np.asarray(q[b, h], np.float64) * scale
            e = np.exp(s - s.max())
            e /= e.sum()
            o[b, h] = e @ V[:, h // (heads // kv)]
            bound[b, h] = (u + g) * (e @ np.abs(V[:, h // (heads // kv)])) + u * np.abs(o[b, h])
    return o, bound


# ---- distillation ----------------------------------------------------------------------------------------------
def distill(z, top, index, temperature, weight=None):
    """Returns (loss, dz)."""
    z, top = np.asarray(z, np.float64), np.asarray(top, np.float64)
    n, m = z.shape
    loss, dz = 0.0, np.zeros((n, m))
    for r in range(n):
        w = 1.0 / n if weight is None else float(weight[r])
        ok = (index[r] >= 0) & (index[r] < m) & (top[r] != -np.inf)
        if not ok.any():
            continue
        t = top[r, ok] / temperature
        a = np.exp(t - t.max())
        a /= a.sum()
        s = z[r] / temperature
        lse = s.max() + np.log(np.exp(s - s.max()).sum())
        with np.errstate(divide="ignore"):
            log_a = np.log(a)
        some = a != 0
        loss += w * temperature ** 2 * (a[some] * (log_a[some] - s[index[r, ok][some]] + lse)).sum()
        dz[r] = np.exp(s - lse)
        np.subtract.at(dz[r], index[r, ok], a)
        dz[r] *= w * temperature
    return loss, dz
