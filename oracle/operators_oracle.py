"""Plain NumPy float64 definitions of the operators around the layer: the policy loss,
the sorting of tokens by expert with its weighted sum, and the 8-bit form of
activations with what is computed from it.  Test infrastructure only, written from the
definitions in the C header and sharing no code with the library or its binding.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------ policy loss --

def token_stats(logits, token, inv_temp=1.0):
    """logp, lse, entropy [T] and p [T, V]; a row without a token in range or with every
    logit at -inf has logp = entropy = 0, lse = -inf, p = 0."""
    z = np.asarray(logits, dtype=np.float64)
    T, V = z.shape
    logp, ent = np.zeros(T), np.zeros(T)
    lse = np.full(T, -np.inf)
    p = np.zeros((T, V))
    for t in range(T):
        y = int(token[t])
        m = -np.inf if np.all(z[t] == -np.inf) else np.max(z[t])
        if not 0 <= y < V or m == -np.inf:
            continue
        if not np.isfinite(m):
            logp[t] = lse[t] = ent[t] = np.nan
            p[t] = np.nan
            continue
        e = np.exp((z[t] - m) * inv_temp)
        S = np.sum(np.sort(e))
        lse[t] = m * inv_temp + np.log(S)
        p[t] = e / S
        logp[t] = (z[t, y] - m) * inv_temp - np.log(S)
        on = p[t] > 0
        ent[t] = -np.sum(p[t][on] * ((z[t][on] - m) * inv_temp - np.log(S)))
    return logp, lse, ent, p


def policy_loss(logits, token, logp_old, adv, logp_ref=None, weight=None, clip_low=0.2,
                clip_high=0.28, kl_coef=0.0, inv_temp=1.0):
    """dict: sums [4], logp, lse, entropy, coef [T], dlogits [T, V]."""
    T, V = np.shape(logits)
    w = np.ones(T) if weight is None else np.asarray(weight, dtype=np.float64)
    token = np.where(w == 0, -1, np.asarray(token))
    logp, lse, ent, p = token_stats(logits, token, inv_temp)
    coef, sums = np.zeros(T), np.zeros(4)
    dl = np.zeros((T, V))
    for t in range(T):
        if lse[t] == -np.inf:
            continue
        A = float(adv[t])
        r = np.exp(logp[t] - float(logp_old[t]))
        lo, hi = 1.0 - clip_low, 1.0 + clip_high
        clipped = bool((A > 0 and r > hi) or (A < 0 and r < lo))
        surr, d_surr = 0.0, 0.0
        if A != 0:
            surr = min(r * A, min(max(r, lo), hi) * A) if r == r else np.nan
            d_surr = 0.0 if clipped else A * r
        kl = d_kl = 0.0
        if logp_ref is not None:
            d = float(logp_ref[t]) - logp[t]
            kl, d_kl = np.expm1(d) - d, -np.expm1(d)
        coef[t] = w[t] * (-d_surr + kl_coef * d_kl)
        sums += w[t] * np.array([-surr + kl_coef * kl, kl, float(clipped), ent[t]])
        dl[t] = -coef[t] * inv_temp * p[t]
        dl[t, int(token[t])] = coef[t] * inv_temp * -np.expm1(logp[t])
    return dict(sums=sums, logp=logp, lse=lse, entropy=ent, coef=coef, dlogits=dl, p=p)


# ------------------------------------------ tokens sorted by expert and back --

def dispatch_plan(idx, N):
    """offsets [N + 1], row_of_route [T, k], route_of_row [T * k]."""
    idx = np.asarray(idx)
    T, k = idx.shape
    rows = [[] for _ in range(N)]
    for q, e in enumerate(idx.reshape(-1).tolist()):
        if 0 <= e < N:
            rows[e].append(q)
    order = [q for per in rows for q in per]
    offsets = np.concatenate([[0], np.cumsum([len(per) for per in rows])]).astype(np.int64)
    row = np.full(T * k, -1, dtype=np.int64)
    route = np.full(T * k, -1, dtype=np.int64)
    for r, q in enumerate(order):
        row[q], route[r] = r, q
    return offsets, row.reshape(T, k), route


def dispatch(x, row_of_route):
    x = np.asarray(x, dtype=np.float64)
    T, k = row_of_route.shape
    xs = np.zeros((T * k, x.shape[1]))
    for t in range(T):
        for s in range(k):
            if row_of_route[t, s] >= 0:
                xs[row_of_route[t, s]] = x[t]
    return xs


def combine(o, row_of_route, gate=None):
    """y [T, d]; without a gate every weight is 1 (the gradient of dispatch)."""
    o = np.asarray(o, dtype=np.float64)
    T, k = row_of_route.shape
    y = np.zeros((T, o.shape[1]))
    for t in range(T):
        for s in range(k):
            if row_of_route[t, s] >= 0:
                y[t] += (1.0 if gate is None else float(gate[t, s])) * o[row_of_route[t, s]]
    return y


def combine_backward(dy, o, row_of_route, gate):
    dy, o = np.asarray(dy, dtype=np.float64), np.asarray(o, dtype=np.float64)
    T, k = row_of_route.shape
    d_o, dgate = np.zeros_like(o), np.zeros((T, k))
    for t in range(T):
        for s in range(k):
            r = row_of_route[t, s]
            if r >= 0:
                d_o[r] = float(gate[t, s]) * dy[t]
                dgate[t, s] = dy[t] @ o[r]
    return d_o, dgate


# ------------------------------------------------- activations kept in 8 bits --

GROUP = 32


def pack(x):
    """q [R, C] int, scale [R, ceil(C / 32)] int of x [R, C] (float32 values)."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape
    G = -(-C // GROUP)
    q, scale = np.zeros((R, C), dtype=np.int64), np.zeros((R, G), dtype=np.int64)
    for g in range(G):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        for r in range(R):
            if not np.all(np.isfinite(part[r])):
                scale[r, g] = 255
                continue
            top = np.max(np.abs(part[r]))
            # top = f 2^e with 1/2 <= f < 1: its fp32 exponent field is e + 126 (0 for subnormals)
            e = int(np.frexp(top)[1]) + 126 if top > 0 else 0
            scale[r, g] = max(e - 6, 1)
            v = np.rint(part[r] * 2.0 ** (127 - int(scale[r, g])))
            q[r, g * GROUP:(g + 1) * GROUP] = np.clip(v, -127, 127)
    return q, scale


def unpack(q, scale):
    q = np.asarray(q, dtype=np.float64)
    s = np.asarray(scale, dtype=np.int64)
    step = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
    return q * np.repeat(step, GROUP, axis=1)[:, :q.shape[1]]


def swiglu(a, u):
    return a / (1 + np.exp(-a)) * u


def swiglu_backward(a, u, dh):
    """da, du, h."""
    sig = 1 / (1 + np.exp(-a))
    return dh * u * sig * (1 + a * (1 - sig)), dh * a * sig, a * sig * u


def weight_grad(dy, x, offsets=None, route_of_row=None, k=1):
    """dW [N, n_out, n_in] and the sums of the terms' magnitudes."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    R = dy.shape[0]
    offsets = [0, R] if offsets is None else list(offsets)
    src = np.arange(R) if route_of_row is None else np.asarray(route_of_row) // k
    out = np.zeros((len(offsets) - 1, dy.shape[1], x.shape[1]))
    mag = np.zeros_like(out)
    for e in range(len(offsets) - 1):
        rows = np.arange(offsets[e], offsets[e + 1])
        rows = rows[(src[rows] >= 0) & (src[rows] < x.shape[0])]
        out[e] = dy[rows].T @ x[src[rows]]
        mag[e] = np.abs(dy[rows]).T @ np.abs(x[src[rows]])
    return out, mag
