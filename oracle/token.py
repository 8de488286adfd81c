"""Float64 definitions of the token attention operators (test infrastructure
only): norms of query and key heads with the position rotation, and
multi-head attention with a window, first tokens that stay visible, ragged
lengths and a relative position bias by buckets, forward and backward.

The optional error bounds are what a kernel may be off by that keeps fp32
statistics and sums, takes P and dS rounded to bfloat16 as matrix operands
and rounds its outputs once.
"""
import numpy as np

U32 = 2.0 ** -24        # half a step of float32, relative
U16 = 2.0 ** -8         # half a step of bfloat16, relative


# ------------------------------------------------------------- norm and rotation
def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, table, pos, rot, interleaved, inverse=False):
    """x (T, H, d); table (n_pos, rot / 2, 2); pos (T,) inside the table."""
    y = x.copy()
    a, b = _pairs(rot, interleaved)
    c, s = table[pos, :, 0][:, None], table[pos, :, 1][:, None]
    if inverse:
        s = -s
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def qknorm_fwd(x, gain, table, pos, rot, interleaved, eps):
    """One of q, k; tokens with a position outside the table give zeros."""
    real = (pos >= 0) & (pos < table.shape[0])
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    y = rotate(n, table, np.where(real, pos, 0), rot, interleaved)
    return np.where(real[:, None, None], y, 0.0)


def qknorm_bwd(x, gain, table, pos, rot, interleaved, eps, dy):
    real = (pos >= 0) & (pos < table.shape[0])
    dn = rotate(np.where(real[:, None, None], dy, 0.0), table, np.where(real, pos, 0), rot, interleaved, True)
    x = np.where(real[:, None, None], x, 0.0)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dgain = (dn * x * r).sum((0, 1))
    t = dn * gain
    return r * (t - x * r * r * (t * x).mean(-1, keepdims=True)), dgain


# ------------------------------------------------------------- buckets
def bucket_of(n, m, max_distance):
    """Bucket of distance n >= 0 among the m of one side, in whole numbers:
    first + the largest e with (n / first)^(m - first) >= (max_distance / first)^e."""
    first = m // 2
    if n < first:
        return n
    e = 0
    while e < m - first - 1 and n ** (m - first) * first ** (e + 1) >= max_distance ** (e + 1) * first ** (m - first):
        e += 1
    return first + e


def bucket_table(n_buckets, max_distance, causal):
    """Buckets of the relative positions -max_distance .. max_distance."""
    m = n_buckets if causal else n_buckets // 2
    one = [bucket_of(n, m, max_distance) for n in range(max_distance + 1)]
    return np.array([one[max(-r, 0)] if causal else one[abs(r)] + (m if r > 0 else 0)
                     for r in range(-max_distance, max_distance + 1)])


# ------------------------------------------------------------- attention
def visible(p, j, lk, causal, window, n_sink):
    """Truth of (len(p), len(j))."""
    p, j = np.asarray(p)[:, None], np.asarray(j)[None, :]
    see = j < lk
    if causal:
        see = see & (j <= p)
    if window:
        see = see & ((np.abs(p - j) < window) | (j < n_sink))
    return see


def mha(q, k, v, scale, causal=False, window=0, n_sink=0, table=None, max_distance=0, len_q=None, len_k=None,
        dout=None):
    """q (B, Sq, Hq, d), k, v (B, Sk, Hk, d), table (Hq, n_buckets).  Returns a
    dict: o and, with dout, dq, dk, dv, dtable; and for each of them an
    elementwise bound "tol.<name>" of a kernel's error (see above)."""
    B, Sq, Hq, d = q.shape
    Sk, Hk = k.shape[1:3]
    G = Hq // Hk
    names = ["o"] + (["dq", "dk", "dv"] if dout is not None else [])
    shape = {"o": q.shape, "dq": q.shape, "dk": k.shape, "dv": v.shape}
    r = {p + n: np.zeros(shape[n]) for n in names for p in ("", "tol.")}
    if dout is not None and table is not None:
        r["dtable"], r["tol.dtable"] = np.zeros(table.shape), np.zeros(table.shape)
    of = bucket_table(table.shape[1], max_distance, causal) if table is not None else None
    for b in range(B):
        lq = Sq if len_q is None else min(max(int(len_q[b]), 0), Sq)
        lk = Sk if len_k is None else min(max(int(len_k[b]), 0), Sk)
        if lq == 0 or lk == 0:
            continue
        p, j = np.arange(lq) + lk - lq, np.arange(lk)
        see = visible(p, j, lk, causal, window, n_sink)
        at = of[np.clip(j[None, :] - p[:, None], -max_distance, max_distance) + max_distance] if of is not None else None
        for h in range(Hq):
            Q, K, V = q[b, :lq, h], k[b, :lk, h // G], v[b, :lk, h // G]
            K, V = np.where(see.any(0)[:, None], K, 0.0), np.where(see.any(0)[:, None], V, 0.0)
            S = scale * (Q @ K.T)
            size = scale * (np.abs(Q) @ np.abs(K).T)            # what the products' rounding goes by
            if at is not None:
                S = S + table[h][at]
                size = size + np.where(np.abs(table[h][at]) < 1e30, np.abs(table[h][at]), 0.0)
            S = np.where(see, S, -np.inf)
            m = S.max(-1, keepdims=True)
            empty = ~np.isfinite(m)
            E = np.exp(S - np.where(empty, 0.0, m))
            L = E.sum(-1, keepdims=True)
            P = E / np.where(L > 0, L, 1.0)
            o = P @ V
            # relative error of a probability: the exponent's, the exponential's and the sum's
            eta = U32 * (2 * (d + 8) * np.where(see, size, 0.0).max(-1, keepdims=True) + lk + 64)
            av = np.abs(V)
            to = U16 * np.abs(o) + (U16 + 2 * eta) * (P @ av)
            r["o"][b, :lq, h], r["tol.o"][b, :lq, h] = o, to
            if dout is None:
                continue
            DO = dout[b, :lq, h]
            ad = np.abs(DO)
            dP = DO @ V.T
            D = (P * dP).sum(-1, keepdims=True)
            dS = P * (dP - D)
            # dP's own rounding, and D's: for dq and dk that of do . o, o of rounded probabilities and kept to twice
            # bfloat16's digits; the bias gradient has its rows' dS sum to zero again, up to the row's fp32 sum
            tp = U32 * (d + 4) * (ad @ av.T)
            to_row = (ad * (U16 * U16 * np.abs(o) + (U16 + 2 * eta) * (P @ av))).sum(-1, keepdims=True)
            ts = P * (tp + to_row + 4 * eta * (np.abs(dP) + np.abs(D)))
            ta = ts + U16 * np.abs(dS)
            mass = (P * (np.abs(dP) + np.abs(D) + to_row)).sum(-1, keepdims=True)
            tr = (P * tp).sum(-1, keepdims=True) + (4 * eta + 2 * U32 * (lk + 8)) * mass
            tt = P * (tp + tr + 4 * eta * (np.abs(dP) + np.abs(D) + to_row))
            aq, ak = np.abs(Q), np.abs(K)
            r["dq"][b, :lq, h] = scale * dS @ K
            r["tol.dq"][b, :lq, h] = scale * (ta + U32 * lk * np.abs(dS)) @ ak
            r["dk"][b, :lk, h // G] += scale * dS.T @ Q
            r["tol.dk"][b, :lk, h // G] += scale * (ta + U32 * lq * G * np.abs(dS)).T @ aq
            r["dv"][b, :lk, h // G] += P.T @ DO
            r["tol.dv"][b, :lk, h // G] += ((U16 + 2 * eta + U32 * lq * G) * P).T @ ad
            if at is not None:
                np.add.at(r["dtable"][h], at, dS)
                np.add.at(r["tol.dtable"][h], at, tt + U32 * (lq * B + 64) * (np.abs(dS) + ts))
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            r["tol." + n] += U16 * (np.abs(r[n]) + r["tol." + n])
        if table is not None:
            r["tol.dtable"] += U32 * np.abs(r["dtable"])
    return r
