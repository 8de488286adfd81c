"""Float64 definitions of the operators around and beside the attention of a
token block (test infrastructure only): the norms before and after a block
with modulation, gate and residual scale, a gated linear recurrence, both
forward and backward, and clipping by the norm of all gradients.

With `tol` the functions also give, under "tol." names, what a kernel may be
off by that computes in fp32 and rounds its outputs once (half a step `uo` of
their type).  A sum over a row goes through at most 8 elements of a lane, 6
exchanges and 16 waves, hence its 40 half steps; reciprocals, roots, 2^x are
off by a step.
"""
import numpy as np

from .token import U16, U32   # noqa: F401  (half steps of bfloat16 and float32)

ROW = 40 * U32                # a sum over a row, and the factor made of it, relative to the sum of magnitudes


# ------------------------------------------------------------- norms around a block
def _norm(t, et, layer, eps):
    """The normed rows, factor, and the normed rows' and the factor's (relative) error from an error et of t."""
    mean = t.mean(-1, keepdims=True) if layer else 0.0
    c = t - mean
    r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    n = c * r
    mabs = np.abs(t).mean(-1, keepdims=True) if layer else 0.0
    # the mean's error moves all elements, each element's rounding after the subtraction
    ec = et + (et.mean(-1, keepdims=True) if layer else 0.0) + ROW * mabs + U32 * np.abs(c)
    er = ROW + r * (np.abs(n) * ec).mean(-1, keepdims=True)
    return n, r, r * ec + np.abs(n) * (er + 2 * U32), er


def _norm_back(dn, edn, n, en, r, er, layer):
    """Gradient of the rows from that of the normed rows, and its error."""
    c1 = dn.mean(-1, keepdims=True) if layer else np.zeros_like(r)
    c2 = (dn * n).mean(-1, keepdims=True)
    m1 = np.abs(dn).mean(-1, keepdims=True) if layer else np.zeros_like(r)
    m2 = np.abs(dn * n).mean(-1, keepdims=True)
    e1 = ROW * m1 + (edn.mean(-1, keepdims=True) if layer else 0.0)
    e2 = ROW * m2 + (edn * np.abs(n) + np.abs(dn) * en).mean(-1, keepdims=True)
    mag = np.abs(dn) + m1 + np.abs(n) * m2
    g = r * (dn - c1 - n * c2)
    return g, r * (edn + e1 + en * m2 + np.abs(n) * e2) + r * mag * (er + 6 * U32)


def blocknorm(x, h, gain_post, gate, gain_pre, scale, shift, lens, *, layer, branch, post, pre, eps, res_scale, shared=False,
              dz=None, dy=None, uz=0.0, uy=0.0):
    """x, h, dz, dy (B, S, D); gains (D,), gate, scale, shift (B or 1, D), each may be None; lens (B,).  A dict of z, y, and
    with dz or dy (None: zero) dx, dh, dgain_post, dgate, dgain_pre, dscale, dshift, and their tolerances.  uz, uy: half steps
    of the stream's and of the other tensors' type."""
    B, S, D = x.shape
    real = (np.arange(S)[None, :] < np.asarray(lens)[:, None])[..., None]
    one, zero = np.ones(D), np.zeros(D)
    row = lambda t, d: d if t is None else t[:, None]  # noqa: E731
    g1, g2 = one if gain_post is None else gain_post, one if gain_pre is None else gain_pre
    gate_, sc, sh = row(gate, one), row(scale, zero), row(shift, zero)
    k, m = res_scale * gate_, g2 * (1 + sc)
    x = np.where(real, x, 0.0)
    out, nil = {}, np.zeros_like(x)
    z, ez = x, nil
    if branch:
        h = np.where(real, h, 0.0)
        hn, rh, eh, erh = _norm(h, nil, layer, eps) if post else (h, None, nil, None)
        v = hn * g1 if post else hn
        z = np.where(real, x + k * v, 0.0)
        ez = np.abs(k * g1 if post else k) * eh + 4 * U32 * (np.abs(x) + np.abs(k * v))
        out["z"], out["tol.z"] = z, np.where(real, uz * np.abs(z) + ez, 0.0)
    if pre:
        n, r, en, er = _norm(z, ez, layer, eps)
        y = np.where(real, n * m + sh, 0.0)
        out["y"] = y
        out["tol.y"] = np.where(real, uy * np.abs(y) + np.abs(m) * en + 4 * U32 * (np.abs(n * m) + np.abs(sh)), 0.0)
    if dz is None and dy is None:
        return out
    dZ = np.where(real, 0.0 if dz is None else dz, 0.0) + nil
    edZ = U32 * np.abs(dZ)
    over = (0, 1) if shared else (1,)
    col = lambda t: t.sum(over).reshape(-1, D)  # noqa: E731
    if pre:
        dy = np.where(real, dy, 0.0)
        t = dy * m
        back, eback = _norm_back(t, 2 * U32 * np.abs(t), n, en, r, er, layer)
        dZ, edZ = np.where(real, dZ + back, 0.0), np.where(real, edZ + eback + U32 * np.abs(back), 0.0)
        # a column's sum: 128 tokens at most in a thread, then in 64 bits
        q, eq = col(dy * n), col(np.abs(dy) * en + 140 * U32 * np.abs(dy * n))
        out["dshift"], out["tol.dshift"] = col(dy), 140 * U32 * col(np.abs(dy))
        out["dscale"], out["tol.dscale"] = g2 * q, np.abs(g2) * (eq + 4 * U32 * np.abs(q))
        w = (1 + sc) * (dy * n).sum(1, keepdims=True)
        ew = np.abs(1 + sc) * (np.abs(dy) * en + 140 * U32 * np.abs(dy * n)).sum(1, keepdims=True)
        out["dgain_pre"], out["tol.dgain_pre"] = w.sum((0, 1)), (ew + 4 * U32 * np.abs(w)).sum((0, 1))
    out["dx"], out["tol.dx"] = dZ, uz * np.abs(dZ) + edZ
    if branch:
        dv = dZ * k
        edv = np.abs(k) * edZ + 3 * U32 * np.abs(dv)
        p, ep = dZ * hn, edZ * np.abs(hn) + np.abs(dZ) * eh + 140 * U32 * np.abs(dZ * hn)
        out["dgate"] = res_scale * g1 * col(p) if post else res_scale * col(p)
        out["tol.dgate"] = np.abs(res_scale * g1 if post else res_scale) * (col(ep) + 4 * U32 * np.abs(col(p)))
        dh, edh = dv, edv
        if post:
            out["dgain_post"] = (k * p).sum((0, 1))
            out["tol.dgain_post"] = (np.abs(k) * (ep + 4 * U32 * np.abs(p))).sum((0, 1))
            dh, edh = _norm_back(dv * g1, edv * np.abs(g1) + U32 * np.abs(dv * g1), hn, eh, rh, erh, layer)
        dh = np.where(real, dh, 0.0)
        out["dh"], out["tol.dh"] = dh, np.where(real, uy * np.abs(dh) + edh, 0.0)
    return out


# ------------------------------------------------------------- gated linear recurrence
def scan(x, r, g, decay, lens, *, sharp, reverse=False, h0=None, dy=None, dht=None, uo=0.0):
    """x, r, g, dy (B, S, D); decay (D,); h0, dht (B, D) or None.  A dict of y, ht, and with dy dx, dr, dg, ddecay, dh0, and
    their tolerances."""
    B, S, D = x.shape
    out = {n: np.zeros((B, S, D)) for n in ("y", "tol.y")}
    out["ht"], out["tol.ht"] = np.zeros((B, D)), np.zeros((B, D))
    if dy is not None:
        for n in ("dx", "dr", "dg"):
            out[n], out["tol." + n] = np.zeros((B, S, D)), np.zeros((B, S, D))
        out["dh0"], out["tol.dh0"] = np.zeros((B, D)), np.zeros((B, D))
        dsum, esum, asum = np.zeros(D), np.zeros(D), np.zeros(D)
    soft = np.log1p(np.exp(-np.abs(decay))) + np.maximum(decay, 0)
    for b in range(B):
        n = int(lens[b])
        at = np.arange(n)[::-1] if reverse else np.arange(n)
        X, R, G = x[b, at], r[b, at], g[b, at]
        sig = lambda v: np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))  # noqa: E731
        s, cs, sg, cg = sig(R), sig(-R), sig(G), sig(-G)
        es, eg = U32 * (10 + 2 * np.abs(R)), U32 * (10 + 2 * np.abs(G))         # relative, of both s and 1 - s
        la = -sharp * soft * s
        el = es + 12 * U32                                                      # relative
        a = np.exp(la)
        ea = np.abs(la) * el + 3 * U32                                          # relative
        p = -np.expm1(2 * la)
        # by the series, or by 1 - a^2 where that is 0.22 at least; relative
        epp = el + 10 * U32 + np.where(2 * la > -0.3, 0.0, (2 * ea + 3 * U32) / np.maximum(p, 0.2))
        w = np.sqrt(p)
        u = w * sg * X
        eu = np.abs(u) * (epp + eg + 8 * U32) + 2e-19 * np.abs(sg * X)
        h, mag, eh = (np.zeros((n + 1, D)) for _ in range(3))
        if h0 is not None:
            h[0], mag[0] = h0[b], np.abs(h0[b])
        for t in range(n):
            h[t + 1] = a[t] * h[t] + u[t]
            mag[t + 1] = a[t] * mag[t] + np.abs(u[t])
            eh[t + 1] = a[t] * (eh[t] + mag[t] * (ea[t] + 4 * U32)) + eu[t]
        eh += 40 * U32 * mag                                                    # joins of parts of the sequence
        out["y"][b, at], out["tol.y"][b, at] = h[1:], uo * np.abs(h[1:]) + eh[1:]
        out["ht"][b], out["tol.ht"][b] = h[n], eh[n] + U32 * np.abs(h[n])
        if dy is None:
            continue
        dY = dy[b, at]
        E, me, ee = (np.zeros((n, D)) for _ in range(3))
        cur, mc, ec = (np.zeros(D) if dht is None else dht[b]), np.zeros(D) if dht is None else np.abs(dht[b]), np.zeros(D)
        for t in range(n - 1, -1, -1):
            E[t], me[t], ee[t] = dY[t] + cur, np.abs(dY[t]) + mc, ec + 4 * U32 * (np.abs(dY[t]) + mc)
            cur, mc, ec = a[t] * E[t], a[t] * me[t], a[t] * (ee[t] + me[t] * (ea[t] + 4 * U32))
        out["dh0"][b], out["tol.dh0"][b] = cur, ec + 41 * U32 * mc
        ee += 40 * U32 * me
        left, right = a * h[:-1], np.where(p > 0, u * a * a / np.where(p > 0, p, 1.0), 0.0)
        dla = E * (left - right)
        edla = ee * (np.abs(left) + np.abs(right)) + me * (a * eh[:-1] + mag[:-1] * a * (ea + 4 * U32)) + \
            me * np.where(p > 0, (eu * a * a + np.abs(u) * a * a * (2 * ea + epp + 8 * U32)) / np.where(p > 0, p, 1.0), 0.0)
        wsg = w * sg
        for name, v, e in (("dx", E * wsg, ee * wsg + np.abs(E) * wsg * (epp + eg + 8 * U32) + 2e-19 * np.abs(E)),
                           ("dg", E * u * cg, (ee * np.abs(u) + np.abs(E) * eu) * cg + np.abs(E * u) * cg * (eg + 8 * U32)),
                           ("dr", dla * la * cs, edla * np.abs(la) * cs + np.abs(dla * la) * cs * (el + es + 8 * U32))):
            out[name][b, at], out["tol." + name][b, at] = v, uo * np.abs(v) + e
        dsum += (dla * s).sum(0)
        # sums of 64 tokens at most in fp32, then in 64 bits
        esum += (edla * s + np.abs(dla) * s * (es + 100 * U32)).sum(0)
    if dy is not None:
        f = sharp / (1 + np.exp(-decay))
        out["ddecay"], out["tol.ddecay"] = -f * dsum, f * (esum + 4 * U32 * np.abs(dsum))
    return out


# ------------------------------------------------------------- clipping
def clip(grads, max_norm, grad_scale=1.0):
    """Norm, factor and the clipped gradients."""
    norm = grad_scale * np.sqrt(sum((g * g).sum() for g in grads))
    factor = grad_scale * (1.0 if norm <= max_norm else max_norm / norm)
    return norm, factor, [factor * g for g in grads]
