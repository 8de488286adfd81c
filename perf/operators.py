"""The attention operators of token models that the framework is timed on.

Three operators that a transformer generator or discriminator needs around
its projections: the norm of every query and key head with the position
rotation in the same pass ("norm"), attention with a sliding window and a few
first tokens that stay visible, and the learned relative position bias by
buckets inside it ("attend", with or without a bias).  A case is one pass:
a forward, a training forward and backward, or the step of one new token over
a cache.  listed() holds the fixed cases, draw() one more of the same ranges,
prepare() / run() / work() their inputs, call and unavoidable work, exact()
the same outputs in float64.  run() computes elementary torch operations in
float32 where `own` is false and calls paragan_2411_03999_amd.lib where it is
true.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # ---- norm and rotation of query and key heads
        # eight sequences take one step each: launch latency
        _norm("norm_step_t8_h32_8_d128", T=8, Hq=32, Hk=8, d=128, rot=128),
        # a training batch of 64 x 64 token grids, heads in one projection buffer
        _norm("norm_fwd_t32768_h8_d64", T=32768, Hq=8, Hk=8, d=64, rot=64),
        # its kind of backward at an odd token count, shared keys, half of each head rotated, adjacent pairs
        _norm("norm_bwd_t15005_h32_8_d128", T=15005, Hq=32, Hk=8, d=128, rot=64, inter=1, bwd=1),
        # float32 training, a head width that is no power of two
        _norm("norm_bwd_f32_t4096_h8_d80", T=4096, Hq=8, Hk=8, d=80, rot=80, bwd=1, f32=1),
        # ---- attention
        # 16 x 16 token grids: many short sequences, every token sees every token, with the bias
        _attend("attend_fwd_b64_s256_h8_d64_bias", B=64, Sq=256, Sk=256, Hq=8, Hk=8, d=64, buckets=32, maxd=128),
        # long causal sequences with shared keys, no window: the matrix products bound it
        _attend("attend_fwd_b2_s8192_h16_4_d128", B=2, Sq=8192, Sk=8192, Hq=16, Hk=4, d=128, causal=1),
        # a padded batch of odd length through a window with sinks
        _attend("attend_fwd_b4_s4099_h16_d64_w512", B=4, Sq=4099, Sk=4099, Hq=16, Hk=16, d=64, causal=1, window=512,
                sink=4, ragged=1),
        # training on 64 x 64 token grids with the bias and its gradient
        _attend("attend_train_b4_s4096_h8_d64_bias", B=4, Sq=4096, Sk=4096, Hq=8, Hk=8, d=64, buckets=32, maxd=128,
                train=1),
        # training through a window with sinks, shared keys, padded batch
        _attend("attend_train_b2_s4096_h16_4_d128_w1024", B=2, Sq=4096, Sk=4096, Hq=16, Hk=4, d=128, causal=1,
                window=1024, sink=16, ragged=1, train=1),
        # training of a small causal model on short padded sequences: latency of the whole pass
        _attend("attend_train_b16_s77_h4_d32_bias", B=16, Sq=77, Sk=77, Hq=4, Hk=4, d=32, causal=1, buckets=16,
                maxd=64, ragged=1, train=1),
        # one new token for each of 32 sequences over caches of up to 8192: the cache is read once
        _attend("attend_step_b32_s8192_h32_8_d128", B=32, Sq=1, Sk=8192, Hq=32, Hk=8, d=128, causal=1, ragged=1),
        # one new token of one long sequence, window, sinks and bias: few keys count, latency
        _attend("attend_step_b1_s32768_h16_2_d64_w1024_bias", B=1, Sq=1, Sk=32768, Hq=16, Hk=2, d=64, causal=1,
                window=1024, sink=4, buckets=32, maxd=128),
    ]


def _norm(name, T, Hq, Hk, d, rot, inter=0, bwd=0, f32=0):
    c = {"kind": "norm", "T": T, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "inter": inter, "bwd": bwd, "f32": f32}
    return {"name": name, **c} if name else c


def _attend(name, B, Sq, Sk, Hq, Hk, d, causal=0, window=0, sink=0, buckets=0, maxd=0, ragged=0, train=0):
    c = {"kind": "attend", "B": B, "Sq": Sq, "Sk": Sk, "Hq": Hq, "Hk": Hk, "d": d, "causal": causal, "window": window,
         "sink": sink, "buckets": buckets, "maxd": maxd, "ragged": ragged, "train": train}
    return {"name": name, **c} if name else c


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _heads(rng):
    hk = rng.choice([1, 2, 4, 8])
    return hk * rng.choice([1, 1, 2, 4]), hk


def draw(rng):
    what = rng.choice(["norm", "norm", "fwd", "fwd", "train", "train", "step", "step"])
    if what == "norm":
        hq, hk = _heads(rng)
        d = 8 * rng.randint(4, 16)
        return _norm(None, T=_log(rng, 1, 40000), Hq=hq, Hk=hk, d=d, rot=16 * rng.randint(0, d // 16),
                     inter=rng.randint(0, 1), bwd=rng.randint(0, 1), f32=int(rng.random() < 0.3))
    while True:
        hq, hk = _heads(rng)
        causal = rng.randint(0, 1)
        c = {"Hq": hq, "Hk": hk, "d": rng.choice([32, 64, 64, 80, 96, 128, 128]), "causal": causal,
             "ragged": rng.randint(0, 1), "train": int(what == "train")}
        if what == "step":
            c.update(B=_log(rng, 1, 64), Sq=rng.choice([1, 1, 1, 2, 4]), Sk=_log(rng, 16, 32768), causal=1)
        else:
            s = _log(rng, 16, 8192)
            c.update(B=_log(rng, 1, 64), Sq=s, Sk=s)
        if rng.random() < 0.5:
            c.update(window=_log(rng, 16, 2048), sink=rng.choice([0, 1, 4, 16, 64]))
        if rng.random() < 0.4:
            c.update(buckets=rng.choice([8, 16, 32, 64]), maxd=rng.choice([64, 128, 256]))
        c = _attend(None, **c)
        most = 1.1e9 if c["train"] else 2.2e9
        kv = c["B"] * c["Sk"] * c["Hk"] * c["d"]
        if c["B"] * c["Hq"] * c["Sq"] * c["Sk"] <= most and kv <= 32 * 8192 * 8 * 128 and \
                work(c)["flops"] <= 5.6e11 and c["Sk"] >= c["Sq"]:
            return c


# ------------------------------------------------------------- inputs
def _lens(c):
    """Keys of each sequence: full, or from full down to half."""
    return [c["Sk"] - (b * c["Sk"]) // (2 * c["B"]) if c["ragged"] else c["Sk"] for b in range(c["B"])]


def _lens_q(c):
    return [n if c["Sq"] == c["Sk"] else c["Sq"] for n in _lens(c)]


def _randn(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "norm":
        T, Hq, Hk, d, rot = c["T"], c["Hq"], c["Hk"], c["d"], c["rot"]
        dt = torch.float32 if c["f32"] else torch.bfloat16
        qkv = _randn(gen, T, (Hq + 2 * Hk) * d, dtype=dt)           # one projection buffer: q | k | v
        s["q"] = qkv[:, :Hq * d].unflatten(1, (Hq, d))
        s["k"] = qkv[:, Hq * d:(Hq + Hk) * d].unflatten(1, (Hk, d))
        s["gq"] = 1 + 0.1 * _randn(gen, d, dtype=torch.float32)
        s["gk"] = 1 + 0.1 * _randn(gen, d, dtype=torch.float32)
        n_pos = 4096
        ang = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * \
            torch.exp(-math.log(1e4) * torch.arange(rot // 2, device=DEV, dtype=torch.float64) / max(rot // 2, 1))
        s["table"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()     # [n_pos][rot / 2][2]
        s["pos"] = torch.randint(0, n_pos, (T,), generator=gen, device=DEV, dtype=torch.int32)
        if c["bwd"]:
            s["dq"], s["dk"] = _randn(gen, T, Hq, d, dtype=dt), _randn(gen, T, Hk, d, dtype=dt)
        return s
    B, Sq, Sk, Hq, Hk, d = (c[n] for n in ("B", "Sq", "Sk", "Hq", "Hk", "d"))
    if Sq == Sk:                                                      # one projection buffer: q | k | v
        qkv = _randn(gen, B, Sq, Hq + 2 * Hk, d)
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    else:                                                             # new tokens over a cache
        s["q"], s["k"], s["v"] = _randn(gen, B, Sq, Hq, d), _randn(gen, B, Sk, Hk, d), _randn(gen, B, Sk, Hk, d)
    s["scale"] = 1.0 / math.sqrt(d)
    s["table"] = 0.5 * _randn(gen, Hq, c["buckets"], dtype=torch.float32) if c["buckets"] else None
    if c["ragged"]:
        s["len_k"] = torch.tensor(_lens(c), device=DEV, dtype=torch.int32)
        s["len_q"] = torch.tensor(_lens_q(c), device=DEV, dtype=torch.int32)
    else:
        s["len_k"] = s["len_q"] = None
    if c["train"]:
        s["do"] = _randn(gen, B, Sq, Hq, d)
    return s


# ------------------------------------------------------------- one pass
def run(s):
    if own:
        return _own_norm(s) if s["case"]["kind"] == "norm" else _own_attend(s)
    return _plain_norm(s) if s["case"]["kind"] == "norm" else _plain_attend(s)


def _own_norm(s):
    from paragan_2411_03999_amd import lib
    c = s["case"]
    if "ctx" not in s:                                                # what a program makes once: handle, plan, buffers
        s["ctx"] = lib.Context()
        T, Hq, Hk, d, dt = c["T"], c["Hq"], c["Hk"], c["d"], s["q"].dtype
        s["desc"] = lib.qknorm_desc(s["q"], s["k"], rot=c["rot"], interleaved=c["inter"], n_pos=s["table"].shape[0],
                                    eps=EPS)
        if c["bwd"]:                                                  # gradients lie as q and k do
            g = torch.empty((T, Hq + 2 * Hk, d), device=DEV, dtype=dt)
            s["oq"], s["ok"] = g[:, :Hq], g[:, Hq:Hq + Hk]
        else:
            s["oq"], s["ok"] = (torch.empty((T, h, d), device=DEV, dtype=dt) for h in (Hq, Hk))
        s["og"] = torch.empty((2, d), device=DEV, dtype=torch.float32)
        s["ws"] = lib.workspace(lib.paragan_qknorm_ws_size(s["desc"]))
    if not c["bwd"]:
        lib.paragan_qknorm_fwd(s["ctx"], s["desc"], s["q"], s["k"], s["gq"], s["gk"], s["table"], s["pos"], s["oq"],
                               s["ok"])
        return s["oq"], s["ok"]
    lib.paragan_qknorm_bwd(s["ctx"], s["desc"], s["q"], s["k"], s["gq"], s["gk"], s["table"], s["pos"], s["dq"],
                           s["dk"], s["oq"], s["ok"], s["og"][0], s["og"][1], s["ws"])
    return s["oq"], s["ok"], s["og"][0], s["og"][1]


def _own_attend(s):
    from paragan_2411_03999_amd import lib
    c = s["case"]
    if "ctx" not in s:
        s["ctx"] = lib.Context()
        s["o"] = torch.empty((c["B"], c["Sq"], c["Hq"], c["d"]), device=DEV, dtype=torch.bfloat16)
        s["desc"] = lib.mha_desc(s["q"], s["k"], s["v"], s["o"], scale=s["scale"], causal=c["causal"],
                                 window=c["window"], n_sink=c["sink"], n_buckets=c["buckets"], max_distance=c["maxd"])
        saved, ws = lib.paragan_mha_sizes(s["desc"])
        s["saved"] = lib.workspace(saved) if c["train"] else None
        s["ws"] = lib.workspace(ws)
        if c["train"]:
            s["g"] = torch.empty((c["B"], c["Sq"], c["Hq"] + 2 * c["Hk"], c["d"]), device=DEV, dtype=torch.bfloat16)
            s["gt"] = torch.empty_like(s["table"]) if c["buckets"] else None
    lib.paragan_mha_fwd(s["ctx"], s["desc"], s["q"], s["k"], s["v"], s["table"], s["len_q"], s["len_k"], s["o"],
                        s["saved"], s["ws"])
    if not c["train"]:
        return s["o"]
    hq, hk = c["Hq"], c["Hk"]
    dq, dk, dv = s["g"][:, :, :hq], s["g"][:, :, hq:hq + hk], s["g"][:, :, hq + hk:]
    lib.paragan_mha_bwd(s["ctx"], s["desc"], s["q"], s["k"], s["v"], s["table"], s["len_q"], s["len_k"], s["o"],
                        s["saved"], s["do"], dq, dk, dv, s["gt"], s["ws"])
    return [s["o"], dq, dk, dv] + ([s["gt"]] if c["buckets"] else [])


def _turn(x, cs, rot, inter, sign):
    """Rotation of the pairs of the first `rot` elements by the angle, or back (sign -1); cs [T][rot / 2][2]."""
    if not rot:
        return x
    co, si = cs[:, None, :, 0], sign * cs[:, None, :, 1]
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * co - b * si, a * si + b * co], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_norm(s):
    c = s["case"]
    cs = s["table"][s["pos"].long()]
    outs, gains = [], []
    for x, g, dy in ((s["q"], s["gq"], s.get("dq")), (s["k"], s["gk"], s.get("dk"))):
        dt, x = x.dtype, x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if dy is None:
            outs.append(_turn(x * r * g, cs, c["rot"], c["inter"], 1.0).to(dt))
            continue
        dn = _turn(dy.float(), cs, c["rot"], c["inter"], -1.0)
        gains.append((dn * x * r).sum((0, 1), dtype=torch.float64).float())
        t = dn * g
        outs.append((r * (t - x * r * r * (t * x).mean(-1, keepdim=True))).to(dt))
    return outs + gains


def _bucket(rel, causal, nb, maxd):
    """Bucket of a key at distance rel (key position - query position): exact distances up to half of a side's
    buckets, logarithmic ones from there to maxd, the last bucket beyond; a side for earlier and one for later keys."""
    half = nb if causal else nb // 2
    n = (-rel).clamp(min=0) if causal else rel.abs()
    first = half // 2
    far = torch.log(n.clamp(min=1).double() / first) / math.log(maxd / first) * (half - first)
    b = torch.where(n < first, n, (first + torch.floor(far + 1e-9).long()).clamp(max=half - 1))
    return b if causal else b + half * (rel > 0)


def _plain_attend(s):
    c = s["case"]
    B, Sq, Sk, Hq, Hk, d = (c[n] for n in ("B", "Sq", "Sk", "Hq", "Hk", "d"))
    G = Hq // Hk
    rows = lambda t: t.float().unflatten(2, (Hk, -1)).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Sq, d)  # noqa: E731
    q, k, v = rows(s["q"]), s["k"].float().transpose(1, 2).contiguous(), s["v"].float().transpose(1, 2).contiguous()
    i, j = torch.arange(Sq, device=DEV)[None, :, None], torch.arange(Sk, device=DEV)[None, None, :]
    p = i + Sk - Sq                                                   # the queries' positions
    if s["len_k"] is not None:
        lk, lq = s["len_k"].long()[:, None, None], s["len_q"].long()[:, None, None]
        p = i + (lk - lq)
        seen = (i < lq) & (j < lk)
    else:
        seen = (j >= 0).expand(1, Sq, Sk)
    dist = p - j
    if c["causal"]:
        seen = seen & (dist >= 0)
    if c["window"]:
        seen = seen & ((dist.abs() < c["window"]) | (j < c["sink"]))
    x = (q @ k.transpose(-1, -2)).unflatten(2, (G, Sq)) * s["scale"]  # [B][Hk][G][Sq][Sk]
    if s["table"] is not None:
        bias = s["table"][:, _bucket(-dist[:1] if Sq == Sk else -dist, c["causal"], c["buckets"], c["maxd"])]
        x += bias.unflatten(0, (Hk, G)).permute(2, 0, 1, 3, 4)
    seen = seen[:, None, None]
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    x.div_(x.sum(-1, keepdim=True).clamp(min=1e-30))
    x = x.flatten(2, 3)                                               # the probabilities, [B][Hk][G Sq][Sk]
    back = lambda t: t.unflatten(2, (G, Sq)).permute(0, 3, 1, 2, 4).reshape(B, Sq, Hq, d).to(torch.bfloat16)  # noqa: E731
    o = x @ v
    if not c["train"]:
        return back(o)
    do = rows(s["do"])
    dv = (x.transpose(-1, -2) @ do).transpose(1, 2).to(torch.bfloat16)
    ds = do @ v.transpose(-1, -2)
    ds.sub_((do * o).sum(-1, keepdim=True)).mul_(x)
    dq = back((ds @ k) * s["scale"])
    dk = ((ds.transpose(-1, -2) @ q) * s["scale"]).transpose(1, 2).to(torch.bfloat16)
    outs = [back(o), dq, dk, dv]
    if s["table"] is not None:
        # sums along the diagonals (one distance each) of every head, then over the buckets' distances
        t = ds.unflatten(2, (G, Sq)).flatten(1, 2).sum(0)             # [Hq][Sq][Sk]: all sequences share positions
        W = Sk + Sq                                                   # rows of W - 1, read as rows of W: column j - i
        t = torch.nn.functional.pad(torch.nn.functional.pad(t, (0, Sq - 1)).flatten(1), (0, Sq)).unflatten(1, (Sq, W))
        t = t.sum(1, dtype=torch.float64)                             # column e: distance e, or e - W
        e = torch.arange(W, device=DEV)
        at = _bucket(torch.where(e < Sk, e, e - W), c["causal"], c["buckets"], c["maxd"])
        outs.append((t @ (at[:, None] == torch.arange(c["buckets"], device=DEV)).double()).float())
    return outs


# ------------------------------------------------------------- unavoidable work
def _pairs(c, b):
    """Visible (query, key) pairs of sequence b, and the keys that some query sees."""
    n, nq = _lens(c)[b], _lens_q(c)[b]
    pairs, lo_all, w = 0, n, c["window"]
    p = torch.arange(nq, dtype=torch.int64) + n - nq
    hi = torch.clamp(p + 1, max=n) if c["causal"] else torch.full_like(p, n)
    lo = torch.zeros_like(p)
    if w:
        lo = torch.clamp(p - w + 1, min=0)
        if not c["causal"]:
            hi = torch.clamp(p + w, max=n)
    sinks = torch.minimum(torch.full_like(p, c["sink"]) if w else torch.zeros_like(p), torch.minimum(lo, hi))
    pairs = int((hi - lo).clamp(min=0).sum() + sinks.sum())
    lo_all = int(lo.min()) if nq else n
    return pairs, (n - lo_all) + min(c["sink"] if w else 0, lo_all)


def work(case):
    c = case
    if c["kind"] == "norm":
        el, n = 4 if c["f32"] else 2, c["T"] * (c["Hq"] + c["Hk"]) * c["d"]
        table = min(c["T"], 4096) * c["rot"] * 4 + 4 * c["T"]
        return {"bytes": float(n * el * (3 if c["bwd"] else 2) + table), "flops": float(n * (14 if c["bwd"] else 8))}
    pairs = keys = rows = 0
    for b in range(c["B"]):
        a, k = _pairs(c, b)
        pairs, keys, rows = pairs + a, keys + k, rows + _lens_q(c)[b]
    qo, kv = 2 * rows * c["Hq"] * c["d"], 2 * keys * c["Hk"] * c["d"]
    return {"bytes": float((4 * qo + 4 * kv) if c["train"] else (2 * qo + 2 * kv)),
            "flops": float((14 if c["train"] else 4) * c["d"] * pairs * c["Hq"])}


# ------------------------------------------------------------- the same outputs in float64
def _exact_norm(s, c):
    import numpy as np
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    tab, pos = n(s["table"]), s["pos"].cpu().numpy()
    z = tab[pos, :, 0] + 1j * tab[pos, :, 1]                          # [T][rot / 2] as unit complex numbers
    rot, res = c["rot"], ([], [])

    def turn(x, w):
        if not rot:
            return x
        y = x.copy()
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
        t = (x[..., lo] + 1j * x[..., hi]) * w[:, None, :]
        y[..., lo], y[..., hi] = t.real, t.imag
        return y

    for x, g, dy in ((n(s["q"]), n(s["gq"]), s.get("dq")), (n(s["k"]), n(s["gk"]), s.get("dk"))):
        rms = np.sqrt(np.einsum("thd,thd->th", x, x) / x.shape[-1] + EPS)[..., None]
        u = x / rms
        if dy is None:
            res[0].append(turn(u * g, z))
            continue
        dn = turn(n(dy), np.conj(z))                                   # the transposed rotation
        res[1].append(np.einsum("thd,thd->d", dn, u))
        du = dn * g
        res[0].append((du - u * (np.einsum("thd,thd->th", du, u) / x.shape[-1])[..., None]) / rms)
    return [torch.from_numpy(np.ascontiguousarray(t)) for t in res[0] + res[1]]


def _exact_buckets(c):
    """Bucket of every distance -maxd .. maxd (clamped there) by whole-number comparisons: the logarithmic bucket
    is the largest e with (n / first)^(half - first) >= (maxd / first)^e."""
    nb, maxd = c["buckets"], c["maxd"]
    half = nb if c["causal"] else nb // 2
    first = half // 2
    m = half - first
    got = []
    for rel in range(-maxd, maxd + 1):
        n = max(-rel, 0) if c["causal"] else abs(rel)
        b = n
        if n >= first:
            e = 0
            while e < m - 1 and n ** m * first ** (e + 1) >= maxd ** (e + 1) * first ** m:
                e += 1
            b = first + e
        got.append(b + (half if rel > 0 and not c["causal"] else 0))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "norm":
        return _exact_norm(s, c)
    Hq, Hk, Sq, Sk, d = c["Hq"], c["Hk"], c["Sq"], c["Sk"], c["d"]
    kw = {"dtype": torch.float64, "device": DEV}
    o = torch.zeros((c["B"], Sq, Hq, d), **kw)
    if c["train"]:
        dq, dk, dv = torch.zeros_like(o), torch.zeros((c["B"], Sk, Hk, d), **kw), torch.zeros((c["B"], Sk, Hk, d), **kw)
    if c["buckets"]:
        of = torch.tensor(_exact_buckets(c), device=DEV)
        dt = torch.zeros((Hq, c["buckets"]), **kw)
    for b in range(c["B"]):
        nk, nq = _lens(c)[b], _lens_q(c)[b]
        pos = torch.arange(nk - nq, nk, device=DEV)
        key = torch.arange(nk, device=DEV)
        rel = key[None, :] - pos[:, None]
        hide = torch.zeros_like(rel, dtype=torch.bool)
        if c["causal"]:
            hide |= rel > 0
        if c["window"]:
            hide |= (rel.abs() >= c["window"]) & (key[None, :] >= c["sink"])
        at = of[rel.clamp(-c["maxd"], c["maxd"]) + c["maxd"]] if c["buckets"] else None
        for h in range(Hq):
            q, k, v = s["q"][b, :nq, h].double(), s["k"][b, :nk, h * Hk // Hq].double(), s["v"][b, :nk, h * Hk // Hq].double()
            z = torch.mm(q, k.t().contiguous()) * s["scale"]
            if c["buckets"]:
                z += s["table"][h].double()[at]
            z[hide] = -math.inf
            P = torch.softmax(z, -1).nan_to_num(0.0)                   # a row without a visible key is zero
            o[b, :nq, h] = torch.mm(P, v)
            if not c["train"]:
                continue
            g = s["do"][b, :nq, h].double()
            dP = torch.mm(g, v.t().contiguous())
            dz = P * (dP - (P * dP).sum(-1, keepdim=True))
            dq[b, :nq, h] = torch.mm(dz, k) * s["scale"]
            dk[b, :nk, h * Hk // Hq] += torch.mm(dz.t().contiguous(), q) * s["scale"]
            dv[b, :nk, h * Hk // Hq] += torch.mm(P.t().contiguous(), g)
            if c["buckets"]:
                dt[h] += torch.zeros(c["buckets"], **kw).index_add_(0, at.flatten(), dz.flatten())
    if not c["train"]:
        return o
    return [o, dq, dk, dv] + ([dt] if c["buckets"] else [])
