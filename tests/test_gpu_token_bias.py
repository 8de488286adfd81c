"""Attention with relative position biases that are large against the scores: the lowest finite value and the usual
masks of -1e4 and below, in rows that see other keys too and in rows that see nothing else, forward and backward.

A bias that a row's keys share shifts its scores and leaves the softmax as it is.  With equal keys the scores of a
row are equal too, so their fp32 sums with the bias round alike and the probabilities are exact; with a bias that
scores vanish in they are equal whatever the keys.  The bounds are therefore those of the definition without that
bias (oracle/token.py)."""
import math

import numpy as np
import pytest

from oracle import token as T
from paragan_2411_03999_amd import lib

from .parity import need_gpu
from .test_gpu_token import held, mha_case

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


def trained(q, k, v, do, table, scale=0.125, **kw):
    """o, dq, dk, dv, dtable of one forward and backward."""
    torch = need_gpu()
    Q, K, V, DO, TB = (t.cuda() for t in (q, k, v, do, table))
    out = {"o": torch.empty_like(Q), "dq": torch.empty_like(Q), "dk": torch.empty_like(K), "dv": torch.empty_like(V),
           "dtable": torch.empty_like(TB)}
    d = lib.mha_desc(Q, K, V, out["o"], scale=scale, n_buckets=table.shape[1], **kw)
    sb, wb = lib.paragan_mha_sizes(d)
    ctx, ws, saved = lib.Context(), lib.workspace(wb), lib.workspace(sb)
    ws.fill_(255)
    lib.paragan_mha_fwd(ctx, d, Q, K, V, TB, None, None, out["o"], saved, ws)
    ws.fill_(255)
    lib.paragan_mha_bwd(ctx, d, Q, K, V, TB, None, None, out["o"], saved, DO, out["dq"], out["dk"], out["dv"], out["dtable"], ws)
    torch.cuda.synchronize()
    return out


def against(out, q, k, v, do, table, scale=0.125, **kw):
    n = lambda t: t.double().numpy()  # noqa: E731
    want = T.mha(n(q), n(k), n(v), scale, table=n(table), dout=n(do), **kw)
    for name, t in out.items():
        held(name, t, want[name], want["tol." + name] + 1e-30)


def inputs(torch, seed, B, Sq, Sk, Hq, Hk, d):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(B, s, h, d, generator=gen).bfloat16() for s, h in ((Sq, Hq), (Sk, Hk), (Sk, Hk), (Sq, Hq))], gen


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("value", [LOWEST, -1e9, -1e5, -2e3])
def test_own_position_masked(value, d):
    """Causal, bucket 0 very low: the first query sees its own key alone and takes all of it, the others take nothing of
    theirs (2^-2885 is zero in float64 too, so the definition gives the same for all four)."""
    torch = need_gpu()
    print("own position masked", value, d, flush=True)
    (q, k, v, do), gen = inputs(torch, 1, 2, 170, 170, 4, 2, d)
    table = torch.randn(4, 8, generator=gen)
    given = table.clone()
    table[:, 0], given[:, 0] = LOWEST, value
    kw = dict(causal=1, max_distance=30)
    against(trained(q, k, v, do, given, **kw), q, k, v, do, table, **kw)


@pytest.mark.parametrize("causal,window", [(0, 0), (1, 0), (1, 90), (0, 90)])
@pytest.mark.parametrize("value", [LOWEST, -1e9, 1e9, -1e8])
def test_rows_of_nothing_else(value, causal, window):
    """Every bucket of one head holds a value that scores vanish in, near the diagonal and past max_distance: its rows are
    means.  The other query head of the same key head has an ordinary bias."""
    torch = need_gpu()
    print("nothing else", value, causal, window, flush=True)
    (q, k, v, do), gen = inputs(torch, 2, 1, 300, 300, 2, 1, 64)
    table = torch.randn(2, 8, generator=gen)
    given = table.clone()
    table[0], given[0] = LOWEST, value
    kw = dict(causal=causal, window=window, max_distance=9)
    against(trained(q, k, v, do, given, **kw), q, k, v, do, table, **kw)


@pytest.mark.parametrize("Sq,Sk", [(150, 150), (40, 150)])
@pytest.mark.parametrize("value", [-1e9, -1e6, -1e5, -1e4, 3e4, 900.0, 500.0])
def test_equal_keys_under_one_bias(value, Sq, Sk):
    """One value in every bucket of a head, equal keys: the probabilities are those of no bias at all."""
    torch = need_gpu()
    print("equal keys", value, Sq, Sk, flush=True)
    (q, k, v, do), gen = inputs(torch, 3, 1, Sq, Sk, 2, 1, 64)
    k[:] = k[:, :1]
    table = torch.randn(2, 16, generator=gen)
    given = table.clone()
    table[1], given[1] = 0.0, value
    kw = dict(causal=1, max_distance=200)                          # no tile lies past it
    against(trained(q, k, v, do, given, **kw), q, k, v, do, table, **kw)


@pytest.mark.parametrize("value", [float(np.finfo(np.float32).max), 2.5e38])
def test_largest_values_stay_finite(value):
    """A value whose multiple by log2(e) passes float32: in one bucket it takes the whole row, in all of them the row is a
    mean; forward, backward and the form for few rows."""
    torch = need_gpu()
    print("largest", value, flush=True)
    (q, k, v, do), gen = inputs(torch, 4, 1, 150, 150, 2, 1, 64)
    table = torch.randn(2, 8, generator=gen)
    table[0], table[1, 0] = value, value
    for causal in (0, 1):
        kw = dict(causal=causal, max_distance=9)
        against(trained(q, k, v, do, table, **kw), q, k, v, do, table, **kw)
        o = torch.empty_like(q).cuda()
        d = lib.mha_desc(q.cuda(), k.cuda(), v.cuda(), o, scale=0.125, n_buckets=8, **kw)
        lib.paragan_mha_fwd(lib.Context(), d, q.cuda(), k.cuda(), v.cuda(), table.cuda(), None, None, o, None,
                            lib.workspace(lib.paragan_mha_sizes(d)[1]))
        against({"o": o}, q, k, v, do, table, **kw)


@pytest.mark.parametrize("case", [
    # Sq, Hq, Hk, d, causal, window, sink, nb, maxd, masked bucket
    (2100, 4, 1, 64, 1, 64, 5, 16, 40, 0), (700, 6, 2, 96, 1, 0, 0, 256, 512, 200), (600, 2, 2, 128, 0, 100, 130, 130, 300, 129),
    (130, 8, 1, 40, 1, 1, 0, 8, 20, 0)])
def test_masked_bucket_in_split_blocks_and_wide_tables(case):
    """A lowest-value bucket of one head of a group: key blocks that are split, tables wider than a wave, a far bucket, and
    rows (window of one) that see it alone."""
    torch = need_gpu()
    Sq, Hq, Hk, d, causal, window, sink, nb, maxd, bucket = case
    print("masked bucket", case, flush=True)
    (q, k, v, do), gen = inputs(torch, 6, 1, Sq, Sq, Hq, Hk, d)
    table = torch.randn(Hq, nb, generator=gen)
    table[Hq - 1, bucket] = LOWEST
    kw = dict(causal=causal, window=window, n_sink=sink, max_distance=maxd)
    against(trained(q, k, v, do, table, **kw), q, k, v, do, table, **kw)


def test_masked_bias_captured_and_replayed():
    """A captured pass whose table changes between replays, from ordinary values to masks and back."""
    torch = need_gpu()
    (q, k, v, do), gen = inputs(torch, 7, 1, 170, 170, 2, 1, 64)
    side = torch.cuda.Stream()
    ctx = lib.Context(side)
    q, k, v, do, table = (t.cuda() for t in (q, k, v, do, torch.randn(2, 8, generator=gen)))
    out = [torch.empty_like(t) for t in (q, q, k, v, table)]
    d = lib.mha_desc(q, k, v, out[0], scale=0.125, causal=1, n_buckets=8, max_distance=30)
    sb, wb = lib.paragan_mha_sizes(d)
    saved, ws = lib.workspace(sb), lib.workspace(wb)

    def run():
        lib.paragan_mha_fwd(ctx, d, q, k, v, table, None, None, out[0], saved, ws)
        lib.paragan_mha_bwd(ctx, d, q, k, v, table, None, None, out[0], saved, do, out[1], out[2], out[3], out[4], ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        run()
    base = table.clone()
    for rep, value in enumerate((LOWEST, None, -1e9, None)):
        table.copy_(base)
        if value is not None:
            table[:, 0] = value
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        for t in out:
            t.fill_(9.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(out, want)), rep


@pytest.mark.parametrize("lq,lk", [([140, 77, 1, 0], [140, 77, 1, 0]), ([140, 90, 7, 3], [30, 0, 50, 129])])
def test_masked_bucket_in_ragged_batches(lq, lk):
    """Padded batches, rows that see nothing among them, with the nearest bucket of two heads at the lowest value."""
    def low(t):
        t = t.clone()
        t[:2, 0] = LOWEST
        return t
    for causal, window in ((1, 0), (1, 20), (0, 20)):
        mha_case(4, 140, 140, 4, 2, 64, causal, window, 3 if window else 0, 16, 60, lq, lk, seed=71, tab=low)
        mha_case(4, 140, 140, 4, 2, 128, causal, window, 3 if window else 0, 16, 60, lq, lk, seed=72, tab=low, train=False)


@pytest.mark.parametrize("value", [LOWEST, -math.inf, -1e4, -40.0])
@pytest.mark.parametrize("causal,window", [(0, 0), (1, 0), (0, 120)])
def test_gradient_of_far_buckets_that_hold_nothing(value, causal, window):
    """The buckets past max_distance take a share of their rows that is zero (or e^-40): so is their gradient, with nothing in
    it of what rounding leaves of the rest."""
    torch = need_gpu()
    print("far buckets", value, causal, window, flush=True)
    (q, k, v, do), gen = inputs(torch, 8, 1, 300, 300, 2, 1, 64)
    table = torch.randn(2, 8, generator=gen)
    table[0, 7], table[1, 7] = value, value
    if not causal:
        table[1, 3] = value
    kw = dict(causal=causal, window=window, max_distance=40)
    out = trained(q, k, v, do, table, **kw)
    against(out, q, k, v, do, table, **kw)
    if value < -100:
        assert not out["dtable"][:, 7].any()
