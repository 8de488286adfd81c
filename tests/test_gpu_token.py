"""GPU parity of the token attention operators with their float64 definitions:
norms of query and key heads with the rotation, attention with window, first
tokens, ragged lengths and relative position bias, forward and backward.

Each output is held to an elementwise bound made of half steps: the outputs'
own rounding (bf16 2^-8, fp32 2^-24), the rounding of P and dS as matrix
operands, and fp32 statistics and sums (oracle/token.py)."""
import math

import numpy as np
import pytest

from oracle import token as T
from paragan_2411_03999_amd import lib

from .parity import need_gpu

pytestmark = pytest.mark.gpu

U16, U32 = T.U16, T.U32


def held(name, got, want, tol):
    got = got.detach().double().cpu().numpy()
    assert np.all(np.isfinite(got)), name + ": not finite"
    bad = np.abs(got - want) - tol
    worst = np.unravel_index(np.argmax(bad), bad.shape)
    print("  %s: max error %.3g, largest share of the bound %.3f" %
          (name, np.abs(got - want).max(), (np.abs(got - want) / np.maximum(tol, 1e-300)).max()), flush=True)
    assert bad[worst] <= 0, "%s%s: %.9g, not %.9g (bound %.3g)" % (name, worst, got[worst], want[worst], tol[worst])


# ------------------------------------------------------------- norm and rotation
def qknorm_case(T_, Hq, Hk, d, rot, inter, f32, pad=0, seed=0, pos_null=False, n_pos=50, scale=1.0, inplace=False):
    torch = need_gpu()
    print("qknorm", dict(T=T_, Hq=Hq, Hk=Hk, d=d, rot=rot, inter=inter, f32=f32, pad=pad, seed=seed), flush=True)
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if f32 else torch.bfloat16
    rn = lambda *s: (torch.randn(s, generator=gen) * scale)  # noqa: E731
    buf = torch.full((T_, (Hq + Hk) * d + pad), float("nan"), dtype=dt)     # q | k, then `pad` elements nobody owns
    buf[:, :(Hq + Hk) * d] = rn(T_, (Hq + Hk) * d).to(dt)
    g = [1 + 0.2 * torch.randn(d, generator=gen) for _ in range(2)]
    ang = torch.rand(n_pos, max(rot // 2, 1), generator=gen, dtype=torch.float64) * 100
    table = torch.stack([ang.cos(), ang.sin()], -1).float()
    pos = torch.randint(-1, n_pos + 1, (T_,), generator=gen, dtype=torch.int32)   # some outside on either side
    if pos_null:
        pos = torch.arange(T_, dtype=torch.int32) % n_pos
    dys = [rn(T_, h, d).to(dt) for h in (Hq, Hk)]
    B = buf.cuda()
    q, k = B[:, :Hq * d].unflatten(1, (Hq, d)), B[:, Hq * d:(Hq + Hk) * d].unflatten(1, (Hk, d))
    G, tab = [t.cuda() for t in g], table.cuda() if rot else None
    P = None if pos_null else pos.cuda()
    ctx = lib.Context()
    # backward first: the forward may overwrite its inputs
    dB = torch.full_like(B, 7.0)
    dq, dk = dB[:, :Hq * d].unflatten(1, (Hq, d)), dB[:, Hq * d:(Hq + Hk) * d].unflatten(1, (Hk, d))
    DY = [t.cuda() for t in dys]
    kw = dict(rot=rot, interleaved=inter, n_pos=n_pos, eps=1e-5)
    desc = lib.qknorm_desc(q, k, **kw)
    dg = torch.full((2, d), 7.0, device="cuda")
    ws = lib.workspace(lib.paragan_qknorm_ws_size(desc))
    lib.paragan_qknorm_bwd(ctx, desc, q, k, G[0], G[1], tab, P, DY[0], DY[1], dq, dk, dg[0], dg[1], ws)
    x0 = [t.detach().double().cpu().numpy() for t in (q, k)]
    if inplace:
        desc, outs = lib.qknorm_desc(q, k, q, k, **kw), (q, k)
    else:
        outs = [torch.full((T_, h, d), 7.0, dtype=dt, device="cuda") for h in (Hq, Hk)]
    lib.paragan_qknorm_fwd(ctx, desc, q, k, G[0], G[1], tab, P, outs[0], outs[1])
    torch.cuda.synchronize()
    if pad:
        assert bool((dB[:, (Hq + Hk) * d:] == 7.0).all())
    uo = U32 if f32 else U16
    tb, pn = table.double().numpy()[:, :rot // 2], pos.numpy()
    for i, n in enumerate("qk"):
        x, gn, dy = x0[i], g[i].double().numpy(), dys[i].double().numpy()
        y = T.qknorm_fwd(x, gn, tb, pn, rot, inter, 1e-5)
        # the size of what is added: |n| turned with |cos|, |sin|
        mag = T.qknorm_fwd(np.abs(x), np.abs(gn), np.abs(tb), pn, rot, inter, 1e-5)
        mag = np.maximum(np.abs(mag), np.abs(T.qknorm_fwd(np.abs(x), np.abs(gn), np.abs(tb) * [1, -1], pn, rot, inter, 1e-5)))
        held(n, outs[i], y, uo * np.abs(y) + U32 * (d / 2 + 16) * mag + 1e-30)
        dx, dgain = T.qknorm_bwd(x, gn, tb, pn, rot, inter, 1e-5, dy)
        real = ((pn >= 0) & (pn < n_pos))[:, None, None]
        xx = np.where(real, x, 0.0)
        r = 1 / np.sqrt((xx * xx).mean(-1, keepdims=True) + 1e-5)
        dn = np.where(real, np.sqrt((dy * dy).sum(-1, keepdims=True)), 0.0) * np.ones(d)    # any element after the turn
        big = r * (dn * np.abs(gn) + np.abs(xx) * r * r * (dn * np.abs(gn) * np.abs(xx)).mean(-1, keepdims=True))
        held("d" + n, (dq, dk)[i], dx, uo * np.abs(dx) + U32 * (d + 24) * big + 1e-30)
        terms = (np.abs(dn * xx * r)).sum((0, 1))
        held("dgain_" + n, dg[i], dgain, U32 * (T_ / 8 + d + 1100) * terms + 1e-30)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("case", [
    (1, 1, 1, 8, 0, 0), (1, 3, 1, 16, 16, 0), (7, 4, 2, 32, 32, 1), (63, 8, 8, 64, 64, 0), (65, 5, 3, 80, 48, 1),
    (33, 32, 8, 128, 128, 0), (130, 6, 1, 128, 64, 1), (17, 2, 2, 256, 256, 0), (9, 3, 3, 200, 176, 0),
    (2000, 4, 4, 24, 16, 1)])
def test_qknorm(case, f32):
    qknorm_case(*case, f32, pad=8, seed=sum(case))


def test_qknorm_many_tokens_wrap_the_table():
    qknorm_case(20011, 3, 1, 64, 32, 0, False, pos_null=True)      # more items than one round of the grid


def test_qknorm_in_place_and_far_values():
    qknorm_case(50, 4, 2, 64, 64, 0, False, inplace=True)
    qknorm_case(20, 4, 2, 40, 16, 1, True, scale=1e6)
    qknorm_case(20, 4, 2, 40, 16, 0, True, scale=1e-6)              # eps decides


def test_qknorm_padding_is_not_read():
    torch = need_gpu()
    q = torch.full((3, 2, 32), float("nan"), dtype=torch.bfloat16, device="cuda")
    q[1] = 1.0
    table = torch.full((2, 16, 2), float("nan"), device="cuda")
    table[1, :, 0], table[1, :, 1] = 1.0, 0.0
    pos = torch.tensor([-5, 1, 2], dtype=torch.int32, device="cuda")
    o = torch.full_like(q, 9.0)
    ok = torch.full_like(q, 9.0)
    one = torch.ones(32, device="cuda")
    d = lib.qknorm_desc(q, q, rot=32, interleaved=0, n_pos=2, eps=1e-6)
    ctx = lib.Context()
    lib.paragan_qknorm_fwd(ctx, d, q, q, one, one, table, pos, o, ok)
    dq, dk, dg = torch.empty_like(q), torch.empty_like(q), torch.empty(2, 32, device="cuda")
    lib.paragan_qknorm_bwd(ctx, d, q, q, one, one, table, pos, q, q, dq, dk, dg[0], dg[1],
                           lib.workspace(lib.paragan_qknorm_ws_size(d)))
    torch.cuda.synchronize()
    for t in (o, ok):
        assert not t[0].any() and not t[2].any() and bool((t[1] == 1.0).all())
    for t in (dq, dk):
        assert not t[0].any() and not t[2].any() and bool(torch.isfinite(t).all())
    assert bool(torch.isfinite(dg).all())


def test_qknorm_gain_sums_beside_a_large_term():
    """Gain gradients that are a sum over tokens, one of them 2^26: every block's partial but one is 256 x 3/256 = 3, below
    half a step of the large one, so joining in 32 bits loses those that meet it.  The blocks' partials are rounded once
    (the large one by 4 at most) and so is the result (by 4)."""
    torch = need_gpu()
    T_, d = 131072, 8
    print("gain sums", T_, flush=True)
    x = torch.ones(T_, 1, d, device="cuda")
    dy = torch.full((T_, 1, d), 3.0 / 256, device="cuda")
    dy[0] = 2.0 ** 26
    one, dg = torch.ones(d, device="cuda"), torch.empty(2, d, device="cuda")
    ds = lib.qknorm_desc(x, x, rot=0, interleaved=0, n_pos=1, eps=1e-12)          # 1 / sqrt(1 + 1e-12) is 1 in float32
    lib.paragan_qknorm_bwd(lib.Context(), ds, x, x, one, one, None, None, dy, dy, torch.empty_like(x), torch.empty_like(x), dg[0],
                           dg[1], lib.workspace(lib.paragan_qknorm_ws_size(ds)))
    torch.cuda.synchronize()
    want = 2.0 ** 26 + (T_ - 1) * 3.0 / 256
    print("  off by", (dg.double() - want).abs().max().item(), flush=True)
    assert bool(((dg.double() - want).abs() <= 8.0).all())


def test_qknorm_least_eps():
    """Zero rows and padding under the least eps taken: zeros, and gradients of zero rows that are r t."""
    torch = need_gpu()
    x = torch.zeros(4, 2, 16, device="cuda")
    x[1] = 1.0
    pos = torch.tensor([0, 0, 0, -1], dtype=torch.int32, device="cuda")
    one, out, dx, dg = torch.ones(16, device="cuda"), torch.empty(2, 4, 2, 16, device="cuda"), torch.empty(2, 4, 2, 16, device="cuda"), torch.empty(2, 16, device="cuda")
    eps = float(np.finfo(np.float32).tiny)
    d = lib.qknorm_desc(x, x, rot=0, interleaved=0, n_pos=1, eps=eps)
    ctx = lib.Context()
    lib.paragan_qknorm_fwd(ctx, d, x, x, one, one, None, pos, out[0], out[1])
    dy = torch.full_like(x, 2.0 ** -20)
    lib.paragan_qknorm_bwd(ctx, d, x, x, one, one, None, pos, dy, dy, dx[0], dx[1], dg[0], dg[1],
                           lib.workspace(lib.paragan_qknorm_ws_size(d)))
    torch.cuda.synchronize()
    for t in range(2):
        assert not out[t][[0, 2, 3]].any() and bool((out[t][1] == 1.0).all())
        # 2^-20 / sqrt(2^-126) = 2^43, a reciprocal root being off by a step at most
        assert bool(((dx[t][[0, 2]] / 2.0 ** 43 - 1).abs() <= 2 * 2.0 ** -23).all()) and not dx[t][3].any()
    assert bool(torch.isfinite(dg).all())


# ------------------------------------------------------------- attention
def mha_case(B, Sq, Sk, Hq, Hk, d, causal=0, window=0, sink=0, nb=0, maxd=0, lq=None, lk=None, train=True, seed=0,
             layout="fused", scale=None, tab=None, poison=True):
    torch = need_gpu()
    print("mha", dict(B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hk=Hk, d=d, causal=causal, window=window, sink=sink, nb=nb, maxd=maxd,
                      lq=lq, lk=lk, train=train, seed=seed, layout=layout), flush=True)
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=gen).bfloat16()  # noqa: E731
    q, k, v, do = rn(B, Sq, Hq, d), rn(B, Sk, Hk, d), rn(B, Sk, Hk, d), rn(B, Sq, Hq, d)
    table = torch.randn(Hq, nb, generator=gen) if nb else None
    if tab is not None:
        table = tab(table)
    scale = scale or 1 / math.sqrt(d)
    n = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    want = T.mha(n(q), n(k), n(v), float(np.float32(scale)), causal, window, sink, n(table), maxd, lq, lk, n(do) if train else None)
    if poison:      # what nobody may read
        for b in range(B):
            k[b, Sk if lk is None else lk[b]:] = float("nan")
            v[b, Sk if lk is None else lk[b]:] = float("inf")
            q[b, Sq if lq is None else lq[b]:] = float("nan")
            do[b, Sq if lq is None else lq[b]:] = float("nan")

    def place(t):   # the same values in another layout
        if layout == "heads":                                    # [B][H][S][d]
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        pad = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2] + 1, t.shape[3]), 7.0, dtype=t.dtype)
        pad[:, :t.shape[1], :t.shape[2]] = t
        return pad.cuda()[:, :t.shape[1], :t.shape[2]]
    Q, K, V, DO = place(q), place(k), place(v), place(do)
    O = place(torch.full_like(q, 5.0))
    t32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    LQ, LK, TB = t32(lq), t32(lk), None if table is None else table.cuda()
    desc = lib.mha_desc(Q, K, V, O, scale=scale, causal=causal, window=window, n_sink=sink, n_buckets=nb, max_distance=maxd)
    sb, wb = lib.paragan_mha_sizes(desc)
    ctx, ws = lib.Context(), lib.workspace(wb)
    ws.fill_(255)
    saved = lib.workspace(sb) if train else None
    lib.paragan_mha_fwd(ctx, desc, Q, K, V, TB, LQ, LK, O, saved, ws)
    out = {"o": O}
    if train:
        ws.fill_(255)
        out.update(dq=place(torch.full_like(q, 5.0)), dk=place(torch.full_like(k, 5.0)), dv=place(torch.full_like(v, 5.0)))
        if nb:
            out["dtable"] = torch.full((Hq, nb), 5.0, device="cuda")
        lib.paragan_mha_bwd(ctx, desc, Q, K, V, TB, LQ, LK, O, saved, DO, out["dq"], out["dk"], out["dv"],
                            out.get("dtable"), ws)
    torch.cuda.synchronize()
    for name, t in out.items():
        held(name, t, want[name], want["tol." + name] + 1e-30)
        if layout != "heads" and name != "dtable":               # the rows and heads around it stay as they were
            base = t._base
            assert bool((base[:, t.shape[1]:] == 7.0).all()) and bool((base[:, :, t.shape[2]:] == 7.0).all()), name
    return out


TRAIN = [
    # B, Sq, Sk, Hq, Hk, d, causal, window, sink, nb, maxd
    (1, 1, 1, 1, 1, 8), (2, 5, 5, 2, 1, 32, 1), (1, 33, 33, 3, 3, 64), (2, 64, 64, 4, 2, 128, 1),
    (1, 127, 127, 2, 2, 96), (1, 300, 300, 2, 1, 80, 1), (1, 257, 257, 4, 1, 64, 0, 0, 0, 32, 128),
    (2, 150, 150, 2, 2, 32, 1, 0, 0, 16, 64), (1, 290, 290, 2, 1, 128, 1, 40, 0), (1, 290, 290, 2, 2, 64, 1, 33, 5),
    (1, 260, 260, 2, 1, 40, 0, 20, 70), (1, 300, 300, 2, 2, 64, 0, 100, 0, 8, 20), (1, 400, 400, 1, 1, 32, 1, 64, 4, 32, 512),
    (1, 1100, 1100, 1, 1, 24, 0, 0, 0, 64, 512), (1, 70, 200, 2, 2, 64, 1), (1, 200, 70, 2, 1, 64, 1),
    (1, 65, 130, 2, 1, 32, 0, 30, 3, 12, 40), (3, 96, 96, 8, 1, 64, 1, 1, 0), (1, 96, 96, 2, 2, 16, 1, 1, 1, 2, 2),
    (1, 513, 513, 2, 2, 128, 0, 0, 0, 32, 128), (1, 600, 600, 1, 1, 128, 1, 100, 200, 16, 50),
    (1, 2100, 2100, 4, 1, 64, 1, 64, 5), (1, 1500, 1500, 2, 2, 32, 0, 90, 130),
    (1, 100, 100, 1, 1, 32, 1, 10, 1000), (1, 100, 100, 1, 1, 32, 0, 1 << 29, 1 << 29), (1, 200, 200, 2, 1, 32, 1, 1 << 29)]


@pytest.mark.parametrize("case", TRAIN, ids=[("-".join(map(str, c))) for c in TRAIN])
def test_mha_train(case):
    mha_case(*case, seed=len(case) + case[1])


@pytest.mark.parametrize("causal,window,sink,nb", [(1, 0, 0, 0), (1, 20, 3, 16), (0, 0, 0, 16), (0, 9, 2, 0)])
def test_mha_ragged(causal, window, sink, nb):
    """Padded batch: full, odd, one token, none; behind the lengths lie NaN and infinities."""
    n = [140, 77, 1, 0]
    mha_case(4, 140, 140, 4, 2, 64, causal, window, sink, nb, 60 if nb else 0, n, n, seed=1)
    mha_case(4, 140, 140, 4, 2, 64, causal, window, sink, nb, 60 if nb else 0, n, n, train=False, layout="heads")


def test_mha_more_queries_than_keys_leaves_empty_rows():
    mha_case(3, 90, 90, 2, 1, 64, 1, 0, 0, 8, 30, [90, 40, 7], [30, 0, 50], seed=3)
    mha_case(2, 90, 90, 2, 1, 32, 1, 10, 4, 0, 0, [90, 12], [30, 12], seed=4)


@pytest.mark.parametrize("causal,window,sink", [(1, 0, 0), (1, 20, 3), (0, 20, 0)])
def test_mha_key_blocks_behind_the_last_key(causal, window, sink):
    """Caches far longer than their sequences, with few queries: the key blocks behind the last key have no query tile to
    walk (the first of their queries would lie past the rows of a head), and their gradients are zeros."""
    mha_case(3, 40, 700, 4, 2, 64, causal, window, sink, 0, 0, [33, 0, 7], [5, 3, 300], seed=21)
    mha_case(3, 40, 700, 2, 1, 128, causal, window, sink, 8, 30, [33, 0, 7], [5, 3, 300], seed=22)


STEP = [
    (1, 1, 1, 1, 1, 8, 1), (3, 1, 40, 4, 4, 64, 1), (2, 1, 1000, 32, 8, 128, 1), (2, 4, 777, 8, 1, 96, 1),
    (1, 1, 5000, 16, 2, 64, 1, 300, 4, 32, 128), (2, 3, 900, 10, 1, 32, 1, 64, 40), (1, 1, 4000, 8, 8, 128, 0, 0, 0, 16, 512),
    (2, 2, 650, 16, 1, 64, 1, 0, 0, 256, 512), (1, 32, 333, 1, 1, 40, 1, 7, 1, 8, 16), (1, 16, 100, 2, 1, 128, 0, 5, 3),
    (1, 100, 2000, 4, 2, 64, 1), (2, 5, 700, 24, 2, 128, 1, 90, 2, 16, 40), (1, 130, 260, 1, 1, 32, 0, 0, 0, 200, 300)]


@pytest.mark.parametrize("case", STEP, ids=[("-".join(map(str, c))) for c in STEP])
def test_mha_step(case):
    """A few new queries over a cache, whole and ragged."""
    mha_case(*case, train=False, seed=5)
    B, Sq, Sk = case[:3]
    lk = [max(1, Sk - 17 * b - Sk // 3) for b in range(B)]
    lq = [Sq if b % 2 == 0 else max(0, Sq - 1) for b in range(B)]
    mha_case(*case, lq=lq, lk=lk, train=False, seed=6, layout="heads")


def test_mha_forward_alone_of_many_rows():
    """Without a backward to follow, and too many rows for the form of few."""
    mha_case(20, 40, 40, 8, 8, 32, 1, 0, 0, 8, 20, train=False, seed=13)
    mha_case(20, 40, 55, 8, 8, 72, 0, 9, 2, lq=[2 * b for b in range(20)], lk=[55 - b for b in range(20)], train=False, seed=14)


def test_mha_step_reads_only_what_is_seen():
    """Old rows of a cache outside the window and the first tokens hold NaN and infinities."""
    torch = need_gpu()
    Sk, w, sink = 700, 50, 3
    print("step with an evicted cache", flush=True)
    gen = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(1, s, h, 64, generator=gen).bfloat16() for s, h in ((1, 4), (Sk, 2), (Sk, 2)))
    n = lambda t: t.double().numpy()  # noqa: E731
    want = T.mha(n(q), n(k), n(v), 0.125, True, w, sink)
    k[:, sink:Sk - w], v[:, sink:Sk - w] = float("nan"), float("inf")
    Q, K, V = q.cuda(), k.cuda(), v.cuda()
    O = torch.empty_like(Q)
    d = lib.mha_desc(Q, K, V, O, scale=0.125, causal=1, window=w, n_sink=sink)
    sb, wb = lib.paragan_mha_sizes(d)
    for saved in (None, lib.workspace(sb)):
        lib.paragan_mha_fwd(lib.Context(), d, Q, K, V, None, None, None, O, saved, lib.workspace(wb))
        held("o", O, want["o"], want["tol.o"])


@pytest.mark.parametrize("S,Hq,Hk,causal", [(1024, 2, 2, 1), (1000, 4, 1, 1), (1003, 6, 2, 0)])
def test_mha_few_heads_visit_only_their_window(S, Hq, Hk, causal):
    """Long sequences of few heads take the form of few rows, whose tiles are of 32 rows: each walks the keys that its own
    queries see, so that a NaN among the values reaches no query further off than a tile of rows and one of keys."""
    torch = need_gpu()
    print("few heads, window", S, Hq, Hk, causal, flush=True)
    gen, w, at = torch.Generator().manual_seed(61), 16, 500
    q, k, v = (torch.randn(1, S, h, 64, generator=gen).bfloat16().cuda() for h in (Hq, Hk, Hk))
    o = [torch.empty_like(q) for _ in range(2)]
    d = lib.mha_desc(q, k, v, o[0], scale=0.125, causal=causal, window=w)
    ws = lib.workspace(lib.paragan_mha_sizes(d)[1])
    for out in o:
        lib.paragan_mha_fwd(lib.Context(), d, q, k, v, None, None, None, out, None, ws)
        torch.cuda.synchronize()
        v[0, at, 0] = float("nan")
    i = torch.arange(S)
    meets = (i - at >= 0 if causal else i - at > -w) & (i - at < w)
    assert bool(torch.isnan(o[1][0, meets, 0]).all())
    far = (i - at).abs() >= w + 64
    assert torch.equal(o[0][0, far], o[1][0, far])


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("Sq,Sk,causal,window,sink,lq,lk", [(65, 130, 0, 30, 3, None, None), (65, 330, 1, 30, 3, None, None),
                                                            (20, 200, 1, 9, 0, [20, 3], [200, 77])])
def test_mha_training_reads_only_what_is_seen(Sq, Sk, causal, window, sink, lq, lk, d):
    """Keys and values that no query sees hold NaN and infinities, beside seen ones: their gradients are zeros."""
    torch = need_gpu()
    print("training, unseen keys", Sq, Sk, causal, window, sink, d, flush=True)
    B, gen = 2, torch.Generator().manual_seed(51)
    q, k, v, do = (torch.randn(B, s, h, d, generator=gen).bfloat16() for s, h in ((Sq, 2), (Sk, 1), (Sk, 1), (Sq, 2)))
    n = lambda t: t.double().numpy()  # noqa: E731
    want = T.mha(n(q), n(k), n(v), 0.125, causal, window, sink, len_q=lq, len_k=lk, dout=n(do))
    for b in range(B):
        nq, nk = (Sq, Sk) if lq is None else (lq[b], lk[b])
        unseen = ~T.visible(np.arange(nq) + nk - nq, np.arange(Sk), nk, causal, window, sink).any(0)
        assert 0 < unseen.sum() < Sk and not want["dk"][b, unseen].any()
        k[b, unseen], v[b, unseen] = float("nan"), float("inf")
    Q, K, V, DO = (t.cuda() for t in (q, k, v, do))
    out = {"o": torch.empty_like(Q), "dq": torch.empty_like(Q), "dk": torch.empty_like(K), "dv": torch.empty_like(V)}
    LQ, LK = (None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lq, lk))
    ds = lib.mha_desc(Q, K, V, out["o"], scale=0.125, causal=causal, window=window, n_sink=sink)
    sb, wb = lib.paragan_mha_sizes(ds)
    ctx, ws, saved = lib.Context(), lib.workspace(wb), lib.workspace(sb)
    lib.paragan_mha_fwd(ctx, ds, Q, K, V, None, LQ, LK, out["o"], saved, ws)
    lib.paragan_mha_bwd(ctx, ds, Q, K, V, None, LQ, LK, out["o"], saved, DO, out["dq"], out["dk"], out["dv"], None, ws)
    torch.cuda.synchronize()
    for name, t in out.items():
        held(name, t, want[name], want["tol." + name] + 1e-30)


def test_mha_lowest_and_infinite_bias():
    """-infinity hides keys (all of them: zeros); the lowest finite value everywhere leaves the softmax of equal scores."""
    torch = need_gpu()

    def hide(t):
        t = t.clone()
        t[0, 3:] = -math.inf          # head 0 sees the nearest three distances
        t[1, :] = -math.inf           # head 1 nothing
        t[2, 1:] = torch.finfo(torch.float32).min
        return t
    for train in (True, False):
        mha_case(1, 70, 70, 3, 3, 32, 1, 0, 0, 8, 30, tab=hide, seed=8, train=train)
    mha_case(1, 1, 70, 3, 1, 32, 1, 0, 0, 8, 30, tab=hide, seed=8, train=False)
    low = torch.full((1, 4), torch.finfo(torch.float32).min, device="cuda")
    for Sq in (1, 50):
        q, k = (torch.randn(1, s, 1, 32, device="cuda").bfloat16() for s in (Sq, 50))
        v = torch.randn(1, 50, 1, 32, device="cuda").bfloat16()
        o = torch.empty_like(q)
        d = lib.mha_desc(q, k, v, o, scale=1e-3, n_buckets=4, max_distance=9)
        lib.paragan_mha_fwd(lib.Context(), d, q, k, v, low, None, None, o, None, lib.workspace(lib.paragan_mha_sizes(d)[1]))
        mean = v.double().mean(1, keepdim=True).expand(1, Sq, 1, 32).cpu().numpy()
        held("o", o, mean, (3 * U16) * np.abs(v.double().cpu().numpy()).mean() + np.zeros_like(mean))


@pytest.mark.parametrize("Sq,Sk,Hq,Hk,causal,window", [(300, 300, 2, 1, 0, 0), (300, 300, 2, 1, 1, 0), (300, 300, 40, 40, 1, 90),
                                                       (1, 300, 4, 2, 1, 0), (3, 3000, 2, 1, 1, 0), (5, 700, 1, 1, 0, 200)])
def test_mha_lowest_bias_alone(Sq, Sk, Hq, Hk, causal, window):
    """The lowest finite value in every bucket: scores vanish in it, near the diagonal and far from it, so that each row is
    the mean of the values that it sees, also where scores pass what an exponential holds."""
    def low(t):
        return torch.full_like(t, torch.finfo(torch.float32).min)
    torch = need_gpu()
    for scale in (None, 8.0):
        mha_case(1, Sq, Sk, Hq, Hk, 64, causal, window, 0, 8, 9, tab=low, train=False, seed=41, scale=scale)


def test_mha_large_scores():
    """Scores of a few hundred: the running maximum moves, nothing overflows."""
    for train in (True, False):
        mha_case(1, 200, 200, 2, 1, 64, 1, scale=8.0, seed=11, train=train)
    mha_case(1, 2, 600, 8, 1, 64, 1, scale=8.0, seed=12, train=False)


@pytest.mark.parametrize("Sq,Sk,Hq,Hk,train,nb", [(150, 150, 2, 1, True, 0), (150, 150, 2, 2, True, 8), (300, 300, 64, 64, False, 0),
                                                  (2, 200, 4, 1, False, 8), (1, 3000, 4, 2, False, 0)])
def test_mha_nan_comes_out(Sq, Sk, Hq, Hk, train, nb):
    """A NaN or infinity in a query, and a NaN in a key, make the outputs of the rows that meet it NaN (forward, backward,
    few rows, few rows with split keys); other rows keep their bits."""
    torch = need_gpu()
    print("nan", Sq, Sk, Hq, Hk, train, nb, flush=True)
    gen = torch.Generator().manual_seed(31)
    q, k, v, do = (torch.randn(1, s, h, 64, generator=gen).bfloat16().cuda() for s, h in ((Sq, Hq), (Sk, Hk), (Sk, Hk), (Sq, Hq)))
    table = torch.randn(Hq, nb, generator=gen).cuda() if nb else None

    def run(q, k):
        o, dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
        dt = torch.empty_like(table) if nb else None
        d = lib.mha_desc(q, k, v, o, scale=0.125, causal=1, n_buckets=nb, max_distance=30 if nb else 0)
        sb, wb = lib.paragan_mha_sizes(d)
        ctx, ws, saved = lib.Context(), lib.workspace(wb), lib.workspace(sb) if train else None
        lib.paragan_mha_fwd(ctx, d, q, k, v, table, None, None, o, saved, ws)
        if train:
            lib.paragan_mha_bwd(ctx, d, q, k, v, table, None, None, o, saved, do, dq, dk, dv, dt, ws)
        torch.cuda.synchronize()
        return o, dq, dk, dv, dt
    ref = run(q, k)
    row, h = Sq // 2, Hq - 1
    hk = h // (Hq // Hk)
    for bad in (float("nan"), float("inf")):
        q2 = q.clone()
        q2[0, row, h, 5] = bad
        got = run(q2, k)
        for i in ((0, 1) if train else (0,)):
            assert bool(torch.isnan(got[i][0, row, h]).all()), i
            same = got[i].clone()
            same[0, row, h] = ref[i][0, row, h]
            assert torch.equal(same, ref[i]), i
        if train:        # every key up to the row's own position
            assert not bool(torch.isfinite(got[2][0, :row + 1, hk].float()).all(-1).any())
            assert bool(torch.isnan(got[3][0, :row + 1, hk]).all())
            assert bool(torch.isnan(got[4][h]).any()) if nb else True
    k2, key = k.clone(), Sk - Sq // 2 - 1
    k2[0, key, hk, 3] = float("nan")
    got = run(q, k2)
    first = key - (Sk - Sq)                                       # the first query that sees it
    for hh in range(Hq):
        if hh // (Hq // Hk) == hk:
            assert bool(torch.isnan(got[0][0, max(first, 0):, hh]).all())
            assert torch.equal(got[0][0, :max(first, 0), hh], ref[0][0, :max(first, 0), hh])
        else:
            assert torch.equal(got[0][:, :, hh], ref[0][:, :, hh])


@pytest.mark.parametrize("nb,maxd,causal", [(32, 128, 1), (32, 128, 0), (2, 2, 1), (4, 500, 0), (64, 100, 1), (256, 512, 0)])
def test_every_bucket(nb, maxd, causal):
    """One query over keys at every distance, equal scores: o is the softmax of the bias alone."""
    torch = need_gpu()
    S, i = 1100, 550
    table = torch.linspace(-3, 3, nb)[None]
    v = torch.randn(1, S, 1, 8, generator=torch.Generator().manual_seed(3)).bfloat16()
    q = torch.zeros(1, S, 1, 8).bfloat16()
    want = T.mha(q.double().numpy(), q.double().numpy(), v.double().numpy(), 1.0, causal, 0, 0, table.double().numpy(), maxd)
    Q, V, TB = q.cuda(), v.cuda(), table.cuda()
    O = torch.empty_like(Q)
    d = lib.mha_desc(Q, Q, V, O, scale=1.0, causal=causal, n_buckets=nb, max_distance=maxd)
    lib.paragan_mha_fwd(lib.Context(), d, Q, Q, V, TB, None, None, O, None, lib.workspace(lib.paragan_mha_sizes(d)[1]))
    held("o", O, want["o"], want["tol.o"])
    # and a single query in the middle through the few-row form
    lk = torch.tensor([i + 1], dtype=torch.int32, device="cuda")
    q1, o1 = Q[:, :1].contiguous(), torch.empty(1, 1, 1, 8, dtype=torch.bfloat16, device="cuda")
    d = lib.mha_desc(q1, Q, V, o1, scale=1.0, causal=causal, n_buckets=nb, max_distance=maxd)
    lib.paragan_mha_fwd(lib.Context(), d, q1, Q, V, TB, None, lk, o1, None, lib.workspace(lib.paragan_mha_sizes(d)[1]))
    w1 = T.mha(q[:, :1].double().numpy(), q.double().numpy(), v.double().numpy(), 1.0, causal, 0, 0, table.double().numpy(),
               maxd, None, [i + 1])
    held("o1", o1, w1["o"], w1["tol.o"])
