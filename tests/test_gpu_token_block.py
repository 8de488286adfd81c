"""GPU parity of the token block's operators with their float64 definitions:
norms around a block with modulation, gate and residual scale, the gated
linear recurrence, forward and backward, and clipping by the norm of all
gradients.

Each output is held to an elementwise bound made of half steps
(oracle/token_block.py).  What no token owns (rows past a sequence's length,
columns between rows) holds NaN on input and must be left alone or zeroed."""
import math

import numpy as np
import pytest

from oracle import token_block as T
from paragan_2411_03999_amd import lib

from .parity import need_gpu
from .test_gpu_token import held

pytestmark = pytest.mark.gpu

U16, U32 = T.U16, T.U32


def num(t):
    return t.detach().double().cpu().numpy()


class Rows:
    """A [B][S][D] tensor inside a wider buffer, NaN (or `fill`) where nobody owns it; head: rows ahead of each sequence."""

    def __init__(self, torch, B, S, D, dt, pad=8, head=1, fill=float("nan")):
        self.buf = torch.full((B, S + head, D + 2 * pad), fill, dtype=dt, device="cuda")
        self.v = self.buf[:, head:, pad:pad + D]
        self.pad, self.head, self.D = pad, head, D

    def set(self, t, lens, rest=float("nan")):
        self.v.copy_(t)
        for b, n in enumerate(lens):
            self.v[b, n:] = rest
        return self

    def untouched(self, fill):
        b = self.buf
        parts = [b[:, :self.head], b[:, :, :self.pad], b[:, :, self.pad + self.D:]]
        return all(bool((p == fill).all()) for p in parts)


# ------------------------------------------------------------- norms around a block
def blocknorm_case(B, S, D, *, layer=0, branch=1, post=0, pre=1, f32=0, res32=0, shared=0, lens=None, rows="all", dz=1, scale=1.0,
                   pad=8, seed=0, repeat=1):
    torch = need_gpu()
    print("blocknorm", dict(B=B, S=S, D=D, layer=layer, branch=branch, post=post, pre=pre, f32=f32, res32=res32, shared=shared, lens=lens,
                            rows=rows, dz=dz, scale=scale, seed=seed), flush=True)
    gen = torch.Generator().manual_seed(seed + 7 * B + S + D)
    dt, rt = torch.float32 if f32 else torch.bfloat16, torch.float32 if f32 or res32 else torch.bfloat16
    rn = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    ln = [S] * B if lens is None else lens
    mk = lambda d: Rows(torch, B, S, D, d, pad)  # noqa: E731
    x, h = mk(rt).set((rn(B, S, D) * scale).to(rt), ln), mk(dt).set((rn(B, S, D) * scale).to(dt), ln) if branch else None
    DZ, DY = mk(rt).set(rn(B, S, D).to(rt), ln), mk(dt).set(rn(B, S, D).to(dt), ln)
    mod = torch.full((1 if shared else B, 3 * D + 16), float("nan"), device="cuda")
    mod[:, 8:3 * D + 8] = 0.5 * rn(1 if shared else B, 3 * D)
    gate, sc, sh = (mod[:, 8 + i * D:8 + (i + 1) * D] for i in range(3))
    g1, g2 = (1 + 0.2 * rn(D).cuda() for _ in range(2))
    have = dict(all="post gate pre scale shift", none="", mod="gate scale shift", gains="post pre", odd="gate shift pre")[rows].split()
    g1 = g1 if post and "post" in have else None
    gate = gate if branch and "gate" in have else None
    g2 = g2 if pre and "pre" in have else None
    sc, sh = sc if pre and "scale" in have else None, sh if pre and "shift" in have else None
    z, y = Rows(torch, B, S, D, rt, pad, fill=7.0), Rows(torch, B, S, D, dt, pad, fill=7.0)
    dx, dh = Rows(torch, B, S, D, rt, pad, fill=7.0), Rows(torch, B, S, D, dt, pad, fill=7.0)
    V = lambda r, on=1: r.v if r is not None and on else None  # noqa: E731
    desc = lib.blocknorm_desc(x.v, V(h), V(z, branch), V(y, pre), gate if gate is not None else sc if sc is not None else sh,
                              kind=layer, post=post, eps=1e-5, res_scale=0.75)
    sb, wb = lib.paragan_blocknorm_sizes(desc)
    saved, ws = lib.workspace(sb), lib.workspace(wb)
    saved.fill_(255), ws.fill_(255)
    L = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    ctx = lib.Context()
    lib.paragan_blocknorm_fwd(ctx, desc, x.v, V(h), g1, gate, g2, sc, sh, L, V(z, branch), V(y, pre), saved)
    dmod = torch.full_like(mod, 7.0)
    dgate, dsc, dsh = (dmod[:, 8 + i * D:8 + (i + 1) * D] for i in range(3))
    dg1, dg2 = torch.full((D,), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda")
    # gradients of rows that are not given are those of ones and zeros, asked for here too; their strides are the descriptor's
    plain = desc.mod_stride == 0 and not shared and B > 1
    if plain:
        dgate, dsc, dsh = (dmod[:1, 8 + i * D:8 + (i + 1) * D] for i in range(3))
    grads = [dg1 if post else None, dgate if branch else None, dg2 if pre else None, dsc if pre else None, dsh if pre else None]
    use_dz = dz or not pre
    for _ in range(repeat):
        lib.paragan_blocknorm_bwd(ctx, desc, x.v, V(h), g1, gate, g2, sc, sh, L, saved, V(DZ, use_dz), V(DY, pre), dx.v, V(dh, branch), *grads, ws)
    torch.cuda.synchronize()
    un = lambda t: None if t is None else num(t)  # noqa: E731
    clean = lambda r: np.nan_to_num(num(r.v))  # noqa: E731
    want = T.blocknorm(clean(x), clean(h) if branch else None, un(g1), un(gate), un(g2), un(sc), un(sh), ln, layer=layer, branch=branch,
                       post=post, pre=pre, eps=float(np.float32(1e-5)), res_scale=0.75, shared=shared or plain,
                       dz=clean(DZ) if use_dz else None, dy=clean(DY) if pre else np.zeros((B, S, D)),
                       uz=U32 if f32 or res32 else U16, uy=U32 if f32 else U16)
    got = dict(z=V(z, branch), y=V(y, pre), dx=dx.v, dh=V(dh, branch), dgain_post=grads[0], dgate=grads[1], dgain_pre=grads[2],
               dscale=grads[3], dshift=grads[4])
    for name, t in got.items():
        if t is not None:
            held(name, t, want[name], want["tol." + name] + 1e-30)
    assert all(r.untouched(7.0) for r in (z, y, dx, dh)) and bool((dmod[:, :8] == 7.0).all()) and bool((dmod[:, 3 * D + 8:] == 7.0).all())


KINDS = [dict(), dict(layer=1), dict(post=1), dict(layer=1, post=1), dict(branch=0), dict(pre=0), dict(pre=0, post=1, layer=1)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("D", [8, 64, 72, 136, 256, 264, 512, 520, 1152, 2048])
def test_blocknorm(kind, D):
    blocknorm_case(3, 11, D, **KINDS[kind], lens=[11, 0, 6], seed=kind)


@pytest.mark.parametrize("types", [dict(f32=1), dict(res32=1)])
@pytest.mark.parametrize("kind", [0, 3, 4, 6])
@pytest.mark.parametrize("D", [40, 200, 1480, 4104, 8192])
def test_blocknorm_types(kind, D, types):
    blocknorm_case(2, 7, D, **KINDS[kind], **types, lens=[7, 5], seed=kind)


@pytest.mark.parametrize("rows", ["none", "mod", "gains", "odd"])
@pytest.mark.parametrize("shared", [0, 1])
def test_blocknorm_rows_not_given(rows, shared):
    blocknorm_case(4, 5, 96, layer=1, post=1, rows=rows, shared=shared)
    blocknorm_case(4, 5, 1032, post=0, rows=rows, shared=shared, dz=0)


@pytest.mark.parametrize("shape", [(1, 1, 8), (1, 1, 8192), (5, 1, 768), (1, 3001, 64), (2, 1501, 520), (70, 3, 136), (300, 1, 40),
                                   (1, 9000, 8), (9, 129, 1152)])
@pytest.mark.parametrize("shared", [0, 1])
def test_blocknorm_shapes(shape, shared):
    blocknorm_case(*shape, layer=shared, post=1, shared=shared, pad=0)


def test_blocknorm_far_values():
    blocknorm_case(2, 9, 320, layer=1, post=1, f32=1, scale=1e6)
    blocknorm_case(2, 9, 320, layer=0, post=1, f32=1, scale=1e-4)        # eps decides
    blocknorm_case(2, 9, 1000, layer=1, post=0, scale=1e4)


def test_blocknorm_in_place():
    """z over x and y over h, as a forward without a backward may have it: the bits of separate outputs."""
    torch = need_gpu()
    for D in (72, 1152):
        x, h, g = torch.randn(2, 300, D, device="cuda").bfloat16(), torch.randn(2, 300, D, device="cuda").bfloat16(), torch.rand(2, D, device="cuda")
        z, y = torch.empty_like(x), torch.empty_like(h)
        ctx = lib.Context()
        kw = dict(kind=lib.NORM_LAYER, post=1, eps=1e-6)
        lib.paragan_blocknorm_fwd(ctx, lib.blocknorm_desc(x, h, z, y, g, **kw), x, h, None, g, None, g, g, None, z, y, None)
        lib.paragan_blocknorm_fwd(ctx, lib.blocknorm_desc(x, h, x, h, g, **kw), x, h, None, g, None, g, g, None, x, h, None)
        torch.cuda.synchronize()
        assert torch.equal(x, z) and torch.equal(h, y)


def test_blocknorm_nan_stays_in_its_row():
    torch = need_gpu()
    x, h = torch.randn(1, 40, 520, device="cuda"), torch.randn(1, 40, 520, device="cuda").bfloat16()
    x[0, 3, 7], h[0, 9, 519], x[0, 20, 0] = float("nan"), float("inf"), float("inf")
    z, y = torch.empty_like(x), torch.empty_like(h)
    lib.paragan_blocknorm_fwd(lib.Context(), lib.blocknorm_desc(x, h, z, y, kind=lib.NORM_RMS, eps=1e-6), x, h, None, None, None, None, None,
                              None, z, y, None)
    bad = (~torch.isfinite(y.float())).any(-1)[0]
    assert bad.nonzero().flatten().tolist() == [3, 9, 20]
    assert bool(torch.isnan(y[0, 3].float()).all())


# ------------------------------------------------------------- recurrence
def scan_case(B, S, D, *, f32=0, reverse=0, lens=None, state=1, sharp=8.0, spread=0, pad=8, seed=0, decay=None, xs=1.0):
    torch = need_gpu()
    print("scan", dict(B=B, S=S, D=D, f32=f32, reverse=reverse, lens=lens, state=state, sharp=sharp, spread=spread, seed=seed), flush=True)
    gen = torch.Generator().manual_seed(seed + 7 * B + S + D)
    dt = torch.float32 if f32 else torch.bfloat16
    rn = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    ln = [S] * B if lens is None else lens
    mk = lambda: Rows(torch, B, S, 3 * D, dt, pad)  # noqa: E731
    buf = mk().set((rn(B, S, 3 * D) * (1 + spread)).to(dt), ln)
    x, r, g = (buf.v[..., i * D:(i + 1) * D] for i in range(3))
    x *= xs
    dec = (torch.rand(D, generator=gen) * 5 - 8 if decay is None else torch.full((D,), decay)).cuda()
    h0, dht = (rn(B, D).cuda() if state else None for _ in range(2))
    dy = Rows(torch, B, S, D, dt, pad).set(rn(B, S, D).to(dt), ln)
    y = Rows(torch, B, S, D, dt, pad, fill=7.0)
    dbuf = Rows(torch, B, S, 3 * D, dt, pad, fill=7.0)
    dx, dr, dg = (dbuf.v[..., i * D:(i + 1) * D] for i in range(3))
    ht, dh0 = (torch.full((B, D), 7.0, device="cuda") if state else None for _ in range(2))
    ddec = torch.full((D,), 7.0, device="cuda")
    desc = lib.scan_desc(x, r, g, y.v, sharp=sharp, reverse=reverse)
    sb, wb = lib.paragan_scan_sizes(desc)
    saved, ws = lib.workspace(sb), lib.workspace(wb)
    saved.fill_(255), ws.fill_(255)
    L = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    ctx = lib.Context()
    # without and with what the backward needs: the same bits
    lib.paragan_scan_fwd(ctx, desc, x, r, g, dec, L, h0, y.v, ht, None, ws)
    first = y.v.clone()
    ws.fill_(255), y.v.fill_(7.0)
    lib.paragan_scan_fwd(ctx, desc, x, r, g, dec, L, h0, y.v, ht, saved, ws)
    ws.fill_(255)
    lib.paragan_scan_bwd(ctx, desc, x, r, g, dec, L, saved, dy.v, dht, dx, dr, dg, ddec, dh0, ws)
    torch.cuda.synchronize()
    assert torch.equal(first, y.v)
    clean = lambda t: np.nan_to_num(num(t))  # noqa: E731
    un = lambda t: None if t is None else num(t)  # noqa: E731
    want = T.scan(clean(x), clean(r), clean(g), num(dec), ln, sharp=sharp, reverse=reverse, h0=un(h0), dy=clean(dy.v), dht=un(dht),
                  uo=U32 if f32 else U16)
    for name, t in (("y", y.v), ("ht", ht), ("dx", dx), ("dr", dr), ("dg", dg), ("ddecay", ddec), ("dh0", dh0)):
        if t is not None:
            held(name, t, want[name], want["tol." + name] + 1e-30)
    assert y.untouched(7.0) and dbuf.untouched(7.0)


@pytest.mark.parametrize("f32", [0, 1])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("shape", [(1, 1, 8), (3, 2, 8), (2, 15, 24), (2, 16, 72), (3, 17, 128), (1, 64, 136), (2, 129, 64), (5, 300, 40),
                                   (1, 1021, 520), (2, 1025, 8)])
def test_scan(shape, reverse, f32):
    scan_case(*shape, f32=f32, reverse=reverse, state=shape[1] % 2)


@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("lens", [[40, 0, 1, 39], [0, 0, 0, 0], [7, 40, 33, 16]])
def test_scan_ragged(lens, reverse):
    scan_case(4, 40, 72, lens=lens, reverse=reverse)
    scan_case(4, 40, 8, lens=lens, reverse=reverse, f32=1, state=0)
    scan_case(4, 700, 136, lens=[n * 17 for n in lens], reverse=reverse)


@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("f32", [0, 1])
def test_scan_lengths_that_cut_chunks(f32, reverse):
    """Lengths that end on, just before and just after a tile, a chunk and a run inside one."""
    for S in (3000, 4096):
        scan_case(6, S, 72, lens=[S, S - 1, 2049, 65, 1, 1537], reverse=reverse, f32=f32, pad=0)
    scan_case(3, 1000, 520, lens=[513, 1000, 129], reverse=reverse, f32=f32, pad=0)


@pytest.mark.parametrize("shape", [(1, 4099, 64), (2, 2500, 264), (1, 8200, 8), (40, 130, 256), (3, 600, 2048)])
def test_scan_long(shape):
    scan_case(*shape, reverse=shape[0] % 2, f32=shape[0] % 2)


def test_scan_many_short_rows():
    scan_case(700, 3, 64)
    scan_case(33, 1, 4096)


def test_scan_far_values():
    scan_case(2, 200, 64, decay=-80.0)               # decays of one to the last bit: the root is far below a step
    scan_case(2, 200, 64, decay=-120.0, f32=1)       # softplus underflows: nothing comes in
    scan_case(2, 200, 64, decay=3.0, f32=1)          # strong decays
    scan_case(2, 200, 64, decay=60.0)                # everything is forgotten at once
    scan_case(2, 200, 64, spread=30, f32=1)          # gates far out on either side
    scan_case(1, 300, 64, sharp=1e-3, f32=1)
    scan_case(1, 300, 64, xs=1e12, f32=1)


def test_scan_state_in_place_and_steps_follow_the_whole():
    """Tokens one at a time over a state in place: each new output is the row that one call over the sequence gives."""
    torch = need_gpu()
    B, S, D = 3, 37, 264
    gen = torch.Generator().manual_seed(5)
    buf = torch.randn(B, S, 3 * D, generator=gen).bfloat16().cuda()
    dec = (torch.rand(D, generator=gen) * 5 - 8).cuda()
    h0 = torch.randn(B, D, generator=gen).cuda()
    want = T.scan(*(num(buf[..., i * D:(i + 1) * D]) for i in range(3)), num(dec), [S] * B, sharp=8.0, h0=num(h0), uo=U16)
    h, ctx = h0.clone(), lib.Context()
    for t0, n in ((0, 20), *((t, 1) for t in range(20, S))):
        x, r, g = (buf[:, t0:t0 + n, i * D:(i + 1) * D] for i in range(3))
        y = torch.empty(B, n, D, dtype=torch.bfloat16, device="cuda")
        d = lib.scan_desc(x, r, g, y, sharp=8.0)
        ws = lib.workspace(lib.paragan_scan_sizes(d)[1])
        lib.paragan_scan_fwd(ctx, d, x, r, g, dec, None, h, y, h, None, ws)
        held("tokens from %d" % t0, y, want["y"][:, t0:t0 + n], want["tol.y"][:, t0:t0 + n])
    held("state", h, want["ht"], want["tol.ht"])


@pytest.mark.parametrize("dims", [(2, 40, 72), (3, 300, 520), (1, 9000, 264), (2, 5000, 1000)])
def test_scan_states_in_place(dims):
    """ht over h0 and dh0 over dht, whole and in chunks: the bits of separate ones."""
    torch = need_gpu()
    B, S, D = dims
    x, r, g, dy = (torch.randn(B, S, D, device="cuda").bfloat16() for _ in range(4))
    dec, h0, dht = torch.rand(D, device="cuda") * 5 - 8, torch.randn(B, D, device="cuda"), torch.randn(B, D, device="cuda")
    y, grads, ddec, ctx = torch.empty_like(x), [torch.empty_like(x) for _ in range(3)], torch.empty(D, device="cuda"), lib.Context()
    d = lib.scan_desc(x, r, g, y, sharp=8.0)
    sb, wb = lib.paragan_scan_sizes(d)
    saved, ws, outs = lib.workspace(sb), lib.workspace(wb), []
    for rep in range(4):
        a, b = h0.clone(), dht.clone()
        ht, dh0 = (a, b) if rep else (torch.empty_like(a), torch.empty_like(b))
        lib.paragan_scan_fwd(ctx, d, x, r, g, dec, None, a, y, ht, saved, ws)
        lib.paragan_scan_bwd(ctx, d, x, r, g, dec, None, saved, dy, b, *grads, ddec, dh0, ws)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (y, ht, *grads, ddec, dh0)])
    assert all(torch.equal(u, v) for o in outs[1:] for u, v in zip(outs[0], o))


def test_scan_nan_reaches_the_tokens_after_it_alone():
    torch = need_gpu()
    for S in (50, 3000):
        for reverse in (0, 1):
            x, r, g = (torch.randn(2, S, 64, device="cuda").bfloat16() for _ in range(3))
            at = S // 3
            x[0, at, 5], r[1, at, 60] = float("inf"), float("nan")
            y = torch.empty_like(x)
            d = lib.scan_desc(x, r, g, y, sharp=8.0, reverse=reverse)
            ws = lib.workspace(lib.paragan_scan_sizes(d)[1])
            lib.paragan_scan_fwd(lib.Context(), d, x, r, g, torch.full((64,), -5.0, device="cuda"), None, None, y, None, None, ws)
            bad = ~torch.isfinite(y.float())
            want = torch.zeros_like(bad)
            span = slice(None, at + 1) if reverse else slice(at, None)
            want[0, span, 5], want[1, span, 60] = True, True
            assert torch.equal(bad, want), (S, reverse)


def test_scan_rows_that_repeat():
    """Gates shared by the batch, one input for all tokens: zero strides in the forward, refused by the backward."""
    torch = need_gpu()
    x, r, g = torch.randn(3, 1, 40, device="cuda").bfloat16(), *(torch.randn(1, 21, 40, device="cuda").bfloat16() for _ in range(2))
    X, R, G = x.expand(3, 21, 40), r.expand(3, 21, 40), g.expand(3, 21, 40)
    y, dec = torch.empty(3, 21, 40, dtype=torch.bfloat16, device="cuda"), torch.full((40,), -4.0, device="cuda")
    d = lib.scan_desc(X, R, G, y, sharp=8.0)
    sb, wb = lib.paragan_scan_sizes(d)
    saved, ws = lib.workspace(sb), lib.workspace(wb)
    lib.paragan_scan_fwd(lib.Context(), d, X, R, G, dec, None, None, y, None, saved, ws)
    want = T.scan(num(X), num(R), num(G), num(dec), [21] * 3, sharp=8.0, uo=U16)
    held("y", y, want["y"], want["tol.y"])
    with pytest.raises(lib.ParaganError, match="overlaps itself"):
        lib.paragan_scan_bwd(lib.Context(), d, X, R, G, dec, None, saved, y, None, X, R, G, dec, None, ws)


# ------------------------------------------------------------- clipping
def clip_case(sizes, limit, *, in_place=0, scale=1.0, at=0, seed=0, grad_scale=1.0):
    torch = need_gpu()
    print("clip", dict(n=len(sizes), limit=limit, in_place=in_place, scale=scale, at=at, grad_scale=grad_scale), flush=True)
    gen = torch.Generator().manual_seed(seed)
    grads, outs, bufs = [], [], []
    for i, (n, bf) in enumerate(sizes):
        dt = torch.bfloat16 if bf else torch.float32
        for o in (0, 1):
            buf = torch.full((n + 24,), 7.0, dtype=dt, device="cuda")
            k = (at + 3 * i + 5 * o) % 11
            (outs if o else grads).append(buf[k:k + n])
            bufs.append((buf, k, n))
        grads[-1].copy_((torch.randn(n, generator=gen) * scale).to(dt))
    G = [num(g) for g in grads]
    norm0 = grad_scale * math.sqrt(sum((g * g).sum() for g in G))
    most = limit * norm0 if norm0 else 1.0
    most = float(np.float32(most))
    plan = lib.ClipPlan(grads, None if in_place else outs)
    norm, ws = torch.full((2,), 9.0, device="cuda"), lib.workspace(plan.ws_bytes)
    ws.fill_(255)
    lib.paragan_clip(lib.Context(), plan, most, grad_scale, norm, ws)
    torch.cuda.synchronize()
    gs = float(np.float32(grad_scale))
    wn, wk, want = T.clip(G, most, gs)
    assert abs(norm[0].item() - wn) <= 2 * U32 * wn and abs(norm[1].item() - wk) <= 2 * U32 * wk, (norm.tolist(), wn, wk)
    for (n, bf), g, o, w in zip(sizes, grads, outs, want):
        # the factor is off by half a step, the product by another, the output by its own
        got = num(g if in_place else o)
        tol = (U16 if bf else 0.0) * np.abs(w) + 3 * U32 * np.abs(w) + 2.0 ** -133      # (half of the smallest bf16)
        assert np.all(np.abs(got - w) <= tol)
    for buf, k, n in bufs:
        assert bool((buf[:k] == 7.0).all()) and bool((buf[k + n:] == 7.0).all())


SETS = {"one": [(1, 0)], "vectors": [(7, 0), (64, 1), (1, 1), (0, 0), (513, 0), (16, 1)], "pieces": [(16384, 0), (16385, 1), (40000, 0), (32768, 1)],
        "many": [(1 + 37 * i % 901, i % 2) for i in range(500)], "large": [(3_000_001, 0), (5_000_003, 1), (20, 0)]}


@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("limit", [0.1, 1.5, math.inf])
@pytest.mark.parametrize("in_place", [0, 1])
def test_clip(name, limit, in_place):
    clip_case(SETS[name], limit, in_place=in_place, at=len(name))


def test_clip_far_values_and_scales():
    clip_case(SETS["vectors"], 0.5, scale=1e30)                  # squares past fp32 on either side
    clip_case(SETS["vectors"], 0.5, scale=1e-30)
    clip_case(SETS["pieces"], 0.5, grad_scale=1.0 / 3)
    clip_case(SETS["pieces"], 2.0, grad_scale=1.0 / 3, in_place=1)
    clip_case([(5, 0), (0, 1)], 1.0, scale=0.0)
    clip_case([(0, 0)], 1.0)


def test_clip_not_finite():
    torch = need_gpu()
    ctx, norm = lib.Context(), torch.zeros(2, device="cuda")
    for bad in (float("nan"), float("inf")):
        a, b = torch.ones(100, device="cuda"), torch.ones(20000, device="cuda").bfloat16()
        b[15000] = bad
        oa, ob = torch.zeros_like(a), torch.zeros_like(b)
        plan = lib.ClipPlan([a, b], [oa, ob])
        lib.paragan_clip(ctx, plan, 1.0, 1.0, norm, lib.workspace(plan.ws_bytes))
        torch.cuda.synchronize()
        if math.isnan(bad):
            assert bool(torch.isnan(norm).all()) and bool(torch.isnan(oa).all()) and bool(torch.isnan(ob).all())
        else:
            assert math.isinf(norm[0].item()) and norm[1].item() == 0.0 and bool((oa == 0).all())
            assert bool(torch.isnan(ob[15000])) and int(torch.isnan(ob).sum()) == 1
