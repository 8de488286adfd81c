"""The token block's operators as a program uses them: norm, recurrence, gate
and residual through forward and backward and the clipping of all their
gradients, repeated calls, captured graphs, two streams, tensors past 32-bit
offsets, and calls that are refused."""
import math

import numpy as np
import pytest

from oracle import token_block as T
from paragan_2411_03999_amd import lib

from .parity import need_gpu
from .test_gpu_token import held
from .test_gpu_token_block import num

pytestmark = pytest.mark.gpu

U16, U32 = T.U16, T.U32
EPS, SHARP = 1e-6, 8.0


class Mixer:
    """Two sublayers' worth of what the operators do: norm of the stream with a condition's scale and shift, recurrence over
    it (its gates given), gated residual with the norm of the next block's input; backward of all, and clipping of every
    gradient of a parameter or of the condition."""

    def __init__(self, torch, ctx, B, S, D, gen, reverse=0, ragged=True):
        self.ctx, self.dims, self.reverse = ctx, (B, S, D), reverse
        rn = lambda *s: torch.randn(s, generator=gen).cuda()  # noqa: E731
        e = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
        self.x0, self.gates = rn(B, S, D).bfloat16(), rn(B, S, 2 * D).bfloat16()
        self.dz, self.dy = rn(B, S, D).bfloat16(), rn(B, S, D).bfloat16()
        self.mod, self.gain, self.decay = 0.3 * rn(B, 5 * D), 1 + 0.1 * rn(3, D), torch.rand(D, generator=gen).cuda() * 5 - 8
        self.h0 = rn(B, D)
        self.lens = [S - 5 * b for b in range(B)] if ragged else [S] * B
        self.len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        f = torch.float32
        # forward: n0 = norm(x0), h = scan(n0), z = x0 + gate norm(h), y = norm(z)
        self.n0, self.h, self.ht, self.z, self.y = e(B, S, D), e(B, S, D), e(B, D, dt=f), e(B, S, D), e(B, S, D)
        self.dh, self.dn0, self.dgates, self.dx1, self.dx0 = (e(B, S, k * D) for k in (1, 1, 2, 1, 1))
        self.dmod, self.dgain, self.ddecay, self.dh0 = e(B, 5 * D, dt=f), e(3, D, dt=f), e(D, dt=f), e(B, D, dt=f)
        c = lambda t, i, n=D: t[..., i * n:(i + 1) * n]  # noqa: E731
        self.c = c
        m = self.mod
        self.d0 = lib.blocknorm_desc(self.x0, None, None, self.n0, c(m, 0), kind=lib.NORM_LAYER, eps=EPS)
        self.ds = lib.scan_desc(self.n0, c(self.gates, 0), c(self.gates, 1), self.h, sharp=SHARP, reverse=reverse)
        self.d1 = lib.blocknorm_desc(self.x0, self.h, self.z, self.y, c(m, 2), kind=lib.NORM_RMS, post=1, eps=EPS, res_scale=0.5)
        sizes = [lib.paragan_blocknorm_sizes(self.d0), lib.paragan_scan_sizes(self.ds), lib.paragan_blocknorm_sizes(self.d1)]
        self.saved = [lib.workspace(s) for s, _ in sizes]
        self.plan = lib.ClipPlan([self.dmod, self.dgain, self.ddecay, self.dh0, self.dgates])
        self.norm = e(2, dt=f)
        self.ws = lib.workspace(max([w for _, w in sizes] + [self.plan.ws_bytes]))

    def fwd(self):
        c, m, g = self.c, self.mod, self.gain
        lib.paragan_blocknorm_fwd(self.ctx, self.d0, self.x0, None, None, None, g[0], c(m, 0), c(m, 1), self.len, None, self.n0, self.saved[0])
        lib.paragan_scan_fwd(self.ctx, self.ds, self.n0, c(self.gates, 0), c(self.gates, 1), self.decay, self.len, self.h0, self.h, self.ht,
                             self.saved[1], self.ws)
        lib.paragan_blocknorm_fwd(self.ctx, self.d1, self.x0, self.h, g[1], c(m, 2), g[2], c(m, 3), c(m, 4), self.len, self.z, self.y,
                                  self.saved[2])

    def bwd(self):
        c, m, g, dm, dg = self.c, self.mod, self.gain, self.dmod, self.dgain
        lib.paragan_blocknorm_bwd(self.ctx, self.d1, self.x0, self.h, g[1], c(m, 2), g[2], c(m, 3), c(m, 4), self.len, self.saved[2], self.dz,
                                  self.dy, self.dx1, self.dh, dg[1], c(dm, 2), dg[2], c(dm, 3), c(dm, 4), self.ws)
        lib.paragan_scan_bwd(self.ctx, self.ds, self.n0, c(self.gates, 0), c(self.gates, 1), self.decay, self.len, self.saved[1], self.dh,
                             None, self.dn0, c(self.dgates, 0), c(self.dgates, 1), self.ddecay, self.dh0, self.ws)
        # the stream's gradient so far comes in as dz
        lib.paragan_blocknorm_bwd(self.ctx, self.d0, self.x0, None, None, None, g[0], c(m, 0), c(m, 1), self.len, self.saved[0], self.dx1,
                                  self.dn0, self.dx0, None, None, None, dg[0], c(dm, 0), c(dm, 1), self.ws)

    def clip(self, most=1.0):
        lib.paragan_clip(self.ctx, self.plan, most, 1.0, self.norm, self.ws)

    def run(self):
        self.fwd()
        self.bwd()
        self.clip()

    def results(self):
        return (self.n0, self.h, self.ht, self.z, self.y, self.dx0, self.dgates, self.dmod, self.dgain, self.ddecay, self.dh0, self.norm)

    def outs(self):
        return [t.clone() for t in self.results()]


@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("dims", [(3, 150, 72), (2, 333, 520)])
def test_block_against_the_definitions(dims, reverse):
    """Each step held to the float64 definition of the same inputs, and the whole to the chain of definitions within the sum
    of the steps' roundings (relative 2-norm)."""
    torch = need_gpu()
    B, S, D = dims
    blk = Mixer(torch, lib.Context(), B, S, D, torch.Generator().manual_seed(1 + D), reverse)
    blk.fwd()
    blk.bwd()
    torch.cuda.synchronize()
    c, m, g = blk.c, blk.mod, blk.gain
    eps = float(np.float32(EPS))
    kw0 = dict(layer=True, branch=0, post=0, pre=1, eps=eps, res_scale=1.0)
    kw1 = dict(layer=False, branch=1, post=1, pre=1, eps=eps, res_scale=0.5)
    a0 = lambda x: (x, None, None, None, num(g[0]), num(c(m, 0)), num(c(m, 1)), blk.lens)  # noqa: E731
    a1 = lambda x, h: (x, h, num(g[1]), num(c(m, 2)), num(g[2]), num(c(m, 3)), num(c(m, 4)), blk.lens)  # noqa: E731
    gates = (num(c(blk.gates, 0)), num(c(blk.gates, 1)), num(blk.decay), blk.lens)
    ks = dict(sharp=SHARP, reverse=reverse, h0=num(blk.h0), uo=U16)
    r0 = T.blocknorm(*a0(num(blk.x0)), **kw0, dz=num(blk.dx1), dy=num(blk.dn0), uz=U16, uy=U16)
    rs = T.scan(num(blk.n0), *gates, dy=num(blk.dh), **ks)
    r1 = T.blocknorm(*a1(num(blk.x0), num(blk.h)), **kw1, dz=num(blk.dz), dy=num(blk.dy), uz=U16, uy=U16)
    dm = blk.dmod
    for name, got, r, key in (("n0", blk.n0, r0, "y"), ("h", blk.h, rs, "y"), ("ht", blk.ht, rs, "ht"), ("z", blk.z, r1, "z"), ("y", blk.y, r1, "y"),
                              ("dx1", blk.dx1, r1, "dx"), ("dh", blk.dh, r1, "dh"), ("dn0", blk.dn0, rs, "dx"), ("dr", c(blk.dgates, 0), rs, "dr"),
                              ("dg", c(blk.dgates, 1), rs, "dg"), ("ddecay", blk.ddecay, rs, "ddecay"), ("dh0", blk.dh0, rs, "dh0"),
                              ("dx0", blk.dx0, r0, "dx"), ("dscale0", c(dm, 0), r0, "dscale"), ("dshift0", c(dm, 1), r0, "dshift"),
                              ("dgate", c(dm, 2), r1, "dgate"), ("dscale1", c(dm, 3), r1, "dscale"), ("dshift1", c(dm, 4), r1, "dshift"),
                              ("dgain0", blk.dgain[0], r0, "dgain_pre"), ("dpost", blk.dgain[1], r1, "dgain_post"), ("dgain2", blk.dgain[2], r1, "dgain_pre")):
        held(name, got, r[key], r["tol." + key] + 1e-30)
    # the chain from the stream on, nothing rounded in between
    n0 = T.blocknorm(*a0(num(blk.x0)), **kw0)["y"]
    h = T.scan(n0, *gates, **ks)["y"]
    r1 = T.blocknorm(*a1(num(blk.x0), h), **kw1, dz=num(blk.dz), dy=num(blk.dy))
    rs = T.scan(n0, *gates, dy=r1["dh"], **ks)
    r0 = T.blocknorm(*a0(num(blk.x0)), **kw0, dz=r1["dx"], dy=rs["dx"])
    rel = lambda got, w: np.linalg.norm(num(got) - w) / np.linalg.norm(w)  # noqa: E731
    errs = dict(y=rel(blk.y, r1["y"]), ht=rel(blk.ht, T.scan(n0, *gates, **ks)["ht"]), dx0=rel(blk.dx0, r0["dx"]), dr=rel(c(blk.dgates, 0), rs["dr"]),
                dg=rel(c(blk.dgates, 1), rs["dg"]), ddecay=rel(blk.ddecay, rs["ddecay"]), dgate=rel(c(dm, 2), r1["dgate"]),
                dscale0=rel(c(dm, 0), r0["dscale"]), dgain0=rel(blk.dgain[0], r0["dgain_pre"]))
    # at most eight roundings to bf16 in a row (n0, h, dx1, dh, dn0 and the output's own among them), each entering once, and
    # those of n0 and h once more through the formulas that use them again
    print("  chain", {k: "%.2e" % v for k, v in errs.items()}, flush=True)
    assert max(errs.values()) < 10 * U16
    # clipping of everything together
    before = [num(t) for t in (blk.dmod, blk.dgain, blk.ddecay, blk.dh0, blk.dgates)]
    n, k, want = T.clip(before, 1.0)
    blk.clip()
    torch.cuda.synchronize()
    assert abs(blk.norm[0].item() - n) <= 2 * U32 * n and n > 1.0
    for t, w in zip((blk.dmod, blk.dgain, blk.ddecay, blk.dh0, blk.dgates), want):
        u = U16 if t.dtype == torch.bfloat16 else 0.0
        assert np.all(np.abs(num(t) - w) <= (u + 3 * U32) * np.abs(w) + 2.0 ** -133)


def test_the_same_call_gives_the_same_bits():
    torch = need_gpu()
    for dims in ((2, 700, 264), (1, 5000, 64), (40, 20, 1032)):
        blk = Mixer(torch, lib.Context(), *dims, torch.Generator().manual_seed(3), ragged=dims[1] > 300)
        blk.run()
        first = blk.outs()
        for _ in range(3):
            blk.ws.fill_(255)
            [s.fill_(255) for s in blk.saved]
            blk.run()
            assert all(torch.equal(a, b) for a, b in zip(first, blk.outs()))


def test_captured_and_replayed():
    """Two captured passes that share a workspace, replayed in turn with eager work between and new inputs."""
    torch = need_gpu()
    side = torch.cuda.Stream()
    ctx = lib.Context(side)
    gen = torch.Generator().manual_seed(4)
    blks = [Mixer(torch, ctx, 2, 130, 136, gen), Mixer(torch, ctx, 1, 2600, 64, gen, reverse=1)]
    ws = max((b.ws for b in blks), key=lambda t: t.numel())
    graphs = []
    for b in blks:
        b.ws = ws
        with torch.cuda.stream(side):
            b.run()                       # once before, as any program does
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.run()
        graphs.append(g)
    for rep in range(3):
        for b, g in zip(blks, graphs):
            b.x0.copy_(torch.randn(b.x0.shape, generator=gen).bfloat16())
            b.gates.copy_(torch.randn(b.gates.shape, generator=gen).bfloat16())
            b.dy.copy_(torch.randn(b.dy.shape, generator=gen).bfloat16())
            b.len.copy_(torch.tensor([max(0, n - 40 * rep) for n in b.lens], dtype=torch.int32))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                b.run()
            torch.cuda.synchronize()
            want = b.outs()
            for t in b.results():
                t.fill_(9.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, b.outs())), rep


def test_steps_captured_over_a_state():
    """One token a replay, the state in place: the outputs of one call over the sequence."""
    torch = need_gpu()
    side = torch.cuda.Stream()
    ctx = lib.Context(side)
    B, S, D = 4, 12, 136
    buf = torch.randn(B, S, 3 * D, device="cuda").bfloat16()
    dec, h = torch.rand(D, device="cuda") * 5 - 8, torch.zeros(B, D, device="cuda")
    tok, y1 = torch.empty(B, 1, 3 * D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, 1, D, dtype=torch.bfloat16, device="cuda")
    part = lambda t, i: t[..., i * D:(i + 1) * D]  # noqa: E731
    d = lib.scan_desc(part(tok, 0), part(tok, 1), part(tok, 2), y1, sharp=SHARP)
    ws = lib.workspace(lib.paragan_scan_sizes(d)[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        lib.paragan_scan_fwd(ctx, d, part(tok, 0), part(tok, 1), part(tok, 2), dec, None, h, y1, h, None, ws)
    h.zero_()
    want = T.scan(*(num(part(buf, i)) for i in range(3)), num(dec), [S] * B, sharp=SHARP, uo=U16)
    for t in range(S):
        tok.copy_(buf[:, t:t + 1])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        held("token %d" % t, y1, want["y"][:, t:t + 1], want["tol.y"][:, t:t + 1])
    held("state", h, want["ht"], want["tol.ht"])


def test_two_streams_at_once():
    torch = need_gpu()
    streams = [torch.cuda.Stream() for _ in range(2)]
    blks = [Mixer(torch, lib.Context(s), 2, 1400, 264, torch.Generator().manual_seed(5 + i)) for i, s in enumerate(streams)]
    torch.cuda.synchronize()
    want = []
    for b in blks:
        b.run()
        torch.cuda.synchronize()
        want.append(b.outs())
    for b in blks:
        b.ws.fill_(255)
    torch.cuda.synchronize()
    for _ in range(5):
        for b in blks:
            b.run()
    torch.cuda.synchronize()
    for b, w in zip(blks, want):
        assert all(torch.equal(x, y) for x, y in zip(w, b.outs()))


@pytest.mark.parametrize("reverse", [0, 1])
def test_scan_past_32_bit_offsets(reverse):
    """Tokens 2 MB apart over sequences of more than 4 GB: whole and in chunks."""
    torch = need_gpu()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    B, S, D, ts = 2, 2500, 8, (1 << 20) - 8
    gen = torch.Generator().manual_seed(6)
    small = [torch.randn(B, S, D, generator=gen).bfloat16() for _ in range(4)]
    big = torch.zeros(B * S * ts, dtype=torch.bfloat16, device="cuda")          # 10 GB
    out = torch.zeros_like(big)
    view = lambda t, off: t.as_strided((B, S, D), (S * ts, ts, 1), off)  # noqa: E731
    x, r, g, dy = (view(big, 8 * i) for i in range(4))
    for v, t in zip((x, r, g, dy), small):
        v.copy_(t)
    y, dx, dr, dg = (view(out, 8 * i) for i in range(4))
    # the gradients lie as x, r, g and dy as y: all have these strides
    dec = (torch.rand(D, generator=gen) * 5 - 8).cuda()
    d = lib.scan_desc(x, r, g, y, sharp=SHARP, reverse=reverse)
    sb, wb = lib.paragan_scan_sizes(d)
    saved, ws, ddec = lib.workspace(sb), lib.workspace(wb), torch.empty(D, device="cuda")
    lens = [S, S - 700]
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ctx = lib.Context()
    lib.paragan_scan_fwd(ctx, d, x, r, g, dec, L, None, y, None, saved, ws)
    lib.paragan_scan_bwd(ctx, d, x, r, g, dec, L, saved, dy, None, dx, dr, dg, ddec, None, ws)
    torch.cuda.synchronize()
    want = T.scan(*(num(t) for t in small[:3]), num(dec), lens, sharp=SHARP, reverse=reverse, dy=num(small[3]), uo=U16)
    for name, t in (("y", y), ("dx", dx), ("dr", dr), ("dg", dg), ("ddecay", ddec)):
        held(name, t.contiguous(), want[name], want["tol." + name] + 1e-30)
    out.view(-1)[:32].zero_()
    assert int(torch.count_nonzero(out[32:ts])) == 0


def test_blocknorm_past_32_bit_offsets():
    """Tokens 32 MB apart."""
    torch = need_gpu()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    B, S, D, ts = 2, 150, 520, (1 << 24) + 8
    gen = torch.Generator().manual_seed(7)
    small = [torch.randn(B, S, D, generator=gen).bfloat16() for _ in range(4)]
    big, out = (torch.zeros(B * S * ts, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    view = lambda t, i: t.as_strided((B, S, D), (S * ts, ts, 1), i * 1024)  # noqa: E731
    x, h, dz, dy = (view(big, i) for i in range(4))
    for v, t in zip((x, h, dz, dy), small):
        v.copy_(t)
    z, y, dx, dh = (view(out, i) for i in range(4))
    gate = torch.randn(B, D, generator=gen).cuda()
    d = lib.blocknorm_desc(x, h, z, y, gate, kind=lib.NORM_LAYER, post=1, eps=EPS)
    sb, wb = lib.paragan_blocknorm_sizes(d)
    saved, ws, dgate = lib.workspace(sb), lib.workspace(wb), torch.empty_like(gate)
    ctx = lib.Context()
    lib.paragan_blocknorm_fwd(ctx, d, x, h, None, gate, None, None, None, None, z, y, saved)
    lib.paragan_blocknorm_bwd(ctx, d, x, h, None, gate, None, None, None, None, saved, dz, dy, dx, dh, None, dgate, None, None, None, ws)
    torch.cuda.synchronize()
    want = T.blocknorm(num(small[0]), num(small[1]), None, num(gate), None, None, None, [S] * B, layer=True, branch=1, post=1, pre=1,
                       eps=float(np.float32(EPS)), res_scale=1.0, dz=num(small[2]), dy=num(small[3]), uz=U16, uy=U16)
    for name, t in (("z", z), ("y", y), ("dx", dx), ("dh", dh), ("dgate", dgate)):
        held(name, t.contiguous(), want[name], want["tol." + name] + 1e-30)


def test_a_sequence_split_by_hand():
    """A sequence in two calls, the state handed on and its gradient handed back: the definition of the whole."""
    torch = need_gpu()
    B, S, D, cut = 2, 300, 72, 111
    gen = torch.Generator().manual_seed(8)
    buf = torch.randn(B, S, 3 * D, generator=gen).cuda()
    dy, dec = torch.randn(B, S, D, generator=gen).cuda(), (torch.rand(D, generator=gen) * 5 - 8).cuda()
    part = lambda t, i, a, b: t[:, a:b, i * D:(i + 1) * D]  # noqa: E731
    y, db, ctx, steps = torch.empty(B, S, D, device="cuda"), torch.empty_like(buf), lib.Context(), []
    h = None
    for a, b in ((0, cut), (cut, S)):
        x, r, g = (part(buf, i, a, b) for i in range(3))
        d = lib.scan_desc(x, r, g, y[:, a:b], sharp=SHARP)
        sb, wb = lib.paragan_scan_sizes(d)
        saved, ws, ht = lib.workspace(sb), lib.workspace(wb), torch.empty(B, D, device="cuda")
        lib.paragan_scan_fwd(ctx, d, x, r, g, dec, None, h, y[:, a:b], ht, saved, ws)
        steps.append((d, saved, ws, x, r, g, a, b))
        h = ht
    back, total = None, torch.zeros(D, device="cuda", dtype=torch.float64)
    for d, saved, ws, x, r, g, a, b in reversed(steps):
        dh0, ddec = torch.empty(B, D, device="cuda"), torch.empty(D, device="cuda")
        lib.paragan_scan_bwd(ctx, d, x, r, g, dec, None, saved, dy[:, a:b], back, *(part(db, i, a, b) for i in range(3)), ddec, dh0, ws)
        back, total = dh0, total + ddec.double()
    torch.cuda.synchronize()
    want = T.scan(*(num(part(buf, i, 0, S)) for i in range(3)), num(dec), [S] * B, sharp=SHARP, h0=np.zeros((B, D)), dy=num(dy), uo=U32)
    for name, t in (("y", y), ("ht", h), ("dx", part(db, 0, 0, S)), ("dr", part(db, 1, 0, S)), ("dg", part(db, 2, 0, S)), ("ddecay", total), ("dh0", back)):
        held(name, t, want[name], want["tol." + name] + 2 * U32 * np.abs(want[name]) + 1e-30)


def test_refused_calls_touch_nothing():
    torch = need_gpu()
    ctx = lib.Context()
    z = lambda *s, dt=torch.bfloat16: torch.full(s, 3.0, dtype=dt, device="cuda")  # noqa: E731
    f = torch.float32
    odd = z(2 * 8 * 32 + 8).view(-1)[1:1 + 2 * 8 * 32].view(2, 8, 32)
    rows, vec, lens = z(2, 32, dt=f), z(32, dt=f), torch.full((2,), 8, dtype=torch.int32, device="cuda")
    x, h, zo, y = (z(2, 8, 32) for _ in range(4))
    d = lib.blocknorm_desc(x, h, zo, y, rows, kind=lib.NORM_RMS, post=1, eps=EPS)
    sb, wb = lib.paragan_blocknorm_sizes(d)
    saved, ws = lib.workspace(sb), lib.workspace(wb)
    fwd = [x, h, vec, rows, vec, rows, rows, lens, zo, y, saved]
    for i, bad in ((0, None), (0, odd), (0, x.float()), (1, None), (1, z(2, 8, 16)), (2, z(16, dt=f)), (3, z(1, 32, dt=f)), (3, vec), (4, vec.double()),
                   (5, z(2, 40, dt=f)[:, :32]), (6, rows.cpu()), (7, lens[:1]), (7, lens.long()), (8, None), (8, odd), (9, None), (9, z(2, 8, 64)[..., :32]),
                   (10, saved[16:])):
        args = list(fwd)
        args[i] = bad
        with pytest.raises(lib.ParaganError):
            lib.paragan_blocknorm_fwd(ctx, d, *args)
    grads = [z(2, 8, 32), z(2, 8, 32), z(32, dt=f), z(2, 32, dt=f), z(32, dt=f), z(2, 32, dt=f), z(2, 32, dt=f)]
    bwd = fwd[:8] + [saved, x, y, *grads, ws]
    for i, bad in ((8, None), (8, saved[8:]), (10, None), (11, None), (11, odd), (12, None), (13, z(8, dt=f)), (14, vec), (17, z(3, 32, dt=f)), (18, None),
                   (18, ws[8:])):
        args = list(bwd)
        args[i] = bad
        with pytest.raises(lib.ParaganError):
            lib.paragan_blocknorm_bwd(ctx, d, *args)
    shared = lib.blocknorm_desc(x, h, zo, y, rows[:1].expand(2, 32), kind=lib.NORM_RMS, eps=EPS)   # one row: given as one
    with pytest.raises(lib.ParaganError):
        lib.paragan_blocknorm_fwd(ctx, shared, x, h, None, rows[:1].expand(2, 32), None, None, None, None, zo, y, None)
    d0 = lib.blocknorm_desc(x, None, None, y, kind=lib.NORM_RMS, eps=EPS)
    for args in ([x, None, None, None, None, None, None, None, saved, None, None, grads[0]] + [None] * 6 + [ws],
                 [x, None, None, None, None, None, None, None, saved, None, y, grads[0], None, grads[2]] + [None] * 4 + [ws]):
        with pytest.raises(lib.ParaganError):
            lib.paragan_blocknorm_bwd(ctx, d0, *args)
    ds = lib.scan_desc(x, x, x, zo, sharp=SHARP)
    sb, wb = lib.paragan_scan_sizes(ds)
    saved, ws, st = lib.workspace(sb), lib.workspace(wb), z(2, 32, dt=f)
    fwd = [x, h, x, vec, lens, st, zo, st, saved, ws]
    for i, bad in ((0, None), (1, odd), (2, x.float()), (3, z(16, dt=f)), (3, None), (4, lens[:1]), (5, z(2, 16, dt=f)), (5, st.bfloat16()), (6, None),
                   (7, z(1, 32, dt=f)), (8, saved[16:]), (9, None), (9, ws[1:])):
        args = list(fwd)
        args[i] = bad
        with pytest.raises(lib.ParaganError):
            lib.paragan_scan_fwd(ctx, ds, *args)
    g3 = [z(2, 8, 32) for _ in range(3)]
    bwd = [x, h, x, vec, lens, saved, y, st, *g3, z(32, dt=f), z(2, 32, dt=f), ws]
    for i, bad in ((5, None), (6, None), (7, z(2, 8, dt=f)), (8, None), (9, odd), (10, z(2, 8, 32, dt=f)), (11, None), (12, vec), (13, None)):
        args = list(bwd)
        args[i] = bad
        with pytest.raises(lib.ParaganError):
            lib.paragan_scan_bwd(ctx, ds, *args)
    a, b = z(100, dt=f), z(100, dt=f)
    for grads_, outs in (([a, a], None), ([a, a[50:]], None), ([a], [b[:50]]), ([a[:60]], [a[40:]]), ([a, b], [b, a]), ([a], [b.bfloat16()]),
                         ([a.view(10, 10).t()], None), ([a.cpu()], None)):
        with pytest.raises(lib.ParaganError):
            lib.ClipPlan(grads_, outs)
    plan, norm = lib.ClipPlan([a], [b]), z(2, dt=f)
    ws = lib.workspace(plan.ws_bytes)
    for args in ((0.0, 1.0, norm, ws), (-1.0, 1.0, norm, ws), (math.nan, 1.0, norm, ws), (1.0, 0.0, norm, ws), (1.0, math.inf, norm, ws),
                 (1.0, math.nan, norm, ws), (1.0, 1.0, norm[:1], ws), (1.0, 1.0, norm.double(), ws), (1.0, 1.0, norm, None), (1.0, 1.0, norm, ws[8:])):
        with pytest.raises(lib.ParaganError):
            lib.paragan_clip(ctx, plan, *args)
    torch.cuda.synchronize()
    assert all(bool((t == 3.0).all()) for t in (zo, y, st, b, norm, *grads, *g3, bwd[11], bwd[12]))


def test_clip_far_and_many():
    """A gradient of more than 2^31 elements, and pieces of very many tensors."""
    torch = need_gpu()
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    big = torch.zeros((1 << 31) + 5, dtype=torch.bfloat16, device="cuda")
    big[-3:], big[0], big[1 << 30] = 2.0, 2.0, 4.0
    small = [torch.full((3,), 1.0, device="cuda") for _ in range(4000)]
    plan = lib.ClipPlan([big] + small)
    norm = torch.zeros(2, device="cuda")
    lib.paragan_clip(lib.Context(), plan, 1.0, 1.0, norm, lib.workspace(plan.ws_bytes))
    torch.cuda.synchronize()
    want = math.sqrt(4 * 4.0 + 16.0 + 12000.0)
    assert abs(norm[0].item() - want) <= 2 * U32 * want
    assert all(abs(t[2].item() - 1 / want) <= 4 * U32 / want for t in (small[0], small[-1]))
    assert abs(big[-1].item() - 2 / want) <= U16 * 2.1 / want and big[5].item() == 0.0
