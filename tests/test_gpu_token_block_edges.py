"""Calls at the edges of what the token block's operators accept."""
import numpy as np
import pytest

from oracle import token_block as T
from paragan_2411_03999_amd import lib

from .parity import need_gpu
from .test_gpu_token import held
from .test_gpu_token_block import Rows, num

pytestmark = pytest.mark.gpu

U16, U32 = T.U16, T.U32


# ------------------------------------------------------------- recurrence over tokens that overlap
def windows(torch, gen, B, S, D, st, lens, dt):
    """[B][S][D] whose tokens lie `st` elements apart, st < D allowed; what no token of a sequence holds is NaN."""
    n = (S - 1) * st + D
    buf = torch.full((B, n + 16), float("nan"), dtype=dt)
    for b, m in enumerate(lens):
        if m:
            buf[b, 8:8 + (m - 1) * st + D] = torch.randn((m - 1) * st + D, generator=gen).to(dt)
    return buf.cuda().as_strided((B, S, D), (n + 16, st, 1), 8)


def overlapping(torch, B, S, D, strides, lens, reverse, f32, seed):
    gen = torch.Generator().manual_seed(seed + S + D)
    dt = torch.float32 if f32 else torch.bfloat16
    x, r, g = (windows(torch, gen, B, S, D, D if st is None else st, lens, dt) for st in strides)
    dec, h0 = (torch.rand(D, generator=gen) * 5 - 8).cuda(), torch.randn(B, D, generator=gen).cuda()
    y, ht = Rows(torch, B, S, D, dt, fill=7.0), torch.full((B, D), 7.0, device="cuda")
    d = lib.scan_desc(x, r, g, y.v, sharp=8.0, reverse=reverse)
    saved, ws = (lib.workspace(n) for n in lib.paragan_scan_sizes(d))
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def run():
        lib.paragan_scan_fwd(lib.Context(), d, x, r, g, dec, L, h0, y.v, ht, saved, ws)
        torch.cuda.synchronize()
        return y, ht
    return x, r, g, dec, h0, run


@pytest.mark.parametrize("f32", [0, 1])
@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("S", [12, 40, 300, 1000])   # a thread a sequence, one tile or two, several, in chunks
@pytest.mark.parametrize("strides", [(8, None, None), (None, 16, 40), (8, 8, 8), (64, 0, 24)])
def test_scan_over_windows(strides, S, reverse, f32):
    """Tokens that overlap (strides between 0 and the width), each with all of its channels, the last ones of a length too."""
    torch = need_gpu()
    B, D = 4, 72
    lens = [S, S - 5, 0, S // 3]
    x, r, g, dec, h0, run = overlapping(torch, B, S, D, strides, lens, reverse, f32, 3)
    y, ht = run()
    clean = lambda t: np.nan_to_num(num(t))  # noqa: E731
    want = T.scan(clean(x), clean(r), clean(g), num(dec), lens, sharp=8.0, reverse=reverse, h0=num(h0), uo=U32 if f32 else U16)
    held("y", y.v, want["y"], want["tol.y"] + 1e-30)
    held("ht", ht, want["ht"], want["tol.ht"] + 1e-30)
    assert y.untouched(7.0)


@pytest.mark.parametrize("reverse", [0, 1])
@pytest.mark.parametrize("S", [40, 1000])
def test_scan_windows_keep_nan_in_their_channels(S, reverse):
    """A NaN that a token past the length would share with the last ones reaches the channels of those that own it."""
    torch = need_gpu()
    B, D, st, cut = 2, 72, 16, S - 9
    for which in range(3):
        x, r, g, dec, h0, run = overlapping(torch, B, S, D, (st, st, st), [cut, S], reverse, 0, 5 + which)
        (x, r, g)[which][0, cut - 1, 50] = float("nan")
        hit = np.zeros((S, D), bool)
        for t in range(cut):
            if 0 <= (cut - 1 - t) * st + 50 < D:
                hit[t, (cut - 1 - t) * st + 50] = True
        order = hit[:cut][::-1] if reverse else hit[:cut]
        after = np.logical_or.accumulate(order, 0)
        want = np.zeros((B, S, D), bool)
        want[0, :cut] = after[::-1] if reverse else after
        y, ht = run()
        assert np.array_equal(np.isnan(num(y.v)), want), (which, "y")
        assert np.array_equal(np.isnan(num(ht)), np.stack([after[-1], np.zeros(D, bool)])), (which, "ht")
