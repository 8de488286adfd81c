"""The float64 definitions of the token block's operators against finite
differences and element-by-element loops, and the refusals of the library's
entry points (no GPU needed)."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from oracle import token_block as T
from paragan_2411_03999_amd import lib

from .test_token_oracle import diff


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lib.LIB_PATH):
        from paragan_2411_03999_amd.build import build
        build()
    return lib.load()


# ------------------------------------------------------------- definitions
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("branch,post,pre", [(1, 0, 1), (1, 1, 1), (0, 0, 1), (1, 0, 0), (1, 1, 0)])
def test_blocknorm_gradient_by_differences(layer, branch, post, pre):
    r = np.random.default_rng(1)
    B, S, D = 2, 3, 8
    n = lambda *s: r.normal(size=s)  # noqa: E731
    x, h, g1, g2 = n(B, S, D), n(B, S, D), n(D), n(D)
    for shared in (False, True):
        gate, scale, shift = (n(1 if shared else B, D) for _ in range(3))
        dz, dy = n(B, S, D), n(B, S, D)
        kw = dict(layer=layer, branch=branch, post=post, pre=pre, eps=0.01, res_scale=0.7, shared=shared)
        args = (x, h, g1 if post else None, gate, g2, scale, shift, [3, 1])

        def f():
            o = T.blocknorm(*args, **kw)
            return np.concatenate([(o["z"] * dz).ravel() if branch else np.zeros(1), (o["y"] * dy).ravel() if pre else np.zeros(1)])
        got = T.blocknorm(*args, **kw, dz=dz if branch else None, dy=dy if pre else None)
        for t, name in ((x, "dx"), (h, "dh"), (g1, "dgain_post"), (gate, "dgate"), (g2, "dgain_pre"), (scale, "dscale"), (shift, "dshift")):
            if name in got:
                assert np.abs(diff(f, t, 1.0) - got[name]).max() < 1e-7, name
        assert not got["dx"][1, 1:].any()


def test_blocknorm_by_loops():
    r = np.random.default_rng(2)
    x, h, gate = r.normal(size=(2, 3, 8)), r.normal(size=(2, 3, 8)), r.normal(size=(2, 8))
    o = T.blocknorm(x, h, None, gate, None, None, None, [3, 2], layer=True, branch=1, post=0, pre=1, eps=0.5, res_scale=2.0)
    for b, s in ((0, 0), (0, 2), (1, 1)):
        z = [x[b, s, c] + 2 * gate[b, c] * h[b, s, c] for c in range(8)]
        mean = sum(z) / 8
        var = sum((v - mean) ** 2 for v in z) / 8
        assert np.allclose(o["z"][b, s], z) and np.allclose(o["y"][b, s], [(v - mean) / math.sqrt(var + 0.5) for v in z])
    assert not o["z"][1, 2].any() and not o["y"][1, 2].any()


@pytest.mark.parametrize("reverse", [False, True])
def test_scan_by_loops_and_differences(reverse):
    r = np.random.default_rng(3)
    B, S, D = 3, 5, 4
    n = lambda *s: r.normal(size=s)  # noqa: E731
    x, rr, g, decay, h0, dy, dht = n(B, S, D), n(B, S, D), n(B, S, D), n(D) - 2, n(B, D), n(B, S, D), n(B, D)
    lens = [5, 0, 3]
    kw = dict(sharp=3.0, reverse=reverse)
    o = T.scan(x, rr, g, decay, lens, h0=h0, dy=dy, dht=dht, **kw)
    for b in range(B):
        for c in range(D):
            h = h0[b, c]
            for i in range(lens[b]):
                t = lens[b] - 1 - i if reverse else i
                a = math.exp(-3.0 * math.log(1 + math.exp(decay[c])) / (1 + math.exp(-rr[b, t, c])))
                h = a * h + math.sqrt(1 - a * a) * x[b, t, c] / (1 + math.exp(-g[b, t, c]))
                assert abs(o["y"][b, t, c] - h) < 1e-12
            assert abs(o["ht"][b, c] - h) < 1e-12
    f = lambda: (lambda v: np.concatenate([(v["y"] * dy).ravel(), (v["ht"] * dht).ravel()]))(T.scan(x, rr, g, decay, lens, h0=h0, **kw))  # noqa: E731
    for t, name in ((x, "dx"), (rr, "dr"), (g, "dg"), (decay, "ddecay"), (h0, "dh0")):
        assert np.abs(diff(f, t, 1.0) - o[name]).max() < 1e-7, name
    assert not o["dx"][1].any() and not o["y"][2, 3:].any() and np.array_equal(o["dh0"][1], dht[1])


def test_clip_formula():
    g = [np.array([3.0]), np.array([0.0, 4.0])]
    norm, k, out = T.clip(g, 2.5)
    assert norm == 5.0 and k == 0.5 and out[1][1] == 2.0
    assert T.clip(g, 5.0)[1] == 1.0 and T.clip(g, 5.0, 2.0)[:2] == (10.0, 1.0) and T.clip(g, math.inf, 2.0)[1] == 2.0


# ------------------------------------------------------------- refusals
def bn(**kw):
    two = C.c_int64 * 2
    st = [two(10 * 64, 64) for _ in range(4)]
    d = lib.BlockNormDesc(4, 10, 64, lib.BF16, lib.BF16, lib.NORM_RMS, 1, 1, 1, 1e-6, 1.0, 192, *st)
    for k, v in kw.items():
        setattr(d, k, two(*v) if k.endswith("stride") and k != "mod_stride" else v)
    return d


def test_blocknorm_refusals(L):
    assert lib.paragan_blocknorm_check(bn()) == lib.OK
    good = (dict(stream_dtype=lib.F32), dict(dtype=lib.F32, stream_dtype=lib.F32), dict(D=8192, x_stride=(81920, 8192), h_stride=(81920, 8192),
            z_stride=(81920, 8192), y_stride=(81920, 8192), mod_stride=8192), dict(mod_stride=0), dict(mod_stride=64), dict(branch=0, post=0),
            dict(pre=0), dict(x_stride=(0, 64)), dict(B=1, z_stride=(0, 64)), dict(res_scale=-2.0), dict(z_stride=(64, 256)),
            dict(B=1, S=2 ** 30))
    for kw in good:
        assert lib.paragan_blocknorm_check(bn(**kw)) == lib.OK, kw
    nan = float("nan")
    bad = (dict(B=0), dict(S=0), dict(S=-1), dict(B=1 << 16, S=1 << 15), dict(B=1, S=2 ** 30 + 1), dict(B=2 ** 20 + 1, S=1), dict(D=0), dict(D=4), dict(D=60), dict(D=8200), dict(dtype=2),
           dict(dtype=lib.F32), dict(stream_dtype=7), dict(kind=2), dict(branch=2), dict(post=-1), dict(pre=3), dict(branch=0), dict(branch=0, post=0, pre=0),
           dict(eps=0.0), dict(eps=1e-39), dict(eps=nan), dict(eps=float("inf")), dict(res_scale=nan), dict(mod_stride=32), dict(mod_stride=100),
           dict(mod_stride=-192), dict(x_stride=(640, -64)), dict(x_stride=(640, 63)), dict(h_stride=(1 << 58, 64)), dict(z_stride=(0, 64)),
           dict(y_stride=(640, 32)), dict(z_stride=(64, 64)), dict(y_stride=(632, 64)))
    for kw in bad:
        assert lib.paragan_blocknorm_check(bn(**kw)) == lib.EINVAL, kw
        assert L.paragan_last_error(None).decode().startswith("blocknorm")
    assert L.paragan_blocknorm_check(None) == lib.EINVAL
    assert L.paragan_blocknorm_fwd(None, *[None] * 12) == lib.EINVAL
    assert L.paragan_blocknorm_bwd(None, *[None] * 20) == lib.EINVAL
    s, w = lib.paragan_blocknorm_sizes(bn())
    assert s >= 4 * 10 * 16 and w > 0
    with pytest.raises(lib.ParaganError):
        lib.paragan_blocknorm_sizes(bn(D=9))


def sc(**kw):
    two = C.c_int64 * 2
    d = lib.ScanDesc(4, 10, 64, lib.BF16, 0, 8.0, two(1920, 192), two(1920, 192), two(1920, 192), two(640, 64))
    for k, v in kw.items():
        setattr(d, k, two(*v) if k.endswith("stride") else v)
    return d


def test_scan_refusals(L):
    assert lib.paragan_scan_check(sc()) == lib.OK
    for kw in (dict(dtype=lib.F32), dict(reverse=1), dict(x_stride=(0, 192)), dict(r_stride=(0, 0)), dict(S=1, y_stride=(64, 0)), dict(sharp=1e-3)):
        assert lib.paragan_scan_check(sc(**kw)) == lib.OK, kw
    nan = float("nan")
    for kw in (dict(B=0), dict(S=0), dict(B=1 << 16, S=1 << 15), dict(B=1, S=2 ** 30 + 1), dict(B=2 ** 22 + 1, S=1), dict(D=0), dict(D=12), dict(D=(1 << 20) + 8), dict(dtype=3), dict(reverse=2),
               dict(sharp=0.0), dict(sharp=-1.0), dict(sharp=nan), dict(sharp=float("inf")), dict(y_stride=(0, 64)), dict(y_stride=(640, 56)),
               dict(x_stride=(1920, 100)), dict(g_stride=(-1920, 192)), dict(r_stride=(1 << 58, 192)), dict(B=1 << 14, D=1 << 17), dict(x_stride=(1 << 28, 1 << 20))):
        assert lib.paragan_scan_check(sc(**kw)) == lib.EINVAL, kw
        assert L.paragan_last_error(None).decode().startswith("scan")
    assert L.paragan_scan_check(None) == lib.EINVAL
    assert L.paragan_scan_fwd(None, *[None] * 11) == lib.EINVAL
    assert L.paragan_scan_bwd(None, *[None] * 15) == lib.EINVAL
    s, w = lib.paragan_scan_sizes(sc())
    assert s > 0 and w > 0


def tensors(*rows):
    arr = (lib.ClipTensor * len(rows))()
    for i, t in enumerate(rows):
        arr[i] = lib.ClipTensor(*t)
    return arr


def clip_sizes(L, arr):
    n, w = C.c_size_t(), C.c_size_t()
    rc = L.paragan_clip_sizes(arr, len(arr), C.byref(n), C.byref(w))
    return rc, n.value, w.value


def test_clip_plan(L):
    """The plan's pieces cover every tensor once, in order."""
    a = 1 << 20
    arr = tensors((a, a, 40000, lib.F32, 0), (a + 160000, a + 160000, 0, lib.F32, 0), (a + 160002, a + 800002, 16385, lib.BF16, 0))
    rc, n, w = clip_sizes(L, arr)
    assert rc == lib.OK and w > 0
    host, d = np.zeros(n, np.uint8), lib.ClipDesc()
    assert L.paragan_clip_plan(arr, 3, C.byref(d), C.c_void_p(host.ctypes.data)) == lib.OK
    assert (d.n_tensors, d.n_elements, d.bytes, d.in_place) == (3, 56385, 160000 + 32770, 0)
    piece = host.view(np.dtype([("src", "u8"), ("dst", "u8"), ("n", "i4"), ("bf16", "i4")]))
    assert len(piece) == d.n_pieces
    for bf16, at, to, n in ((0, a, a, 40000), (1, a + 160002, a + 800002, 16385)):
        for p in piece[piece["bf16"] == bf16]:
            assert p["src"] == at and p["dst"] == to and 0 < p["n"] <= n
            n -= int(p["n"])
            at, to = at + int(p["n"]) * (2 if bf16 else 4), to + int(p["n"]) * (2 if bf16 else 4)
        assert n == 0
    assert list(piece["bf16"]) == sorted(piece["bf16"])


def test_clip_refusals(L):
    a = 1 << 20
    for arr in (tensors((a, a, 10, 5, 0)), tensors((a, a, -1, lib.F32, 0)), tensors((0, a, 4, lib.F32, 0)), tensors((a, 0, 4, lib.F32, 0)),
                tensors((a + 2, a + 2, 4, lib.F32, 0)), tensors((a + 1, a + 1, 4, lib.BF16, 0)), tensors((a, a, 4, lib.F32, 1)),
                tensors((a, a, (1 << 40) + 1, lib.F32, 0)),
                tensors((a, a, 10, lib.F32, 0), (a, a, 10, lib.F32, 0)),                    # named twice
                tensors((a, a, 10, lib.F32, 0), (a + 36, a + 36, 10, lib.F32, 0)),          # overlap
                tensors((a, a + 8, 10, lib.F32, 0)),                                        # an output on its own gradient
                tensors((a, a + 4000, 10, lib.F32, 0), (a + 400, a + 4036, 10, lib.F32, 0)),
                tensors((a, a + 400, 10, lib.F32, 0), (a + 400, a + 400, 10, lib.F32, 0))):  # an output on another gradient
        assert clip_sizes(L, arr)[0] == lib.EINVAL
        assert L.paragan_last_error(None).decode().startswith("clip")
        assert L.paragan_clip_plan(arr, len(arr), C.byref(lib.ClipDesc()), C.c_void_p(1 << 20)) == lib.EINVAL
    assert L.paragan_clip_sizes(None, 1, None, None) == lib.EINVAL
    ok = tensors((a, a, 10, lib.F32, 0))
    assert L.paragan_clip_sizes(ok, 0, None, None) == lib.EINVAL
    assert L.paragan_clip_plan(ok, 1, None, None) == lib.EINVAL
    assert L.paragan_clip_plan(ok, 1, C.byref(lib.ClipDesc()), None) == lib.EINVAL
    assert L.paragan_clip(None, None, None, 1.0, 1.0, None, None) == lib.EINVAL


def test_step_clip_refusals(L):
    n = C.c_size_t()
    assert L.paragan_grad_clip_size(C.byref(n)) == lib.OK and n.value >= 16 and L.paragan_grad_clip_size(None) == lib.EINVAL
    assert L.paragan_set_grad_clip(None, 1.0, 1.0, C.c_void_p(256)) == lib.EINVAL


def test_binding_refuses_before_the_library():
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    x, h = z(2, 5, 16), z(2, 5, 16)
    kw = dict(kind=lib.NORM_RMS, eps=1e-6)
    for args in ((x, h, None, h, None), (x, None, None, None, None), (x, h, z(2, 5, 8), h, None), (x, h, x.float(), h, None),
                 (x, h, x, z(2, 5, 16, dt=torch.float16), None), (x, z(2, 16, 5).transpose(1, 2), x, h, None), (x, h, x, h, z(3, 16)),
                 (x, h, x, h, z(2, 8)), (x[0], h[0], x[0], h[0], None)):
        with pytest.raises(lib.ParaganError):
            lib.blocknorm_desc(*args, **kw)
    d = lib.blocknorm_desc(x, h, x, h, z(2, 48, dt=torch.float32)[:, 16:32], **kw)
    assert d.mod_stride == 48 and lib.blocknorm_desc(x, h, x, h, z(1, 16), **kw).mod_stride == 0
    for args in ((x, h, h, x.float()), (x, h, h, z(2, 5, 8)), (x.half(),) * 4, (z(2, 16, 5).transpose(1, 2),) * 4):
        with pytest.raises(lib.ParaganError):
            lib.scan_desc(*args, sharp=8.0)
    for g, o in (([], None), ([x], []), ([x], [h.float()]), ([x.transpose(0, 1)], None), ([x], None), ([x.half()], None)):
        with pytest.raises(lib.ParaganError):
            lib.ClipPlan(g, o)
