"""The float64 definitions of the token attention operators against finite
differences and element-by-element loops, and the refusals of the library's
entry points (no GPU needed)."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from oracle import token as T
from paragan_2411_03999_amd import lib


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lib.LIB_PATH):
        from paragan_2411_03999_amd.build import build
        build()
    return lib.load()


def diff(f, x, dy, eps=1e-6):
    """Gradient of sum(f() * dy) in the elements of x by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        up = (f() * dy).sum()
        x[i] = old - eps
        g[i] = ((up - (f() * dy).sum()) / (2 * eps))
        x[i] = old
    return g


@pytest.mark.parametrize("inter", [False, True])
def test_qknorm_gradient_by_differences(inter):
    r = np.random.default_rng(1)
    x, gain, dy = r.normal(size=(4, 2, 24)), r.normal(size=24), r.normal(size=(4, 2, 24))
    ang = r.normal(size=(5, 8))
    table = np.stack([np.cos(ang), np.sin(ang)], -1)
    pos = np.array([3, -1, 5, 0])          # two of the four are padding
    f = lambda: T.qknorm_fwd(x, gain, table, pos, 16, inter, 1e-3)  # noqa: E731
    assert not f()[1].any() and not f()[2].any()
    dx, dg = T.qknorm_bwd(x, gain, table, pos, 16, inter, 1e-3, dy)
    assert np.abs(diff(f, x, dy) - dx).max() < 1e-7
    assert np.abs(diff(f, gain, dy) - dg).max() < 1e-7


def test_rotation_turns_pairs():
    x = np.zeros((1, 1, 16))
    x[0, 0, 1] = 2.0
    t = np.zeros((1, 8, 2))
    t[0, :, 0], t[0, :, 1] = 0.6, 0.8
    y = T.rotate(x, t, np.array([0]), 16, False)
    assert np.allclose(y[0, 0, 1], 1.2) and np.allclose(y[0, 0, 9], 1.6)
    y = T.rotate(x, t, np.array([0]), 16, True)       # second of the pair (0, 1)
    assert np.allclose(y[0, 0, 0], -1.6) and np.allclose(y[0, 0, 1], 1.2)
    assert np.allclose(T.rotate(y, t, np.array([0]), 16, True, inverse=True), x)


@pytest.mark.parametrize("nb,maxd,causal", [(32, 128, True), (32, 128, False), (8, 16, False), (2, 512, True),
                                            (64, 100, True), (256, 512, False)])
def test_buckets_follow_the_real_formula(nb, maxd, causal):
    m = nb if causal else nb // 2
    first = m // 2
    one = [T.bucket_of(n, m, maxd) for n in range(maxd + 40)]
    assert one[:first] == list(range(first)) and one[maxd] == m - 1 and one == sorted(one)
    for n in range(first, maxd):
        e = math.log(n / first) / math.log(maxd / first) * (m - first)
        if abs(e - round(e)) > 1e-9:
            assert one[n] == min(m - 1, first + math.floor(e)), n


@pytest.mark.parametrize("causal,window,sink,nb", [(True, 0, 0, 0), (True, 3, 2, 4), (False, 2, 1, 8), (False, 0, 0, 4)])
def test_mha_by_loops_and_differences(causal, window, sink, nb):
    r = np.random.default_rng(2)
    B, Sq, Sk, Hq, Hk, d, maxd = 2, 4, 6, 4, 2, 3, 5
    q, k, v, do = r.normal(size=(B, Sq, Hq, d)), r.normal(size=(B, Sk, Hk, d)), r.normal(size=(B, Sk, Hk, d)), None
    do = r.normal(size=q.shape)
    table = r.normal(size=(Hq, nb)) if nb else None
    lq, lk = [4, 2], [6, 1]                # the second: one key, two queries, the first of them before it
    kw = dict(causal=causal, window=window, n_sink=sink, table=table, max_distance=maxd, len_q=lq, len_k=lk)
    got = T.mha(q, k, v, 0.7, dout=do, **kw)
    of = T.bucket_table(nb, maxd, causal) if nb else None
    for b in range(B):
        for i in range(Sq):
            for h in range(Hq):
                p, num, den = i + lk[b] - lq[b], np.zeros(d), 0.0
                for j in range(lk[b]):
                    if i >= lq[b] or (causal and j > p) or (window and abs(p - j) >= window and j >= sink):
                        continue
                    s = 0.7 * q[b, i, h] @ k[b, j, h // 2]
                    if nb:
                        s += table[h, of[min(max(j - p, -maxd), maxd) + maxd]]
                    num, den = num + math.exp(s) * v[b, j, h // 2], den + math.exp(s)
                assert np.allclose(got["o"][b, i, h], num / den if den else 0.0, atol=1e-12)
    f = lambda: T.mha(q, k, v, 0.7, **kw)["o"]  # noqa: E731
    for x, n in ((q, "dq"), (k, "dk"), (v, "dv")) + (((table, "dtable"),) if nb else ()):
        assert np.abs(diff(f, x, do) - got[n]).max() < 1e-8, n


# ------------------------------------------------------------- refusals
def qk(**kw):
    d = lib.QkNormDesc(100, 8, 2, 64, 64, 0, 256, lib.BF16, 1e-6, 512, 128, 512, 128)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_qknorm_refusals(L):
    assert lib.paragan_qknorm_check(qk()) == lib.OK
    assert lib.paragan_qknorm_check(qk(dtype=lib.F32, interleaved=1, rot=0, T=(1 << 31) - 1)) == lib.OK
    assert lib.paragan_qknorm_check(qk(d=8, rot=0)) == lib.OK
    bad = [dict(T=0), dict(T=1 << 31), dict(Hq=0), dict(Hk=0), dict(Hk=-1), dict(d=0), dict(d=60), dict(d=264, ldq=9999),
           dict(rot=-16), dict(rot=8), dict(rot=80), dict(interleaved=2), dict(n_pos=0), dict(dtype=2), dict(eps=0.0),
           dict(eps=float("nan")), dict(eps=float("inf")), dict(ldq=511), dict(ldk=120), dict(ldqo=516), dict(ldko=0),
           dict(ldq=1 << 62), dict(ldk=-128)]
    for b in bad:
        assert lib.paragan_qknorm_check(qk(**b)) == lib.EINVAL, b
        assert b"qknorm" in L.paragan_last_error(None)
    assert L.paragan_qknorm_check(None) == lib.EINVAL
    assert lib.paragan_qknorm_ws_size(qk()) > 0
    assert L.paragan_qknorm_ws_size(C.byref(qk()), None) == lib.EINVAL
    assert L.paragan_qknorm_fwd(None, C.byref(qk()), *[None] * 8) == lib.EINVAL
    assert L.paragan_qknorm_bwd(None, C.byref(qk()), *[None] * 13) == lib.EINVAL


def mh(**kw):
    st = lambda s, h: (C.c_int64 * 3)(s * h * 64, h * 64, 64)  # noqa: E731
    d = lib.MhaDesc(2, 100, 100, 8, 2, 64, 1, 16, 4, 32, 128, 0.125, st(100, 8), st(100, 2), st(100, 2), st(100, 8))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def s3(*v):
    return (C.c_int64 * 3)(*v)


def test_mha_refusals(L):
    assert lib.paragan_mha_check(mh()) == lib.OK
    ok = [dict(window=0), dict(n_buckets=0, max_distance=0), dict(causal=0), dict(d=8), dict(n_buckets=256, max_distance=512),
          dict(k_stride=s3(0, 128, 64)), dict(k_stride=s3(1 << 32, (1 << 24) - 8, 64)), dict(window=1 << 29, n_sink=1 << 29), dict(q_stride=s3(0, 0, 0)),            # broadcast inputs of a forward
          dict(o_stride=s3(64 * 100 * 8, 64, 6400)), dict(n_buckets=2, max_distance=2),
          dict(B=1, Hq=2, Hk=1, Sk=1 << 29, Sq=1, k_stride=s3(0, 64, 64), o_stride=s3(0, 0, 64))]
    for g in ok:
        assert lib.paragan_mha_check(mh(**g)) == lib.OK, (g, L.paragan_last_error(None))
    bad = [dict(B=0), dict(Sq=0), dict(Sk=0), dict(Hq=0), dict(Hk=0), dict(Hk=3), dict(d=0), dict(d=4), dict(d=136),
           dict(causal=2), dict(window=-1), dict(n_sink=-1), dict(n_buckets=-2), dict(n_buckets=1), dict(n_buckets=257),
           dict(causal=0, n_buckets=2), dict(causal=0, n_buckets=33), dict(max_distance=513), dict(max_distance=16),
           dict(max_distance=0), dict(scale=0.0), dict(scale=1e-38), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
           dict(q_stride=s3(51200, 512, 60)), dict(k_stride=s3(-128, 128, 64)), dict(v_stride=s3(1 << 62, 128, 64)),
           dict(o_stride=s3(0, 512, 64)), dict(o_stride=s3(51200, 512, 56)), dict(Sq=(1 << 29) + 8), dict(window=(1 << 29) + 1), dict(n_sink=(1 << 29) + 1), dict(k_stride=s3(1 << 32, 1 << 24, 64)), dict(B=1 << 30),
           dict(Sq=1 << 29, Sk=1 << 29)]
    for b in bad:
        assert lib.paragan_mha_check(mh(**b)) == lib.EINVAL, b
        assert b"mha" in L.paragan_last_error(None)
    assert L.paragan_mha_check(None) == lib.EINVAL
    saved, ws = lib.paragan_mha_sizes(mh())
    assert saved >= 2 * 8 * 100 * 4 and ws > 0 and saved % 256 == 0
    assert L.paragan_mha_fwd(None, C.byref(mh()), *[None] * 9) == lib.EINVAL
    assert L.paragan_mha_bwd(None, C.byref(mh()), *[None] * 14) == lib.EINVAL


def test_mha_workspaces_stay_in_proportion(L):
    """Half a long sequence as first tokens of a short window would give millions of pieces of key blocks; many
    sequences of one new token need no partials."""
    one = dict(B=1, Hq=1, Hk=1, n_buckets=0, max_distance=0)
    for n in (1 << 20, 1 << 22):
        st = s3(64 * n, 64, 64)
        d = mh(Sq=n, Sk=n, window=16, n_sink=n // 2, q_stride=st, k_stride=st, v_stride=st, o_stride=st, **one)
        assert lib.paragan_mha_check(d) == lib.OK
        assert lib.paragan_mha_sizes(d)[1] < 2 * 4 * n + (3 << 29)
    d = mh(B=4096, Sq=1, Sk=4096, n_buckets=0, max_distance=0, q_stride=s3(512, 512, 64), o_stride=s3(512, 512, 64),
           k_stride=s3(4096 * 128, 128, 64), v_stride=s3(4096 * 128, 128, 64))
    assert lib.paragan_mha_sizes(d)[1] < 64 << 20


def test_descriptors_refuse_tensors_that_do_not_belong_together():
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    d = lib.mha_desc(z(2, 5, 4, 32), z(2, 7, 2, 32), z(2, 7, 2, 32), z(2, 5, 4, 32), scale=0.1)
    assert (d.B, d.Sq, d.Sk, d.Hq, d.Hk, d.d) == (2, 5, 7, 4, 2, 32) and list(d.q_stride) == [640, 128, 32]
    for q, k, v, o in ((z(2, 5, 4, 32), z(1, 7, 2, 32), z(2, 7, 2, 32), z(2, 5, 4, 32)),
                       (z(2, 5, 4, 32), z(2, 7, 2, 32), z(2, 7, 2, 16), z(2, 5, 4, 32)),
                       (z(2, 5, 4, 32), z(2, 7, 2, 32), z(2, 7, 2, 32), z(2, 4, 4, 32)),
                       (z(2, 5, 4, 32, dt=torch.float32), z(2, 7, 2, 32), z(2, 7, 2, 32), z(2, 5, 4, 32)),
                       (z(2, 5, 32, 4).transpose(2, 3), z(2, 7, 2, 32), z(2, 7, 2, 32), z(2, 5, 4, 32))):
        with pytest.raises(lib.ParaganError):
            lib.mha_desc(q, k, v, o, scale=0.1)
    d = lib.qknorm_desc(z(9, 6, 16)[:, :4], z(9, 2, 16), rot=16, interleaved=0, n_pos=3, eps=1e-6)
    assert (d.T, d.Hq, d.Hk, d.d, d.ldq, d.ldk, d.ldqo) == (9, 4, 2, 16, 96, 32, 64)
    for q, k in ((z(9, 4, 16), z(8, 2, 16)), (z(9, 4, 16), z(9, 2, 8)), (z(9, 4, 16), z(9, 2, 16, dt=torch.float32)),
                 (z(9, 4, 16, dt=torch.float16), z(9, 2, 16, dt=torch.float16)),
                 (z(4, 9, 16).transpose(0, 1), z(9, 2, 16))):
        with pytest.raises(lib.ParaganError):
            lib.qknorm_desc(q, k, rot=0, interleaved=0, n_pos=1, eps=1e-6)


def test_mha_tensors_are_held_to_the_descriptor():
    """Tensors that lie elsewhere than the descriptor says, or are too short, are refused before any pointer is passed on;
    other views of the same memory are as good (these stop at not being on the GPU)."""
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    qkv = z(2, 7, 8, 32)                                          # one projection buffer, and its gradient's views
    q, k, v, o = qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:], z(2, 7, 4, 32)
    d = lib.mha_desc(q, k, v, o, scale=0.1, n_buckets=8, max_distance=20)
    g = torch.empty_like(qkv)
    put = lambda t, name: lib._placed(d, lib._mha_dims, (name,), t)[0]  # noqa: E731
    for t, kind in ((g[:, :, :4], "dq"), (g[:, :, 4:6], "dk"), (g[:, :, 6:], "dv"), (torch.empty_like(o), "dout"), (q, "q"),
                    (k, "k"), (v, "v"), (o, "o"), (z(14, 128), "o"), (z(2, 7, 2, 64), "o"), (z(2, 7, 1, 4, 32), "o")):
        with pytest.raises(lib.ParaganError, match="on the GPU"):
            put(t, kind)
    for t, kind in ((torch.empty_like(k), "dk"), (z(2, 7, 2, 32), "dv"), (z(2, 7, 4, 32), "dq"), (g[:, :, :2], "q"),
                    (g[:, :, :4], "o"), (z(2, 7, 4, 32, dt=torch.float32), "o"), (z(2, 7, 4, 32, dt=torch.float16), "o"),
                    (z(2, 6, 4, 32), "o"), (z(2, 4, 7, 32).transpose(1, 2), "o"), (g[:1, :, :4], "q"), (z(2 * 7 * 4 * 32), "q")):
        with pytest.raises(lib.ParaganError, match="not where the descriptor says"):
            put(t, kind)
    d.Sq, d.Sk = 6, 6                                             # a descriptor changed afterwards
    with pytest.raises(lib.ParaganError, match="not where"):
        put(torch.empty_like(o), "o")
    one = lib.mha_desc(z(1, 1, 1, 8), z(1, 9, 1, 8), z(1, 9, 1, 8), z(1, 1, 1, 8), scale=1.0)
    with pytest.raises(lib.ParaganError, match="on the GPU"):
        lib._placed(one, lib._mha_dims, ("o",), z(8))
    with pytest.raises(lib.ParaganError, match="on the GPU"):     # strides of single elements mean nothing
        lib._placed(one, lib._mha_dims, ("o",), z(3, 5, 2, 8)[:1, :1, :1])
    f = torch.float32
    for t, n in ((z(4, 8, dt=f), (32, 8)), (z(32, dt=f), (32, 8)), (z(6, 8, dt=f), (32, 8)), (z(9, dt=f), (9,)), (z(0, dt=f), (0,))):
        with pytest.raises(lib.ParaganError, match="on the GPU"):
            lib._hold("table", t, "float32", *n)
    for t, n in ((z(3, 8, dt=f), (32, 8)), (z(8, 4, dt=f), (32, 8)), (z(4, 9, dt=f), (32, 8)), (z(31, dt=f), (32, 8)), (z(8, dt=f), (9,))):
        with pytest.raises(lib.ParaganError, match="must hold"):
            lib._hold("table", t, "float32", *n)
    assert put(None, "q") is None


def test_qknorm_tensors_are_held_to_the_descriptor():
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    x = z(6, 9, 16)                                               # q of 4 heads, k of 2, others'
    q, k = x[:, :4], x[:, 4:6]
    kw = dict(rot=16, interleaved=0, n_pos=5, eps=1e-6)
    for bad in ((z(6, 4, 16, dt=torch.float32), None), (z(5, 4, 16), None), (z(6, 2, 16), None), (None, z(6, 4, 16)),
                (None, z(6, 2, 8)), (None, z(6, 2, 16, dt=torch.float16))):
        with pytest.raises(lib.ParaganError, match="an output differs"):
            lib.qknorm_desc(q, k, *bad, **kw)
    d = lib.qknorm_desc(q, k, **kw)
    put = lambda t, name: lib._placed(d, lib._qknorm_dims, (name,), t)  # noqa: E731
    for t, name in ((q, "q"), (k, "k"), (torch.empty_like(x)[:, :4], "dq"), (torch.empty_like(x)[:, 4:6], "dk"), (z(6, 4, 16), "qo"),
                    (z(2, 3, 4, 16), "dqo"), (z(6, 32), "ko"), (z(6, 1, 2, 16), "dko"), (z(2, 3, 9, 16)[:, :, :4], "dq")):
        with pytest.raises(lib.ParaganError, match="on the GPU"):
            put(t, name)
    for t, name in ((z(6, 4, 16), "dq"), (z(6, 2, 16), "dk"), (x[:, :4], "qo"), (z(6, 4, 16), "ko"), (z(5, 4, 16), "qo"),
                    (z(6, 4, 16, dt=torch.float32), "dqo"), (z(2, 4, 9, 16)[:, :3, :4], "dq"), (z(4, 6, 16).transpose(0, 1), "qo")):
        with pytest.raises(lib.ParaganError, match="not where the descriptor says"):
            put(t, name)
    f = torch.float32
    for name, t in (("gain_q", z(8, dt=f)), ("gain_k", z(15, dt=f)), ("dgain_q", z(2, dt=f)), ("table", z(4, 8, 2, dt=f)),
                    ("pos", z(5, dt=torch.int32))):
        with pytest.raises(lib.ParaganError, match="must hold"):
            put(t, name)
    for name, t in (("gain_q", z(16, dt=f)), ("dgain_k", z(16, dt=f)), ("table", z(5, 8, 2, dt=f)), ("pos", z(9, dt=torch.int32))):
        with pytest.raises(lib.ParaganError, match="on the GPU"):
            put(t, name)
    one = lib.qknorm_desc(z(1, 3, 8), z(1, 1, 8), rot=0, interleaved=0, n_pos=1, eps=1e-6)
    with pytest.raises(lib.ParaganError, match="on the GPU"):      # a single token has no stride to speak of
        lib._placed(one, lib._qknorm_dims, ("q",), z(4, 9, 8)[:1, :3])


def test_qknorm_refuses_an_eps_that_the_hardware_takes_for_zero(L):
    least = float(np.finfo(np.float32).tiny)
    assert lib.paragan_qknorm_check(qk(eps=least)) == lib.OK
    for eps in (np.nextafter(np.float32(least), np.float32(0)), 1e-39, 1e-45, -least):
        assert lib.paragan_qknorm_check(qk(eps=float(eps))) == lib.EINVAL, eps
