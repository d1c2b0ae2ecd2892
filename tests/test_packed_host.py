"""Refusals of the packed attention's and the rotary positions' entry points, and the bands: nothing is launched (no GPU)."""
import ctypes
import math

import paper_2608_01127_amd as mw
from paper_2608_01127_amd import _lib

A = 0x10000
U = 0x10008


def err():
    return mw.load().mw_last_error().decode()


def batch(**kw):
    x = dict(cu_q=A, cu_k=A, plan=A, N=3, total_q=100, total_k=100, H=4, Hkv=2, D=64, chunk_len=1, backward=1)
    x.update(kw)
    return _lib.mw_packed(*x.values())


def init(p=True, cu_q=A, cu_k=A, plan=A, n=1 << 40, N=3, total_q=100, total_k=100, H=4, Hkv=2, D=64, chunk_len=1, backward=1):
    p = ctypes.byref(_lib.mw_packed()) if p else None
    return mw.load().mw_packed_init(p, cu_q, cu_k, plan, n, N, total_q, total_k, H, Hkv, D, chunk_len, backward, None)


def fwd(p=None, q=A, k=A, v=A, o=A, lse=A, scale=0.125, ws=A, n=1 << 40, strides=None, null=False):
    p = None if null else ctypes.byref(p or batch())
    return mw.load().mw_packed_attn_fwd(q, k, v, p, o, lse, scale, ws, n, strides, None)


def bwd(p=None, q=A, k=A, v=A, o=A, d_o=A, lse=A, dq=A, dk=A, dv=A, scale=0.125, ws=A, n=1 << 40, strides=None, null=False):
    p = None if null else ctypes.byref(p or batch())
    return mw.load().mw_packed_attn_bwd(q, k, v, o, d_o, lse, p, dq, dk, dv, scale, ws, n, strides, None)


BAD_SIZES = [dict(N=0), dict(total_q=0), dict(total_k=0), dict(H=0), dict(Hkv=0), dict(chunk_len=0), dict(H=5)]
TOO_LARGE = [dict(D=0), dict(D=96), dict(D=256), dict(N=(1 << 16) + 1), dict(total_q=(1 << 23) + 1), dict(total_k=(1 << 24) + 1),
             dict(H=1 << 15)]


def test_struct_layouts():
    assert ctypes.sizeof(_lib.mw_packed) == 56 and _lib.mw_packed.N.offset == 24
    assert ctypes.sizeof(_lib.mw_rope_band) == 56 and _lib.mw_rope_band.theta.offset == 8
    assert _lib.mw_rope_bands.axis.offset == 52 and _lib.mw_rope_bands.freq.offset == 120
    assert ctypes.sizeof(_lib.mw_rope_bands) == 120 + 8 * 64


def test_plan_refusals():
    assert init(p=False) == mw.MW_EINVAL
    for name in ("cu_q", "cu_k", "plan"):
        assert init(**{name: None}) == mw.MW_EINVAL
    assert init(plan=U) == mw.MW_EALIGN and init(cu_q=A + 2) == mw.MW_EALIGN and init(cu_k=A + 1) == mw.MW_EALIGN
    for bad in BAD_SIZES:
        assert init(**bad) == mw.MW_EINVAL
    for bad in TOO_LARGE:
        assert init(**bad) == mw.MW_EUNSUPPORTED
    size = mw.load().mw_packed_plan_bytes
    need = size(3, 100, 100, 4, 2, 64, 1, 1)
    assert need > size(3, 100, 100, 4, 2, 64, 1, 0) > 0
    assert init(n=need - 1) == mw.MW_EINVAL and "plan" in err()
    assert size(0, 100, 100, 4, 2, 64, 1, 1) == 0 and size(3, 100, 100, 4, 3, 64, 1, 1) == 0


def test_refusals():
    for f in (fwd, bwd):
        assert f(null=True) == mw.MW_EINVAL
        for name in ("cu_q", "cu_k", "plan"):
            assert f(batch(**{name: None})) == mw.MW_EINVAL and "not initialised" in err()
        for name in ("q", "k", "v", "o", "lse"):
            assert f(**{name: None}) == mw.MW_EINVAL and f"{name} is NULL" in err()
            assert f(**{name: U}) == mw.MW_EALIGN
        for bad in BAD_SIZES:
            assert f(batch(**bad)) == mw.MW_EINVAL
        for bad in TOO_LARGE:
            assert f(batch(**bad)) == mw.MW_EUNSUPPORTED
        for s in (0.0, -1.0, float("nan"), float("inf")):
            assert f(scale=s) == mw.MW_EINVAL
        assert f(ws=U) == mw.MW_EALIGN
    for name in ("d_o", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: None}) == mw.MW_EINVAL and bwd(**{name: U}) == mw.MW_EALIGN
    assert bwd(batch(backward=0)) == mw.MW_EINVAL and "without its backward" in err()
    need = mw.load().mw_packed_attn_bwd_workspace_size(ctypes.byref(batch()))
    assert need >= 2 * 4 * 4 * 100 and bwd(n=need - 1) == mw.MW_EINVAL and "workspace" in err()
    long = batch(total_k=100000)
    need = mw.load().mw_packed_attn_workspace_size(ctypes.byref(long))
    assert need > 0 and fwd(long, n=need - 1) == mw.MW_EINVAL and fwd(long, ws=None) == mw.MW_EINVAL
    assert mw.load().mw_packed_attn_workspace_size(ctypes.byref(batch())) == 0  # too few keys to cut
    assert mw.load().mw_packed_attn_bwd_workspace_size(ctypes.byref(batch(backward=0))) == 0


def test_stride_refusals():
    def strides(n, **bad):
        arr = (_lib.mw_strides * n)()
        for i in range(n):
            arr[i] = _lib.mw_strides(-5, 64, 256)  # (b is not used)
        for i, s in bad.values():
            arr[i] = _lib.mw_strides(0, *s)
        return arr

    for f, n, outputs in ((fwd, 4, (3,)), (bwd, 8, (5, 6, 7))):
        for i in range(n):
            assert f(strides=strides(n, x=(i, (64, 56)))) == mw.MW_EINVAL   # rows overlap
            assert f(strides=strides(n, x=(i, (68, 512)))) == mw.MW_EALIGN
            assert f(strides=strides(n, x=(i, (-64, 512)))) == mw.MW_EINVAL
        for i in outputs:
            assert f(strides=strides(n, x=(i, (0, 256)))) == mw.MW_EINVAL and "overlaps" in err()


def bands(*bs, halves=0, gain=1.0, n=None, out=True):
    arr = (_lib.mw_rope_band * max(1, len(bs)))()
    for x, b in zip(arr, bs):
        for name, v in {"theta": 1e4, "factor": 1.0, **b}.items():
            setattr(x, name, v)
    r = _lib.mw_rope_bands()
    st = mw.load().mw_rope_bands_init(ctypes.byref(r) if out else None, arr, len(bs) if n is None else n, halves, gain)
    return st, r


def test_bands():
    one = dict(dim_offset=0, dim_count=64)
    st, r = bands(one)
    assert st == mw.MW_OK and (r.n_bands, r.n_pairs, r.n_axes, r.halves, r.gain) == (1, 32, 1, 0, 1.0)
    for i in range(32):
        assert abs(r.freq[i] * 2 * math.pi - 1e4 ** (-2 * i / 64)) <= 1e-15
    st, r = bands(dict(one, factor=4.0))
    assert all(abs(r.freq[i] * 8 * math.pi - 1e4 ** (-2 * i / 64)) <= 1e-15 for i in range(32))
    st, r = bands(dict(one, factor=8.0, trained_len=8192.0, turns_lo=1.0, turns_hi=32.0), dict(dim_offset=64, dim_count=10, axis=2),
                  halves=1, gain=-0.5)
    assert st == mw.MW_OK and (r.n_pairs, r.n_axes, r.halves, r.gain) == (37, 3, 1, -0.5)
    for i in range(32):
        f = 1e4 ** (-2 * i / 64)
        k = min(1.0, max(0.0, (8192 * f / (2 * math.pi) - 1) / 31))
        assert abs(r.freq[i] * 2 * math.pi - f * (k + (1 - k) / 8)) <= 1e-15
    assert list(r.axis[:37]) == [0] * 32 + [2] * 5
    bad = [dict(one, dim_offset=-2), dict(one, dim_offset=1), dict(one, dim_count=0), dict(one, dim_count=3),
           dict(one, dim_offset=66), dict(one, dim_count=2 ** 31 - 2, dim_offset=2 ** 31 - 2), dict(one, theta=0.0),
           dict(one, theta=float("nan")), dict(one, theta=float("inf")), dict(one, axis=4), dict(one, axis=-1), dict(one, factor=0.0),
           dict(one, factor=float("inf")), dict(one, turns_lo=2.0, turns_hi=1.0), dict(one, turns_hi=1.0),
           dict(one, turns_lo=float("nan"))]
    for b in bad:
        assert bands(b)[0] == mw.MW_EINVAL, b
    assert bands(one, dict(dim_offset=62, dim_count=4))[0] == mw.MW_EINVAL and "share" in err()
    assert bands(one, n=0)[0] == mw.MW_EINVAL and bands(one, n=5)[0] == mw.MW_EINVAL and bands(one, out=False)[0] == mw.MW_EINVAL
    assert bands(one, halves=2)[0] == mw.MW_EINVAL
    for g in (0.0, float("nan"), float("inf")):
        assert bands(one, gain=g)[0] == mw.MW_EINVAL


def rope(q=A, k=A, q_out=A, k_out=A, b=None, pos=A, pos_bytes=8, pos_strides=(0, 0, 1), first=0, inverse=0, strides=None, B=1, H=2,
         Hkv=2, T=5, D=64, null=False):
    if b is None:
        b = bands(dict(dim_offset=0, dim_count=64))[1]
    ps = None
    if pos_strides is not None:
        ps = (_lib.mw_strides * 1)(_lib.mw_strides(*pos_strides))
    return mw.load().mw_rope_apply(q, k, q_out, k_out, None if null else ctypes.byref(b), pos, pos_bytes, ps, first, inverse,
                                   strides, B, H, Hkv, T, D, None)


def test_rope_refusals():
    for name in ("q", "q_out"):
        assert rope(**{name: None}) == mw.MW_EINVAL and rope(**{name: U}) == mw.MW_EALIGN
    assert rope(k=None) == mw.MW_EINVAL and rope(k_out=None) == mw.MW_EINVAL
    assert rope(k=U) == mw.MW_EALIGN and rope(k_out=U) == mw.MW_EALIGN
    assert rope(null=True) == mw.MW_EINVAL and rope(b=_lib.mw_rope_bands()) == mw.MW_EINVAL
    for name in ("B", "H", "Hkv", "T"):
        assert rope(**{name: 0}) == mw.MW_EINVAL
    for D in (0, 96, 256):
        assert rope(D=D) == mw.MW_EUNSUPPORTED
    assert rope(T=(1 << 24) + 1) == mw.MW_EUNSUPPORTED and rope(B=1 << 20, T=1 << 10) == mw.MW_EUNSUPPORTED
    assert rope(H=1 << 15) == mw.MW_EUNSUPPORTED and rope(Hkv=1 << 15) == mw.MW_EUNSUPPORTED
    assert rope(inverse=2) == mw.MW_EINVAL
    assert rope(pos_bytes=2) == mw.MW_EINVAL and rope(pos=A + 4) == mw.MW_EALIGN and rope(pos=A + 2, pos_bytes=4) == mw.MW_EALIGN
    assert rope(pos_strides=None) == mw.MW_EINVAL and rope(pos_strides=(0, 0, -1)) == mw.MW_EINVAL
    wide = bands(dict(dim_offset=0, dim_count=72))[1]
    assert rope(b=wide) == mw.MW_EINVAL and "within the head" in err()
    two = bands(dict(dim_offset=0, dim_count=32), dict(dim_offset=32, dim_count=32, axis=1))[1]
    assert rope(b=two, pos=None) == mw.MW_EINVAL and "several axes" in err()
    wrong = bands(dict(dim_offset=0, dim_count=64))[1]
    wrong.n_pairs = 31
    assert rope(b=wrong) == mw.MW_EINVAL
    s = lambda *x: (_lib.mw_strides * 4)(*[_lib.mw_strides(*y) for y in x])
    good = (640, 320, 64)
    assert rope(strides=s(good, good, (640, 64, 128), good)) == mw.MW_EINVAL and "must have its strides" in err()
    for i in range(4):
        assert rope(strides=s(*[(640, 324, 64) if j == i else good for j in range(4)])) == mw.MW_EALIGN
    assert rope(q_out=2 * A, strides=s(good, good, (640, 0, 64), good)) == mw.MW_EINVAL and "overlaps" in err()


def test_binding_of_bands():
    import pytest
    r = mw.rope_bands([dict(dim_offset=0, dim_count=8)], halves=True, gain=2.0)
    assert (r.n_pairs, r.halves, r.gain) == (4, 1, 2.0)
    with pytest.raises(mw.MWError):
        mw.rope_bands([])
    with pytest.raises(ValueError):
        mw.rope_bands([dict(dim_offset=0, dim_count=8, base=3.0)])
