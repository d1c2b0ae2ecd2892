"""Refusals of the cross attention's entry points: arguments are checked before anything is launched (no GPU)."""
import paper_2608_01127_amd as mw
from paper_2608_01127_amd import _lib

A = 0x10000
U = 0x10008


def err():
    return mw.load().mw_last_error().decode()


def fwd(q=A, k=A, v=A, kv_len=None, o=A, lse=A, strides=None, B=1, H=4, Hkv=2, T=8, M=8, D=64, scale=0.125, ws=None, n=0):
    return mw.load().mw_cross_attn_fwd(q, k, v, kv_len, o, lse, strides, B, H, Hkv, T, M, D, scale, ws, n, None)


def bwd(q=A, k=A, v=A, kv_len=None, o=A, d_o=A, lse=A, dq=A, dk=A, dv=A, ws=A, n=1 << 40, strides=None, B=1, H=4, Hkv=2,
        T=8, M=8, D=64, scale=0.125):
    return mw.load().mw_cross_attn_bwd(q, k, v, kv_len, o, d_o, lse, dq, dk, dv, ws, n, strides, B, H, Hkv, T, M, D, scale,
                                       None)


def test_refusals():
    for f in (fwd, bwd):
        for name in ("q", "k", "v", "o"):
            assert f(**{name: None}) == mw.MW_EINVAL and f"{name} is NULL" in err()
            assert f(**{name: U}) == mw.MW_EALIGN
        for name in ("B", "H", "Hkv", "T", "M"):
            assert f(**{name: 0}) == mw.MW_EINVAL
        assert f(H=5) == mw.MW_EINVAL and "multiple" in err()
        assert f(H=2, Hkv=4) == mw.MW_EINVAL
        for D in (0, 63, 96, 256):
            assert f(D=D) == mw.MW_EUNSUPPORTED
        assert f(T=1 << 24) == mw.MW_EUNSUPPORTED  # times two query heads a key head
        assert f(M=(1 << 24) + 1) == mw.MW_EUNSUPPORTED
        for s in (0.0, -1.0, float("nan"), float("inf")):
            assert f(scale=s) == mw.MW_EINVAL
        assert f(kv_len=U) == mw.MW_EALIGN
    for name in ("d_o", "lse", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: None}) == mw.MW_EINVAL and "NULL" in err()
        assert bwd(**{name: U}) == mw.MW_EALIGN
    assert fwd(lse=U) == mw.MW_EALIGN and fwd(ws=U, n=64) == mw.MW_EALIGN
    need = mw.mw_cross_attn_bwd_workspace_size(1, 4, 2, 8, 8, 64)
    assert bwd(n=need - 1) == mw.MW_EINVAL and "workspace" in err()


def test_stride_refusals():
    def strides(n, **bad):
        arr = (_lib.mw_strides * n)()
        for i in range(n):
            arr[i] = _lib.mw_strides(4 * 8 * 64, 8 * 64, 64)
        for i, s in bad.values():
            arr[i] = _lib.mw_strides(*s)
        return arr

    for f, n, outputs in ((fwd, 4, (3,)), (bwd, 8, (5, 6, 7))):
        for i in range(n):
            assert f(strides=strides(n, x=(i, (2048, 512, 63)))) == mw.MW_EINVAL   # rows overlap
            assert f(strides=strides(n, x=(i, (2048, 516, 64)))) == mw.MW_EALIGN
            assert f(strides=strides(n, x=(i, (2048, -512, 64)))) == mw.MW_EINVAL
        for i in outputs:
            assert f(strides=strides(n, x=(i, (2048, 0, 64)))) == mw.MW_EINVAL and "overlaps" in err()


def test_workspace_sizes():
    size = mw.mw_cross_attn_workspace_size
    assert size(1, 4, 4, 1, 1, 64) == 0                       # one key: nothing to split
    assert size(1, 4, 4, 8, 20000, 64) > 0                    # few rows over many keys
    assert size(8, 16, 16, 20000, 128, 128) == 0              # many rows
    assert size(1, 5, 2, 8, 8, 64) == 0 and size(1, 4, 4, 8, 8, 96) == 0
    rows = 2 * 4 * 100 * 4
    assert mw.mw_cross_attn_bwd_workspace_size(2, 4, 2, 100, 50, 64) >= 2 * rows
    assert mw.mw_cross_attn_bwd_workspace_size(2, 4, 3, 100, 50, 64) == 0
