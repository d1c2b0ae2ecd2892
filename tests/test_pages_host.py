"""Refusals and host bookkeeping of the paged cache that need no GPU: everything here returns before a launch."""
import ctypes

import pytest

import paper_2608_01127_amd as mw
from paper_2608_01127_amd import _lib

A = 0x10000
U = 0x10008


def err():
    return mw.load().mw_last_error().decode()


def seqs(*s):
    return (ctypes.c_int32 * len(s))(*s)


class Cache:
    def __init__(self, P=8, H=2, L=64, D=64, N=4, W=4):
        n = mw.load().mw_kvpages_host_bytes(P, N, W)
        self.host = (ctypes.c_int32 * (n // 4))()
        self.c = _lib.mw_kvpages()
        self.status = mw.load().mw_kvpages_init(ctypes.byref(self.c), A, A, A, A, A, A, ctypes.addressof(self.host), n, P, H,
                                                L, D, N, W)

    def append(self, s=seqs(0), k=A, v=A, strides=None, t=1, n=None):
        return mw.load().mw_kvpages_append(ctypes.byref(self.c), s, len(s) if n is None else n, k, v, strides, t, None)

    def attend(self, q=A, k=A, v=A, nq=1, ql=1, s=seqs(0), n=None, H=2, flags=0, o=A, lse=A, scale=0.1, ws=None, wsn=0,
               strides=None):
        return mw.load().mw_chunk_attn_paged(q, k, v, nq, ql, ctypes.byref(self.c), s, len(s) if n is None else n, H, flags,
                                             o, lse, scale, ws, wsn, strides, None)


def test_init():
    f = mw.load().mw_kvpages_init
    host = (ctypes.c_int32 * 4096)()
    h = ctypes.addressof(host)
    c = _lib.mw_kvpages()
    ref = ctypes.byref(c)
    ok = (8, 2, 64, 64, 4, 4)

    def init(ptrs=(A,) * 6, host=h, n=16384, sizes=ok, ref=ref):
        return f(ref, *ptrs, host, n, *sizes)

    assert init() == mw.MW_OK and mw.load().mw_kvpages_n_free(ref) == 8
    assert init(ref=None) == mw.MW_EINVAL and init(host=None) == mw.MW_EINVAL
    for i in range(6):
        assert init(ptrs=tuple(None if j == i else A for j in range(6))) == mw.MW_EINVAL
        assert init(ptrs=tuple(U if j == i else A for j in range(6))) == mw.MW_EALIGN
        assert init(sizes=tuple(0 if j == i else s for j, s in enumerate(ok))) in (mw.MW_EINVAL, mw.MW_EUNSUPPORTED)
    assert init(sizes=(8, 2, 65, 64, 4, 4)) == mw.MW_EINVAL and "multiple of 64" in err()
    assert init(sizes=(8, 2, 64, 96, 4, 4)) == mw.MW_EUNSUPPORTED
    assert init(sizes=(8, 2, 64, 64, 4, (1 << 18) + 1)) == mw.MW_EUNSUPPORTED
    assert init(n=mw.load().mw_kvpages_host_bytes(8, 4, 4) - 4) == mw.MW_EINVAL and "host block" in err()
    assert mw.load().mw_kvpages_host_bytes(0, 4, 4) == 0


def test_uninitialised_caches_are_refused():
    lib = mw.load()
    c = _lib.mw_kvpages()
    ref = ctypes.byref(c)
    for r in (None, ref):
        assert lib.mw_kvpages_len(r, 0) == mw.MW_EINVAL and lib.mw_kvpages_n_free(r) == mw.MW_EINVAL
        assert lib.mw_kvpages_append(r, seqs(0), 1, A, A, None, 1, None) == mw.MW_EINVAL
        assert lib.mw_kvpages_fork(r, 0, 1, None) == mw.MW_EINVAL and lib.mw_kvpages_copy(r, 0, 1, None) == mw.MW_EINVAL
        assert lib.mw_kvpages_free(r, seqs(0), 1, None) == mw.MW_EINVAL
        assert lib.mw_kvpages_evict(r, 0, 0, 1, None) == mw.MW_EINVAL and lib.mw_kvpages_compact(r, None) == mw.MW_EINVAL
        assert lib.mw_chunk_attn_paged(A, A, A, 1, 1, r, seqs(0), 1, 2, 0, A, A, 0.1, None, 0, None, None) == mw.MW_EINVAL
        assert lib.mw_chunk_attn_paged_workspace_size(r, seqs(0), 1, 2, 1, 1) == 0
    x = Cache()
    x.c.W = 5  # not what was initialised
    assert lib.mw_kvpages_n_free(ctypes.byref(x.c)) == mw.MW_EINVAL and "corrupt" in err()


def test_append_refusals_leave_the_cache_as_it_was():
    x = Cache()
    before = bytes(x.host)
    assert x.append(k=None) == mw.MW_EINVAL and x.append(v=U) == mw.MW_EALIGN
    assert x.append(t=0) == mw.MW_EINVAL and x.append(n=0) == mw.MW_EINVAL
    assert x.append(s=seqs(4)) == mw.MW_EINVAL and x.append(s=seqs(-1)) == mw.MW_EINVAL
    assert x.append(s=seqs(1, 2, 1)) == mw.MW_EINVAL and "twice" in err()
    assert x.append(t=4 * 64 + 1) == mw.MW_EFULL and "row" in err()
    assert x.append(s=seqs(0, 1, 2), t=3 * 64) == mw.MW_EFULL and "9 pages are needed and 8 are free" in err()
    assert mw.load().mw_kvpages_append(ctypes.byref(x.c), seqs(*range(4)), 300, A, A, None, 1, None) == mw.MW_EUNSUPPORTED
    bad = (_lib.mw_strides * 2)(_lib.mw_strides(128, 64, 64), _lib.mw_strides(128, 64, 60))
    assert x.append(strides=bad) == mw.MW_EINVAL
    assert bytes(x.host) == before


def test_sequence_operations_refuse():
    lib = mw.load()
    x = Cache()
    ref = ctypes.byref(x.c)
    before = bytes(x.host)
    for f in (lib.mw_kvpages_fork, lib.mw_kvpages_copy):
        assert f(ref, 0, 0, None) == mw.MW_EINVAL and f(ref, 0, 4, None) == mw.MW_EINVAL and f(ref, -1, 0, None) == mw.MW_EINVAL
        assert f(ref, 0, 1, None) == mw.MW_OK  # an empty sequence: nothing to do
    assert lib.mw_kvpages_evict(ref, 0, 0, 1, None) == mw.MW_EEMPTY and lib.mw_kvpages_evict(ref, 0, -1, 0, None) == mw.MW_EINVAL
    assert lib.mw_kvpages_evict(ref, 0, 0, 0, None) == mw.MW_OK
    assert lib.mw_kvpages_free(ref, seqs(1, 1), 2, None) == mw.MW_EINVAL
    assert lib.mw_kvpages_page_of(ref, 0, 0) == mw.MW_EINVAL and lib.mw_kvpages_len(ref, 9) == mw.MW_EINVAL
    assert lib.mw_kvpages_compact(ref, None) == 0
    assert bytes(x.host) == before


def test_attention_refusals():
    x = Cache()
    for kw in (dict(q=None), dict(o=None), dict(k=None), dict(v=None), dict(nq=0), dict(ql=0), dict(H=3), dict(H=0),
               dict(flags=2), dict(scale=0.0), dict(scale=float("nan")), dict(s=seqs(4)), dict(n=0)):
        assert x.attend(**kw) == mw.MW_EINVAL, kw
    for kw in (dict(q=U), dict(k=U), dict(v=U), dict(o=U), dict(lse=U), dict(ws=U)):
        assert x.attend(**kw) == mw.MW_EALIGN, kw
    for kw in (dict(nq=65), dict(ql=1 << 25), dict(n=257, s=seqs(*([0] * 257)))):
        assert x.attend(**kw) == mw.MW_EUNSUPPORTED, kw
    flat = lambda heads, t: _lib.mw_strides(heads * 64, t, 64)
    bad = (_lib.mw_strides * 4)(flat(2, 64), flat(2, 64), flat(2, 64), flat(2, 0))
    assert x.attend(strides=bad) == mw.MW_EINVAL and "overlaps" in err()


def test_struct_layout():
    assert ctypes.sizeof(_lib.mw_kvpages) == 7 * 8 + 6 * 4
    assert _lib.mw_kvpages.host.offset == 48 and _lib.mw_kvpages.W.offset == 76


@pytest.mark.parametrize("bad", [(0, 2, 64, 64, 4, 4), (8, 0, 64, 64, 4, 4), (8, 2, 64, 64, 0, 4)])
def test_python_class_refuses_sizes_before_it_allocates(bad):
    import torch
    if not torch.cuda.is_available():
        with pytest.raises(mw.MWError):
            mw.KVPages(*bad, device="cpu")


def test_sequence_numbers_that_a_c_int_does_not_hold_are_refused():
    """ctypes would keep the low 32 bits: 2^32 would name sequence 0."""
    for f in (lambda s: _lib._seqs([s]), _lib._int32):
        for bad, kind in ((1 << 32, ValueError), (-(1 << 31) - 1, ValueError), (1.5, TypeError)):
            with pytest.raises(kind):
                f(bad)
    assert list(_lib._seqs([0, 255])) == [0, 255] and _lib._int32(-1) == -1
