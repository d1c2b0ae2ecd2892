"""Refusals and host bookkeeping of the eviction by weight that need no GPU: everything here returns before a launch."""
import ctypes

import paper_2608_01127_amd as mw
from paper_2608_01127_amd import _lib
from test_pages_host import Cache, err, seqs

A = 0x10000
U = 0x10008


def weigh(c, s=seqs(0), n=None, q=A, lse=A, H=2, T=1, w=A, add=1, scale=0.1, ws=None, wsn=0, strides=None):
    return mw.load().mw_kvpages_weigh(ctypes.byref(c.c), s, len(s) if n is None else n, q, lse, H, T, w, add, scale, ws, wsn,
                                      strides, None)


def evict(c, s=seqs(0), n=None, w=A, keep=10, first=0, recent=0, ws=A, wsn=1 << 40):
    return mw.load().mw_kvpages_evict_weighted(ctypes.byref(c.c), s, len(s) if n is None else n, w, keep, first, recent, ws, wsn,
                                               None)


def hold(c, seq, tokens):
    """Tokens in the host's books, as an append leaves them (nothing is launched): pages in order from the front."""
    P, N, W, L = c.c.P, c.c.N, c.c.W, c.c.L
    refs, lens, table = 4, 4 + 2 * P, 4 + 2 * P + N
    page = c.host[1]
    for w in range(-(-tokens // L)):
        c.host[table + seq * W + w] = page
        c.host[refs + page] = 1
        page += 1
        c.host[2] -= 1
    c.host[1] = page
    c.host[lens + seq] = tokens
    assert mw.load().mw_kvpages_len(ctypes.byref(c.c), seq) == tokens


def test_refusals():
    c = Cache()
    null = type("C", (), {"c": None})
    for f in (weigh, evict):
        assert f(c, s=seqs(4)) == mw.MW_EINVAL and f(c, s=seqs(-1)) == mw.MW_EINVAL and f(c, n=0) == mw.MW_EINVAL
        assert f(c, s=seqs(1, 0, 1)) == mw.MW_EINVAL and "twice" in err()
        assert f(c, w=None) == mw.MW_EINVAL and f(c, w=U) == mw.MW_EALIGN
        assert f(c, s=seqs(*[0] * 257)) == mw.MW_EUNSUPPORTED
        broken = Cache()
        broken.host[0] = 1
        assert f(broken) == mw.MW_EINVAL
    for name in ("q", "lse"):
        assert weigh(c, **{name: None}) == mw.MW_EINVAL and weigh(c, **{name: U}) == mw.MW_EALIGN
    assert weigh(c, ws=U) == mw.MW_EALIGN
    for H in (0, 3):
        assert weigh(c, H=H) == mw.MW_EINVAL
    assert weigh(c, T=0) == mw.MW_EINVAL and weigh(c, T=(1 << 24) + 1) == mw.MW_EUNSUPPORTED
    assert weigh(c, H=1 << 15) == mw.MW_EUNSUPPORTED
    assert weigh(c, add=2) == mw.MW_EINVAL
    for s in (0.0, float("nan"), float("inf")):
        assert weigh(c, scale=s) == mw.MW_EINVAL
    st = lambda *x: (_lib.mw_strides * 1)(_lib.mw_strides(*x))
    assert weigh(c, strides=st(128, 64, 60)) == mw.MW_EINVAL and weigh(c, strides=st(128, 68, 64)) == mw.MW_EALIGN
    assert evict(c, keep=0) == mw.MW_EINVAL and evict(c, keep=257) == mw.MW_EINVAL
    assert evict(c, first=-1) == mw.MW_EINVAL and evict(c, first=11) == mw.MW_EINVAL
    assert evict(c, recent=-1) == mw.MW_EINVAL and evict(c, first=5, recent=6) == mw.MW_EINVAL
    assert evict(c, ws=None) == mw.MW_EINVAL and evict(c, ws=U) == mw.MW_EALIGN
    need = mw.load().mw_kvpages_evict_weighted_workspace_size(ctypes.byref(c.c), seqs(0), 1, 10, 0)
    assert need >= 120 and evict(c, wsn=need - 1) == mw.MW_EINVAL and "workspace" in err()


def test_nothing_to_do_is_not_launched():
    c = Cache()
    assert weigh(c) == mw.MW_OK and evict(c) == mw.MW_OK  # empty sequences
    hold(c, 1, 100)
    assert evict(c, s=seqs(0, 1), keep=100) == mw.MW_OK and evict(c, s=seqs(1), keep=256) == mw.MW_OK
    assert mw.load().mw_kvpages_n_free(ctypes.byref(c.c)) == 6


def test_too_few_pages_changes_nothing():
    c = Cache(P=7)
    hold(c, 0, 200)
    hold(c, 1, 130)  # none is free
    before = bytes(c.host)
    assert evict(c, s=seqs(0), keep=100) == mw.MW_EFULL and "2 pages are needed and 0 are free" in err()
    assert bytes(c.host) == before


def test_workspace_sizes():
    c = Cache(L=128, W=100, P=400)
    size = lambda keep, first, *s: mw.load().mw_kvpages_evict_weighted_workspace_size(ctypes.byref(c.c), seqs(*s), len(s), keep, first)
    assert size(1000, 0, 0) >= 12 * 1000 and size(1000, 0, 0, 1) >= 24 * 1000
    assert size(1000, 300, 0) < size(1000, 200, 0) < size(1000, 100, 0)  # whole pages of the anchor stay
    assert size(0, 0, 0) == 0 and size(10, 11, 0) == 0
    f = lambda H, T, *s: mw.load().mw_kvpages_weigh_workspace_size(ctypes.byref(c.c), seqs(*s), len(s), H, T)
    hold(c, 0, 5000)
    assert f(2, 1, 0) == 0 and f(2, 4000, 0) > 0 and f(3, 4000, 0) == 0


def test_no_workspace_for_weights_is_above_its_limit():
    """At any lengths, which it does not grow with: one of 64 MiB serves every call."""
    c = Cache(L=1024, W=10000, P=40000)
    f = lambda H, T, *s: mw.load().mw_kvpages_weigh_workspace_size(ctypes.byref(c.c), seqs(*s), len(s), H, T)
    sizes = {}
    for n in (1, 64, 5000, 19200, 64000, 131072, 133000, 700_000, 4_000_000):
        c = Cache(L=1024, W=10000, P=40000)
        hold(c, 0, n)
        hold(c, 1, n // 3 + 1)
        for H, T in ((2, 1), (2, 40), (16, 4800), (128, 60000), (2, 1 << 20)):
            for s in ((0,), (1, 0)):
                size = sizes[n, H, s] = f(H, T, *s)
                assert 0 <= size <= 64 << 20 and size % 256 == 0
    assert any(sizes[a, H, s] > sizes[b, H, s] for a, H, s in sizes for b in (700_000, 4_000_000) if a < b)
