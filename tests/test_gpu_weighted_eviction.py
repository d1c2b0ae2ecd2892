"""Eviction from the paged cache by accumulated attention weight: the weights against 64-bit values, what stays and its
pages against a model of the cache, and a rollout that uses both."""
import math

import pytest

from attention_bounds import attention64, check
from test_gpu_pages import BLOCK, Model, make, randn, tokens

pytestmark = pytest.mark.gpu


def weights_of(mw, cache, model, seqs, q, lse, H, **kw):
    """mw_kvpages_weigh into rows of markers against 64-bit values, within a bound that counts roundings: scores in 32
    bits (2^-22 of the products' magnitudes), the exponent's sum with the LSE (2^-23 of both), the hardware's 2^x (2^-22), and a
    sum of at most 64 partial sums, each of n / 64 terms (2^-24 a step)."""
    import torch
    d = cache.desc
    w = torch.full((d.N, d.W * d.L), 3.0, device="cuda")
    old = kw.pop("old", 0.0)
    w[seqs] = old
    mw.mw_kvpages_weigh(cache, seqs, q, lse, w, **kw)
    torch.cuda.synchronize()
    sc = kw.get("scale") or 1 / math.sqrt(d.D)
    G = H // d.H
    for s in range(d.N):
        n = model.lens[s]
        if s not in seqs:
            assert bool((w[s] == 3).all())
            continue
        assert bool((w[s, n:] == old).all())
        b = seqs.index(s)
        k = model.values(s)[0]
        want = torch.zeros(n, dtype=torch.float64, device="cuda")
        off = torch.zeros_like(want)
        rows = 0
        for h in range(H):
            x = q[b, h].double()
            l = lse[b, h].double()[:, None]
            p = torch.exp(torch.where(l == -math.inf, -math.inf, (x @ k[h // G].t()) * sc - torch.where(l == -math.inf, 0.0, l)))
            size = sc * (x.abs() @ k[h // G].abs().t()) + torch.where(l.isfinite(), l, 0.0).abs()
            want += p.sum(0)
            off += (p * (2.0 ** -22 * (1 + 2 * size))).sum(0)
            rows += x.shape[0]
        off += 2.0 ** -24 * (rows / 32 + 64) * want + 1e-37
        if kw.get("add", True):
            want = want + old
            off = off + 2.0 ** -24 * want.abs()
        check(f"weights s={s}", w[s, :n], want, off)
    return w


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("L", [64, 192])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (6, 2), (16, 2)])
def test_weights(mw, D, L, H, Hkv):
    """One row to several tiles of them, lengths of one, a block's edge and beyond; the call's own LSE, and add."""
    import torch
    lens = [1, 63, 64, 200, 450]
    N, W = 6, 8
    cache, model = make(mw, 40, Hkv, L, D, N, W)
    for s, n in enumerate(lens):
        k, v = tokens((1, Hkv, n, D), 10 + s), tokens((1, Hkv, n, D), 20 + s)
        k = (k.float() / 16).bfloat16()
        mw.mw_kvpages_append(cache, [s], k, v)
        model.append([s], k, v)
    for T, seqs, layout in ((1, [4, 0, 2], "bhtd"), (33, [3, 1], "bthd"), (7, [0, 1, 2, 3, 4, 5], "bthd")):
        print(f"[case] weigh D={D} L={L} H={H} Hkv={Hkv} T={T} {seqs}", flush=True)
        q = randn((len(seqs), H, T, D), 30 + T, layout)
        kn, vn = randn((len(seqs), Hkv, T, D), 31 + T), randn((len(seqs), Hkv, T, D), 32 + T)
        _, lse = mw.mw_chunk_attn_paged(q, kn, vn, 1, T, cache, seqs, want_lse=True)
        weights_of(mw, cache, model, seqs, q, lse, H, add=False)
        weights_of(mw, cache, model, seqs, q, lse, H, old=0.25)
        _, alone = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, seqs, want_lse=True)
        w = weights_of(mw, cache, model, seqs, q, alone, H, add=False)
        for s in seqs:  # the rows' weights over what they see sum to one: as many as rows
            if model.lens[s]:
                assert abs(float(w[s, :model.lens[s]].sum()) - H * T) <= H * T * 2.0 ** -12


@pytest.mark.parametrize("D", [64, 72, 128])
def test_rows_that_weigh_nothing(mw, D):
    """An LSE of -inf (a row that saw nothing) or +inf."""
    import torch
    cache, model = make(mw, 8, 2, 64, D, 2, 4)
    k, v = randn((1, 2, 100, D), 1), randn((1, 2, 100, D), 2)
    mw.mw_kvpages_append(cache, [1], k, v)
    model.append([1], k, v)
    q = randn((1, 4, 40, D), 3)
    lse = torch.randn(1, 4, 40, device="cuda") + 5
    lse[0, 1] = -math.inf
    lse[0, 2, ::3] = -math.inf
    lse[0, 3, 5] = math.inf
    weights_of(mw, cache, model, [1], q, lse, 4, add=False)
    weights_of(mw, cache, model, [1], q, lse, 4, add=False, scale=0.5)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv,T", [(8, 8, 600), (6, 2, 400), (5, 1, 77)])
def test_rows_staged_for_several_blocks(mw, D, H, Hkv, T):
    """One query head to a key head, an odd number of them; strided rows, a last step partly filled, lengths that end
    within a group of blocks."""
    cache, model = make(mw, 260, Hkv, 128, D, 3, 80)
    for s, m in enumerate((9001, 130, 4000)):
        k, v = randn((1, Hkv, m, D), 70 + s), randn((1, Hkv, m, D), 80 + s)
        mw.mw_kvpages_append(cache, [s], k, v)
        model.append([s], k, v)
    q = randn((3, H, T, D), 61, "bthd")
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, [2, 0, 1], want_lse=True)
    lse[0, 0, ::7] = -math.inf
    weights_of(mw, cache, model, [2, 0, 1], q, lse, H, old=0.5)


def test_pages_beyond_32_bits(mw):
    """A pool of more than 2^32 bytes: weights and eviction of a sequence in its last pages."""
    import torch
    H, D, L, n = 16, 128, 640, 60_000
    cache = mw.KVPages(3900, H, L, D, 2, 3800)
    k, v = randn((1, H, n, D), 1), randn((1, H, n, D), 2)
    for _ in range(40):  # 2.4 million tokens in front
        mw.mw_kvpages_append(cache, [0], k, v)
    model = Model(cache, 3900, H, L, D, 2, 3800)
    model.rows[0], model.lens[0] = list(range(3750)), 2_400_000
    x, y = tokens((1, H, 1500, D), 3), tokens((1, H, 1500, D), 4)
    mw.mw_kvpages_append(cache, [1], x, y)
    model.append([1], x, y)
    assert cache.page_of(1, 0) == 3750 and 3750 * H * L * D > 2**32
    q = (randn((1, H, 90, D), 5).float() / 64).bfloat16()
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, 90, cache, [1], want_lse=True)
    w = torch.zeros((2, 3800 * L), device="cuda")
    mw.mw_kvpages_weigh(cache, [1], q, lse, w)
    torch.cuda.synchronize()
    kk = model.values(1)[0]
    want = torch.zeros(1500, dtype=torch.float64, device="cuda")
    for h in range(H):
        want += torch.softmax(q[0, h].double() @ kk[h].t() * D ** -0.5, -1).sum(0)
    # (scores of up to 2^7 in 32 bits: 2^-16 of a weight)
    assert bool(((w[1, :1500].double() - want).abs() <= 2.0 ** -14 * want + 1e-30).all())
    before = w.clone()
    mw.mw_kvpages_evict_weighted(cache, [1], w, 700, first=100, recent=50)
    torch.cuda.synchronize()
    stay = torch.tensor(kept(before[1, :1500].tolist(), 1500, 700, 100, 50), device="cuda")
    assert torch.equal(w[1, :700], before[1][stay]) and not bool(w[1, 700:].any())
    assert [cache.page_of(1, i) for i in range(2)] == [3753, 3754] and cache.len(1) == 700 and cache.n_free == 3900 - 3752
    old = kk[:, stay]
    for p, at in ((3753, 0), (3754, 640)):
        m = min(640, 700 - at)
        scale = cache.k_scales[p].double().repeat_interleave(BLOCK, -1)[:, :m, None]
        got = cache.k_pages[p, :, :m].view(torch.float8_e4m3fn).double() * scale
        exact = old[:, at:at + m]
        # codes change only where a finer block's become subnormal in the new one: half a step of 2^-9 of its scale
        assert bool(((got - exact).abs() <= 2.0 ** -10 * scale).all())


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("n", [70, 3000])
def test_many_rows_are_divided(mw, D, n):
    """Rows of a call divided among workgroups, and not (no workspace of that size); two members of unlike lengths."""
    import torch
    H, Hkv, T = 8, 4, 700
    cache, model = make(mw, 120, Hkv, 64, D, 2, 50)
    for s, m in enumerate((n, max(1, n // 3))):
        k, v = randn((1, Hkv, m, D), 40 + s), randn((1, Hkv, m, D), 50 + s)
        mw.mw_kvpages_append(cache, [s], k, v)
        model.append([s], k, v)
    q = randn((2, H, T, D), 60, "bthd")
    assert mw.mw_kvpages_weigh_workspace_size(cache, [0, 1], H, T) > 0
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, [0, 1], want_lse=True)
    a = weights_of(mw, cache, model, [0, 1], q, lse, H, add=False)
    b = weights_of(mw, cache, model, [1, 0], q.flip(0), lse.flip(0).contiguous(), H, add=False,
                   workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    again = weights_of(mw, cache, model, [0, 1], q, lse, H, add=False)
    assert torch.equal(a, again)


def kept(w, n, keep, first, recent):
    """Places that stay, in order (ties: lowest index; a NaN is the lightest)."""
    w = [(-math.inf if x != x else x) for x in w[:n]]
    nan = [x != x for x in w]
    mid = sorted(range(first, n - recent), key=lambda j: (-w[j], j))[:keep - first - recent]
    return sorted([*range(first), *mid, *range(n - recent, n)])


def evict(mw, cache, model, seqs, weights, keep, first=0, recent=0):
    """The call, and the same on the model."""
    import torch
    before = weights.clone()
    L = model.L
    w0, w1 = first // L, -(-keep // L)
    mw.mw_kvpages_evict_weighted(cache, seqs, weights, keep, first=first, recent=recent)
    torch.cuda.synchronize()
    jobs = [s for s in seqs if model.lens[s] > keep]
    new = model.take(len(jobs) * (w1 - w0))
    assert len(new) == len(jobs) * (w1 - w0)
    source = {s: (list(model.rows[s]), model.lens[s]) for s in jobs}
    for i, s in enumerate(jobs):
        row, n = source[s]
        stay = kept(before[s].tolist(), n, keep, first, recent)
        assert len(stay) == keep and stay[:first] == list(range(first))
        pages = new[i * (w1 - w0):(i + 1) * (w1 - w0)]
        moved = torch.tensor(stay[w0 * L:], device="cuda", dtype=torch.long)
        where = torch.tensor(row, device="cuda")[moved // L]
        for x in range(2):
            value = model.code[x][where, :, moved % L].double() * torch.exp2(model.exp[x][where, :, moved % L // BLOCK].double())[..., None]
            for c in range(0, len(moved), BLOCK):
                val = value[c:c + BLOCK].transpose(0, 1)  # [H, t, D]
                model.write(x, pages[c // L], c % L, val)
        want = before[s].clone()
        want[:keep] = before[s][torch.tensor(stay, device="cuda")]
        want[keep:n] = 0
        assert torch.equal(weights[s].nan_to_num(nan=1e9), want.nan_to_num(nan=1e9)), f"weights of sequence {s}"
        model.rows[s] = row[:w0] + pages
        model.lens[s] = keep
    for s in range(len(model.lens)):
        if s not in jobs:
            assert torch.equal(weights[s].nan_to_num(nan=1e9), before[s].nan_to_num(nan=1e9))
    model.verify()


def filled(mw, lens, H, L, D, N, W, P, seed=1):
    cache, model = make(mw, P, H, L, D, N, W)
    for s, n in enumerate(lens):
        if n:
            k, v = tokens((1, H, n, D), seed + s), tokens((1, H, n, D), seed + 50 + s)
            mw.mw_kvpages_append(cache, [s], k, v)
            model.append([s], k, v)
    return cache, model


def some_weights(cache, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.exp(2 * torch.randn(cache.desc.N, cache.desc.W * cache.desc.L, device="cuda", generator=g))
    return torch.where(torch.rand(w.shape, device="cuda", generator=g) < 0.2, 0.0, w.bfloat16().float())


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("L", [64, 192])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (64, 0, 64), (100, 30, 20), (200, 192, 0), (192, 192, 0), (257, 70, 187),
                                               (399, 0, 1)])
def test_what_stays(mw, D, L, keep, first, recent):
    """Several sequences, some of them short enough to be left alone; ties; nothing chosen by weight; a cut only."""
    cache, model = filled(mw, [400, 63, 0, 401, 577], 3, L, D, 6, 10, 60)
    w = some_weights(cache, keep)
    evict(mw, cache, model, [4, 0, 2, 1, 3], w, keep, first, recent)
    # and again, on what is left, and more tokens behind
    k, v = tokens((2, 3, 70, D), 90), tokens((2, 3, 70, D), 91)
    mw.mw_kvpages_append(cache, [0, 4], k, v)
    model.append([0, 4], k, v)
    evict(mw, cache, model, [0, 4], some_weights(cache, keep + 1), max(1, keep // 2), first // 2, recent // 2)


def test_equal_infinite_and_nan_weights(mw):
    import torch
    cache, model = filled(mw, [300, 300, 300, 300, 300], 2, 64, 64, 5, 6, 60)
    w = torch.zeros(5, 6 * 64, device="cuda")
    w[0] = 1.0                                     # all equal: the front ones
    w[1, 50:80] = float("nan")
    w[1, 100:103] = float("inf")
    w[1, 7:300:9] = -1.0
    w[2, ::2] = -0.0                               # equal to 0
    w[2, 200:210] = 1e-45                          # the least above 0
    w[3] = float("nan")
    w[4] = -torch.arange(6 * 64, device="cuda")
    w[4, 299] = -float("inf")
    evict(mw, cache, model, [0, 1, 2, 3, 4], w, 123, 0, 0)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_branches_keep_their_common_pages(mw, D):
    """The other branches read what they did; the anchor's whole pages stay shared; freed pages are those nobody reads."""
    cache, model = filled(mw, [500], 2, 64, D, 4, 9, 40)
    for s in (1, 2):
        mw.mw_kvpages_fork(cache, 0, s)
        model.rows[s], model.lens[s] = list(model.rows[0]), model.lens[0]
    evict(mw, cache, model, [1, 2], some_weights(cache, 5), 250, 150, 60)
    assert model.rows[1][:2] == model.rows[0][:2] == model.rows[2][:2] and model.rows[1][2] != model.rows[0][2]
    evict(mw, cache, model, [0], some_weights(cache, 6), 130, 0, 130)
    mw.mw_kvpages_free(cache, [0, 1])
    model.drop([0, 1])
    model.verify()


def test_too_few_pages(mw):
    import torch
    cache, model = filled(mw, [200, 200], 2, 64, 64, 2, 4, 10)  # two pages are free
    w = some_weights(cache, 7)
    before = w.clone()
    with pytest.raises(mw.MWError) as e:
        mw.mw_kvpages_evict_weighted(cache, [0, 1], w, 100)
    assert e.value.code == mw.MW_EFULL
    torch.cuda.synchronize()
    assert torch.equal(w, before)
    model.verify()
    evict(mw, cache, model, [0], w, 100)
    evict(mw, cache, model, [1], w, 100)


def test_long_sequences(mw):
    """More tokens than are held in LDS, and more pages than travel in one launch."""
    cache, model = filled(mw, [40001, 33100], 1, 64, 64, 2, 640, 2300)
    w = some_weights(cache, 8)
    evict(mw, cache, model, [0, 1], w, 33001, 1000, 501)
    evict(mw, cache, model, [0, 1], w, 20000, 0, 0)


def test_codes_that_were_finer(mw):
    """A token of a small block beside one of a large block: its codes are rounded again, and become subnormal or 0."""
    import torch
    H, D = 1, 64
    cache, model = make(mw, 8, H, 64, D, 1, 6)
    k, v = randn((1, H, 192, D), 1), randn((1, H, 192, D), 2)
    gain = torch.tensor([1.0, 2.0 ** 12, 2.0 ** -11], device="cuda").repeat_interleave(64).view(1, 1, 192, 1)
    k, v = (k.float() * gain).bfloat16(), (v.float() * gain).bfloat16()
    mw.mw_kvpages_append(cache, [0], k, v)
    model.append([0], k, v)
    w = torch.zeros(1, 6 * 64, device="cuda")
    w[0, ::3] = 1.0
    evict(mw, cache, model, [0], w, 64)


def test_a_rollout_that_drops_its_lightest_tokens(mw):
    """Positions, attention of the packed prompts, commit, single tokens over the pages with their weights, eviction, and
    the attention over what is left: every step against 64-bit values."""
    import torch
    H, Hkv, D, L, lens = 4, 2, 128, 64, [300, 211]
    T = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(9)
    x = {n: torch.randn(T, h, D, device="cuda", generator=g).bfloat16() for n, h in (("q", H), ("k", Hkv), ("v", Hkv))}
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=D)], halves=True)
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
    view = lambda t: t.transpose(0, 1)[None]
    mw.mw_rope_apply(view(x["q"]), view(x["k"]), rb, pos, q_out=view(x["q"]), k_out=view(x["k"]))
    cu = torch.tensor([0, *lens], device="cuda").cumsum(0).to(torch.int32)
    pack = mw.Packed(cu, T, H, Hkv, D)
    o, lse = mw.mw_packed_attn_fwd(x["q"], x["k"], x["v"], pack)
    cache, model = make(mw, 24, Hkv, L, D, 2, 8)
    at = 0
    for s, n in enumerate(lens):
        i = slice(at, at + n)
        at += n
        causal = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        for h in range(H):
            want = attention64(x["q"][i, h], x["k"][i, h // 2], x["v"][i, h // 2], causal, D ** -0.5)
            check(f"o {s} {h}", o[i, h], *want["o"])
        k, v = view(x["k"][i]), view(x["v"][i])
        mw.mw_kvpages_append(cache, [s], k, v)
        model.append([s], k, v)
    w = torch.zeros(2, 8 * L, device="cuda")
    total = torch.zeros(2, 8 * L, dtype=torch.float64, device="cuda")
    for step in range(3):
        q, k, v = (torch.randn(2, h, 1, D, device="cuda", generator=g).bfloat16() for h in (H, Hkv, Hkv))
        at = torch.tensor([[model.lens[0]], [model.lens[1]]], device="cuda")
        q, k = mw.mw_rope_apply(q, k, rb, at)
        o, lse = mw.mw_chunk_attn_paged(q, k, v, 1, 1, cache, [0, 1], want_lse=True)
        mw.mw_kvpages_weigh(cache, [0, 1], q, lse, w)
        torch.cuda.synchronize()
        for s in (0, 1):
            kk, vv = model.values(s)
            for h in range(H):
                a = torch.cat([kk[h // 2], k[s, h // 2].double()])
                c = torch.cat([vv[h // 2], v[s, h // 2].double()])
                none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
                want = attention64(q[s, h], a, c, none, D ** -0.5)
                check(f"o {step} {s} {h}", o[s, h], *want["o"])
                p = torch.exp((q[s, h].double() @ a.t())[0] * D ** -0.5 - want["lse"][0])
                total[s, :model.lens[s]] += p[:-1]
        # (32-bit sums of probabilities of at most 1, a few 2^-22 off each)
        assert bool(((w.double() - total).abs() <= 3 * H * 2.0 ** -19).all())
        mw.mw_kvpages_append(cache, [0, 1], k, v)
        model.append([0, 1], k, v)
    model.verify()
    evict(mw, cache, model, [0, 1], w, 150, 10, 20)
    q = torch.randn(2, H, 1, D, device="cuda", generator=g).bfloat16()
    o, _ = mw.mw_chunk_attn_paged(q, None, None, 1, 1, cache, [0, 1])
    for s in (0, 1):
        kk, vv = model.values(s)
        for h in range(H):
            none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
            check("o", o[s, h], *attention64(q[s, h], kk[h // 2], vv[h // 2], none, D ** -0.5)["o"])


def test_refusals_of_the_binding(mw):
    import torch
    cache, _ = filled(mw, [100, 100], 2, 64, 64, 2, 4, 12)
    w = torch.zeros(2, 256, device="cuda")
    q, lse = randn((2, 4, 3, 64), 1), torch.zeros(2, 4, 3, device="cuda")
    for bad in (w[:1], w.double(), w.cpu(), w.t().contiguous().t()):
        with pytest.raises(ValueError):
            mw.mw_kvpages_weigh(cache, [0, 1], q, lse, bad)
        with pytest.raises(ValueError):
            mw.mw_kvpages_evict_weighted(cache, [0, 1], bad, 50)
    with pytest.raises(ValueError):
        mw.mw_kvpages_weigh(cache, [0, 1], q, lse[:1], w)
    with pytest.raises(ValueError):
        mw.mw_kvpages_weigh(cache, [0], q, lse, w)
    with pytest.raises(mw.MWError):
        mw.mw_kvpages_weigh(cache, [1, 1], q, lse, w)
    with pytest.raises(mw.MWError):
        mw.mw_kvpages_evict_weighted(cache, [0, 0], w, 50)
    graph = torch.cuda.CUDAGraph()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(graph):
        w.add_(1.0)
        with pytest.raises(mw.MWError):
            mw.mw_kvpages_weigh(cache, [0, 1], q, lse, w, workspace=ws)
        with pytest.raises(mw.MWError):
            mw.mw_kvpages_evict_weighted(cache, [0, 1], w, 50, workspace=ws)


@pytest.mark.parametrize("H,T,n", [(8, 700, 3000), (256, 40, 500)])
def test_weights_with_a_workspace_of_another_size(mw, H, T, n):
    """One sized for other lengths: smaller ones divide the rows into what fits, larger ones change nothing."""
    import torch
    Hkv, D = 4, 64
    cache, model = make(mw, 120, Hkv, 64, D, 1, 50)
    k, v = randn((1, Hkv, n, D), 41), randn((1, Hkv, n, D), 51)
    mw.mw_kvpages_append(cache, [0], k, v)
    model.append([0], k, v)
    q = randn((1, H, T, D), 60)
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, [0], want_lse=True)
    need, one = mw.mw_kvpages_weigh_workspace_size(cache, [0], H, T), -(-n // 64) * 256
    assert need >= 3 * one
    whole = weights_of(mw, cache, model, [0], q, lse, H, add=False)
    for nbytes in (need + 1024, need, need - 16, 2 * one, 2 * one - 16, one, 16):
        print(f"[case] weigh {n} tokens, workspace of {nbytes} of {need} bytes", flush=True)
        space = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")  # (as fp32: NaN)
        w = weights_of(mw, cache, model, [0], q, lse, H, add=False, workspace=space[:nbytes])
        parts = int((~space[:nbytes // 4 * 4].view(torch.float32).isnan()).sum()) // n
        assert parts == 0 if nbytes < 2 * one else 2 <= parts <= nbytes // one
        assert bool((space[nbytes:] == 255).all())
        if nbytes >= need:
            assert torch.equal(w, whole)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv,T,n", [(4, 2, 40, 100), (8, 8, 600, 3000), (6, 2, 400, 5000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_that_weigh_nothing_may_hold_anything(mw, D, H, Hkv, T, n, bad):
    """Rows of LSE -inf, next to others and in rows of their own: the weights are those with any other queries there."""
    import torch
    cache, model = make(mw, 2 * n // 64 + 4, Hkv, 64, D, 2, n // 64 + 1)
    for s, m in enumerate((n, n // 3)):
        mw.mw_kvpages_append(cache, [s], randn((1, Hkv, m, D), 1 + s), randn((1, Hkv, m, D), 3 + s))
    q = randn((2, H, T, D), 5, "bthd")
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, [0, 1], want_lse=True)
    none = torch.zeros((2, H, T), dtype=torch.bool, device="cuda")
    none[0, :, 1::2] = none[1, 0] = none[1, :, -5:] = none[1, 1, 7] = True
    none[0, -1, 30:] = True
    lse[none] = -math.inf
    runs = []
    for x in (q, torch.where(none[..., None], bad, q.float()).bfloat16()):
        w = torch.zeros((2, cache.desc.W * 64), device="cuda")
        mw.mw_kvpages_weigh(cache, [0, 1], x, lse, w)
        runs.append(w)
    torch.cuda.synchronize()
    assert bool(runs[0].isfinite().all()) and bool((runs[0][0, :n] > 0).any())
    assert torch.equal(*runs)


@pytest.mark.parametrize("k", [5, 40, 100, 140])
def test_a_nan_is_lighter_than_minus_infinity(mw, k):
    """Rows of both, and of finite weights, so that the cut falls within each of the three."""
    import torch
    cache, _ = filled(mw, [200], 2, 64, 64, 1, 4, 12)
    g = torch.Generator().manual_seed(k)
    kind = torch.randint(0, 3, (256,), generator=g)
    w = torch.where(kind == 0, math.nan, torch.where(kind == 1, -math.inf, -torch.rand(256, generator=g)))
    order = sorted(range(3, 190), key=lambda j: (bool(w[j].isnan()), 0.0 if w[j].isnan() else -float(w[j]), j))
    stay = sorted([0, 1, 2, *order[:k], *range(190, 200)])
    got = w.cuda()[None].clone()
    before = [cache.k_pages.clone(), cache.k_scales.clone()]
    rows = [cache.page_of(0, i) for i in range(4)]
    mw.mw_kvpages_evict_weighted(cache, [0], got, k + 13, first=3, recent=10)
    torch.cuda.synchronize()
    want = torch.zeros(256)
    want[:k + 13] = w[stay]
    want[200:] = w[200:]
    assert torch.equal(got[0].cpu().nan_to_num(nan=1e9), want.nan_to_num(nan=1e9))
    value = lambda pages, scales, p, t: pages[p, :, t].view(torch.float8_e4m3fn).float() * scales[p]
    for i, j in enumerate(stay):
        new = value(cache.k_pages, cache.k_scales, cache.page_of(0, i // 64), i % 64)
        step = cache.k_scales[cache.page_of(0, i // 64)] * 2.0 ** -10  # (codes that become subnormal)
        assert bool(((new - value(*before, rows[j // 64], j % 64)).abs() <= step).all()), (i, j)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_weights_of_many_heads_of_a_key_head(mw, D):
    cache, model = make(mw, 12, 1, 64, D, 2, 6)
    for s, n in enumerate((300, 65)):
        k, v = randn((1, 1, n, D), 1 + s), randn((1, 1, n, D), 3 + s)
        mw.mw_kvpages_append(cache, [s], k, v)
        model.append([s], k, v)
    for H, T in ((16384, 1), (257, 3), (4095, 2)):
        q = randn((2, H, T, D), 5, "bthd")
        _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, T, cache, [1, 0], want_lse=True)
        weights_of(mw, cache, model, [1, 0], q, lse, H, old=0.5)


def test_as_many_sequences_as_a_call_names(mw):
    """256 of them, several empty or short; runs of pages in several launches; one token that stays of each."""
    H, D, L = 1, 64, 64
    lens = [(37 * s) % 201 for s in range(256)]
    cache, model = filled(mw, lens, H, L, D, 256, 5, 1400)
    q = randn((256, 2, 3, D), 5)
    seqs = [(s * 101 + 7) % 256 for s in range(256)]
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, 3, cache, seqs, want_lse=True)
    weights_of(mw, cache, model, seqs, q, lse, 2, add=False)
    w = some_weights(cache, 3)
    evict(mw, cache, model, seqs, w, 130, 65, 30)
    evict(mw, cache, model, seqs, w, 1)


def test_pages_of_the_largest_size(mw):
    """65536 tokens a page: blocks are found by a product's high word."""
    H, D, L = 1, 64, 1 << 16
    cache, model = filled(mw, [70_001, 131_072], H, L, D, 2, 2, 8)
    q = randn((2, 3, 2, D), 5)
    q = (q.float() / 256).bfloat16()
    _, lse = mw.mw_chunk_attn_paged(q, None, None, 1, 2, cache, [0, 1], want_lse=True)
    weights_of(mw, cache, model, [0, 1], q, lse, 3, add=False)
    evict(mw, cache, model, [1, 0], some_weights(cache, 4), 65_999, 65_537, 200)
