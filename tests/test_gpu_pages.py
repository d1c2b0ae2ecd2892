"""The paged 8-bit cache: pages, codes and scales against a model of them in torch, and the attention over it
against 64-bit values of what the codes stand for."""
import math
import random

import pytest

from attention_bounds import attention64, check

pytestmark = pytest.mark.gpu
BLOCK = 64


def randn(shape, seed, layout="bhtd"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, T, D = shape
    if layout == "bthd":
        return torch.randn(B, T, H, D, device="cuda", generator=g).bfloat16().transpose(1, 2)
    return torch.randn(B, H, T, D, device="cuda", generator=g).bfloat16()


def tokens(shape, seed, layout="bhtd"):
    """Tokens whose magnitude changes from token to token by up to 2^8 either way."""
    import torch
    x = randn(shape, seed, layout)
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    return (x.float() * torch.exp2(torch.randint(-8, 9, (shape[0], 1, shape[2], 1), device="cuda", generator=g))).bfloat16()


class Model:
    """What the cache holds, written apart from the library: per sequence a list of page numbers and its length;
    codes as the numbers they stand for over their scale."""

    def __init__(self, cache, P, H, L, D, N, W):
        import torch
        self.P, self.H, self.L, self.D, self.W = P, H, L, D, W
        self.cache = cache
        self.code = [torch.zeros(P, H, L, D, device="cuda") for _ in range(2)]
        self.exp = [torch.full((P, H, L // BLOCK), -1000, device="cuda") for _ in range(2)]
        self.rows = [[] for _ in range(N)]
        self.lens = [0] * N

    def users(self, page):
        return sum(r.count(page) for r in self.rows)

    def take(self, n, held=()):
        used = {p for r in self.rows for p in r} | set(held)
        return [p for p in range(self.P) if p not in used][:n]

    def append(self, seqs, k, v):
        t = k.shape[2]
        shared = {s: self.rows[s][-1] for s in seqs
                  if self.lens[s] % self.L and self.users(self.rows[s][-1]) > 1}
        held = set(shared.values())
        for i, s in enumerate(seqs):
            if s in shared:
                new = self.take(1, held)[0]
                old = self.rows[s][-1]
                n = self.lens[s] % self.L
                for x in range(2):
                    self.code[x][new, :, :n] = self.code[x][old, :, :n]
                    nb = -(-n // BLOCK)
                    self.exp[x][new, :, :nb] = self.exp[x][old, :, :nb]
                self.rows[s][-1] = new
            total = self.lens[s] + t
            self.rows[s] += self.take(-(-total // self.L) - len(self.rows[s]), held)
            pos, at = self.lens[s], 0
            while at < t:
                page, off = self.rows[s][pos // self.L], pos % self.L
                n = min(BLOCK - off % BLOCK, t - at)
                for x, src in enumerate((k, v)):
                    self.write(x, page, off, src[i, :, at:at + n].float())
                pos, at = pos + n, at + n
            self.lens[s] = total

    def write(self, x, page, off, val):
        import torch
        blk, first = off // BLOCK, off % BLOCK == 0
        top = val.abs().nan_to_num(0.0, posinf=float("inf")).amax((1, 2)).double()
        e = torch.ceil(torch.log2(top.clamp(2.0 ** -140, 2.0 ** 127) / 448))
        e = torch.where(top > 448 * torch.exp2(e), e + 1, torch.where(top <= 224 * torch.exp2(e), e - 1, e))
        e = e.clamp(-100, 100).long()
        old = self.exp[x][page, :, blk]
        if not first:
            lo = off // BLOCK * BLOCK
            grown = torch.maximum(e, old)
            self.code[x][page, :, lo:off] = self.round(torch.ldexp(self.code[x][page, :, lo:off].double(),
                                                                   (old - grown)[:, None, None]))
            e = grown
        self.exp[x][page, :, blk] = e
        self.code[x][page, :, off:off + val.shape[1]] = self.round(torch.ldexp(val.double(), -e[:, None, None]))

    @staticmethod
    def round(y):
        import torch
        return y.clamp(-448, 448).float().to(torch.float8_e4m3fn).float()

    def drop(self, seqs):
        for s in seqs:
            self.rows[s], self.lens[s] = [], 0

    def verify(self):
        import torch
        torch.cuda.synchronize()
        c = self.cache
        assert c.lens.tolist() == self.lens
        live = {p for r in self.rows for p in r}
        assert c.n_free == self.P - len(live)
        table = c.table.tolist()
        for s, r in enumerate(self.rows):
            assert table[s][:len(r)] == r and c.len(s) == self.lens[s]
            assert [c.page_of(s, w) for w in range(len(r))] == r
            for w, page in enumerate(r):
                n = min(self.L, self.lens[s] - w * self.L)
                nb = -(-n // BLOCK)
                for x, (pages, scales) in enumerate(((c.k_pages, c.k_scales), (c.v_pages, c.v_scales))):
                    got = pages[page, :, :n].view(torch.float8_e4m3fn).float()
                    want = self.code[x][page, :, :n]
                    assert torch.equal(got.nan_to_num(nan=1e9), want.nan_to_num(nan=1e9)), f"codes of sequence {s} page {w}"
                    assert torch.equal(scales[page, :, :nb].double(), torch.exp2(self.exp[x][page, :, :nb].double()))

    def values(self, s):
        """K and V of a sequence as the codes stand for them, [H, len, D] in 64 bits."""
        import torch
        out = []
        for x in range(2):
            if not self.rows[s]:
                out.append(torch.zeros(self.H, 0, self.D, dtype=torch.float64, device="cuda"))
                continue
            e = self.exp[x][self.rows[s]].double().repeat_interleave(BLOCK, -1)[..., None]
            y = self.code[x][self.rows[s]].double() * torch.exp2(e)  # [pages, H, L, D]
            out.append(y.transpose(0, 1).reshape(self.H, -1, self.D)[:, :self.lens[s]])
        return out


def make(mw, P, H, L, D, N, W, fill=0x7F):
    cache = mw.KVPages(P, H, L, D, N, W)
    for t in (cache.k_pages, cache.v_pages):
        t.fill_(fill)  # NaN codes: what no token has reached must never be read
    for t in (cache.k_scales, cache.v_scales):
        t.fill_(float("nan"))
    cache.table.fill_(-1)
    return cache, Model(cache, P, H, L, D, N, W)


def put(mw, cache, model, seqs, t, seed, layout="bhtd", make_tokens=tokens):
    k, v = (make_tokens((len(seqs), model.H, t, model.D), seed + i, layout) for i in range(2))
    mw.mw_kvpages_append(cache, seqs, k, v)
    model.append(seqs, k, v)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("L", [64, 192])
def test_appends_of_odd_lengths_fill_pages_and_blocks(mw, D, L):
    print(f"[case] append D={D} L={L}", flush=True)
    cache, model = make(mw, 40, 2, L, D, 3, 12)
    for i, (seqs, t) in enumerate((([0], 1), ([0], 62), ([0, 1], 1), ([1, 0, 2], 65), ([2], 64), ([2], 63), ([2, 0], 200),
                                   ([1], 1), ([1], 7))):
        put(mw, cache, model, seqs, t, 100 * i, "bthd" if i % 2 else "bhtd")
        model.verify()


@pytest.mark.parametrize("D", [64, 128])
def test_special_values(mw, D):
    """Zeros, values that underflow, the largest that fit, infinities and NaN; a NaN does not touch the scale."""
    import torch
    cache, model = make(mw, 8, 1, 64, D, 2, 4)
    special = [0.0, -0.0, 448.0, -448.0, 449.0, 1e-30, -3e38, 3e38, float("inf"), float("-inf"), float("nan"), 2.0 ** -133]

    def fixed(values):
        def f(shape, seed, layout):
            x = torch.zeros(shape, device="cuda")
            for i, val in enumerate(values):
                x[..., i % shape[2], i] = val
            return x.bfloat16()
        return f

    put(mw, cache, model, [0], 64, 0, make_tokens=fixed([0.0]))           # a block of zeros
    put(mw, cache, model, [0], 5, 0, make_tokens=fixed(special[:6]))      # then ordinary ones
    put(mw, cache, model, [0], 3, 0, make_tokens=fixed([1e4, float("nan")]))  # the scale grows over older codes
    put(mw, cache, model, [1], 9, 0, make_tokens=fixed(special))
    put(mw, cache, model, [1], 56, 0, make_tokens=fixed([1e-38] * 4))
    model.verify()


def test_a_growing_scale_rounds_older_codes_again(mw):
    import torch
    cache, model = make(mw, 4, 3, 128, 64, 1, 2)
    for i in range(30):
        grow = lambda shape, seed, layout: (randn(shape, seed, layout).float() * 2.0 ** (i % 11)).bfloat16()
        put(mw, cache, model, [0], 1 + i % 5, 10 * i, make_tokens=grow)
    model.verify()


@pytest.mark.parametrize("D", [64, 72])
def test_forks_share_pages_and_copy_them_on_write(mw, D):
    cache, model = make(mw, 40, 2, 128, D, 6, 8)
    put(mw, cache, model, [0], 300, 1)
    for dst in (1, 2, 5):
        mw.mw_kvpages_fork(cache, 0, dst)
        model.rows[dst], model.lens[dst] = list(model.rows[0]), model.lens[0]
    model.verify()
    put(mw, cache, model, [1, 2], 40, 2)       # both copy the shared last page
    model.verify()
    put(mw, cache, model, [0], 100, 3)         # shared with 5 still
    put(mw, cache, model, [5], 10, 4)          # now its own: written in place
    model.verify()
    mw.mw_kvpages_fork(cache, 1, 3)
    model.rows[3], model.lens[3] = list(model.rows[1]), model.lens[1]
    put(mw, cache, model, [1, 3], 1, 5)        # every sharer is in the call: both copy, the old page is free
    model.verify()
    mw.mw_kvpages_free(cache, [0, 2])
    model.drop([0, 2])
    model.verify()
    mw.mw_kvpages_copy(cache, 1, 0)
    pages = model.take(len(model.rows[1]))
    for x in range(2):
        model.code[x][pages] = model.code[x][model.rows[1]]
        model.exp[x][pages] = model.exp[x][model.rows[1]]
    model.rows[0], model.lens[0] = pages, model.lens[1]
    model.verify()


def test_full_pools_refuse_and_stay_as_they_were(mw):
    import torch
    cache, model = make(mw, 5, 1, 64, 64, 3, 4)
    put(mw, cache, model, [0, 1], 100, 1)
    k = torch.zeros(2, 1, 100, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(mw.MWError) as e:
        mw.mw_kvpages_append(cache, [0, 1], k, k)
    assert e.value.code == mw.MW_EFULL
    mw.mw_kvpages_fork(cache, 0, 2)
    model.rows[2], model.lens[2] = list(model.rows[0]), model.lens[0]
    for f, code in ((lambda: mw.mw_kvpages_copy(cache, 0, 1), mw.MW_EINVAL), (lambda: mw.mw_kvpages_fork(cache, 1, 2), mw.MW_EINVAL),
                    (lambda: mw.mw_kvpages_evict(cache, 0, 0, 2), mw.MW_EEMPTY),
                    (lambda: mw.mw_kvpages_append(cache, [0], k[:1].expand(1, 1, 100, 64), k[:1, :, :99]), ValueError)):
        with pytest.raises((mw.MWError, ValueError)) as e:
            f()
        assert e.type is code or e.value.code == code
    model.verify()
    put(mw, cache, model, [0], 1, 3)  # the last free page takes the copy of the shared one
    assert cache.n_free == 0
    with pytest.raises(mw.MWError):
        mw.mw_kvpages_append(cache, [1], k[:1], k[:1])
    mw.mw_kvpages_free(cache, [2])
    model.drop([2])
    with pytest.raises(mw.MWError):
        mw.mw_kvpages_copy(cache, 0, 2)  # two pages are needed
    model.verify()


@pytest.mark.parametrize("L", [64, 128])
def test_random_operations(mw, L):
    """300 operations of all kinds against the model, the pool often nearly full."""
    rng = random.Random(L)
    P, N, W = 40, 6, 10
    cache, model = make(mw, P, 1, L, 64, N, W)
    done = {}
    for i in range(300):
        kind = rng.choice(["append"] * 4 + ["fork", "copy", "free", "free", "evict", "compact"])
        s, d = rng.randrange(N), rng.choice([x for x in range(N) if not model.lens[x]] or [0])
        try:
            if kind == "append":
                seqs = rng.sample(range(N), rng.randint(1, 3))
                t = rng.choice([1, 3, 30, 64, 100, 200])
                k, v = (tokens((len(seqs), 1, t, 64), 10 * i + j) for j in range(2))
                mw.mw_kvpages_append(cache, seqs, k, v)
                model.append(seqs, k, v)
            elif kind == "fork":
                mw.mw_kvpages_fork(cache, s, d)
                model.rows[d], model.lens[d] = list(model.rows[s]), model.lens[s]
            elif kind == "copy":
                mw.mw_kvpages_copy(cache, s, d)
                pages = model.take(len(model.rows[s]))
                for x in range(2):
                    model.code[x][pages] = model.code[x][model.rows[s]]
                    model.exp[x][pages] = model.exp[x][model.rows[s]]
                model.rows[d], model.lens[d] = pages, model.lens[s]
            elif kind == "free":
                mw.mw_kvpages_free(cache, [s])
                model.drop([s])
            elif kind == "evict":
                full = model.lens[s] // L
                first = rng.randint(0, full)
                n = rng.randint(0, full - first)
                mw.mw_kvpages_evict(cache, s, first, n)
                del model.rows[s][first:first + n]
                model.lens[s] -= n * L
            else:
                live = sorted({p for r in model.rows for p in r})
                holes = [p for p in range(len(live)) if p not in live]
                move = dict(zip([p for p in live if p >= len(live)], holes))
                assert mw.mw_kvpages_compact(cache) == len(move)
                for src, dst in move.items():
                    for x in range(2):
                        model.code[x][dst] = model.code[x][src]
                        model.exp[x][dst] = model.exp[x][src]
                model.rows = [[move.get(p, p) for p in r] for r in model.rows]
            done[kind] = done.get(kind, 0) + 1
        except mw.MWError as e:
            assert e.code in (mw.MW_EFULL, mw.MW_EINVAL), e
        if i % 10 == 9:
            model.verify()
    model.verify()
    assert len(done) == 6 and min(done.values()) >= 5, done


def test_operations_of_more_pages_than_one_launch_names(mw):
    """900 pages appended, copied, and compacted at once; an eviction that moves a long row."""
    L, n = 64, 900
    cache, model = make(mw, 2 * n + 8, 1, L, 64, 3, n + 4)
    k, v = (randn((1, 1, n * L + 10, 64), i) for i in (1, 2))
    mw.mw_kvpages_append(cache, [0], k, v)
    mw.mw_kvpages_copy(cache, 0, 1)
    model.append([0], k, v)
    pages = model.take(n + 1)
    for x in range(2):
        model.code[x][pages] = model.code[x][model.rows[0]]
        model.exp[x][pages] = model.exp[x][model.rows[0]]
    model.rows[1], model.lens[1] = pages, model.lens[0]
    mw.mw_kvpages_evict(cache, 1, 3, 2)
    del model.rows[1][3:5]
    model.lens[1] -= 2 * L
    mw.mw_kvpages_free(cache, [0])
    model.drop([0])
    assert mw.mw_kvpages_compact(cache) == n - 1
    live = sorted(model.rows[1])
    move = dict(zip([p for p in live if p >= n - 1], [p for p in range(n - 1) if p not in live]))
    for src, dst in move.items():
        for x in range(2):
            model.code[x][dst] = model.code[x][src]
            model.exp[x][dst] = model.exp[x][src]
    model.rows[1] = [move.get(p, p) for p in model.rows[1]]
    model.verify()


# ------------------------------------------------------------------------------- attention

def attend(mw, cache, model, seqs, nq, ql, H, flags, seed=0, layout="bhtd", queued=True, split=True, scale=None):
    import torch
    D, G = model.D, H // model.H
    T, B = nq * ql, len(seqs)
    print(f"[case] paged D={D} L={model.L} lens={[model.lens[s] for s in seqs]} nq={nq} ql={ql} H={H}/{model.H} "
          f"flags={flags} queued={queued}", flush=True)
    q = randn((B, H, T, D), seed, layout)
    k, v = (randn((B, model.H, T, D), seed + i, layout) for i in (1, 2)) if queued else (None, None)
    o, lse = mw.mw_chunk_attn_paged(q, k, v, nq, ql, cache, seqs, flags=flags, want_lse=True, split=split, scale=scale)
    torch.cuda.synchronize()
    c = torch.arange(T, device="cuda") // ql
    hidden = c[None, :] > c[:, None] if flags == 0 else c[None, :] != c[:, None]
    for b, s in enumerate(seqs):
        K, V = model.values(s)
        old = torch.zeros((T, K.shape[1]), dtype=torch.bool, device="cuda")
        for hk in range(model.H):
            kk, vv, hid = K[hk], V[hk], old
            if queued:
                kk, vv = torch.cat([kk, k[b, hk].double()]), torch.cat([vv, v[b, hk].double()])
                hid = torch.cat([old, hidden], 1)
            rows = q[b, hk * G:(hk + 1) * G].reshape(G * T, D)
            want = attention64(rows, kk, vv, hid.repeat(G, 1), 1 / math.sqrt(D) if scale is None else scale)
            check(f"o b={b} hk={hk}", o[b, hk * G:(hk + 1) * G].reshape(G * T, D), *want["o"])
            check(f"lse b={b} hk={hk}", lse[b, hk * G:(hk + 1) * G].reshape(-1), *want["lse"])
    return o, lse


def filled(mw, H, L, D, lens, seed=0, W=None, make_tokens=randn):
    W = W or -(-max(max(lens), 1) // L) + 2
    cache, model = make(mw, sum(-(-n // L) for n in lens) + 3, H, L, D, len(lens), W)
    # committed in turns, so that the sequences' pages are mixed
    at = [0] * len(lens)
    while any(a < n for a, n in zip(at, lens)):
        for s, n in enumerate(lens):
            t = min(n - at[s], 150)
            if t > 0:
                put(mw, cache, model, [s], t, seed + at[s] + 7 * s, make_tokens=make_tokens)
                at[s] += t
    return cache, model


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("nq,ql,flags", [(1, 1, 0), (3, 1, 0), (1, 33, 0), (3, 70, 0), (3, 70, 1), (2, 130, 1), (5, 13, 0)])
def test_queues_over_ragged_histories(mw, D, nq, ql, flags):
    """Histories of zero, one, a block's and a page's edges and ordinary ones; unread places hold NaN codes."""
    cache, model = filled(mw, 2, 128, D, [0, 1, 64, 128, 129, 500], seed=D)
    attend(mw, cache, model, list(range(6)), nq, ql, 2, flags, seed=nq * ql)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv", [(3, 1), (8, 2), (40, 1)])
@pytest.mark.parametrize("nq,ql,flags", [(1, 1, 0), (4, 1, 0), (2, 40, 1)])
def test_shared_heads(mw, D, H, Hkv, nq, ql, flags):
    cache, model = filled(mw, Hkv, 64, D, [700, 130], seed=H)
    attend(mw, cache, model, [0, 1], nq, ql, H, flags, seed=H, layout="bthd")


@pytest.mark.parametrize("D", [64, 72, 128])
def test_cached_tokens_alone_and_repeated_sequences(mw, D):
    cache, model = filled(mw, 2, 64, D, [0, 333], seed=3)
    attend(mw, cache, model, [1, 0, 1], 1, 20, 4, 0, queued=False)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_long_histories_are_split(mw, D):
    cache, model = filled(mw, 1, 192, D, [6000, 10], seed=5)
    assert mw.mw_chunk_attn_paged_workspace_size(cache, [0, 1], 1, 1, 1) > 0
    a = attend(mw, cache, model, [0, 1], 1, 1, 1, 0, seed=5)
    b = attend(mw, cache, model, [0, 1], 1, 1, 1, 0, seed=5, split=False)
    attend(mw, cache, model, [0, 1], 1, 100, 2, 1, seed=6)


@pytest.mark.parametrize("D", [64, 128])
def test_blocks_of_very_different_magnitude(mw, D):
    def spread(shape, seed, layout):
        return (tokens(shape, seed, layout).float() * 0.25).bfloat16()
    cache, model = filled(mw, 2, 64, D, [400], seed=6, make_tokens=spread)
    attend(mw, cache, model, [0], 1, 40, 2, 0, seed=7, scale=0.02)


def test_many_rows_per_head(mw):
    cache, model = filled(mw, 1, 64, 128, [300, 641], seed=8)
    attend(mw, cache, model, [0, 1], 2, 333, 2, 0, seed=8)
    attend(mw, cache, model, [0, 1], 2, 333, 1, 1, seed=9, layout="bthd")


def test_offsets_beyond_32_bits(mw):
    """Pages of a pool of more than 4 GiB of codes: the last ones are written, copied and read."""
    import torch
    H, L, D = 16, 2048, 128
    P = (1 << 32) // (H * L * D) + 4
    cache = mw.KVPages(P, H, L, D, P + 1, 2)
    k1, v1 = randn((1, H, L, D), 1), randn((1, H, L, D), 2)
    for s in range(P - 2):
        mw.mw_kvpages_append(cache, [s], k1[:, :, :1], v1[:, :, :1])  # one token takes a page
    k, v = randn((1, H, 100, D), 3), randn((1, H, 100, D), 4)
    mw.mw_kvpages_append(cache, [P - 2], k, v)
    mw.mw_kvpages_copy(cache, P - 2, P - 1)
    assert cache.page_of(P - 2, 0) == P - 2 and cache.page_of(P - 1, 0) == P - 1 and cache.n_free == 0
    torch.cuda.synchronize()
    small = mw.KVPages(1, H, 128, D, 1, 1)
    mw.mw_kvpages_append(small, [0], k, v)
    q = randn((1, H, 3, D), 5)
    want, _ = mw.mw_chunk_attn_paged(q, None, None, 1, 3, small, [0])
    for s in (P - 2, P - 1):
        got, _ = mw.mw_chunk_attn_paged(q, None, None, 1, 3, cache, [s])
        assert torch.equal(got, want)
    for s in range(0, P - 2, 200):
        mw.mw_kvpages_free(cache, list(range(s, min(s + 200, P - 2))))
    assert mw.mw_kvpages_compact(cache) == 2
    for s in (P - 2, P - 1):
        got, _ = mw.mw_chunk_attn_paged(q, None, None, 1, 3, cache, [s])
        assert torch.equal(got, want)


def test_captured_calls_follow_the_cache(mw):
    """A captured attention, replayed while sequences grow, branch, roll and move between the replays, equals
    eager calls each time (its key ranges were planned for the lengths at the capture)."""
    import torch
    H, L, D = 2, 64, 64
    cache, model = filled(mw, H, L, D, [1500, 700, 0], seed=9, W=60)
    q, k, v = (randn((2, h, 8, D), 20 + i) for i, h in enumerate((4, H, H)))
    o, lse = torch.empty_like(q), torch.empty((2, 4, 8), device="cuda")
    ws = torch.empty(mw.mw_chunk_attn_paged_workspace_size(cache, [0, 1], 4, 1, 8), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: mw.mw_chunk_attn_paged(q, k, v, 1, 8, cache, [0, 1], out=o, lse=lse, workspace=ws)
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    t = lambda n, i: (randn((1, H, n, D), 50 + i), randn((1, H, n, D), 60 + i))
    steps = [lambda: None, lambda: mw.mw_kvpages_append(cache, [0], *t(130, 0)), lambda: mw.mw_kvpages_evict(cache, 0, 1, 9),
             lambda: mw.mw_kvpages_free(cache, [1]), lambda: mw.mw_kvpages_fork(cache, 0, 1),
             lambda: mw.mw_kvpages_append(cache, [1], *t(3, 1)), lambda: mw.mw_kvpages_compact(cache)]
    for step in steps:
        step()
        o.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        got = (o.clone(), lse.clone())
        call()
        torch.cuda.synchronize()
        # an eager call may divide longer keys otherwise: equal up to roundings
        assert torch.allclose(got[0].float(), o.float(), atol=2.0 ** -7 * 4) and torch.allclose(got[1], lse, atol=1e-4)
        again = mw.mw_chunk_attn_paged(q, k, v, 1, 8, cache, [0, 1], split=False)[0]
        assert torch.allclose(again.float(), o.float(), atol=2.0 ** -7 * 4)


def test_operations_refuse_a_stream_under_capture(mw):
    """They change the books on the host, which a replay does not; a refusal leaves the cache and the capture alone."""
    import torch
    H, L, D = 2, 64, 64
    cache, model = filled(mw, H, L, D, [200, 0, 0], seed=4)
    k, v = randn((1, H, 5, D), 1), randn((1, H, 5, D), 2)
    x = torch.zeros(64, device="cuda")
    free = cache.n_free
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for op in (lambda: mw.mw_kvpages_append(cache, [0], k, v), lambda: mw.mw_kvpages_fork(cache, 0, 1),
                   lambda: mw.mw_kvpages_copy(cache, 0, 1), lambda: mw.mw_kvpages_free(cache, [0]),
                   lambda: mw.mw_kvpages_evict(cache, 0, 0, 1), lambda: mw.mw_kvpages_compact(cache)):
            with pytest.raises(mw.MWError, match="captured"):
                op()
        x += 1
    for n in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, torch.full_like(x, n + 1.0))
    assert cache.n_free == free and cache.len(0) == 200 and cache.len(1) == 0
    model.verify()
    mw.mw_kvpages_append(cache, [0], k, v)  # and outside a capture they run as before
    assert cache.len(0) == 205


# ------------------------------------------------------------------------------- together

@pytest.mark.parametrize("D", [64, 128])
def test_conditioned_branching_rollout(mw, D):
    """A rollout as a server runs it: history committed, branched, every branch stepped with a queue that attends to
    its own history and, through cross attention, to its own prompt; the best branch kept, the window rolled
    behind an anchor, the pool compacted."""
    import torch
    H, L, ql = 2, 64, 40
    cache, model = make(mw, 60, H, L, D, 4, 16)
    put(mw, cache, model, [0], 200, 1, make_tokens=randn)
    prompt = [randn((3, H, 50, D), 2 + i) for i in range(2)]
    kv_len = torch.tensor([50, 0, 17], dtype=torch.int32, device="cuda")
    none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
    for step in range(3):
        for s in (1, 2, 3):
            mw.mw_kvpages_fork(cache, 0, s)
            model.rows[s], model.lens[s] = list(model.rows[0]), model.lens[0]
        x, lse = attend(mw, cache, model, [1, 2, 3], 2, ql, H, 0, seed=30 + step)
        y, yl = mw.mw_cross_attn_fwd(x, *prompt, kv_len=kv_len)
        for b, n in enumerate(kv_len.tolist()):
            for h in range(H):
                want = attention64(x[b, h], prompt[0][b, h, :n], prompt[1][b, h, :n], none, 1 / math.sqrt(D))
                check(f"cross b={b} h={h}", y[b, h], *want["o"])
                check(f"cross lse b={b} h={h}", yl[b, h], *want["lse"])
        done = (x[:, :, :ql].contiguous(), (x + y)[:, :, :ql].contiguous())  # the finished chunk
        mw.mw_kvpages_append(cache, [1, 2, 3], *done)
        model.append([1, 2, 3], *done)
        model.verify()
        best = 1 + step
        mw.mw_kvpages_free(cache, [0] + [s for s in (1, 2, 3) if s != best])
        model.drop([0] + [s for s in (1, 2, 3) if s != best])
        mw.mw_kvpages_fork(cache, best, 0)
        model.rows[0], model.lens[0] = list(model.rows[best]), model.lens[best]
        mw.mw_kvpages_free(cache, [best])
        model.drop([best])
        mw.mw_kvpages_evict(cache, 0, 1, 1)  # the page behind the anchor
        del model.rows[0][1:2]
        model.lens[0] -= L
        moved = mw.mw_kvpages_compact(cache)
        live = sorted(model.rows[0])
        move = dict(zip([p for p in live if p >= len(live)], [p for p in range(len(live)) if p not in live]))
        assert moved == len(move)
        for src, dst in move.items():
            for i in range(2):
                model.code[i][dst] = model.code[i][src]
                model.exp[i][dst] = model.exp[i][src]
        model.rows[0] = [move.get(p, p) for p in model.rows[0]]
        model.verify()
