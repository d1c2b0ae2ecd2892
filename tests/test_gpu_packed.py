"""Attention of packed sequences forward and backward against 64-bit values, at the lengths, masks, strides and shared
heads where it can go wrong."""
import math

import pytest

from attention_bounds import attention64, check

pytestmark = pytest.mark.gpu


def randn(shape, seed, layout="thd"):
    """bf16 [T,H,D], or a view of that shape."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, H, D = shape
    if layout == "thd":
        return torch.randn(T, H, D, device="cuda", generator=g).bfloat16()
    if layout == "htd":
        return torch.randn(H, T, D, device="cuda", generator=g).bfloat16().transpose(0, 1)
    wide = torch.randn(T, H, D + 8, device="cuda", generator=g).bfloat16()  # rows with a gap behind them
    return wide[..., :D]


def edges(lens, first=0):
    import torch
    return (torch.tensor([0, *lens], device="cuda").cumsum(0) + first).to(torch.int32)


def hidden_of(nq, nk, chunk):
    import torch
    at = torch.arange(nk - nq, nk, device="cuda").view(nq, 1)
    j = torch.arange(nk, device="cuda").view(1, nk)
    return (j // chunk > torch.div(at, chunk, rounding_mode="floor")) | (at < 0)


def verify(mw, nk, H, Hkv, D, chunk=1, nq=None, layout="thd", backward=True, scale=None, seed=1, behind=0, bad=None):
    """behind: tokens behind the last sequence; bad: a value that those and the sequences of no queries hold."""
    import torch
    print(f"[case] packed nk={nk} nq={nq} H={H} Hkv={Hkv} D={D} chunk={chunk} {layout} behind={behind}", flush=True)
    nq_ = nk if nq is None else nq
    Tq, Tk = max(1, sum(nq_) + behind), max(1, sum(nk) + behind)
    q, do = randn((Tq, H, D), seed, layout), randn((Tq, H, D), seed + 1, layout)
    k, v = randn((Tk, Hkv, D), seed + 2, layout), randn((Tk, Hkv, D), seed + 3, layout)
    if bad is not None:
        for t, n in ((q, nq_), (do, nq_), (k, nk), (v, nk)):
            t[sum(n):] = bad
    cu_q = edges(nq_)
    pack = mw.Packed(cu_q, Tq, H, Hkv, D, chunk_len=chunk, cu_k=None if nq is None else edges(nk), total_k=Tk, backward=backward)
    mark = lambda t: torch.full_like(t, 7.0)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack, scale=scale, out=mark(q), lse=torch.full((H, Tq), 7.0, device="cuda"))
    got = {"o": o, "lse": lse}
    if backward:
        got["dq"], got["dk"], got["dv"] = mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack, scale=scale, dq=mark(q), dk=mark(k),
                                                                dv=mark(v))
    torch.cuda.synchronize()
    for name, t in got.items():  # what no sequence has is left as it was
        n = sum(nk) if name in ("dk", "dv") else sum(nq_)
        assert bool(((t[:, n:] if name == "lse" else t[n:]) == 7).all()), name
    sc = 1 / math.sqrt(D) if scale is None else scale
    G = H // Hkv
    q0 = k0 = 0
    for s, (a, b) in enumerate(zip(nq_, nk)):
        i, j = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        if a == 0:
            if backward:
                assert not bool(got["dk"][j].any()) and not bool(got["dv"][j].any())
            continue
        hidden = hidden_of(a, b, chunk).repeat(G, 1)
        for hk in range(Hkv):
            h = slice(hk * G, (hk + 1) * G)
            rows = lambda t: t[i, h].transpose(0, 1).reshape(G * a, -1)
            want = attention64(rows(q), k[j, hk], v[j, hk], hidden, sc, rows(do) if backward else None)
            for name, (value, bound) in want.items():
                x = got[name]
                x = x[j, hk] if name in ("dk", "dv") else x[h, i].reshape(-1) if name == "lse" else rows(x)
                check(f"{name} s={s} hk={hk}", x, value, bound)
    return got


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("chunk", [1, 7, 64, 100000])
@pytest.mark.parametrize("lens", [[1], [0, 2, 63], [64, 65, 0, 1], [129, 31, 200], [333]])
def test_small_and_odd_lengths(mw, D, chunk, lens):
    verify(mw, lens, 2, 2, D, chunk=chunk, seed=sum(lens) + chunk % 97)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv", [(3, 1), (4, 2), (8, 1), (10, 2), (6, 1)])
@pytest.mark.parametrize("chunk", [1, 33])
def test_shared_heads(mw, D, H, Hkv, chunk):
    verify(mw, [50, 1, 130], H, Hkv, D, chunk=chunk, layout="htd", seed=H + chunk)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("chunk", [1, 20, 1000])
def test_queries_that_are_the_newest_tokens(mw, D, chunk):
    """Fewer queries than keys, as many, none, and none of the keys; more queries than keys (the first ones see nothing)."""
    verify(mw, [70, 200, 1, 64, 90], 4, 2, D, chunk=chunk, nq=[1, 33, 1, 64, 0], seed=5)
    verify(mw, [70, 0, 10, 1], 2, 1, D, chunk=chunk, nq=[100, 5, 140, 2], seed=6)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_tokens_of_no_sequence_are_neither_read_nor_written(mw, D, bad):
    verify(mw, [65, 127, 3], 2, 2, D, seed=7, behind=70, bad=bad)
    verify(mw, [300, 17], 4, 1, D, chunk=50, nq=[2, 17], seed=8, behind=3, bad=bad)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_a_sequence_of_nan_stays_its_own(mw, D):
    import torch
    lens, H = [40, 70, 100], 2
    q, k, v, do = (randn((210, H, D), 10 + i) for i in range(4))
    pack = mw.Packed(edges(lens), 210, H, H, D, backward=True)
    runs = []
    for bad in (None, float("nan")):
        if bad is not None:
            for t in (q, k, v, do):
                t[40:110] = bad
        o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
        runs.append([o, lse.t(), *mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)])
    torch.cuda.synchronize()
    for a, b in zip(*runs):
        assert torch.equal(a[:40], b[:40]) and torch.equal(a[110:], b[110:])
        assert bool(b[40:110].isnan().any())


@pytest.mark.parametrize("D", [64, 72, 128])
def test_long_keys_of_few_rows_are_cut(mw, D):
    for nk, nq in (([6001], [1]), ([3001, 7, 1999], [1, 1, 1]), ([4000, 30], [40, 30])):
        assert mw.mw_packed_attn_workspace_size(mw.Packed(edges(nq), sum(nq), 4, 2, D, cu_k=edges(nk), total_k=sum(nk))) > 0
        verify(mw, nk, 4, 2, D, nq=nq, seed=sum(nk))


@pytest.mark.parametrize("D", [64, 72, 128])
def test_cut_tiles_of_every_size_are_joined_whole(mw, D):
    """Tiles of 64 and of 128 rows and keys, every row and key of them, cut along long keys or rows."""
    for H, nk, nq in ((2, [6000], [64]), (1, [5000, 4000], [64, 63]), (2, [4100], [2050]), (1, [3000], [3000])):
        pack = mw.Packed(edges(nq), sum(nq), H, 1, D, cu_k=edges(nk), total_k=sum(nk), backward=True)
        assert mw.mw_packed_attn_workspace_size(pack) > 0
        verify(mw, nk, H, 1, D, nq=nq, seed=sum(nk) + H)
    verify(mw, [700, 64], 8, 1, D, seed=12)      # rows of many heads: key tiles are cut
    verify(mw, [2000, 1100], 16, 8, D, seed=13)  # tiles of 128 at some widths


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("chunk", [1, 600])
def test_long_sequences(mw, D, chunk):
    """Whole steps, steps on the diagonal and cut tiles of both directions."""
    verify(mw, [2111, 777, 90], 2, 1, D, chunk=chunk, seed=9)


@pytest.mark.parametrize("D,H,Hkv,chunk,lens", [(64, 8, 8, 64, [3471, 2406, 1997]), (72, 4, 1, 1, [3091, 2664, 1849]),
                                                (128, 4, 2, 1, [8, 1353, 2, 2523, 1706]), (72, 2, 2, 64, [4763, 4353])])
def test_fewer_tiles_than_places(mw, D, H, Hkv, chunk, lens):
    """Tiles cut into more items than run at once, and into fewer; parts of uneven number."""
    verify(mw, lens, H, Hkv, D, chunk=chunk, seed=60)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_many_sequences(mw, D):
    import torch
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 40, (1500,), generator=g).tolist()
    H, T = 2, sum(lens)
    q, k, v, do = (randn((T, H, D), 20 + i) for i in range(4))
    pack = mw.Packed(edges(lens), T, H, H, D, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    dq, dk, dv = mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)
    # one sequence alone gives the same rows: its tiles' steps are its own
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    for s in (0, 700, 1023, 1024, 1025, 1499):
        if lens[s] == 0:
            continue
        i = slice(at[s], at[s + 1])
        one = mw.Packed(edges([lens[s]]), lens[s], H, H, D, backward=True)
        o1, lse1 = mw.mw_packed_attn_fwd(q[i], k[i], v[i], one)
        g1 = mw.mw_packed_attn_bwd(q[i], k[i], v[i], o1, do[i], lse1, one)
        hidden = hidden_of(lens[s], lens[s], 1)
        for h in range(H):
            want = attention64(q[i, h], k[i, h], v[i, h], hidden, D ** -0.5, do[i, h])
            for name, a, b in zip(("o", "dq", "dk", "dv"), (o, dq, dk, dv), (o1, *g1)):
                check(f"{name} s={s}", a[i, h], *want[name])
                check(f"{name} s={s} alone", b[:, h], *want[name])
            check(f"lse s={s}", lse[h, i], *want["lse"])


@pytest.mark.parametrize("D", [64, 72, 128])
def test_strided_results_equal_contiguous_ones_and_repeat(mw, D):
    import torch
    lens, H, Hkv = [300, 170, 1], 4, 2
    T = sum(lens)
    pack = mw.Packed(edges(lens), T, H, Hkv, D, chunk_len=50, backward=True)
    t = [randn((T, H, D), 50, "htd"), randn((T, Hkv, D), 51, "gap"), randn((T, Hkv, D), 52, "htd"), randn((T, H, D), 53, "gap")]
    runs = []
    for x in (t, [y.contiguous() for y in t], t):
        q, k, v, do = x
        o, lse = torch.empty_like(t[0]), torch.empty((H, T), device="cuda")
        mw.mw_packed_attn_fwd(q, k, v, pack, out=o, lse=lse)
        runs.append((o.contiguous(), lse, *mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)))
    torch.cuda.synchronize()
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_keys_shared_between_heads(mw, D):
    """A head stride of 0 reads as the expanded copy; each key head's gradient is its own."""
    import torch
    T, H = 150, 3
    q, do = randn((T, H, D), 60), randn((T, H, D), 61)
    k, v = (randn((T, 1, D), 62 + i).expand(T, H, D) for i in range(2))
    pack = mw.Packed(edges([100, 50]), T, H, H, D, backward=True)
    runs = []
    for kk, vv in ((k, v), (k.contiguous(), v.contiguous())):
        o, lse = mw.mw_packed_attn_fwd(q, kk, vv, pack)
        runs.append((o, lse, *mw.mw_packed_attn_bwd(q, kk, vv, o, do, lse, pack)))
    torch.cuda.synchronize()
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_outputs_stay_within_their_views(mw):
    import torch
    lens, H, D = [37, 45], 2, 72
    T = sum(lens)
    q, k, v, do = (randn((T, H, D), 65 + i) for i in range(4))
    pack = mw.Packed(edges(lens), T, H, H, D, backward=True)
    mark = lambda: torch.full((T + 3, H, D + 8), 7.0, device="cuda", dtype=torch.bfloat16)
    o, dq, dk, dv = (mark() for _ in range(4))
    cut = lambda x: x[:T, :, :D]
    _, lse = mw.mw_packed_attn_fwd(q, k, v, pack, out=cut(o))
    mw.mw_packed_attn_bwd(q, k, v, cut(o), do, lse, pack, dq=cut(dq), dk=cut(dk), dv=cut(dv))
    torch.cuda.synchronize()
    for x in (o, dq, dk, dv):
        assert bool((x[..., D:] == 7).all()) and bool((x[T:] == 7).all()) and not bool((cut(x) == 7).all())


def test_one_sequence_is_block_causal_attention(mw):
    """The same rows through mw_block_causal_attn_*, within both kernels' bounds."""
    import torch
    T, H, D, chunk = 700, 4, 128, 120
    q, k, v, do = (randn((T, H, D), 75 + i) for i in range(4))
    pack = mw.Packed(edges([T]), T, H, H, D, chunk_len=chunk, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    grads = mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)
    view = lambda t: t.transpose(0, 1)[None]
    o1, lse1 = mw.mw_block_causal_attn_fwd(view(q), view(k), view(v), chunk)
    grads1 = mw.mw_block_causal_attn_bwd(view(q), view(k), view(v), o1, view(do), lse1, chunk)
    hidden = hidden_of(T, T, chunk)
    for h in range(H):
        want = attention64(q[:, h], k[:, h], v[:, h], hidden, D ** -0.5, do[:, h])
        for name, a, b in zip(("o", "dq", "dk", "dv"), (o, *grads), (o1, *grads1)):
            check(name, a[:, h], b[0, h], 2 * want[name][1])
        check("lse", lse[h], lse1[0, h], 2 * want["lse"][1])


def test_large_scores(mw):
    for scale in (8.0, 1e-4):
        verify(mw, [300, 40], 2, 1, 128, scale=scale, backward=False, seed=9)
        verify(mw, [1000], 2, 1, 64, nq=[1], scale=scale, backward=False, seed=9)


def test_gradient_against_differences(mw):
    """The loss sum(dO * O) along random directions: the gradients' inner products with them against central
    differences of the 64-bit forward."""
    import torch
    lens, H, Hkv, D, chunk = [20, 11], 2, 1, 64, 4
    T = sum(lens)
    x = [randn((T, h, D), 70 + i) for i, h in enumerate((H, Hkv, Hkv))]
    do = randn((T, H, D), 73)
    pack = mw.Packed(edges(lens), T, H, Hkv, D, chunk_len=chunk, backward=True)
    o, lse = mw.mw_packed_attn_fwd(*x, pack)
    grads = mw.mw_packed_attn_bwd(*x, o, do, lse, pack)

    def loss(q, k, v):
        total, at = 0.0, 0
        for n in lens:
            i = slice(at, at + n)
            at += n
            for h in range(H):
                s = (q[i, h] @ k[i, 0].t() / 8.0).masked_fill(hidden_of(n, n, chunk), float("-inf"))
                total += float((torch.softmax(s, -1) @ v[i, 0] * do[i, h].double()).sum())
        return total

    x = [t.double() for t in x]
    for i, name in enumerate("qkv"):
        u = randn(tuple(x[i].shape), 80 + i).double()
        h = 1e-5
        up, down = ([t + (h * s * u if j == i else 0) for j, t in enumerate(x)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        got = float((grads[i].double() * u).sum())
        # roundings of the gradient's terms: at most 2^-6 of its 1-norm against |u|, and they add in 2-norm
        off = 2.0 ** -6 * float((grads[i].double() * u).norm())
        print(f"[slope] d{name}: {got:.6f} against {slope:.6f}, allowed {off:.6f}", flush=True)
        assert abs(got - slope) <= off


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H", [3, 12])
def test_gradients_of_rows_of_few_keys_keep_their_precision(mw, D, H):
    """Many short sequences, so that most rows see few keys: next to those keys' dP - Delta the rounding of O to bf16
    would not be small, so Delta must not come from it.  What is left is the rounding of dS and that of the gradient itself:
    relative errors of at most 2^-8 each, spread over their interval, so 2^-8 / sqrt(3) in the mean square at most
    and sqrt(2) of that together, for sums of independent terms (random inputs) too."""
    import torch
    lens, Hkv = [5, 2, 17, 40, 9, 3] * 8, 3
    T, G = sum(lens), H // 3
    q, do = randn((T, H, D), 1), randn((T, H, D), 2)
    k, v = randn((T, Hkv, D), 3), randn((T, Hkv, D), 4)
    pack = mw.Packed(edges(lens), T, H, Hkv, D, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    got = dict(zip(("dq", "dk", "dv"), mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)))
    want = {n: torch.zeros(t.shape, dtype=torch.float64) for n, t in got.items()}
    q, do, k, v = (t.double().cpu() for t in (q, do, k, v))
    at = 0
    for n in lens:
        i = slice(at, at + n)
        at += n
        hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
        for h in range(H):
            P = torch.softmax((q[i, h] @ k[i, h // G].t() / math.sqrt(D)).masked_fill(hidden, float("-inf")), -1)
            dP = do[i, h] @ v[i, h // G].t()
            dS = P * (dP - (P * dP).sum(-1, keepdim=True)) / math.sqrt(D)
            want["dq"][i, h] = dS @ k[i, h // G]
            want["dk"][i, h // G] += dS.t() @ q[i, h]
            want["dv"][i, h // G] += P.t() @ do[i, h]
    for name, w in want.items():
        g = got[name].double().cpu()
        print(f"[precision] {name}: {((g - w).norm() / w.norm()).item():.2e}", flush=True)
        assert (g - w).norm() <= 2.0 ** -8 * math.sqrt(2 / 3) * w.norm(), name


@pytest.mark.parametrize("D,H,Hkv,chunk", [(128, 12, 6, 600), (72, 16, 16, 1), (64, 24, 8, 1)])
def test_rows_that_fill_the_card(mw, D, H, Hkv, chunk):
    verify(mw, [4800, 2399, 1, 700], H, Hkv, D, chunk=chunk, layout="thd", seed=40)


def test_side_stream_and_graph_replays(mw):
    """A captured plan, forward and backward, replayed over new inputs and lengths with eager work between, equals
    eager calls; two graphs that share workspaces, replayed in turn, too."""
    import torch
    H, Hkv, D, T, N = 4, 2, 64, 900, 4
    q, do = (torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.empty((T, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    pack = mw.Packed(cu, T, H, Hkv, D, chunk_len=30, backward=True)
    outs = [[torch.zeros_like(q), torch.zeros((H, T), device="cuda"), torch.zeros_like(q), torch.zeros_like(k),
             torch.zeros_like(v)] for _ in range(2)]
    ws = torch.empty(max(16, mw.mw_packed_attn_workspace_size(pack)), dtype=torch.uint8, device="cuda")
    ws_b = torch.empty(mw.mw_packed_attn_bwd_workspace_size(pack), dtype=torch.uint8, device="cuda")

    def load(seed):
        for i, t in enumerate((q, do, k, v)):
            t.copy_(randn(tuple(t.shape), seed + i))
        cu.copy_(torch.tensor([0, seed % 90, 500, 500 + seed % 77, T - seed % 5], dtype=torch.int32))

    def step(x):
        pack.update()
        mw.mw_packed_attn_fwd(q, k, v, pack, out=x[0], lse=x[1], workspace=ws)
        mw.mw_packed_attn_bwd(q, k, v, x[0], do, x[1], pack, workspace=ws_b, dq=x[2], dk=x[3], dv=x[4])

    load(101)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for x in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(x)
        graphs.append(g)
    for seed in (203, 311, 477):
        load(seed)
        for t in (t for x in outs for t in x):
            t.fill_(9.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        eager = [torch.full_like(t, 9.0) for t in outs[0]]
        step(eager)
        torch.cuda.synchronize()
        for x in outs:
            for a, b in zip(x, eager):
                assert torch.equal(a, b)


@pytest.mark.parametrize("D,H,Hkv,lens", [(128, 4, 2, [1500, 7, 2600]), (64, 12, 4, [4100, 900]), (72, 3, 3, [5, 3000])])
def test_two_calls_at_once_share_a_plan(mw, D, H, Hkv, lens):
    """Both directions on two streams, eagerly and as two graphs replayed together, against one after the other."""
    import torch
    T = sum(lens)
    pack = mw.Packed(edges(lens), T, H, Hkv, D, backward=True)
    sets = []
    for seed in (70, 80):
        q, do = randn((T, H, D), seed), randn((T, H, D), seed + 1)
        k, v = randn((T, Hkv, D), seed + 2), randn((T, Hkv, D), seed + 3)
        work = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
                for n in (mw.mw_packed_attn_workspace_size(pack), mw.mw_packed_attn_bwd_workspace_size(pack))]
        out = [torch.empty_like(q), torch.empty((H, T), device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)]
        sets.append((q, k, v, do, work, out))

    def run(x):
        q, k, v, do, work, out = x
        mw.mw_packed_attn_fwd(q, k, v, pack, out=out[0], lse=out[1], workspace=work[0])
        mw.mw_packed_attn_bwd(q, k, v, out[0], do, out[1], pack, workspace=work[1], dq=out[2], dk=out[3], dv=out[4])

    want = []
    for x in sets:
        run(x)
        torch.cuda.synchronize()
        want.append([t.clone() for t in x[5]])
    streams = [torch.cuda.Stream() for _ in sets]
    graphs = []
    for s, x in zip(streams, sets):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            run(x)
        graphs.append(g)
    for eager in (True, False, True, False):
        for x in sets:
            for t in x[5]:
                t.fill_(9.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for s, x, g in zip(streams, sets, graphs):
                with torch.cuda.stream(s):
                    if eager:
                        run(x)
                    else:
                        g.replay()
        torch.cuda.synchronize()
        for x, w in zip(sets, want):
            assert all(torch.equal(a, b) for a, b in zip(x[5], w))


def test_places_out_of_range_stay_within_the_tensors(mw):
    """Lengths that overrun the tensors are cut, descending ones empty; what lies around the outputs is left alone."""
    import torch
    H, D, T = 2, 64, 100
    wide = [torch.full((T + 200, H, D), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    o, dq, dk, dv = (w[100:100 + T] for w in wide)
    q, k, v, do = (randn((T, H, D), 90 + i) for i in range(4))
    cu = torch.tensor([-5, 50, 300, 20, 90, 2**31 - 1], device="cuda").to(torch.int32)
    pack = mw.Packed(cu, T, H, H, D, backward=True)
    lse = torch.full((H, T), 7.0, device="cuda")
    mw.mw_packed_attn_fwd(q, k, v, pack, out=o, lse=lse)
    mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for w in wide:
        assert bool((w[:100] == 7).all()) and bool((w[100 + T:] == 7).all())
    hidden = hidden_of(50, 50, 1)  # the first sequence is not touched by the others
    check("o", o[:20, 0], *(x[:20] for x in attention64(q[:50, 0], k[:50, 0], v[:50, 0], hidden, D ** -0.5)["o"]))


def test_two_plans_of_a_batch_give_the_same_bits(mw):
    """Where the plan puts an item is decided by atomics, what the item computes is not."""
    import torch
    lens, H, Hkv, D = [3000, 2, 700, 0, 1111, 40], 4, 2, 128
    T = sum(lens)
    q, do = randn((T, H, D), 95), randn((T, H, D), 96)
    k, v = randn((T, Hkv, D), 97), randn((T, Hkv, D), 98)
    runs = []
    for _ in range(3):
        pack = mw.Packed(edges(lens), T, H, Hkv, D, backward=True)
        o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
        runs.append((o, lse, *mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)))
    torch.cuda.synchronize()
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_heads_far_apart(mw, D):
    """Query heads of a key head more than 2^32 bytes apart read as their copies."""
    import torch
    T, H, far = 200, 3, 2**30 + 64
    big = [torch.empty(2 * far + T * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, do = (b.as_strided((T, H, D), (D, far, 1)) for b in big)
    q.copy_(randn((T, H, D), 101))
    do.copy_(randn((T, H, D), 102))
    k, v = randn((T, 1, D), 103), randn((T, 1, D), 104)
    pack = mw.Packed(edges([150, 50]), T, H, 1, D, backward=True)
    runs = []
    for x, y in ((q, do), (q.contiguous(), do.contiguous())):
        o, lse = mw.mw_packed_attn_fwd(x, k, v, pack, out=torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda"))
        runs.append((o, lse, *mw.mw_packed_attn_bwd(x, k, v, o, y, lse, pack)))
    torch.cuda.synchronize()
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits(mw):
    """Keys of more than 2^32 bytes: single tokens at the end of a long and of a short sequence."""
    import torch
    Hkv, D, nk = 16, 128, [1_100_000, 777]
    Tk = sum(nk)
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v = (torch.empty((Tk, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        for i in range(0, Tk, 1 << 17):
            t[i:i + (1 << 17)] = torch.randn((min(Tk, i + (1 << 17)) - i, Hkv, D), device="cuda", generator=g).bfloat16()
    q = randn((4, 32, D), 8)
    pack = mw.Packed(edges([1, 3]), 4, 32, Hkv, D, cu_k=edges(nk), total_k=Tk)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    torch.cuda.synchronize()
    for i, j, h in ((slice(0, 1), slice(0, nk[0]), 31), (slice(1, 4), slice(nk[0], Tk), 0), (slice(1, 4), slice(nk[0], Tk), 31)):
        n = j.stop - j.start
        want = attention64(q[i, h], k[j, h // 2], v[j, h // 2], hidden_of(i.stop - i.start, n, 1), D ** -0.5)
        check(f"o {h}", o[i, h], *want["o"])
        check(f"lse {h}", lse[h, i], *want["lse"])


def test_refusals_of_the_binding(mw):
    import torch
    T, H, D = 10, 2, 64
    q = randn((T, H, D), 1)
    pack = mw.Packed(edges([T]), T, H, H, D)
    with pytest.raises(TypeError):
        mw.mw_packed_attn_fwd(q.float(), q, q, pack)
    for bad in (q[:5], q[:, :1], q.cpu()):
        with pytest.raises(ValueError):
            mw.mw_packed_attn_fwd(bad, q, q, pack)
        with pytest.raises(ValueError):
            mw.mw_packed_attn_fwd(q, q, bad, pack)
    with pytest.raises(ValueError):
        mw.mw_packed_attn_fwd(q, q, q, pack, lse=torch.empty((T, H), device="cuda"))
    o, lse = mw.mw_packed_attn_fwd(q, q, q, pack)
    with pytest.raises(mw.MWError):
        mw.mw_packed_attn_bwd(q, q, q, o, q, lse, pack)  # planned without the backward
    with pytest.raises(ValueError):
        mw.Packed(edges([T]).long(), T, H, H, D)
    with pytest.raises(ValueError):
        mw.Packed(edges([T]), T, H, H, D, cu_k=edges([T, 0]))
    with pytest.raises(mw.MWError):
        mw.Packed(edges([T]), T, 3, 2, D)
    with pytest.raises(mw.MWError):
        mw.Packed(edges([T]), T, H, H, 96)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("scale", [8.0, 1e-4])
@pytest.mark.parametrize("nk,nq,chunk", [([300, 40], None, 1), ([700, 200], [90, 200], 50)])
def test_gradients_at_large_and_small_scales(mw, D, scale, nk, nq, chunk):
    """LSE of some hundreds, and of nearly equal scores.  Beside the roundings that attention64 counts, a probability is off by
    those of its score and of the LSE in 32 bits: the score's sum 2^-22 of its products' magnitudes, LSE and LSE log2 e half a step
    each and their difference with the score one (together 2^-22 of |LSE| and the magnitudes), and the LSE's own error, in
    which the scores' come again."""
    import torch
    H, Hkv = 4, 2
    nq_ = nk if nq is None else nq
    Tq, Tk, G = sum(nq_), sum(nk), H // Hkv
    q, do = randn((Tq, H, D), 1), randn((Tq, H, D), 2)
    k, v = randn((Tk, Hkv, D), 3), randn((Tk, Hkv, D), 4)
    pack = mw.Packed(edges(nq_), Tq, H, Hkv, D, chunk_len=chunk, cu_k=edges(nk), total_k=Tk, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack, scale=scale)
    got = dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack, scale=scale))))
    torch.cuda.synchronize()
    q0 = k0 = 0
    for s, (a, b) in enumerate(zip(nq_, nk)):
        i, j = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        hidden = hidden_of(a, b, chunk).repeat(G, 1)
        for hk in range(Hkv):
            h = slice(hk * G, (hk + 1) * G)
            rows = lambda t: t[i, h].transpose(0, 1).reshape(G * a, -1).double()
            x, y, g, c = rows(q), rows(do), k[j, hk].double(), v[j, hk].double()
            want = attention64(x, g, c, hidden, scale, y)
            p = torch.exp(((x @ g.t()) * scale).masked_fill(hidden, -math.inf) - want["lse"][0][:, None])
            size = scale * (x.abs() @ g.abs().t())
            off = p * 2.0 ** -21 * (size + size.masked_fill(hidden, 0).amax(-1, keepdim=True) + want["lse"][0].abs()[:, None])
            off_o = off @ c.abs()
            off_ds = off * ((y @ c.t()) - (y * want["o"][0]).sum(-1, keepdim=True)).abs() + p * (y.abs() * off_o).sum(-1, keepdim=True)
            more = {"o": off_o, "lse": torch.zeros_like(want["lse"][1]), "dq": scale * off_ds @ g.abs(),
                    "dk": scale * off_ds.t() @ x.abs(), "dv": off.t() @ y.abs()}
            for name, (value, bound) in want.items():
                z = got[name]
                z = z[j, hk] if name in ("dk", "dv") else z[h, i].reshape(-1) if name == "lse" else rows(z)
                check(f"{name} s={s} hk={hk}", z, value, bound + more[name])


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,lens,nq", [(257, [40, 3], None), (4096, [9], None), (16384, [70, 2], [3, 2])])
def test_many_heads_of_a_key_head(mw, D, H, lens, nq):
    """Tiles and steps that hold a part of one token's heads."""
    verify(mw, lens, H, 1, D, nq=nq, seed=H)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv", [(16384, 16384), (16383, 5461)])
def test_many_key_heads(mw, D, H, Hkv):
    """More key heads than places for workgroups; some of them against 64-bit values."""
    import torch
    lens, T, G = [1, 0, 66, 5], 72, H // Hkv
    q, do = randn((T, H, D), 1), randn((T, H, D), 2)
    k, v = randn((T, Hkv, D), 3), randn((T, Hkv, D), 4)
    pack = mw.Packed(edges(lens), T, H, Hkv, D, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    dq, dk, dv = mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)
    torch.cuda.synchronize()
    at = 0
    for n in lens:
        i = slice(at, at + n)
        at += n
        for hk in (0, 1, Hkv // 2, Hkv - 2, Hkv - 1) if n else ():
            h = slice(hk * G, (hk + 1) * G)
            rows = lambda t: t[i, h].transpose(0, 1).reshape(G * n, -1)
            want = attention64(rows(q), k[i, hk], v[i, hk], hidden_of(n, n, 1).repeat(G, 1), D ** -0.5, rows(do))
            got = dict(o=rows(o), lse=lse[h, i].reshape(-1), dq=rows(dq), dk=dk[i, hk], dv=dv[i, hk])
            for name, (value, bound) in want.items():
                check(f"{name} n={n} hk={hk}", got[name], value, bound)


def test_as_many_sequences_as_there_may_be(mw):
    """2^16 of them, one token or none each, but for a few: every row's output is that of its own keys."""
    import torch
    N, H, D = 1 << 16, 2, 64
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 2, (N,), generator=g)
    lens[[0, 1000, 65535]] = torch.tensor([3, 300, 129])
    T = int(lens.sum())
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(torch.int32).cuda()
    q, k, v, do = (randn((T, H, D), 30 + i) for i in range(4))
    pack = mw.Packed(cu, T, H, H, D, backward=True)
    o, lse = mw.mw_packed_attn_fwd(q, k, v, pack)
    dq, dk, dv = mw.mw_packed_attn_bwd(q, k, v, o, do, lse, pack)
    torch.cuda.synchronize()
    one = torch.repeat_interleave(lens, lens).cuda() == 1
    assert torch.equal(o[one], v[one]) and torch.equal(dv[one], do[one])
    s = (q.double() * k.double()).sum(-1) / 8
    assert bool(((lse.t().double() - s).abs()[one] <= 2.0 ** -20 * (1 + s.abs() + (q.double() * k.double()).abs().sum(-1) / 8)[one]).all())
    # (dP - Delta is rounding: sums of 64 products in 32 bits, in two orders)
    size = (do.double().abs() * v.double().abs()).sum(-1, keepdim=True) * 2.0 ** -18
    assert bool((dq.double().abs() <= size * k.double().abs())[one].all()) and bool((dk.double().abs() <= size * q.double().abs())[one].all())
    for s in (0, 1000, 65535):
        i = slice(int(cu[s]), int(cu[s + 1]))
        n = i.stop - i.start
        for h in range(H):
            want = attention64(q[i, h], k[i, h], v[i, h], hidden_of(n, n, 1), 0.125, do[i, h])
            for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
                check(f"{name} s={s} h={h}", t[i, h], *want[name])
