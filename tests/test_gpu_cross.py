"""Cross attention forward and backward against 64-bit values, at the sizes, strides, lengths and shared heads
where it can go wrong."""
import math

import pytest

from attention_bounds import attention64, check

pytestmark = pytest.mark.gpu


def randn(shape, seed, layout="bhtd"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, T, D = shape
    if layout == "bhtd":
        return torch.randn(B, H, T, D, device="cuda", generator=g).bfloat16()
    if layout == "bthd":
        return torch.randn(B, T, H, D, device="cuda", generator=g).bfloat16().transpose(1, 2)
    wide = torch.randn(B, T, H, D + 8, device="cuda", generator=g).bfloat16()  # rows with a gap behind them
    return wide[..., :D].transpose(1, 2)


def verify(mw, B, H, Hkv, T, M, D, lens=None, layout="bhtd", backward=True, scale=None, seed=1, garbage=None):
    import torch
    print(f"[case] cross B={B} H={H} Hkv={Hkv} T={T} M={M} D={D} lens={lens} {layout}", flush=True)
    q, do = randn((B, H, T, D), seed, layout), randn((B, H, T, D), seed + 1, layout)
    k, v = randn((B, Hkv, M, D), seed + 2, layout), randn((B, Hkv, M, D), seed + 3, layout)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    n = [M] * B if lens is None else [min(max(x, 0), M) for x in lens]
    if garbage is not None:
        for b in range(B):
            k[b, :, n[b]:] = garbage
            v[b, :, n[b]:] = garbage
    o, lse = mw.mw_cross_attn_fwd(q, k, v, kv_len=kv_len, scale=scale)
    got = {"o": o, "lse": lse}
    if backward:
        got["dq"], got["dk"], got["dv"] = mw.mw_cross_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len, scale=scale)
    torch.cuda.synchronize()
    sc = 1 / math.sqrt(D) if scale is None else scale
    G = H // Hkv
    none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
    for b in range(B):
        for hk in range(Hkv):
            rows = lambda t: t[b, hk * G:(hk + 1) * G].reshape(G * T, -1)
            want = attention64(rows(q), k[b, hk, :n[b]], v[b, hk, :n[b]], none, sc, rows(do) if backward else None)
            for name, (value, bound) in want.items():
                if name in ("dk", "dv"):
                    x = got[name][b, hk]
                    assert not bool(x[n[b]:].any()), f"{name} of padding states"
                    check(f"{name} b={b} hk={hk}", x[:n[b]], value, bound)
                else:
                    x = got[name][b, hk * G:(hk + 1) * G].reshape(G * T, -1)
                    check(f"{name} b={b} hk={hk}", x.squeeze(-1) if name == "lse" else x, value, bound)
    return got


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("T,M", [(1, 1), (1, 77), (2, 63), (31, 64), (33, 65), (64, 127), (65, 129), (130, 200), (257, 1)])
def test_small_and_odd_lengths(mw, D, T, M):
    verify(mw, 1, 2, 2, T, M, D, seed=10 * T + M)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("H,Hkv", [(3, 1), (4, 2), (8, 1), (6, 2)])
@pytest.mark.parametrize("T,M", [(1, 50), (40, 96), (111, 130)])
def test_shared_heads(mw, D, H, Hkv, T, M):
    verify(mw, 2, H, Hkv, T, M, D, lens=[M, M // 2], layout="bthd", seed=H + T)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_padded_batches_never_read_their_padding(mw, D):
    """Lengths of zero, one, a tile's edge and the whole, also given as negative or beyond M; the padding is NaN."""
    verify(mw, 6, 2, 2, 70, 200, D, lens=[0, 1, 64, 128, 999, -3], garbage=float("nan"), seed=3)
    verify(mw, 2, 4, 2, 70, 200, D, lens=[65, 199], garbage=float("inf"), layout="gap", seed=4)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_long_states_few_rows_are_split(mw, D):
    need = mw.mw_cross_attn_workspace_size(1, 4, 2, 5, 6001, D)
    assert need > 0
    verify(mw, 1, 4, 2, 5, 6001, D, lens=[5990], seed=5)
    verify(mw, 2, 2, 2, 100, 3001, D, lens=[2999, 7], seed=6)  # one member's ranges are mostly empty


@pytest.mark.parametrize("D", [64, 72, 128])
def test_many_rows_are_cut_into_slices(mw, D):
    verify(mw, 1, 2, 1, 2111, 150, D, lens=[141], layout="bthd", seed=7)
    verify(mw, 2, 2, 2, 1500, 33, D, lens=[33, 0], seed=8)


def test_large_scores_and_scales(mw):
    """Scores that differ by far more than the exponential's range, raised late in the walk, and tiny ones."""
    import torch
    for scale in (8.0, 1e-4):
        verify(mw, 1, 2, 2, 70, 300, 128, scale=scale, backward=False, seed=9)
    q, k, v = randn((1, 1, 64, 64), 20), randn((1, 1, 256, 64), 21), randn((1, 1, 256, 64), 22)
    k[:, :, 255] = q[:, :, 5:6].squeeze(2) * 30  # the last key outweighs all before it
    o, lse = mw.mw_cross_attn_fwd(q, k, v)
    none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
    for name, (value, bound) in attention64(q[0, 0], k[0, 0], v[0, 0], none, 0.125).items():
        check(name, (o if name == "o" else lse)[0, 0], value, bound)


def test_a_visible_nan_is_not_hidden(mw):
    import torch
    q, k, v = randn((2, 1, 5, 64), 30), randn((2, 1, 70, 64), 31), randn((2, 1, 70, 64), 32)
    v[0, 0, 3, 7] = float("nan")
    o, lse = mw.mw_cross_attn_fwd(q, k, v)
    assert bool(o[0, 0, :, 7].isnan().all()) and bool(o[1].isfinite().all()) and bool(lse.isfinite().all())


def test_states_shared_between_batch_members_and_heads(mw):
    """Broadcast k and v (strides of 0) read as their expanded copies; each member's gradient is its own."""
    import torch
    B, H, T, M, D = 3, 2, 50, 90, 64
    q, do = randn((B, H, T, D), 40), randn((B, H, T, D), 41)
    k1, v1 = randn((1, 1, M, D), 42), randn((1, 1, M, D), 43)
    k, v = k1.expand(B, H, M, D), v1.expand(B, H, M, D)
    o, lse = mw.mw_cross_attn_fwd(q, k, v)
    g = mw.mw_cross_attn_bwd(q, k, v, o, do, lse)
    oc, lc = mw.mw_cross_attn_fwd(q, k.contiguous(), v.contiguous())
    gc = mw.mw_cross_attn_bwd(q, k.contiguous(), v.contiguous(), oc, do, lc)
    torch.cuda.synchronize()
    assert torch.equal(o, oc) and torch.equal(lse, lc)
    for a, b in zip(g, gc):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_strided_results_equal_contiguous_ones_and_repeat(mw, D):
    import torch
    B, H, Hkv, T, M = 2, 4, 2, 300, 170
    kv_len = torch.tensor([170, 81], dtype=torch.int32, device="cuda")
    t = [randn((B, H, T, D), 50, "bthd"), randn((B, Hkv, M, D), 51, "gap"), randn((B, Hkv, M, D), 52, "bthd"),
         randn((B, H, T, D), 53, "gap")]
    runs = []
    for x in (t, [y.contiguous() for y in t], t):
        q, k, v, do = x
        o = torch.empty_like(t[0])
        lse = torch.empty((B, H, T), device="cuda")
        mw.mw_cross_attn_fwd(q, k, v, kv_len=kv_len, out=o, lse=lse)
        runs.append((o.contiguous(), lse, *mw.mw_cross_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len)))
    torch.cuda.synchronize()
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


def test_outputs_stay_within_their_views(mw):
    """A gap behind each row of o, dq, dk and dv is left as it was."""
    import torch
    B, H, T, M, D = 1, 2, 37, 45, 72
    q, k, v, do = (randn((B, H, n, D), 60 + i) for i, n in enumerate((T, M, M, T)))
    mark = lambda n: torch.full((B, H, n + 3, D + 8), 7.0, device="cuda", dtype=torch.bfloat16)
    o, dq, dk, dv = mark(T), mark(T), mark(M), mark(M)
    cut = lambda x, n: x[:, :, :n, :D]
    _, lse = mw.mw_cross_attn_fwd(q, k, v, out=cut(o, T))
    mw.mw_cross_attn_bwd(q, k, v, cut(o, T), do, lse, dq=cut(dq, T), dk=cut(dk, M), dv=cut(dv, M))
    torch.cuda.synchronize()
    for x, n in ((o, T), (dq, T), (dk, M), (dv, M)):
        assert bool((x[..., D:] == 7).all()) and bool((x[:, :, n:] == 7).all()) and not bool((cut(x, n) == 7).all())


def test_gradient_against_differences(mw):
    """The loss sum(dO * O) along random directions: the gradients' inner products with them against central
    differences of the 64-bit forward."""
    import torch
    B, H, Hkv, T, M, D = 1, 2, 1, 20, 30, 64
    q, k, v, do = (randn((B, h, n, D), 70 + i) for i, (h, n) in enumerate(((H, T), (Hkv, M), (Hkv, M), (H, T))))
    o, lse = mw.mw_cross_attn_fwd(q, k, v)
    grads = mw.mw_cross_attn_bwd(q, k, v, o, do, lse)

    def loss(q, k, v):
        s = torch.matmul(q, k.expand(B, H, M, D).transpose(-1, -2).contiguous()) / 8.0
        return float((torch.softmax(s, -1) @ v.expand(B, H, M, D).contiguous() * do.double()).sum())

    x = [t.double() for t in (q, k, v)]
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


def test_side_stream_and_graph_replays(mw):
    """A captured forward and backward, replayed over new inputs with eager work between, equals eager calls; two
    graphs that share a workspace, replayed in turn, too."""
    import torch
    B, H, Hkv, T, M, D = 2, 4, 2, 600, 130, 64
    q, do = (torch.empty((B, H, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.empty((B, Hkv, M, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    outs = [[torch.empty_like(q), torch.empty((B, H, T), device="cuda"), torch.empty_like(q), torch.empty_like(k),
             torch.empty_like(v)] for _ in range(2)]
    ws = torch.empty(max(16, mw.mw_cross_attn_workspace_size(B, H, Hkv, T, M, D)), dtype=torch.uint8, device="cuda")
    ws_b = torch.empty(mw.mw_cross_attn_bwd_workspace_size(B, H, Hkv, T, M, D), dtype=torch.uint8, device="cuda")

    def load(seed):
        for i, t in enumerate((q, do, k, v)):
            t.copy_(randn(tuple(t.shape), seed + i))
        kv_len.copy_(torch.tensor([M - seed % 50, seed % M], dtype=torch.int32))

    def step(x):
        mw.mw_cross_attn_fwd(q, k, v, kv_len=kv_len, out=x[0], lse=x[1], workspace=ws)
        mw.mw_cross_attn_bwd(q, k, v, x[0], do, x[1], kv_len=kv_len, workspace=ws_b, dq=x[2], dk=x[3], dv=x[4])

    load(100)
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
    for seed in (200, 300, 400):
        load(seed)
        for t in (t for x in outs for t in x):
            t.fill_(9.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        eager = [torch.empty_like(t) for t in outs[0]]
        step(eager)
        torch.cuda.synchronize()
        for x in outs:
            for a, b in zip(x, eager):
                assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("M,lens", [(2, None), (5, None), (40, None), (64, None), (1000, [2, 900]), (1000, [64, 7])])
def test_gradients_of_few_states_keep_their_precision(mw, D, M, lens):
    """Next to a few states' dP - Delta the rounding of O to bf16 would not be small, so Delta must not come from it.
    What is left is the rounding of dS and that of the gradient itself: relative errors of at most 2^-8 each, spread
    over their interval, so 2^-8 / sqrt(3) in the mean square at most and sqrt(2) of that together, for sums of
    independent terms (random inputs) too."""
    import torch
    B, H, T = 2, 3, 700
    n = lens or [M, M]
    q, do = randn((B, H, T, D), 1), randn((B, H, T, D), 2)
    k, v = randn((B, H, M, D), 3), randn((B, H, M, D), 4)
    kv_len = torch.tensor(n, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_cross_attn_fwd(q, k, v, kv_len=kv_len)
    got = dict(zip(("dq", "dk", "dv"), mw.mw_cross_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len)))
    for b in range(B):
        q64, k64, v64, d64 = (x[b].double().cpu() for x in (q, k[:, :, :n[b]], v[:, :, :n[b]], do))
        kt, vt = k64.transpose(1, 2).contiguous(), v64.transpose(1, 2).contiguous()
        P = torch.softmax(q64 @ kt / math.sqrt(D), -1)
        dP = d64 @ vt
        dS = P * (dP - (P * dP).sum(-1, keepdim=True)) / math.sqrt(D)
        want = dict(dq=dS @ k64, dk=dS.transpose(1, 2).contiguous() @ q64, dv=P.transpose(1, 2).contiguous() @ d64)
        for name, w in want.items():
            g = got[name][b].double().cpu()
            g = g if name == "dq" else g[:, :n[b]]
            assert (g - w).norm() <= 2.0 ** -8 * math.sqrt(2 / 3) * w.norm(), (name, b, ((g - w).norm() / w.norm()).item())


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("M,lens", [(300, [290, 41]), (64, [64, 64])])
def test_rows_that_fill_the_card(mw, D, M, lens):
    """Several rounds of the largest row tiles, whole key steps and partly filled ones, members of unlike lengths."""
    verify(mw, 2, 6, 3, 9001, M, D, lens=lens, layout="bthd", seed=40 + M)
