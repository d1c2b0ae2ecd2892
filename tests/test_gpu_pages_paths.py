"""Paths of the paged attention and of the append that only large calls take: row tiles of 128 rows whole and in
ranges, key ranges beyond one lookup of 256 blocks, more members than a wave has lanes, and appends in several
launches.  Values and bounds as in test_gpu_pages.py."""
import ctypes
import math

import pytest

import paper_2608_01127_amd as mw_lib
from attention_bounds import attention64, check
from test_gpu_pages import attend, filled, make, put, randn

# (members' lengths, key heads, query heads, queued chunks, q_len, tokens of a page) and the plan of the call with a
# workspace: rows of a tile, key ranges
WHOLE = ([200, 77], 3, 24, 3, 500, 64)
CUT = ([300, 0, 129], 3, 6, 2, 900, 128)
PLANS = [(64, WHOLE, 128, False), (72, WHOLE, 128, False), (128, WHOLE, 128, False),
         (64, CUT, 128, True), (72, CUT, 128, True), (128, CUT, 128, True)]


class Plan(ctypes.Structure):  # mw::RowsPlan
    _fields_ = [("bm", ctypes.c_int), ("n_splits", ctypes.c_int), ("chunk", ctypes.c_int)]


def rows_plan(D, shape, ws):
    lens, Hkv, H, nq, ql, _ = shape
    fn = mw_lib.load()["_ZN2mw9rows_planEibiixm"]  # mw::rows_plan(int, bool, int, int, long long, size_t)
    fn.restype = Plan
    fn.argtypes = [ctypes.c_int, ctypes.c_bool, ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t]
    return fn(D, True, len(lens) * Hkv, nq * ql * (H // Hkv), max(lens) + nq * ql, ws)


@pytest.mark.parametrize("D,shape,bm,cut", PLANS)
def test_the_shapes_below_take_the_tiles_they_are_for(D, shape, bm, cut):
    plan = rows_plan(D, shape, 1 << 62)
    assert (plan.bm, plan.n_splits > 1) == (bm, cut)


@pytest.mark.gpu
@pytest.mark.parametrize("D,shape,bm,cut", PLANS)
@pytest.mark.parametrize("flags", [0, 1])
def test_large_row_tiles(mw, D, shape, bm, cut, flags):
    lens, Hkv, H, nq, ql, L = shape
    cache, model = filled(mw, Hkv, L, D, lens, seed=D + flags)
    need = mw.mw_chunk_attn_paged_workspace_size(cache, list(range(len(lens))), H, nq, ql)
    assert (need > 0) == cut
    attend(mw, cache, model, list(range(len(lens))), nq, ql, H, flags, seed=D, layout="bthd" if flags else "bhtd")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("nq,ql,H,flags", [(1, 65, 2, 0), (3, 40, 4, 1)])
def test_many_rows_without_a_workspace(mw, D, nq, ql, H, flags):
    """The direct stores of O and LSE, where a workspace would cut the keys into ranges."""
    cache, model = filled(mw, 2, 64, D, [1000, 0, 191], seed=D)
    assert mw.mw_chunk_attn_paged_workspace_size(cache, [0, 1, 2], H, nq, ql) > 0
    attend(mw, cache, model, [0, 1, 2], nq, ql, H, flags, seed=nq, split=False)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("ql", [1, 20])
def test_one_range_of_more_blocks_than_one_lookup(mw, D, ql):
    """33000 and 16484 tokens are 516 and 258 blocks of one workgroup, which looks 256 up at a time; 20 tokens of two
    heads are 40 rows, two row blocks."""
    lens = [33000, 16484, 3, 16384]
    cache, model = make(mw, 520 + 260 + 260 + 4, 1, 64, D, 4, 520)
    for s, n in enumerate(lens):
        put(mw, cache, model, [s], n, 100 * s, make_tokens=randn)
    attend(mw, cache, model, [0, 1, 2, 3], 1, ql, 2, 0, seed=D, split=False)
    attend(mw, cache, model, [1, 0], 1, ql, 2, 0, seed=D + 1, queued=False, split=False)


@pytest.mark.gpu
@pytest.mark.parametrize("B", [64, 65, 130, 256])
@pytest.mark.parametrize("D,ql,H", [(64, 1, 1), (72, 33, 1), (128, 2, 4), (64, 70, 1)])
def test_as_many_members_as_a_call_may_name(mw, B, D, ql, H):
    """Ragged members, every seventh empty, each sequence named several times; 70 rows a member go to the row tiles."""
    cache, model = filled(mw, 1, 64, D, [(0 if i % 7 == 3 else 1 + 53 * i) for i in range(19)], seed=B)
    seqs = [(5 * b + b // 19) % 19 for b in range(B)]
    attend(mw, cache, model, seqs, 1, ql, H, 0, seed=B)
    attend(mw, cache, model, seqs[::-1], 1, ql, H, 0, seed=B + 1, split=False, layout="bthd")


def pages_plan(D, R, blocks, Hkv, ws=1 << 62):
    fn = mw_lib.load()["_ZN2mw10pages_planEiiPKiiim"]  # mw::pages_plan(int, int, const int*, int, int, size_t)
    fn.restype = Plan
    fn.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.c_int, ctypes.c_int, ctypes.c_size_t]
    return fn(D, R, (ctypes.c_int * len(blocks))(*blocks), len(blocks), Hkv, ws)


@pytest.mark.parametrize("n", [32, 63, 64, 65, 128, 256])
@pytest.mark.parametrize("D,R", [(64, 1), (72, 4), (128, 1)])
def test_one_long_member_is_cut_however_many_short_ones_there_are(n, D, R):
    plan = pages_plan(D, R, [2] * (n // 2) + [248] + [2] * (n - n // 2 - 1), 16)
    assert plan.n_splits >= 4 and plan.n_splits == -(-248 // plan.chunk)
    assert pages_plan(D, R, [2] * (n - 1) + [248], 16, 0).n_splits == 1  # without a workspace


@pytest.mark.parametrize("n", [64, 128, 256])
def test_members_of_one_length_that_fill_the_card_are_not_cut(n):
    for blocks in (1, 3, 4, 100, 248):
        assert pages_plan(128, 1, [blocks] * n, 16).n_splits == 1
    assert pages_plan(128, 1, [0] * n, 16).n_splits == 1


@pytest.mark.parametrize("blocks", [[250000] + [1] * 255, [250000] * 2, [5], [0, 0], [4, 1]])
@pytest.mark.parametrize("Hkv,R", [(1, 64), (16, 64), (3, 1)])
def test_partials_of_long_members_stay_within_a_gibibyte(blocks, Hkv, R):
    plan = pages_plan(128, R, blocks, Hkv)
    assert 1 <= plan.chunk and plan.n_splits == max(1, -(-max(blocks) // plan.chunk))
    assert plan.n_splits == 1 or plan.n_splits * len(blocks) * Hkv * R * 130 * 4 <= 1 << 30


def test_a_workspace_of_the_size_asked_for_gets_the_plan_it_was_asked_for():
    import random
    rng = random.Random(1)
    for _ in range(400):
        D, R, Hkv = rng.choice([64, 72, 128]), rng.choice([1, 5, 32, 64]), rng.choice([1, 3, 16])
        top = int(2 ** rng.uniform(0, 18))
        blocks = [rng.choice([top, rng.randint(0, top), 1]) for _ in range(int(2 ** rng.uniform(0, 8)))]
        free = pages_plan(D, R, blocks, Hkv)
        exact = free.n_splits * len(blocks) * Hkv * R * (D + 2) * 4 if free.n_splits > 1 else 0
        for ws in (exact, exact + 100):
            plan = pages_plan(D, R, blocks, Hkv, ws)
            assert (plan.n_splits, plan.chunk) == (free.n_splits, free.chunk), (D, R, Hkv, blocks)
        less = pages_plan(D, R, blocks, Hkv, exact // 2)
        assert less.n_splits == 1 or less.n_splits * len(blocks) * Hkv * R * (D + 2) * 4 <= exact // 2


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("ql,flags", [(1, 0), (1, 1), (3, 0), (3, 1)])
def test_as_many_queued_chunks_as_a_call_may_have(mw, D, ql, flags):
    cache, model = filled(mw, 1, 64, D, [90, 0, 64], seed=D)
    attend(mw, cache, model, [0, 1, 2], 64, ql, 1, flags, seed=ql)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("rows", [1, 40, 100])
def test_a_smaller_workspace_gives_fewer_ranges(mw, D, rows):
    """Down to one byte less than two ranges take; the results stay within their bounds, and what lies behind the
    workspace is left as it was."""
    import torch
    n = 5000
    cache, model = filled(mw, 1, 64, D, [n], seed=D)
    q = randn((1, 1, rows, D), 1)
    k, v = (t[None] for t in model.values(0))
    kb, vb = k.bfloat16(), v.bfloat16()  # exact: codes times powers of two
    none = torch.zeros((1, 1), dtype=torch.bool, device="cuda")
    want = attention64(q[0, 0], k[0, 0], v[0, 0], none, 1 / math.sqrt(D))
    one = rows * (D + 2) * 4  # bytes of one range
    for need, call in ((mw.mw_chunk_attn_paged_workspace_size(cache, [0], 1, 1, rows),
                        lambda ws, lse: mw.mw_chunk_attn_paged(q, None, None, 1, rows, cache, [0], lse=lse, workspace=ws)[0]),
                       (mw.mw_cross_attn_workspace_size(1, 1, 1, rows, n, D),
                        lambda ws, lse: mw.mw_cross_attn_fwd(q, kb, vb, lse=lse, workspace=ws)[0])):
        assert need >= 4 * one and need % one == 0
        for size in (need, need - 1, need // 2, 2 * one, 2 * one - 1):
            buf = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
            lse = torch.empty((1, 1, rows), device="cuda")
            o = call(buf[:size], lse)
            check(f"o with {size} of {need} bytes", o[0, 0], *want["o"])
            check(f"lse with {size} of {need} bytes", lse[0, 0], *want["lse"])
            assert bool((buf[size:] == 0xA5).all())


@pytest.mark.gpu
@pytest.mark.parametrize("D,ql,Hkv", [(64, 1, 16), (72, 8, 16), (128, 33, 16)])
def test_one_long_member_among_many_short_ones(mw, D, ql, Hkv):
    cache, model = filled(mw, Hkv, 64, D, [7000, 70, 0, 130], seed=D)
    seqs = [1, 2, 3] * 10 + [0] + [3, 1, 2] * 11
    assert mw.mw_chunk_attn_paged_workspace_size(cache, seqs, Hkv, 1, ql) > 0
    attend(mw, cache, model, seqs, 1, ql, Hkv, 0, seed=D)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [32, 33, 70])
@pytest.mark.parametrize("D", [64, 72])
def test_appends_to_more_sequences_than_one_launch_names(mw, n, D):
    """All fork from one partly filled page, which each copies on write, in one launch or another; then pages enough
    for several launches, so that a sequence's tokens are cut between two."""
    L = 128
    cache, model = make(mw, 22 * n + 40, 2, L, D, n + 1, 24)
    put(mw, cache, model, [0], 200, 1)
    for s in range(1, n + 1):
        mw.mw_kvpages_fork(cache, 0, s)
        model.rows[s], model.lens[s] = list(model.rows[0]), model.lens[0]
    put(mw, cache, model, list(range(n, 0, -1)), 30, 2)
    model.verify()
    put(mw, cache, model, list(range(1, n + 1)), 17 * L + 5, 3, layout="bthd")
    model.verify()


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72, 128])
def test_replays_over_a_changing_cache_against_the_codes(mw, D):
    """A captured attention, replayed while sequences grow, roll, empty, branch and move: O and LSE of each replay
    against 64-bit values of what the cache then holds, in the bounds of an eager call.  (Averages of 1000 tokens
    are of the size of 0.04: an absolute bar of a few hundredths would not see a page of wrong values.)"""
    import torch
    H, L, ql = 2, 64, 8
    cache, model = filled(mw, H, L, D, [1500, 700, 0], seed=D, W=60)
    q, k, v = (randn((2, h, ql, D), 20 + i) for i, h in enumerate((2 * H, H, H)))
    o, lse = torch.empty_like(q), torch.empty((2, 2 * H, ql), device="cuda")
    ws = torch.empty(mw.mw_chunk_attn_paged_workspace_size(cache, [0, 1], 2 * H, 1, ql), dtype=torch.uint8, device="cuda")
    call = lambda: mw.mw_chunk_attn_paged(q, k, v, 1, ql, cache, [0, 1], out=o, lse=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()

    def append(s, n, seed):
        put(mw, cache, model, [s], n, seed, make_tokens=randn)

    def evict(s, first, n):
        mw.mw_kvpages_evict(cache, s, first, n)
        del model.rows[s][first:first + n]
        model.lens[s] -= n * L

    def free(s):
        mw.mw_kvpages_free(cache, [s])
        model.drop([s])

    def fork(s, d):
        mw.mw_kvpages_fork(cache, s, d)
        model.rows[d], model.lens[d] = list(model.rows[s]), model.lens[s]

    def compact():
        live = sorted({p for r in model.rows for p in r})
        move = dict(zip([p for p in live if p >= len(live)], [p for p in range(len(live)) if p not in live]))
        assert mw.mw_kvpages_compact(cache) == len(move) > 0
        for src, dst in move.items():
            for x in range(2):
                model.code[x][dst] = model.code[x][src]
                model.exp[x][dst] = model.exp[x][src]
        model.rows = [[move.get(p, p) for p in r] for r in model.rows]

    steps = [("as captured", lambda: None), ("grown", lambda: append(0, 130, 50)), ("rolled", lambda: evict(0, 1, 9)),
             ("emptied", lambda: free(1)), ("branched", lambda: fork(0, 1)), ("written", lambda: append(1, 3, 60)),
             ("moved", compact), ("longer than captured", lambda: append(1, 900, 70))]
    none = torch.zeros((2 * ql, 1), dtype=torch.bool, device="cuda")
    for name, step in steps:
        step()
        o.fill_(5.0)
        lse.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        print(f"[step] {name}: {model.lens}", flush=True)
        for b in range(2):
            K, V = model.values(b)
            for hk in range(H):
                rows = lambda t: t[b, 2 * hk:2 * hk + 2].reshape(2 * ql, -1)
                want = attention64(rows(q), torch.cat([K[hk], k[b, hk].double()]), torch.cat([V[hk], v[b, hk].double()]),
                                   none, 1 / math.sqrt(D))
                check(f"o {name} b={b} hk={hk}", rows(o), *want["o"])
                check(f"lse {name} b={b} hk={hk}", rows(lse).squeeze(-1), *want["lse"])
