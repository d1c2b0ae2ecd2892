"""Cross attention, attention over a paged 8-bit cache and the cache's page operations, as passes
that a timing program can prepare, run and check.

Kinds of pass:

  cross   serving: the forward of one cross attention layer, video tokens over an encoder's states;
  train   its forward and backward;
  paged   cached attention over pages of e4m3 keys and values with a scale for each 64 tokens and
          head, the queued tokens' own keys beside it;
  branch  a rollout's history forked into several branches, each of which commits its next tokens
          (quantised; the shared last page is copied on write);
  select  one of two rollouts dropped, the pool compacted, and the kept one copied whole.

With `own` false, run() computes the same in elementary torch operations in 32 bits.  exact() is
the definition in 64 bits.  Widths, head counts, chunk and window sizes are those of this repository's
configurations and tests (1B: 12 heads of 128; 0.5B: 16 of 72; chunks of 600, 1320 and 2640 tokens).
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 64  # tokens that share a scale


def listed():
    return [
        # a single new token's rows over a short prompt, guidance pair with an empty (dropped) condition:
        # the launch is what counts
        dict(name="cross_one", kind="cross", B=2, H=12, Hkv=12, T=1, M=77, D=64, lens="empty", layout="bthd"),
        # a rollout step of the 1B model: 8 in-flight chunks over 512 padded states, guidance pair
        dict(name="cross_stream_1b", kind="cross", B=2, H=12, Hkv=12, T=4800, M=512, D=128, lens="ragged", layout="bthd"),
        # few rows over the long states of a past video, four query heads to a key head
        dict(name="cross_long", kind="cross", B=1, H=16, Hkv=4, T=64, M=15840, D=128, lens="full", layout="bhtd"),
        # odd everything: the 0.5B head width, a ragged batch with an empty member, a prompt of 77 states
        dict(name="train_odd_d72", kind="train", B=3, H=5, Hkv=5, T=2999, M=77, D=72, lens="empty", layout="bhtd"),
        # shared key heads at head width 64: one chunk of 1320 tokens conditioned on another
        dict(name="train_shared_d64", kind="train", B=2, H=12, Hkv=4, T=1320, M=1320, D=64, lens="ragged", layout="bthd"),
        # the 1B model's training window over 512 states
        dict(name="train_1b", kind="train", B=1, H=12, Hkv=12, T=19200, M=512, D=128, lens="full", layout="bthd"),
        # one token of eight ragged sequences, four query heads to a key head: bound by reading the cache
        dict(name="paged_one", kind="paged", B=8, H=16, Hkv=4, D=128, len=15840, L=128, nq=1, ql=1, mode=0, layout="bthd"),
        # 64 queued tokens over a full 6 x 2640-token window
        dict(name="paged_64", kind="paged", B=1, H=16, Hkv=16, D=128, len=15840, L=64, nq=1, ql=64, mode=0, layout="bhtd"),
        # the 0.5B width: odd lengths, three queued chunks, each seeing the history and itself
        dict(name="paged_odd_d72", kind="paged", B=3, H=16, Hkv=16, D=72, len=3601, L=192, nq=3, ql=333, mode=1, layout="bthd"),
        # a rollout step of the 1B model: guidance pair, 8 in-flight chunks, 24 cached chunks and the anchor
        dict(name="paged_stream_1b", kind="paged", B=2, H=12, Hkv=12, D=128, len=14700, L=64, nq=8, ql=600, mode=0, layout="bthd"),
        # four branches of a 1B rollout, one chunk each
        dict(name="branch_1b", kind="branch", H=12, D=128, len=3900, L=128, n=4, t=600, layout="bthd"),
        # best of two 1B rollouts of 24 chunks and the anchor
        dict(name="select_1b", kind="select", H=12, D=128, len=14700, L=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges; lengths are spread over their logarithm."""
    while True:
        kind = rng.choice(["cross", "train", "train", "paged", "paged", "branch", "select"])
        D = rng.choice([64, 72, 128])
        layout = rng.choice(["bhtd", "bthd"])
        Hkv = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
        H = Hkv * rng.choice([1, 1, 2, 4, 8])
        B = rng.choice([1, 2, 3, 8])
        if kind in ("cross", "train"):
            case = dict(kind=kind, B=B, H=H, Hkv=Hkv, T=_log_int(rng, 1, 20000), M=_log_int(rng, 1, 16000), D=D,
                        lens=rng.choice(["full", "ragged", "empty"]), layout=layout)
        elif kind == "paged":
            nq = rng.choice([1, 1, 3, 8])
            case = dict(kind=kind, B=B, H=H, Hkv=Hkv, D=D, len=_log_int(rng, 1, 16000), L=rng.choice([64, 128, 192, 640]),
                        nq=nq, ql=_log_int(rng, 1, 640), mode=rng.choice([0, 0, 1]), layout=layout)
        elif kind == "branch":
            case = dict(kind=kind, H=Hkv, D=D, len=_log_int(rng, 1, 16000), L=rng.choice([64, 128, 192, 640]),
                        n=rng.randint(1, 8), t=_log_int(rng, 1, 2640), layout=layout)
        else:
            case = dict(kind=kind, H=Hkv, D=D, len=_log_int(rng, 64, 16000), L=rng.choice([64, 128, 192, 640]))
        # the 1B stream and training passes are the largest; the plain scores of a case stay within 16 GB
        rows = case["H"] * case.get("B", 1) * (case.get("T") or case.get("nq", 0) * case.get("ql", 0))
        keys = case.get("M") or case.get("len", 0) + case.get("nq", 0) * case.get("ql", 0)
        if work(case)["flops"] <= (2e11 if kind == "train" else 6e11) and work(case)["bytes"] <= 5e8 and rows * keys <= 4e9:
            return case


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, B, H, T, D, layout="bhtd"):
    """bf16 N(0,1) activations as a [B,H,T,D] tensor, or such a view of a [B,T,H,D] one."""
    if layout == "bthd":
        return torch.randn(B, T, H, D, device=DEV, generator=g).to(torch.bfloat16).transpose(1, 2)
    return torch.randn(B, H, T, D, device=DEV, generator=g).to(torch.bfloat16)


def _kv_lens(case):
    """Valid states of each batch member: padded batches end at different places, a dropped condition at 0."""
    B, M = case["B"], case["M"]
    n = [M if case["lens"] == "full" else max(1, M - (b * M) // (2 * B)) for b in range(B)]
    if case["lens"] == "empty":
        n[-1] = 0
    return n


def _seq_lens(case):
    """Cached tokens of each sequence."""
    return [max(0, case["len"] - (b * case["len"]) // (2 * case["B"])) for b in range(case["B"])]


def _history(g, n, H, T, D, layout="bhtd"):
    """K and V of n sequences' tokens; the values' magnitude differs between heads and drifts over the tokens."""
    k, v = _randn(g, n, H, T, D, layout), _randn(g, n, H, T, D, layout)
    gain = torch.exp2(torch.rand(1, H, 1, 1, device=DEV, generator=g) * 2 - 1)
    drift = torch.exp2(torch.sin(torch.arange(T, device=DEV) / 300.0)).view(1, 1, T, 1)
    return k, (v.float() * gain * drift).to(torch.bfloat16)


def _inputs(case, seed):
    """Every random tensor of a case, from the seed alone (shared by prepare and exact)."""
    g, kind, D = _gen(seed), case["kind"], case["D"]
    if kind in ("cross", "train"):
        x = dict(q=_randn(g, case["B"], case["H"], case["T"], D, case["layout"]))
        x["k"], x["v"] = (_randn(g, case["B"], case["Hkv"], case["M"], D, case["layout"]) for _ in range(2))
        if kind == "train":
            x["do"] = _randn(g, case["B"], case["H"], case["T"], D, case["layout"])
        return x
    if kind == "paged":
        T = case["nq"] * case["ql"]
        x = dict(q=_randn(g, case["B"], case["H"], T, D, case["layout"]))
        x["k"], x["v"] = (_randn(g, case["B"], case["Hkv"], T, D, case["layout"]) for _ in range(2))
        x["hist"] = _history(g, case["B"], case["Hkv"], case["len"], D)
        return x
    if kind == "branch":
        x = dict(hist=_history(g, 1, case["H"], case["len"], D))
        x["k"], x["v"] = _history(g, case["n"], case["H"], case["t"], D, case["layout"])
        return x
    return dict(hist=_history(g, 2, case["H"], case["len"], D))


def _exponent(amax):
    """Least e with amax <= 448 * 2^e, within [-100, 100]."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax == 0, -100, e).clamp(-100, 100)


def _encode(x, e):
    """e4m3 codes of x (32 bits) at scale 2^e."""
    return torch.ldexp(x, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _paged(x, n, L):
    """[n,H,T,D] -> [n, pages, H, L, D] in 32 bits, zeros behind the last token."""
    b, H, T, D = x.shape
    W = -(-T // L)
    y = torch.zeros(b, H, W * L, D, device=DEV)
    y[:, :, :T] = x
    return y.view(b, H, W, L, D).transpose(1, 2)


def _quantise(x, lens, L):
    """Codes [n, pages, H, L, D] and exponents [n, pages, H, L / 64] of the first lens[i] tokens of each sequence."""
    T = x.shape[2]
    keep = torch.arange(T, device=DEV).view(1, 1, T, 1) < torch.tensor(lens, device=DEV).view(-1, 1, 1, 1)
    y = _paged(torch.where(keep, x.float(), 0.0), len(lens), L)
    n, W, H, _, D = y.shape
    e = _exponent(y.view(n, W, H, L // BLOCK, BLOCK * D).abs().amax(-1))
    return _encode(y, e.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1)), e


def _plain_pool(case, lens, hist, n_seqs, n_pages, W):
    """The pool as tensors: codes [P,H,L,D], scales [P,H,L/64], the page table and the lengths.  Pages are
    taken lowest first, sequence by sequence."""
    L = case["L"]
    s = {}
    table = torch.zeros(n_seqs, W, dtype=torch.int32, device=DEV)
    length = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
    used = [-(-n // L) for n in lens]
    at = 0
    for i, w in enumerate(used):
        table[i, :w] = torch.arange(at, at + w, device=DEV)
        length[i] = lens[i]
        at += w
    for name, x in zip("kv", hist):
        codes, e = _quantise(x, lens, L)
        pool = torch.zeros(n_pages, *codes.shape[2:], dtype=torch.float8_e4m3fn, device=DEV)
        scale = torch.zeros(n_pages, *e.shape[2:], device=DEV)
        for i, w in enumerate(used):
            p = table[i, :w].long()
            pool.view(torch.uint8)[p] = codes[i, :w].view(torch.uint8)
            # blocks that hold no token yet have no scale
            filled = torch.arange(w * L // BLOCK, device=DEV).view(w, 1, -1) < -(-lens[i] // BLOCK)
            scale[p] = torch.where(filled, torch.ldexp(torch.ones_like(scale[p]), e[i, :w]), 0.0)
        s[name + "_pages"], s[name + "_scales"] = pool, scale
    s["table"], s["lens"] = table, length
    return s


def prepare(case, seed):
    x = _inputs(case, seed)
    kind, D = case["kind"], case["D"]
    s = dict(case=case, **x)
    if own:
        import paper_2608_01127_amd as mw
        s["mw"] = mw
    if kind in ("cross", "train"):
        B, H, Hkv, T, M = (case[n] for n in ("B", "H", "Hkv", "T", "M"))
        s["kv_len"] = torch.tensor(_kv_lens(case), dtype=torch.int32, device=DEV)
        if own:
            s["o"] = torch.empty_like(x["q"])
            s["lse"] = torch.empty((B, H, T), dtype=torch.float32, device=DEV)
            n = mw.mw_cross_attn_workspace_size(B, H, Hkv, T, M, D)
            s["ws"] = torch.empty(max(16, n), dtype=torch.uint8, device=DEV)
            if kind == "train":
                s["dq"], s["dk"], s["dv"] = (torch.empty_like(x[n]) for n in "qkv")
                n = mw.mw_cross_attn_bwd_workspace_size(B, H, Hkv, T, M, D)
                s["ws_b"] = torch.empty(n, dtype=torch.uint8, device=DEV)
        return s
    L, hist = case["L"], x["hist"]
    lens = _seq_lens(case) if kind == "paged" else [case["len"]] * (1 if kind == "branch" else 2)
    grown = case["len"] + case.get("t", 0)
    W = -(-grown // L)
    n_seqs = {"paged": case.get("B", 1), "branch": 1 + case.get("n", 0), "select": 2}[kind]
    used = sum(-(-n // L) for n in lens)
    n_pages = used + (case["n"] * (W - case["len"] // L) if kind == "branch" else 0)
    s["pages_of"] = (used, n_pages, W)
    s["turn"] = 0
    if own:
        cache = mw.KVPages(n_pages, case.get("Hkv") or case["H"], L, D, n_seqs, W)
        for t in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales, cache.table):
            t.zero_()  # what no token has reached is returned too
        for i, n in enumerate(lens):
            if n:
                mw.mw_kvpages_append(cache, [i], hist[0][i:i + 1, :, :n], hist[1][i:i + 1, :, :n])
        s["cache"] = cache
        if kind == "paged":
            T = case["nq"] * case["ql"]
            s["seqs"] = list(range(n_seqs))
            s["o"] = torch.empty_like(x["q"])
            s["lse"] = torch.empty((case["B"], case["H"], T), dtype=torch.float32, device=DEV)
            n = mw.mw_chunk_attn_paged_workspace_size(cache, s["seqs"], case["H"], case["nq"], case["ql"])
            s["ws"] = torch.empty(max(16, n), dtype=torch.uint8, device=DEV)
    else:
        s.update(_plain_pool(case, lens, hist, n_seqs, n_pages, W))
    return s


# ------------------------------------------------------------------------------- the pass

def _softmax(s, hidden):
    """Probabilities and LSE of score rows; a row that sees no key has zeros and -inf."""
    s = s.masked_fill(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    return p / torch.where(l == 0, 1.0, l), (m + torch.log(l)).squeeze(-1)


def _groups(x, Hkv):
    """[B,H,T,D] -> 32 bits [B,Hkv,G*T,D]: the query heads of each key head one after another."""
    B, H, T, D = x.shape
    return x.float().reshape(B, Hkv, H // Hkv * T, D)


def _plain_cross(s):
    case = s["case"]
    B, H, Hkv, T, M, D = (case[n] for n in ("B", "H", "Hkv", "T", "M", "D"))
    scale = 1.0 / math.sqrt(D)
    hidden = (torch.arange(M, device=DEV).view(1, M) >= s["kv_len"].view(B, 1)).view(B, 1, 1, M)
    q, k, v = _groups(s["q"], Hkv), s["k"].float(), s["v"].float()
    p, lse = _softmax(q @ k.transpose(-1, -2).contiguous() * scale, hidden)
    o = p @ v
    out = {"o": o.view(B, H, T, D).to(torch.bfloat16), "lse": lse.view(B, H, T)}
    if case["kind"] == "cross":
        return out
    do = _groups(s["do"], Hkv)
    ds = (do @ v.transpose(-1, -2).contiguous() - (do * o).sum(-1, keepdim=True)) * p
    out["dq"] = (ds @ k * scale).view(B, H, T, D).to(torch.bfloat16)
    out["dk"] = (ds.transpose(-1, -2).contiguous() @ q * scale).to(torch.bfloat16)
    out["dv"] = (p.transpose(-1, -2).contiguous() @ do).to(torch.bfloat16)
    return out


def _gather(s, name):
    """The cached tokens of every sequence, [B,H,W*L,D] in 32 bits; zeros behind a sequence's last token."""
    page = s["table"].long()
    codes, scale = s[name + "_pages"].view(torch.uint8)[page].view(torch.float8_e4m3fn), s[name + "_scales"][page]
    x = codes.float() * scale.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1)  # [B,W,H,L,D]
    B, W, H, L, D = x.shape
    x = x.transpose(1, 2).reshape(B, H, W * L, D)
    keep = torch.arange(W * L, device=DEV).view(1, 1, W * L, 1) < s["lens"].view(B, 1, 1, 1)
    return torch.where(keep, x, 0.0)


def _queue_hidden(case):
    """[T,T]: which queued keys a queued row does not see."""
    c = torch.arange(case["nq"] * case["ql"], device=DEV) // case["ql"]
    return c.view(1, -1) > c.view(-1, 1) if case["mode"] == 0 else c.view(1, -1) != c.view(-1, 1)


def _plain_paged(s):
    case = s["case"]
    B, H, Hkv, D = (case[n] for n in ("B", "H", "Hkv", "D"))
    T = case["nq"] * case["ql"]
    k = torch.cat([_gather(s, "k"), s["k"].float()], dim=2)
    v = torch.cat([_gather(s, "v"), s["v"].float()], dim=2)
    C = k.shape[2] - T
    old = (torch.arange(C, device=DEV).view(1, C) >= s["lens"].view(B, 1)).view(B, 1, 1, C).expand(B, 1, T, C)
    hidden = torch.cat([old, _queue_hidden(case).expand(B, 1, T, T)], dim=-1).repeat(1, 1, H // Hkv, 1)
    p, lse = _softmax(_groups(s["q"], Hkv) @ k.transpose(-1, -2).contiguous() * (1.0 / math.sqrt(D)), hidden)
    return {"o": (p @ v).view(B, H, T, D).to(torch.bfloat16), "lse": lse.view(B, H, T)}


_POOL = ("k_pages", "v_pages", "k_scales", "v_scales", "table", "lens")


def _plain_commit(s, name, new, pages, first, keep):
    """Quantises `new` [n,H,t,D] behind `keep` tokens of the page that the branches share (sequence 0's page
    number `first` in its row), into each branch's own pages [n, w]."""
    L = s["case"]["L"]
    n, w = pages.shape
    pool, scale = s[name + "_pages"].view(torch.uint8), s[name + "_scales"]
    H, D = pool.shape[1], pool.shape[3]
    T = keep + new.shape[2]
    x = torch.zeros(n, H, w * L, D, device=DEV)
    x[:, :, keep:T] = new.float()
    e = _exponent(x.view(n, H, -1, BLOCK * D).abs().amax(-1))
    at = torch.arange(w * L, device=DEV)
    nb = -(-keep // BLOCK)  # blocks that hold old tokens
    if keep:
        src = s["table"][0, first].long()
        old = scale[src][:, :nb]
        eo = torch.frexp(old)[1].to(e.dtype) - 1
        part = torch.where(torch.arange(nb, device=DEV) < keep // BLOCK, eo, torch.maximum(eo, e[:, :, :nb]))
        e = torch.cat([part, e[:, :, nb:]], dim=-1)
        x[:, :, :keep] = (pool.view(torch.float8_e4m3fn)[src].float() * scale[src].repeat_interleave(BLOCK, -1).unsqueeze(-1))[:, :keep]
    codes = _encode(x, e.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1)).view(torch.uint8)
    to = pages.long().repeat_interleave(L, dim=1)[:, :T].reshape(-1)
    row = (at % L)[:T].repeat(n)
    pool[to, :, row] = codes[:, :, :T].transpose(1, 2).reshape(n * T, H, D)
    b = torch.arange(-(-T // BLOCK), device=DEV)
    per = L // BLOCK
    to = pages.long()[:, b // per].reshape(-1)
    scale[to, :, (b % per).repeat(n)] = torch.ldexp(torch.ones_like(e), e)[:, :, b].transpose(1, 2).reshape(-1, H)


def _plain_branch(s):
    case = s["case"]
    n, L = case["n"], case["L"]
    used, _, W = s["pages_of"]
    first = case["len"] // L
    w = W - first  # pages that each branch has of its own
    s["table"][1:, :used] = s["table"][0, :used]
    s["table"][1:, first:W] = torch.arange(used, used + n * w, dtype=torch.int32, device=DEV).view(n, w)
    s["lens"][1:] = case["len"] + case["t"]
    for name in "kv":
        _plain_commit(s, name, s[name], s["table"][1:, first:W], first, case["len"] % L)
    return {name: s[name] for name in _POOL}


def _plain_select(s):
    used = s["pages_of"][0] // 2
    keep = 1 - s["turn"]  # the sequence in the upper pages
    s["turn"] = keep
    for name in _POOL[:4]:
        s[name][:used] = s[name][used:2 * used]  # compaction
        s[name][used:2 * used] = s[name][:used]  # the copy
    pages = torch.arange(2 * used, dtype=torch.int32, device=DEV)
    s["table"][keep, :used] = pages[:used]
    s["table"][1 - keep, :used] = pages[used:]
    s["lens"][1 - keep] = s["lens"][keep]
    return {name: s[name] for name in _POOL}


def _own_pool(cache):
    return {"k_pages": cache.k_pages.view(torch.float8_e4m3fn), "v_pages": cache.v_pages.view(torch.float8_e4m3fn),
            "k_scales": cache.k_scales, "v_scales": cache.v_scales, "table": cache.table, "lens": cache.lens}


def _run_own(s):
    mw, case = s["mw"], s["case"]
    kind = case["kind"]
    if kind in ("cross", "train"):
        mw.mw_cross_attn_fwd(s["q"], s["k"], s["v"], kv_len=s["kv_len"], out=s["o"], lse=s["lse"], workspace=s["ws"])
        if kind == "cross":
            return {n: s[n] for n in ("o", "lse")}
        mw.mw_cross_attn_bwd(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], kv_len=s["kv_len"], workspace=s["ws_b"],
                             dq=s["dq"], dk=s["dk"], dv=s["dv"])
        return {n: s[n] for n in ("o", "lse", "dq", "dk", "dv")}
    cache = s["cache"]
    if kind == "paged":
        mw.mw_chunk_attn_paged(s["q"], s["k"], s["v"], case["nq"], case["ql"], cache, s["seqs"], flags=case["mode"],
                               out=s["o"], lse=s["lse"], workspace=s["ws"])
        return {n: s[n] for n in ("o", "lse")}
    if kind == "branch":
        ids = list(range(1, 1 + case["n"]))
        mw.mw_kvpages_free(cache, ids)
        for i in ids:
            mw.mw_kvpages_fork(cache, 0, i)
        mw.mw_kvpages_append(cache, ids, s["k"], s["v"])
    else:
        drop = s["turn"]
        keep = 1 - drop
        s["turn"] = keep
        mw.mw_kvpages_free(cache, [drop])
        mw.mw_kvpages_compact(cache)
        mw.mw_kvpages_copy(cache, keep, drop)
    return _own_pool(cache)


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind in ("cross", "train"):
        return _plain_cross(s)
    return {"paged": _plain_paged, "branch": _plain_branch, "select": _plain_select}[kind](s)


# ------------------------------------------------------------------------------- its work

def work(case):
    D, kind = case["D"], case["kind"]
    if kind in ("cross", "train"):
        B, H, Hkv, T = (case[n] for n in ("B", "H", "Hkv", "T"))
        keys = sum(_kv_lens(case))
        pairs = H * T * keys
        n_q, n_k = B * H * T, Hkv * keys
        if kind == "cross":  # q, k, v in, o and lse out
            return {"bytes": n_q * (4 * D + 4) + n_k * 4 * D, "flops": 4 * D * pairs}
        # forward as above; backward: q, o, do, lse, k, v in, dq, dk, dv out (padding states' too)
        return {"bytes": n_q * (12 * D + 8) + n_k * 8 * D + B * Hkv * case["M"] * 4 * D, "flops": 14 * D * pairs}
    if kind == "paged":
        B, H, Hkv, nq, ql = (case[n] for n in ("B", "H", "Hkv", "nq", "ql"))
        T, cached = nq * ql, sum(_seq_lens(case))
        pairs = H * (T * cached + B * ql * ql * (nq * (nq + 1) // 2 if case["mode"] == 0 else nq))
        # codes and scales of the cached tokens, q, k, v in; o, lse out
        return {"bytes": Hkv * cached * (2 * D + 8 / BLOCK) + B * T * (H * (4 * D + 4) + Hkv * 4 * D), "flops": 4 * D * pairs}
    if kind == "branch":
        token = case["H"] * 2 * D
        # new tokens read in 16 bits and written in 8; the shared page's tokens read and written
        return {"bytes": case["n"] * token * (3 * case["t"] + 2 * (case["len"] % case["L"])), "flops": 0}
    return {"bytes": 4 * case["len"] * case["H"] * 2 * D, "flops": 0}  # moved once, copied once


# ------------------------------------------------------------------------------- 64-bit values

def _exact_rows(q, k, v, hidden, scale):
    """O, LSE and P of full rows in 64 bits; `hidden` broadcasts over the scores."""
    s = (q @ k.t()) * scale
    s.masked_fill_(hidden, -math.inf)
    lse = torch.logsumexp(s, dim=-1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return p @ v, lse, p


def _exact_cross(case, x):
    B, H, Hkv, T, M, D = (case[n] for n in ("B", "H", "Hkv", "T", "M", "D"))
    scale, G = 1.0 / math.sqrt(D), H // Hkv
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)
    out = {"o": new(B, H, T, D), "lse": new(B, H, T)}
    if case["kind"] == "train":
        out.update(dq=new(B, H, T, D), dk=new(B, Hkv, M, D), dv=new(B, Hkv, M, D))
    for b, n in enumerate(_kv_lens(case)):
        for h in range(H):
            k, v = x["k"][b, h // G, :n].double(), x["v"][b, h // G, :n].double()
            for r in range(0, T, 4096):
                i = slice(r, min(T, r + 4096))
                q = x["q"][b, h, i].double()
                none = torch.zeros((), dtype=torch.bool, device=DEV)
                o, lse, p = _exact_rows(q, k, v, none, scale)
                out["o"][b, h, i], out["lse"][b, h, i] = o, lse
                if case["kind"] == "train" and n:
                    do = x["do"][b, h, i].double()
                    ds = (do @ v.t() - (do * o).sum(-1, keepdim=True)) * p
                    out["dq"][b, h, i] = ds @ k * scale
                    out["dk"][b, h // G, :n] += ds.t() @ q * scale
                    out["dv"][b, h // G, :n] += p.t() @ do
    return out


def _exact_codes(x):
    """What [H,T,D] tokens read as after one commit, in 64 bits: the nearest e4m3 multiples of a power of two
    for each 64 tokens and head."""
    H, T, D = x.shape
    y = torch.nn.functional.pad(x.double(), (0, 0, 0, -T % BLOCK)).view(H, -1, BLOCK * D)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0))  # exact at powers of two times 1.75
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 224.0 * torch.exp2(e), e - 1, e)).clamp(-100, 100)
    y = (y / torch.exp2(e)).float().to(torch.float8_e4m3fn).double() * torch.exp2(e)
    return y.view(H, -1, D)[:, :T]


def _exact_paged(case, x):
    B, H, Hkv, D, nq, ql = (case[n] for n in ("B", "H", "Hkv", "D", "nq", "ql"))
    T, G = nq * ql, H // Hkv
    o = torch.zeros((B, H, T, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((B, H, T), dtype=torch.float64, device=DEV)
    queue = _queue_hidden(case)
    for b, n in enumerate(_seq_lens(case)):
        k, v = (_exact_codes(t[b, :, :n]) if n else t[b, :, :0].double() for t in x["hist"])
        for h in range(H):
            kk = torch.cat([k[h // G], x["k"][b, h // G].double()])
            vv = torch.cat([v[h // G], x["v"][b, h // G].double()])
            hidden = torch.cat([torch.zeros((T, n), dtype=torch.bool, device=DEV), queue], dim=1)
            o[b, h], lse[b, h], _ = _exact_rows(x["q"][b, h].double(), kk, vv, hidden, 1.0 / math.sqrt(D))
    return {"o": o, "lse": lse}


def _exact_pool(case, x):
    """The pages after one pass, written from the tokens themselves."""
    L, H, D = case["L"], case["H"], case["D"]
    grown = case["len"] + case.get("t", 0)
    W = -(-grown // L)
    first, old = case["len"] // L, -(-case["len"] // L)
    branch = case["kind"] == "branch"
    n_pages = old + case["n"] * (W - first) if branch else 2 * old
    out = {}
    for j, name in enumerate("kv"):
        codes = torch.zeros((n_pages, H, L, D), dtype=torch.float64, device=DEV)
        scale = torch.zeros((n_pages, H, L // BLOCK), dtype=torch.float64, device=DEV)

        def put(pages, tokens, settled):
            """`tokens` [H,t,D], of which the first `settled` were committed before the others."""
            for c in range(0, tokens.shape[1], BLOCK):
                t = tokens[:, c:c + BLOCK].double()
                m, e = torch.frexp(t.abs().amax((1, 2)))
                s = torch.exp2(torch.where(m > 0.875, e - 8, e - 9).double())
                page, at = pages[c // L], c % L
                if c < settled < c + t.shape[1]:  # committed in two parts: the old ones are encoded twice
                    n = settled - c
                    m, e = torch.frexp(t[:, :n].abs().amax((1, 2)))
                    s0 = torch.exp2(torch.where(m > 0.875, e - 8, e - 9).double())[:, None, None]
                    t = torch.cat([(t[:, :n] / s0).float().to(torch.float8_e4m3fn).double() * s0, t[:, n:]], dim=1)
                codes[page, :, at:at + t.shape[1]] = (t / s[:, None, None]).float().to(torch.float8_e4m3fn).double()
                scale[page, :, at // BLOCK] = s

        hist = x["hist"][j]
        if branch:
            put(list(range(old)), hist[0], case["len"])
            for i in range(case["n"]):
                own_pages = [old + i * (W - first) + w for w in range(W - first)]
                put(own_pages, torch.cat([hist[0][:, first * L:], x[name][i]], dim=1), case["len"] - first * L)
        else:  # both hold the second sequence
            put(list(range(old)), hist[1], case["len"])
            put(list(range(old, 2 * old)), hist[1], case["len"])
            tail = case["len"] % L  # rows behind the last token: whole pages move, all of them zeros there
            assert tail == 0 or not codes[old - 1, :, tail:].any()
        out[name + "_pages"], out[name + "_scales"] = codes, scale
    out["table"] = out["lens"] = None
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] in ("cross", "train"):
        return _exact_cross(case, x)
    return _exact_paged(case, x) if case["kind"] == "paged" else _exact_pool(case, x)
