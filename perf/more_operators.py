"""Attention of packed sequences, rotary positions, and eviction from the paged cache by accumulated
attention weight, as passes that a timing program can prepare, run and check.

Kinds of pass:

  packed  serving: attention of sequences of different lengths, one behind the other in one tensor, without
          padding; each query token sees the keys of chunks up to its own (chunks of one token: the token-causal
          rule), and with `new` > 0 only the last `new` tokens of each sequence are queries (new = 1: one token);
  train   its forward and backward;
  rope    rotary positions applied to queries and keys;
  turn    the same and, from the gradients of the rotated tensors, those of the tensors before;
  weigh   for every cached token of a paged cache the attention weight it got, summed over rows and heads;
  evict   rollouts forked, and of each branch all but its anchor, its newest tokens and the heaviest others
          dropped (the kept ones are packed into pages of the branch's own).

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
        # one new token of eight ragged sequences, four query heads to a key head: bound by reading the keys
        dict(name="packed_one", kind="packed", lens="15840,14001,12673,9900,8191,7920,3333,64", new=1, chunk=1, H=16, Hkv=4,
             D=128, layout="thd"),
        # short prompts of odd lengths, one of them empty: launches and small tiles count
        dict(name="packed_short_d64", kind="packed", lens="77,300,1,0,129,513", new=0, chunk=1, H=12, Hkv=4, D=64, layout="thd"),
        # prompts of a serving batch, token-causal, four query heads to a key head
        dict(name="packed_prompts", kind="packed", lens="8100,4799,2640,2111,1320,229,1", new=0, chunk=1, H=16, Hkv=4, D=128,
             layout="thd"),
        # odd everything: the 0.5B width, clips of different lengths in chunks of 333 tokens, head-major tensors
        dict(name="train_odd_d72", kind="train", lens="2999,1001,77,640", new=0, chunk=333, H=16, Hkv=16, D=72, layout="htd"),
        # token-causal training on packed texts, shared key heads, head width 64
        dict(name="train_text_d64", kind="train", lens="4096,2050,1024,700,256,66", new=0, chunk=1, H=24, Hkv=8, D=64,
             layout="thd"),
        # the 1B model's training window of 19200 tokens as clips of 16, 9, 6 and 1 chunks of 600
        dict(name="train_clips_1b", kind="train", lens="9600,5400,3600,600", new=0, chunk=600, H=12, Hkv=12, D=128, layout="thd"),
        # one token of eight sequences far into a stretched context, half layout: the launch is what counts
        dict(name="rope_one", kind="rope", B=8, T=1, H=16, Hkv=4, D=128, form="halves", first=0, far=120000, layout="bthd"),
        # queries and keys of the 1B model's training window, three axes of positions, interleaved; and the gradients
        dict(name="turn_axes_1b", kind="turn", B=1, T=19200, H=12, Hkv=12, D=128, form="axes", first=0, far=0, layout="bthd"),
        # one token of eight ragged sequences: bound by reading the keys' codes
        dict(name="weigh_one", kind="weigh", B=8, H=16, Hkv=4, D=128, len=15840, L=128, T=1, layout="bthd"),
        # a rollout step of the 1B model: guidance pair, 8 in-flight chunks over 24 cached chunks and the anchor
        dict(name="weigh_stream_1b", kind="weigh", B=2, H=12, Hkv=12, D=128, len=14700, L=64, T=4800, layout="bthd"),
        # two ragged branches at the 0.5B width, odd anchor and window
        dict(name="evict_odd_d72", kind="evict", n=2, H=16, D=72, len=3601, L=192, keep=1777, first=301, recent=599),
        # half of the 6 x 2640-token window of four branches, the one-frame anchor and the newest chunk kept
        dict(name="evict_window", kind="evict", n=4, H=16, D=128, len=15840, L=64, keep=7920, first=300, recent=2640),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges; lengths are spread over their logarithm."""
    while True:
        kind = rng.choice(["packed", "packed", "train", "train", "rope", "turn", "weigh", "evict"])
        D = rng.choice([64, 72, 128])
        Hkv = rng.choice([1, 2, 3, 4, 8, 12, 16])
        H = Hkv * rng.choice([1, 1, 2, 4, 8])
        if kind in ("packed", "train"):
            n = rng.choice([1, 2, 3, 5, 8, 17, 40])
            lens = [_log_int(rng, 1, 16000) if rng.random() < 0.95 else 0 for _ in range(n)]
            new = rng.choice([0, 0, 1, 1, 7, 64]) if kind == "packed" else 0
            case = dict(kind=kind, lens=",".join(map(str, lens)), new=new, chunk=rng.choice([1, 1, 1, 64, 333, 600, 2640]),
                        H=H, Hkv=Hkv, D=D, layout=rng.choice(["thd", "htd"]))
            tokens = sum(lens)
            if not 0 < tokens <= 20000 * (8 if new else 1):
                continue
        elif kind in ("rope", "turn"):
            form = rng.choice(["halves", "interleaved", "axes", "part"])
            case = dict(kind=kind, B=rng.choice([1, 2, 3, 8]), T=_log_int(rng, 1, 20000), H=H, Hkv=Hkv, D=D, form=form,
                        first=rng.choice([0, 1234]), far=rng.choice([0, 0, 120000, 1000000]), layout=rng.choice(["bhtd", "bthd"]))
        elif kind == "weigh":
            case = dict(kind=kind, B=rng.choice([1, 2, 3, 8]), H=H, Hkv=Hkv, D=D, len=_log_int(rng, 8, 16000),
                        L=rng.choice([64, 128, 192, 640]), T=_log_int(rng, 1, 4800), layout=rng.choice(["bhtd", "bthd"]))
        else:
            length = _log_int(rng, 64, 16000)
            keep = rng.randint(1, length - 1)
            first = rng.choice([0, rng.randint(0, keep // 2)])
            case = dict(kind=kind, n=rng.choice([1, 2, 4]), H=Hkv, D=D, len=length, L=rng.choice([64, 128, 192, 640]), keep=keep,
                        first=first, recent=rng.randint(0, (keep - first) // 2 + 1) if keep > first else 0)
        # the 1B training, stream and rotary passes are the largest
        w = work(case)
        most = {"packed": (3e11, 5e8), "train": (1.9e12, 5e8), "rope": (1e9, 4.7e8), "turn": (1e9, 4.7e8), "weigh": (4e11, 2e8),
                "evict": (1, 2.7e8)}[kind]
        if w["flops"] <= most[0] and w["bytes"] <= most[1]:
            return case


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _lens(case):
    """Keys and queries of each packed sequence."""
    nk = [int(n) for n in case["lens"].split(",")]
    return nk, [min(n, case["new"]) if case["new"] else n for n in nk]


def _packed(g, T, H, D, layout):
    """bf16 N(0,1) activations as a [T,H,D] tensor, or such a view of a [H,T,D] one."""
    if layout == "htd":
        return torch.randn(H, T, D, device=DEV, generator=g).to(torch.bfloat16).transpose(0, 1)
    return torch.randn(T, H, D, device=DEV, generator=g).to(torch.bfloat16)


def _randn(g, B, H, T, D, layout="bhtd"):
    """bf16 N(0,1) activations as a [B,H,T,D] tensor, or such a view of a [B,T,H,D] one."""
    if layout == "bthd":
        return torch.randn(B, T, H, D, device=DEV, generator=g).to(torch.bfloat16).transpose(1, 2)
    return torch.randn(B, H, T, D, device=DEV, generator=g).to(torch.bfloat16)


def _cached_lens(case):
    """Cached tokens of each sequence."""
    if case["kind"] == "evict":
        return [case["len"] - (b * (case["len"] - case["keep"])) // (2 * case["n"]) for b in range(case["n"])]
    return [max(1, case["len"] - (b * case["len"]) // (2 * case["B"])) for b in range(case["B"])]


def _history(g, n, H, T, D):
    """K and V of n sequences' tokens; the values' magnitude differs between heads and drifts over the tokens."""
    k, v = _randn(g, n, H, T, D), _randn(g, n, H, T, D)
    gain = torch.exp2(torch.rand(1, H, 1, 1, device=DEV, generator=g) * 2 - 1)
    drift = torch.exp2(2 * torch.sin(torch.arange(T, device=DEV) / 30.0)).view(1, 1, T, 1)
    return k, (v.float() * gain * drift).to(torch.bfloat16)


def _bands(case):
    """Bands of the head: (first dimension, dimensions, base, axis, scaling), scaling None or (factor, trained
    length, least and most turns of the ramp)."""
    D, form = case["D"], case["form"]
    if form == "axes":  # time, height, width: the 3-axis split
        side = 2 * (D // 6)
        return [(0, D - 2 * side, 1e4, 0, None), (D - 2 * side, side, 1e4, 1, None), (D - side, side, 1e4, 2, None)]
    if form == "halves":
        return [(0, D, 5e5, 0, (8.0, 8192.0, 1.0, 32.0))]
    if form == "part":  # half of the head turns, positions divided by four
        return [(0, D // 2, 1e4, 0, (4.0, 0.0, 0.0, 0.0))]
    return [(0, D, 1e4, 0, None)]


def _is_halves(case):
    return case["form"] in ("halves", "part")


def _gain(case):
    return 0.1 * math.log(8.0) + 1.0 if case["form"] == "halves" else 1.0


def _inputs(case, seed):
    """Every random tensor of a case, from the seed alone (shared by prepare and exact)."""
    g, kind, D = _gen(seed), case["kind"], case["D"]
    if kind in ("packed", "train"):
        nk, nq = _lens(case)
        x = dict(q=_packed(g, sum(nq), case["H"], D, case["layout"]))
        x["k"], x["v"] = (_packed(g, sum(nk), case["Hkv"], D, case["layout"]) for _ in range(2))
        if kind == "train":
            x["do"] = _packed(g, sum(nq), case["H"], D, case["layout"])
        return x
    if kind in ("rope", "turn"):
        B, T = case["B"], case["T"]
        names = [("q", case["H"]), ("k", case["Hkv"])] + ([("dq", case["H"]), ("dk", case["Hkv"])] if kind == "turn" else [])
        x = {n: _randn(g, B, h, T, D, case["layout"]) for n, h in names}
        t = torch.arange(T, device=DEV) + case["first"]
        if case["far"]:  # sequences at places of their own
            t = t + torch.randint(0, case["far"], (B, 1), device=DEV, generator=g)
        if case["form"] == "axes":  # frames of 15 x 20 cells
            t = torch.stack([t // 300, t % 300 // 20, t % 20])
        x["pos"] = t
        return x
    if kind == "weigh":
        x = dict(q=_randn(g, case["B"], case["H"], case["T"], D, case["layout"]))
        x["hist"] = _history(g, case["B"], case["Hkv"], case["len"], D)
        # the rows' LSE as an attention call has left it: over the cached tokens and keys of their own
        x["lse"] = torch.rand(case["B"], case["H"], case["T"], device=DEV, generator=g) * 2.0
        G = case["H"] // case["Hkv"]
        for b, n in enumerate(_cached_lens(case)):
            k, _ = _exact_codes(x["hist"][0][b, :, :n])
            for h in range(case["H"]):
                x["lse"][b, h] += torch.logsumexp(x["q"][b, h].double() @ k[h // G].t() * D ** -0.5, -1).float()
        return x
    x = dict(hist=_history(g, case["n"], case["H"], case["len"], D))
    # heavy-tailed sums, equal ones among them
    w = torch.exp(2.0 * torch.randn(case["n"], case["len"], device=DEV, generator=g)).to(torch.bfloat16).float()
    x["weights"] = torch.where(torch.rand(w.shape, device=DEV, generator=g) < 0.05, 0.0, w)
    return x


def _exponent(amax):
    """Least e with amax <= 448 * 2^e, within [-100, 100]."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax == 0, -100, e).clamp(-100, 100)


def _encode(x, e):
    """e4m3 codes of x (32 bits) at scale 2^e."""
    return torch.ldexp(x, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _quantise(x, lens, L):
    """Codes [n, pages, H, L, D] and exponents [n, pages, H, L / 64] of the first lens[i] tokens of each sequence."""
    n, H, T, D = x.shape
    keep = torch.arange(T, device=DEV).view(1, 1, T, 1) < torch.tensor(lens, device=DEV).view(-1, 1, 1, 1)
    W = -(-T // L)
    y = torch.zeros(n, H, W * L, D, device=DEV)
    y[:, :, :T] = torch.where(keep, x.float(), 0.0)
    y = y.view(n, H, W, L, D).transpose(1, 2)
    e = _exponent(y.reshape(n, W, H, L // BLOCK, BLOCK * D).abs().amax(-1))
    return _encode(y, e.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1)), e


def _plain_pool(L, lens, hist, n_seqs, n_pages, W):
    """The pool as tensors: codes [P,H,L,D], scales [P,H,L/64], the page table and the lengths.  Pages are
    taken lowest first, sequence by sequence."""
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


def _cached(s, i, name):
    """The cached tokens of sequence i, [H,len,D] in 32 bits."""
    n = s["n_cached"][i]
    L = s["case"]["L"]
    page = s["table"][i, :-(-n // L)].long()
    codes, scale = s[name + "_pages"].view(torch.uint8)[page].view(torch.float8_e4m3fn), s[name + "_scales"][page]
    x = codes.float() * scale.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1)  # [w,H,L,D]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def prepare(case, seed):
    x = _inputs(case, seed)
    kind, D = case["kind"], case["D"]
    s = dict(case=case, **x)
    if own:
        import paper_2608_01127_amd as mw
        s["mw"] = mw
    if kind in ("packed", "train"):
        nk, nq = _lens(case)
        H, Hkv, Tq, Tk = case["H"], case["Hkv"], sum(nq), sum(nk)
        if own:
            edges = lambda n: torch.tensor([0, *n], device=DEV).cumsum(0).to(torch.int32)
            cu_q = edges(nq)
            s["pack"] = mw.Packed(cu_q, Tq, H, Hkv, D, chunk_len=case["chunk"], cu_k=edges(nk) if case["new"] else None,
                                  total_k=Tk, backward=kind == "train")
            s["o"], s["lse"] = torch.empty_like(x["q"]), torch.empty((H, Tq), dtype=torch.float32, device=DEV)
            s["ws"] = torch.empty(max(16, mw.mw_packed_attn_workspace_size(s["pack"])), dtype=torch.uint8, device=DEV)
            if kind == "train":
                s["dq"], s["dk"], s["dv"] = (torch.empty_like(x[n]) for n in "qkv")
                s["ws_b"] = torch.empty(mw.mw_packed_attn_bwd_workspace_size(s["pack"]), dtype=torch.uint8, device=DEV)
        return s
    if kind in ("rope", "turn"):
        if own:
            s["bands"] = mw.rope_bands([dict(dim_offset=a, dim_count=d, theta=base, axis=axis) if sc is None else
                                        dict(dim_offset=a, dim_count=d, theta=base, axis=axis, factor=sc[0], trained_len=sc[1],
                                             turns_lo=sc[2], turns_hi=sc[3]) for a, d, base, axis, sc in _bands(case)],
                                       halves=_is_halves(case), gain=_gain(case))
            for n in x:
                if n != "pos":
                    s[n + "_out"] = torch.empty_like(x[n])
        return s
    L, lens, hist = case["L"], _cached_lens(case), x["hist"]
    W = -(-case["len"] // L)
    used = sum(-(-n // L) for n in lens)
    n = len(lens)
    evict = kind == "evict"
    n_seqs = 2 * n if evict else n
    n_pages = used + (n * (-(-case["keep"] // L) - case["first"] // L) if evict else 0)
    s["n_cached"] = lens
    if own:
        cache = mw.KVPages(n_pages, case.get("Hkv") or case["H"], L, D, n_seqs, W)
        for t in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales, cache.table):
            t.zero_()  # what no token has reached is returned too
        for i, m in enumerate(lens):
            mw.mw_kvpages_append(cache, [i], hist[0][i:i + 1, :, :m], hist[1][i:i + 1, :, :m])
        s["cache"] = cache
        s["seqs"] = list(range(n, 2 * n)) if evict else list(range(n))
    else:
        s.update(_plain_pool(L, lens, hist, n_seqs, n_pages, W))
    if evict:
        w = torch.zeros((2 * n, W * L), dtype=torch.float32, device=DEV)
        w[:n, :case["len"]] = x["weights"]
        s["weights"] = w
        if own:
            need = mw.mw_kvpages_evict_weighted_workspace_size(cache, s["seqs"], case["keep"], first=case["first"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        return s
    s["weights"] = torch.zeros((n, W * L), dtype=torch.float32, device=DEV)
    if own:
        need = mw.mw_kvpages_weigh_workspace_size(cache, s["seqs"], case["H"], case["T"])
        s["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------- the pass

def _softmax(s, hidden):
    """Probabilities and LSE of score rows; a row that sees no key has zeros and -inf."""
    s = s.masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return p.div_(torch.where(l == 0, 1.0, l)), (m + torch.log(l)).squeeze(-1)


def _hidden(case, nq, nk):
    """[nq,nk]: which keys a row does not see."""
    at = torch.arange(nk - nq, nk, device=DEV).view(nq, 1)
    j = torch.arange(nk, device=DEV).view(1, nk)
    return (j // case["chunk"] > at // case["chunk"]) | (at < 0)


def _plain_packed(s):
    case = s["case"]
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    G, scale = H // Hkv, 1.0 / math.sqrt(D)
    nk, nq = _lens(case)
    train = case["kind"] == "train"
    out = {"o": torch.empty_like(s["q"]), "lse": torch.empty((H, sum(nq)), device=DEV)}
    if train:
        out.update({"d" + n: torch.empty_like(s[n]) for n in "qkv"})
    q0 = k0 = 0
    for mq, mk in zip(nq, nk):
        i, j = slice(q0, q0 + mq), slice(k0, k0 + mk)
        q0, k0 = q0 + mq, k0 + mk
        if mq == 0 and mk == 0:
            continue
        hidden = _hidden(case, mq, mk).repeat(G, 1)
        rows = lambda t, h: t[i, h].float().transpose(0, 1).reshape(-1, D)  # query heads one after another
        back = lambda t: t.view(G, mq, -1).transpose(0, 1)
        for hk in range(Hkv):
            h = slice(hk * G, (hk + 1) * G)
            q, k, v = rows(s["q"], h), s["k"][j, hk].float(), s["v"][j, hk].float()
            p, lse = _softmax(q @ k.t().contiguous() * scale, hidden)
            o = p @ v
            out["o"][i, h] = back(o).to(torch.bfloat16)
            out["lse"][h, i] = lse.view(G, mq)
            if not train:
                continue
            do = rows(s["do"], h)
            out["dv"][j, hk] = (p.t().contiguous() @ do).to(torch.bfloat16)
            ds = (do @ v.t().contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
            out["dq"][i, h] = back(ds @ k * scale).to(torch.bfloat16)
            out["dk"][j, hk] = (ds.t().contiguous() @ q * scale).to(torch.bfloat16)
    return out


def _angles(case, pos):
    """cos and sin [B or 1, 1, T, pairs] in 64 bits, and the dimensions of each pair."""
    cos, sin, first, second = [], [], [], []
    axes = pos if case["form"] == "axes" else pos.unsqueeze(0)
    for a, d, base, axis, sc in _bands(case):
        i = torch.arange(d // 2, device=DEV, dtype=torch.float64)
        f = torch.pow(torch.tensor(base, dtype=torch.float64, device=DEV), -2.0 * i / d)
        if sc is not None:
            factor, trained, lo, hi = sc
            ramp = ((trained * f / (2 * math.pi) - lo) / (hi - lo)).clamp(0.0, 1.0) if hi > lo else torch.zeros_like(f)
            f = f * (ramp + (1.0 - ramp) / factor)
        t = axes[axis].double().unsqueeze(-1) * f
        t = t.view(-1, 1, *t.shape[-2:])
        cos.append(torch.cos(t))
        sin.append(torch.sin(t))
        e = torch.arange(d // 2, device=DEV)
        first.append(a + (e if _is_halves(case) else 2 * e))
        second.append(a + (e + d // 2 if _is_halves(case) else 2 * e + 1))
    return torch.cat(cos, -1), torch.cat(sin, -1), torch.cat(first), torch.cat(second)


def _turn(x, cos, sin, a, b, gain):
    y = x.clone()
    y[..., a] = gain * (x[..., a] * cos - x[..., b] * sin)
    y[..., b] = gain * (x[..., b] * cos + x[..., a] * sin)
    return y


def _plain_rope(s):
    case = s["case"]
    cos, sin, a, b = _angles(case, s["pos"])
    cos, sin = cos.float(), sin.float()
    out = {}
    for n in ("q", "k", "dq", "dk"):
        if n in s:
            back = n.startswith("d")
            out[n] = _turn(s[n].float(), cos, -sin if back else sin, a, b, _gain(case)).to(torch.bfloat16)
    return out


def _scores(s, b, hk):
    """Score rows of one sequence and key head over its cached tokens, [G*T, len] in 32 bits."""
    case = s["case"]
    G, D = case["H"] // case["Hkv"], case["D"]
    k = _cached(s, b, "k")[hk]
    q = s["q"][b, hk * G:(hk + 1) * G].float().reshape(-1, D)
    return q @ k.t().contiguous() * (1.0 / math.sqrt(D))


def _plain_weigh(s):
    case = s["case"]
    G = case["H"] // case["Hkv"]
    for b, n in enumerate(s["n_cached"]):
        w = torch.zeros(n, dtype=torch.float64, device=DEV)
        for hk in range(case["Hkv"]):
            lse = s["lse"][b, hk * G:(hk + 1) * G].reshape(-1, 1)
            w += _scores(s, b, hk).sub_(lse).exp_().sum(0, dtype=torch.float64)
        s["weights"][b, :n] = w.float()
    return {"weights": s["weights"]}


_POOL = ("k_pages", "v_pages", "k_scales", "v_scales", "table", "lens")


def _kept(w, case):
    """Tokens that stay, in order: the anchor, the newest, and the heaviest of the others (ties: lowest index)."""
    n, first, recent = w.shape[0], case["first"], case["recent"]
    mid = torch.sort(w[first:n - recent], descending=True, stable=True).indices[:case["keep"] - first - recent]
    stay = torch.cat([torch.arange(first, device=DEV), first + mid, torch.arange(n - recent, n, device=DEV)])
    return torch.sort(stay).values


def _plain_evict(s):
    case = s["case"]
    n, L, H, D, keep = case["n"], case["L"], case["H"], case["D"], case["keep"]
    at = sum(-(-m // L) for m in s["n_cached"])
    w0, w1 = case["first"] // L, -(-keep // L)  # pages that stay shared, and all pages of a branch
    s["weights"][n:] = s["weights"][:n]
    for i, m in enumerate(s["n_cached"]):
        stay = _kept(s["weights"][i, :m], case)
        row = s["table"][n + i]
        row[:-(-m // L)] = s["table"][i, :-(-m // L)]
        pages = torch.arange(at, at + w1 - w0, dtype=torch.int32, device=DEV)
        at += w1 - w0
        moved = stay[w0 * L:]
        for name in "kv":
            x = torch.zeros((w1 - w0) * L, H, D, device=DEV)
            x[:keep - w0 * L] = _cached(s, i, name)[:, moved].transpose(0, 1)
            x = x.view(w1 - w0, L, H, D).transpose(1, 2)
            e = _exponent(x.reshape(w1 - w0, H, L // BLOCK, BLOCK * D).abs().amax(-1))
            codes = _encode(x, e.repeat_interleave(BLOCK, dim=-1).unsqueeze(-1))
            s[name + "_pages"].view(torch.uint8)[pages.long()] = codes.view(torch.uint8)
            filled = torch.arange((w1 - w0) * L // BLOCK, device=DEV).view(w1 - w0, 1, -1) < -(-(keep - w0 * L) // BLOCK)
            s[name + "_scales"][pages.long()] = torch.where(filled, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e), 0.0)
        row[w0:w1] = pages
        s["lens"][n + i] = keep
        w = s["weights"][n + i]
        w[:keep] = w[:m][stay]
        w[keep:m] = 0.0
    return {name: s[name] for name in (*_POOL, "weights")}


def _run_own(s):
    mw, case = s["mw"], s["case"]
    kind = case["kind"]
    if kind in ("packed", "train"):
        mw.mw_packed_attn_fwd(s["q"], s["k"], s["v"], s["pack"], out=s["o"], lse=s["lse"], workspace=s["ws"])
        if kind == "packed":
            return {n: s[n] for n in ("o", "lse")}
        mw.mw_packed_attn_bwd(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["pack"], workspace=s["ws_b"], dq=s["dq"],
                              dk=s["dk"], dv=s["dv"])
        return {n: s[n] for n in ("o", "lse", "dq", "dk", "dv")}
    if kind in ("rope", "turn"):
        mw.mw_rope_apply(s["q"], s["k"], s["bands"], s["pos"], q_out=s["q_out"], k_out=s["k_out"])
        out = {n: s[n + "_out"] for n in ("q", "k")}
        if kind == "turn":
            mw.mw_rope_apply(s["dq"], s["dk"], s["bands"], s["pos"], inverse=True, q_out=s["dq_out"], k_out=s["dk_out"])
            out.update({n: s[n + "_out"] for n in ("dq", "dk")})
        return out
    cache = s["cache"]
    if kind == "weigh":
        mw.mw_kvpages_weigh(cache, s["seqs"], s["q"], s["lse"], s["weights"], add=False, workspace=s["ws"])
        return {"weights": s["weights"]}
    n = case["n"]
    mw.mw_kvpages_free(cache, s["seqs"])
    for i in range(n):
        mw.mw_kvpages_fork(cache, i, n + i)
    s["weights"][n:] = s["weights"][:n]
    mw.mw_kvpages_evict_weighted(cache, s["seqs"], s["weights"], case["keep"], first=case["first"], recent=case["recent"],
                                 workspace=s["ws"])
    return {"k_pages": cache.k_pages.view(torch.float8_e4m3fn), "v_pages": cache.v_pages.view(torch.float8_e4m3fn),
            "k_scales": cache.k_scales, "v_scales": cache.v_scales, "table": cache.table, "lens": cache.lens,
            "weights": s["weights"]}


def run(s):
    if own:
        return _run_own(s)
    return {"packed": _plain_packed, "train": _plain_packed, "rope": _plain_rope, "turn": _plain_rope, "weigh": _plain_weigh,
            "evict": _plain_evict}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------- its work

def _visible(nq, nk, L):
    """Visible pairs of one sequence and head: row at place p sees min(nk, (p // L + 1) L) keys."""
    full = lambda p: (lambda c, r: L * L * c * (c + 1) // 2 + r * L * (c + 1))(p // L, p % L)  # places 0..p-1, no end
    lo, hi = max(0, nk - nq), nk
    edge = (nk - 1) // L * L if nk else 0  # from here on a row sees all keys
    return (full(min(hi, edge)) - full(min(lo, edge))) + nk * (hi - max(lo, edge))


def work(case):
    D, kind = case["D"], case["kind"]
    if kind in ("packed", "train"):
        H, Hkv = case["H"], case["Hkv"]
        nk, nq = _lens(case)
        pairs = H * sum(_visible(a, b, case["chunk"]) for a, b in zip(nq, nk))
        n_q, n_k = H * sum(nq), Hkv * sum(nk)
        if kind == "packed":  # q, k, v in, o and lse out
            return {"bytes": n_q * (4 * D + 4) + n_k * 4 * D, "flops": 4 * D * pairs}
        # forward as above; backward: q, o, do, lse, k, v in, dq, dk, dv out
        return {"bytes": n_q * (12 * D + 8) + n_k * 12 * D, "flops": 14 * D * pairs}
    if kind in ("rope", "turn"):
        n = (2 if kind == "turn" else 1) * case["B"] * case["T"] * (case["H"] + case["Hkv"])
        return {"bytes": n * 4 * D, "flops": 3 * n * sum(b[1] for b in _bands(case))}
    lens = _cached_lens(case)
    if kind == "weigh":
        # codes and scales of the keys, q, lse in; the weights out
        return {"bytes": case["Hkv"] * sum(lens) * (D + 4 / BLOCK) + case["B"] * case["H"] * case["T"] * (2 * D + 4) + 4 * sum(lens),
                "flops": 2 * D * case["H"] * case["T"] * sum(lens)}
    moved = case["keep"] - case["first"] // case["L"] * case["L"]
    # the weights read and written, the kept tokens' codes read and written
    return {"bytes": sum(8 * n for n in lens) + case["n"] * moved * case["H"] * 4 * D, "flops": 0}


# ------------------------------------------------------------------------------- 64-bit values

def _exact_packed(case, x):
    H, Hkv, D, L = case["H"], case["Hkv"], case["D"], case["chunk"]
    G, scale = H // Hkv, D ** -0.5
    nk, nq = _lens(case)
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)
    out = {"o": new(sum(nq), H, D), "lse": new(H, sum(nq))}
    train = case["kind"] == "train"
    if train:
        out.update(dq=new(sum(nq), H, D), dk=new(sum(nk), Hkv, D), dv=new(sum(nk), Hkv, D))
    q0 = k0 = 0
    for mq, mk in zip(nq, nk):
        for h in range(H):
            k, v = x["k"][k0:k0 + mk, h // G].double(), x["v"][k0:k0 + mk, h // G].double()
            for r in range(0, mq, 4096):
                n = min(4096, mq - r)
                i = slice(q0 + r, q0 + r + n)
                place = torch.arange(r, r + n, device=DEV) + (mk - mq)
                sees = torch.where(place < 0, 0, torch.clamp((torch.div(place, L, rounding_mode="floor") + 1) * L, max=mk))
                top = int(sees.max())
                q = x["q"][i, h].double()
                s = (q @ k[:top].t()) * scale
                s[torch.arange(top, device=DEV)[None] >= sees[:, None]] = -math.inf
                lse = torch.logsumexp(s, -1) if top else torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
                p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
                o = p @ v[:top]
                out["o"][i, h], out["lse"][h, i] = o, lse
                if train and top:
                    do = x["do"][i, h].double()
                    ds = p * (do @ v[:top].t() - (do * o).sum(1)[:, None])
                    out["dq"][i, h] = scale * (ds @ k[:top])
                    out["dk"][k0:k0 + top, h // G] += scale * (ds.t() @ q)
                    out["dv"][k0:k0 + top, h // G] += p.t() @ do
        q0, k0 = q0 + mq, k0 + mk
    return out


def _exact_rope(case, x):
    """Each pair as a complex number times that of its angle."""
    out = {}
    for n in ("q", "k", "dq", "dk"):
        if n not in x:
            continue
        y = x[n].double()
        sign = -1.0 if n.startswith("d") else 1.0
        for a, d, base, axis, sc in _bands(case):
            pos = (x["pos"][axis] if case["form"] == "axes" else x["pos"]).double()
            band = y[..., a:a + d]
            z = band.unflatten(-1, (2, d // 2)).transpose(-1, -2) if _is_halves(case) else band.unflatten(-1, (d // 2, 2))
            z = torch.view_as_complex(z.contiguous())
            w = []
            for i in range(d // 2):
                f = float(base) ** (-2.0 * i / d)
                if sc is not None:
                    turns = sc[1] * f / (2.0 * math.pi)
                    r = min(1.0, max(0.0, (turns - sc[2]) / (sc[3] - sc[2]))) if sc[3] > sc[2] else 0.0
                    f = r * f + (1.0 - r) * f / sc[0]
                w.append(sign * f)
            t = pos[..., None] * torch.tensor(w, dtype=torch.float64, device=DEV)
            t = t[:, None] if t.dim() == 3 else t[None, None]
            z = torch.view_as_real(z * torch.polar(torch.full_like(t, _gain(case)), t))
            y[..., a:a + d] = (z.transpose(-1, -2) if _is_halves(case) else z).flatten(-2)
        out[n] = y
    return out


def _exact_codes(x):
    """What [H,T,D] tokens read as after one commit, in 64 bits: the nearest e4m3 multiples of a power of two
    for each 64 tokens and head.  Also those powers, [H, ceil(T / 64)]."""
    H, T, D = x.shape
    y = torch.nn.functional.pad(x.double(), (0, 0, 0, -T % BLOCK)).view(H, -1, BLOCK * D)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0))  # exact at powers of two times 1.75
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 224.0 * torch.exp2(e), e - 1, e)).clamp(-100, 100)
    y = (y / torch.exp2(e)).float().to(torch.float8_e4m3fn).double() * torch.exp2(e)
    return y.view(H, -1, D)[:, :T], torch.exp2(e).squeeze(-1)


def _exact_weigh(case, x):
    G, D, L = case["H"] // case["Hkv"], case["D"], case["L"]
    out = torch.zeros((case["B"], -(-case["len"] // L) * L), dtype=torch.float64, device=DEV)
    for b, n in enumerate(_cached_lens(case)):
        k, _ = _exact_codes(x["hist"][0][b, :, :n])
        for h in range(case["H"]):
            s = x["q"][b, h].double() @ k[h // G].t() * D ** -0.5
            out[b, :n] += torch.exp(s - x["lse"][b, h].double()[:, None]).sum(0)
    return {"weights": out}


def _exact_evict(case, x):
    n, L, H, D, keep = case["n"], case["L"], case["H"], case["D"], case["keep"]
    lens = _cached_lens(case)
    W = -(-case["len"] // L)
    w0, w1 = case["first"] // L, -(-keep // L)
    used = sum(-(-m // L) for m in lens)
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)
    out = {}
    P = used + n * (w1 - w0)
    for name in "kv":
        out[name + "_pages"], out[name + "_scales"] = new(P, H, L, D), new(P, H, L // BLOCK)
    weights = new(2 * n, W * L)
    weights[:n, :case["len"]] = x["weights"].double()
    weights[n:] = weights[:n]

    def put(name, page, tokens):
        """Values [H,t,D] into pages from `page` on; what they read as."""
        y, scale = _exact_codes(tokens)
        for c in range(scale.shape[1]):
            t = y[:, BLOCK * c:BLOCK * (c + 1)]
            p, at = page + BLOCK * c // L, BLOCK * c % L
            out[name + "_pages"][p, :, at:at + t.shape[1]] = t / scale[:, c, None, None]
            out[name + "_scales"][p, :, at // BLOCK] = scale[:, c]
        return y

    at, branch = 0, used
    for i, m in enumerate(lens):
        w = x["weights"][i, :m].tolist()
        order = sorted(range(case["first"], m - case["recent"]), key=lambda j: (-w[j], j))
        stay = sorted([*range(case["first"]), *order[:keep - case["first"] - case["recent"]], *range(m - case["recent"], m)])
        moved = torch.tensor(stay, device=DEV)[w0 * L:]
        for j, name in enumerate("kv"):
            values = put(name, at, x["hist"][j][i, :, :m])
            put(name, branch, values[:, moved])
        at += -(-m // L)
        branch += w1 - w0
        weights[n + i, :keep] = x["weights"][i, torch.tensor(stay, device=DEV)].double()
        weights[n + i, keep:m] = 0.0
    out.update(table=None, lens=None, weights=weights)
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    return {"packed": _exact_packed, "train": _exact_packed, "rope": _exact_rope, "turn": _exact_rope, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["kind"]](case, x)
