"""Rotary positions against 64-bit values: bands, layouts, scalings, positions, strides, in place, and the inverse."""
import math

import pytest

pytestmark = pytest.mark.gpu

FORMS = {
    "interleaved": lambda D: ([dict(dim_offset=0, dim_count=D)], False, 1.0),
    "halves": lambda D: ([dict(dim_offset=0, dim_count=D, theta=5e5, factor=8.0, trained_len=8192.0, turns_lo=1.0, turns_hi=32.0)],
                         True, 0.1 * math.log(8.0) + 1.0),
    "part": lambda D: ([dict(dim_offset=D // 4 * 2 - 16, dim_count=D // 2, factor=4.0)], True, 1.0),
    "odd halves": lambda D: ([dict(dim_offset=2, dim_count=22), dict(dim_offset=24, dim_count=6, axis=1)], True, 1.0),
    "axes": lambda D: ([dict(dim_offset=0, dim_count=D - 4 * (D // 6)), dict(dim_offset=D - 4 * (D // 6), dim_count=2 * (D // 6), axis=1),
                        dict(dim_offset=D - 2 * (D // 6), dim_count=2 * (D // 6), axis=2, theta=100.0)], False, 1.0),
    "axes halves": lambda D: ([dict(dim_offset=0, dim_count=D - 4 * (D // 6)),
                               dict(dim_offset=D - 4 * (D // 6), dim_count=2 * (D // 6), axis=1),
                               dict(dim_offset=D - 2 * (D // 6), dim_count=2 * (D // 6), axis=2)], True, 0.5),
}


def randn(shape, seed, layout="bhtd"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, T, D = shape
    if layout == "bhtd":
        return torch.randn(B, H, T, D, device="cuda", generator=g).bfloat16()
    if layout == "bthd":
        return torch.randn(B, T, H, D, device="cuda", generator=g).bfloat16().transpose(1, 2)
    return torch.randn(B, T, H, D + 8, device="cuda", generator=g).bfloat16()[..., :D].transpose(1, 2)


def want64(x, bands, halves, gain, pos, inverse=False):
    """64-bit values and how far bf16 outputs may be off: half a step (2^-8 of the value at most), and what 32-bit sines,
    cosines and products may move (2^-21 of the pair's magnitudes: a fraction of a turn in 32 bits, 2 pi 2^-26 absolute,
    the functions' and three products' roundings, 2^-23 each at most)."""
    import torch
    x = x.double()
    y, off = x.clone(), torch.zeros_like(x)
    for b in bands:
        a, n = b["dim_offset"], b["dim_count"]
        i = torch.arange(n // 2, device=x.device, dtype=torch.float64)
        f = b.get("theta", 1e4) ** (-2 * i / n)
        s = b.get("factor", 1.0)
        if s != 1.0:
            lo, hi = b.get("turns_lo", 0.0), b.get("turns_hi", 0.0)
            r = ((b["trained_len"] * f / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1) if hi > lo else 0.0
            f = f * (r + (1 - r) / s)
        p = pos[b.get("axis", 0)].double()
        t = p[..., None] * f * (-1 if inverse else 1)
        t = t[:, None] if t.dim() == 3 else t[None, None]
        e = torch.arange(n // 2, device=x.device)
        u, w = (a + e, a + n // 2 + e) if halves else (a + 2 * e, a + 2 * e + 1)
        xu, xw = x[..., u], x[..., w]
        y[..., u] = gain * (xu * t.cos() - xw * t.sin())
        y[..., w] = gain * (xw * t.cos() + xu * t.sin())
        big = abs(gain) * (xu.abs() + xw.abs()) * 2.0 ** -21
        # the position times the frequency in turns is rounded to 64 bits
        big = big + abs(gain) * (xu.abs() + xw.abs()) * (p.abs().max() * 2.0 ** -50)
        off[..., u] = off[..., w] = big
    bound = torch.where(off > 0, 2.0 ** -8 * y.abs() + off, 0.0)
    return y, bound


def verify(got, want):
    y, bound = want
    d = (got.double() - y).abs()
    assert bool((d <= bound).all()), float((d - bound).max())


def positions(axes, B, T, kind, dtype, seed=5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = ((axes,) if axes > 1 else ()) + ((B, T) if kind == "members" else (T,))
    top = 2 ** 31 - 1 if kind == "members" else 5000
    return torch.randint(-top if kind == "members" else 0, top, shape, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("kind,dtype", [("shared", "int32"), ("members", "int64")])
def test_forms_and_positions(mw, D, form, kind, dtype):
    import torch
    bands, halves, gain = FORMS[form](D)
    axes = 1 + max(b.get("axis", 0) for b in bands)
    rb = mw.rope_bands(bands, halves=halves, gain=gain)
    for B, H, Hkv, T, layout in ((1, 1, 1, 1, "bhtd"), (2, 3, 1, 37, "bthd"), (3, 4, 2, 130, "gap"), (1, 16, 16, 5, "bhtd")):
        print(f"[case] rope {form} D={D} {kind} {B} {H} {Hkv} {T} {layout}", flush=True)
        q, k = randn((B, H, T, D), 1, layout), randn((B, Hkv, T, D), 2, layout)
        pos = positions(axes, B, T, kind, getattr(torch, dtype))
        rows = pos if axes > 1 else pos[None]
        for inverse in (False, True):
            qo, ko = mw.mw_rope_apply(q, k, rb, pos, inverse=inverse)
            torch.cuda.synchronize()
            verify(qo, want64(q, bands, halves, gain, rows, inverse))
            verify(ko, want64(k, bands, halves, gain, rows, inverse))


@pytest.mark.parametrize("form", list(FORMS))
def test_in_place_equals_out_of_place(mw, form):
    import torch
    D = 128
    bands, halves, gain = FORMS[form](D)
    axes = 1 + max(b.get("axis", 0) for b in bands)
    rb = mw.rope_bands(bands, halves=halves, gain=gain)
    for layout in ("bhtd", "bthd", "gap"):
        q, k = randn((2, 5, 300, D), 3, layout), randn((2, 3, 300, D), 4, layout)
        pos = positions(axes, 2, 300, "shared", torch.int64)
        qo, ko = mw.mw_rope_apply(q, k, rb, pos)
        q_, k_ = randn((2, 5, 300, D), 3, layout), randn((2, 3, 300, D), 4, layout)
        mw.mw_rope_apply(q_, k_, rb, pos, q_out=q_, k_out=k_)
        one, none = mw.mw_rope_apply(q, None, rb, pos)
        torch.cuda.synchronize()
        assert torch.equal(q_, qo) and torch.equal(k_, ko) and torch.equal(one, qo) and none is None


def test_positions_by_number(mw):
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=64)])
    q, k = randn((2, 3, 50, 64), 5), randn((2, 1, 50, 64), 6)
    a = mw.mw_rope_apply(q, k, rb, first=1234567)
    b = mw.mw_rope_apply(q, k, rb, torch.arange(1234567, 1234617, device="cuda"))
    c = mw.mw_rope_apply(q, k, rb, first=0)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(c[0][:, :, 0], q[:, :, 0]) and not torch.equal(c[0][:, :, 1], q[:, :, 1])


def test_a_view_of_positions(mw):
    """Strided and expanded positions read as their copies."""
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=128)], halves=True)
    q = randn((3, 2, 40, 128), 7)
    pos = torch.randint(0, 9999, (40, 3), device="cuda")
    a = mw.mw_rope_apply(q, None, rb, pos.t())[0]
    b = mw.mw_rope_apply(q, None, rb, pos.t().contiguous())[0]
    c = mw.mw_rope_apply(q, None, rb, pos[:, 0].expand(3, 40))[0]
    d = mw.mw_rope_apply(q, None, rb, pos[:, 0].contiguous())[0]
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(c, d)


def test_outputs_stay_within_their_views(mw):
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=44)], halves=True)
    q, k = randn((2, 2, 33, 72), 8), randn((2, 1, 33, 72), 9)
    wide = [torch.full((2, h, 36, 80), 7.0, device="cuda", dtype=torch.bfloat16) for h in (2, 1)]
    cut = [w[:, :, :33, :72] for w in wide]
    mw.mw_rope_apply(q, k, rb, q_out=cut[0], k_out=cut[1])
    torch.cuda.synchronize()
    for w, c, x in zip(wide, cut, (q, k)):
        assert bool((w[..., 72:] == 7).all()) and bool((w[:, :, 33:] == 7).all())
        assert torch.equal(c[..., 44:], x[..., 44:])


def test_gradient_is_the_transpose(mw):
    """The map is linear: sum(g R x) = sum(x R^T g), and differences along random directions are the map itself."""
    import torch
    for form in FORMS:
        bands, halves, gain = FORMS[form](128)
        axes = 1 + max(b.get("axis", 0) for b in bands)
        rb = mw.rope_bands(bands, halves=halves, gain=gain)
        pos = positions(axes, 2, 60, "shared", torch.int32)
        rows = pos if axes > 1 else pos[None]
        x, g, u = (randn((2, 3, 60, 128), 20 + i) for i in range(3))
        grad = mw.mw_rope_apply(g, None, rb, pos, inverse=True)[0].double()
        loss = lambda t: (want64(t, bands, halves, gain, rows)[0] * g.double()).sum()
        h = 2.0 ** -10
        slope = float(loss(x.double() + h * u.double()) - loss(x.double() - h * u.double())) / (2 * h)
        got = float((grad * u.double()).sum())
        off = 2.0 ** -8 * float((grad * u.double()).norm()) * 4  # roundings of independent terms, four deviations
        assert abs(got - slope) <= off, (form, got, slope, off)


def test_cached_keys_shifted_are_keys_at_the_earlier_position(mw):
    """Keys turned to position p, committed to the ring and re-shifted by n, are the keys at p - n: two roundings apart."""
    import torch
    B, H, L, D, n = 1, 2, 64, 128, 3
    side = 2 * (D // 6)
    band = dict(dim_offset=0, dim_count=D - 2 * side)
    rb = mw.rope_bands([band])
    k, v = randn((B, H, L, D), 30), randn((B, H, L, D), 31)
    cache = mw.KVCache(2, B, H, L, D)
    kp = mw.mw_rope_apply(k, None, rb, first=10)[0]
    mw.mw_kvcache_append(cache, kp, v)
    mw.mw_kvcache_rope_shift(cache, n, 0, D - 2 * side)
    direct = mw.mw_rope_apply(k, None, rb, first=10 - n)[0]
    torch.cuda.synchronize()
    pair = k.double().unflatten(-1, (D // 2, 2)).norm(dim=-1).repeat_interleave(2, -1)
    assert bool(((cache.k_slots[0].double() - direct.double()).abs() <= (2 + math.sqrt(2)) * 2.0 ** -8 * pair).all())


def test_long_and_wide(mw):
    import torch
    bands, halves, gain = FORMS["axes"](128)
    rb = mw.rope_bands(bands)
    T = 9001
    t = torch.arange(T, device="cuda")
    pos = torch.stack([t // 300, t % 300 // 20, t % 20])
    q, k = randn((1, 12, T, 128), 40, "bthd"), randn((1, 12, T, 128), 41, "bthd")
    qo, ko = mw.mw_rope_apply(q, k, rb, pos)
    torch.cuda.synchronize()
    verify(qo, want64(q, bands, halves, gain, pos))
    verify(ko, want64(k, bands, halves, gain, pos))


@pytest.mark.parametrize("form", ["interleaved", "halves", "odd halves", "part"])
@pytest.mark.parametrize("H,Hkv", [(61, 7), (60, 1), (1, 62), (64, 0)])
def test_tokens_of_many_heads_in_a_row(mw, form, H, Hkv):
    """Heads in groups, of which the last ones may hold none of q or of k, and the last block fewer tokens."""
    import torch
    B, T, D = 2, 8197, 72
    bands, halves, gain = FORMS[form](D)
    axes = 1 + max(b.get("axis", 0) for b in bands)
    rb = mw.rope_bands(bands, halves=halves, gain=gain)
    q, k = randn((B, H, T, D), 50), randn((B, Hkv, T, D), 51) if Hkv else None
    pos = positions(axes, B, T, "members", torch.int64)
    rows = pos if axes > 1 else pos[None]
    qo, ko = mw.mw_rope_apply(q, k, rb, pos)
    torch.cuda.synchronize()
    for x, y in ((q, qo), (k, ko)):
        if x is not None:
            for b in range(B):
                verify(y[b:b + 1], want64(x[b:b + 1], bands, halves, gain, rows[:, b:b + 1]))
    mw.mw_rope_apply(q, k, rb, pos, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(q, qo) and (k is None or torch.equal(k, ko))


@pytest.mark.parametrize("D", [64, 72])
def test_heads_of_another_order_and_far_apart(mw, D):
    """q by head, k by token; heads whose distance passes 32 bits of bytes."""
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=D)], halves=True)
    B, H, T = 1, 3, 1000
    q, k = randn((B, H, T, D), 52), randn((B, 2, T, D), 53, "bthd")
    qo, ko = mw.mw_rope_apply(q, k, rb)
    far = torch.empty(2 * (1 << 31) + T * D, dtype=torch.bfloat16, device="cuda").as_strided((B, H, T, D), (0, 1 << 31, D, 1))
    far.copy_(q)
    out = torch.empty_like(q)
    mw.mw_rope_apply(far, k, rb, q_out=out)
    mw.mw_rope_apply(q, k, rb, q_out=far)
    torch.cuda.synchronize()
    bands = [dict(dim_offset=0, dim_count=D)]
    pos = torch.arange(T, device="cuda")[None]
    verify(qo, want64(q, bands, True, 1.0, pos))
    verify(ko, want64(k, bands, True, 1.0, pos))
    assert torch.equal(out, qo) and torch.equal(far, qo)


def test_side_stream_and_graph_replays(mw):
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=128)], halves=True)
    q, k = (torch.empty((2, h, 70, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    pos = torch.zeros((2, 70), dtype=torch.int64, device="cuda")
    out = [torch.empty_like(q), torch.empty_like(k)]

    def load(seed):
        q.copy_(randn(tuple(q.shape), seed))
        k.copy_(randn(tuple(k.shape), seed + 1))
        pos.copy_(torch.arange(140).view(2, 70) * seed)

    load(3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mw.mw_rope_apply(q, k, rb, pos, q_out=out[0], k_out=out[1])
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mw.mw_rope_apply(q, k, rb, pos, q_out=out[0], k_out=out[1])
    for seed in (5, 77, 1001):
        load(seed)
        for t in out:
            t.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, mw.mw_rope_apply(q, k, rb, pos)):
            assert torch.equal(a, b)


def test_refusals_of_the_binding(mw):
    import torch
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=64)])
    q, k = randn((2, 3, 50, 64), 5), randn((2, 1, 50, 64), 6)
    with pytest.raises(TypeError):
        mw.mw_rope_apply(q.float(), k, rb)
    for bad in (k[:1], k[:, :, :49], k.cpu()):
        with pytest.raises(ValueError):
            mw.mw_rope_apply(q, bad, rb)
    for bad in (torch.zeros(49, dtype=torch.int64, device="cuda"), torch.zeros(50, device="cuda"), torch.zeros(50, dtype=torch.int64),
                torch.zeros((1, 2, 50), dtype=torch.int64, device="cuda")):
        with pytest.raises(ValueError):
            mw.mw_rope_apply(q, k, rb, bad)
    with pytest.raises(mw.MWError):
        mw.mw_rope_apply(q, k, mw.rope_bands([dict(dim_offset=0, dim_count=66)]))
    two = mw.rope_bands([dict(dim_offset=0, dim_count=32), dict(dim_offset=32, dim_count=32, axis=1)])
    with pytest.raises(mw.MWError):
        mw.mw_rope_apply(q, k, two)
    with pytest.raises(mw.MWError):  # an output in its input's place, with other strides
        mw.mw_rope_apply(q, k, rb, q_out=q.as_strided(q.shape, (9600, 64, 192, 1)))


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("factor", [1.0, 8.0])
def test_far_positions(mw, halves, factor):
    """Positions beyond 2^31 against angles of 60 digits: off by |position| 2^-50 radians at most (the roundings of the exponent, the
    power, 2 pi, the position and the product with it, 2^-53 of the angle each and 2^-52 for the power), and 2^-21 for the 32-bit part."""
    import torch
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    D, H = 64, 3
    pos = [0, 1, -1, 2**31 - 1, 2**31, -2**31 - 1, 2**32 + 12345, 10**10 + 7, -(10**11) - 3, 2**38 + 1, -2**40 + 1, 2**40 + 987654321]
    f = [Decimal(10000) ** (Decimal(-2 * i) / D) / Decimal(factor) for i in range(D // 2)]
    angle = torch.tensor([[float((p * x) % (2 * pi)) for x in f] for p in pos], dtype=torch.float64)
    x = randn((1, H, len(pos), D), 70)
    rb = mw.rope_bands([dict(dim_offset=0, dim_count=D, factor=factor)], halves=halves)
    p = torch.tensor(pos, device="cuda")
    got = mw.mw_rope_apply(x, None, rb, p)[0]
    one = torch.stack([mw.mw_rope_apply(x[:, :, i:i + 1], None, rb, first=n)[0][:, :, 0] for i, n in enumerate(pos)], 2)
    torch.cuda.synchronize()
    assert torch.equal(got, one)
    c, s = angle.cos().cuda(), angle.sin().cuda()
    e = torch.arange(D // 2, device="cuda")
    a, b = (e, e + D // 2) if halves else (2 * e, 2 * e + 1)
    xa, xb = x.double()[..., a], x.double()[..., b]
    off = (xa.abs() + xb.abs()) * (2.0 ** -21 + p.double().abs()[:, None] * 2.0 ** -50)
    for at, y in ((a, xa * c - xb * s), (b, xb * c + xa * s)):
        assert bool(((got.double()[..., at] - y).abs() <= 2.0 ** -8 * y.abs() + off).all())


@pytest.mark.parametrize("form", ["interleaved", "halves", "odd halves"])
@pytest.mark.parametrize("B,H,Hkv,T,layout", [(1, 16384, 3, 2, "bhtd"), (2, 5, 16384, 3, "bthd"), (70000, 2, 1, 1, "bhtd"),
                                              (1, 3000, 3000, 17, "bhtd")])
def test_many_heads_and_members(mw, form, B, H, Hkv, T, layout):
    import torch
    D = 72
    bands, halves, gain = FORMS[form](D)
    axes = 1 + max(b.get("axis", 0) for b in bands)
    rb = mw.rope_bands(bands, halves=halves, gain=gain)
    q, k = randn((B, H, T, D), 60, layout), randn((B, Hkv, T, D), 61, layout)
    pos = positions(axes, B, T, "members", torch.int32)
    qo, ko = mw.mw_rope_apply(q, k, rb, pos)
    torch.cuda.synchronize()
    rows = pos if axes > 1 else pos[None]
    verify(qo, want64(q, bands, halves, gain, rows))
    verify(ko, want64(k, bands, halves, gain, rows))
