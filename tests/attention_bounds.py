"""64-bit values of softmax attention over an explicit mask, and how far bf16 kernels may be from them.

The bounds count roundings.  A kernel rounds the probabilities to bf16 before the product with V (at most
2^-8 relative each), and its result to bf16 (2^-8 of the value); scores, statistics and sums are held in 32
bits, for which 2^-12 relative of the probabilities is allowed (sums of at most 128 products of the scores,
2^-24 each, scaled by their magnitude, and the exponential).  The backward reads O and dO in bf16 for
Delta, rounds dS to bf16 and the gradients to bf16.
"""
import torch

HALF = 2.0 ** -8   # half a step of bf16, relative
FP32 = 2.0 ** -12  # what 32-bit scores and exponentials may move a probability by, relative


def attention64(q, k, v, hidden, scale, do=None):
    """q [R,D], k, v [M,D], hidden [R,M] (or broadcast): 64-bit o, lse and their bounds, with do [R,D] also the
    gradients and theirs, as a dict name -> (value, bound)."""
    q, k, v = q.double(), k.double(), v.double()
    hidden = hidden.expand(q.shape[0], k.shape[0])
    seen = ~hidden.all(0)  # keys that no row sees may hold anything
    k, v = (torch.where(seen[:, None], t, 0.0) for t in (k, v))
    s = (q @ k.t()) * scale
    s = s.masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == float("-inf"), 0.0, lse)[:, None])
    o = p @ v
    pv = p @ v.abs()
    top = (q.abs() @ k.abs().t()).amax(-1) * scale if k.shape[0] else torch.zeros_like(lse)
    out = {"o": (o, (HALF + FP32) * pv + HALF * o.abs() + 1e-30),
           "lse": (lse, 2.0 ** -20 * (1 + torch.where(lse.isfinite(), lse, 0.0).abs() + top))}
    if do is None:
        return out
    do = do.double()
    dp = do @ v.t()
    delta = (do * o).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    off_delta = (do.abs() * out["o"][1]).sum(-1, keepdim=True)
    off_dp = 2.0 ** -20 * (do.abs() @ v.abs().t())
    off_ds = p * (off_delta + off_dp) + (HALF + FP32) * ds.abs()
    dq, dk, dv = ds @ k * scale, ds.t() @ q * scale, p.t() @ do
    off_ds = off_ds * (1 + HALF)
    out["dq"] = (dq, scale * (off_ds @ k.abs()) + HALF * dq.abs() + 1e-30)
    out["dk"] = (dk, scale * (off_ds.t() @ q.abs()) + HALF * dk.abs() + 1e-30)
    out["dv"] = (dv, (HALF + FP32) * (p.t() @ do.abs()) + HALF * dv.abs() + 1e-30)
    return out


def check(name, got, want, bound):
    """Every element within its bound; infinities equal."""
    got, want = got.double(), want.double()
    fine = want.isfinite()
    assert torch.equal(got[~fine], want[~fine]), f"{name}: non-finite values differ"
    assert bool(got[fine].isfinite().all()), f"{name}: non-finite values"
    over = ((got - want).abs() / bound)[fine]
    worst = float(over.max()) if over.numel() else 0.0
    print(f"[bound] {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.3f} times the bound"
