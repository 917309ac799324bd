"""Attention rows in 64 bits, with the bounds that a kernel's roundings allow (shared by the
tests of the packed prompts and of the 8-bit store)."""
import torch

U_OUT = 2.0 ** -8  # rounding to bf16: half a unit in the last of 8 bits


def attend64(q, k, v, seen, scale):
    """q [r, d], k, v [n, d] in 64 bits, row i sees the keys j < seen[i].  Returns o, lse, and per
    output sum_j p_j |v_j| and per row the largest sum_c |q_c k_c| * scale (both over seen keys)."""
    r, n = q.shape[0], k.shape[0]
    hid = torch.arange(n, device=q.device)[None] >= seen[:, None]
    any_seen = (seen > 0)[:, None]
    x = (scale * (q @ k.T)).masked_fill(hid, float("-inf"))
    mag = (scale * (q.abs() @ k.abs().T)).masked_fill(hid, 0.0).amax(1) if n else q.new_zeros(r)
    if n == 0:
        return torch.zeros_like(q), q.new_full((r,), float("-inf")), torch.zeros_like(q), mag
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(any_seen[:, 0], lse, torch.zeros_like(lse))[:, None])
    p = torch.where(any_seen, p, torch.zeros_like(p))
    return p @ v, lse, p @ v.abs(), mag


def check_rows(o, lse, want, u_weights, extra=0.0):
    """o (bf16), lse (fp32) of some rows against attend64's answer.  A logit is off by at most
    ex = 2^-20 of sum |q k| (fp32 sums of d <= 128 products, the exponential's 2^-22, the scales)
    plus `extra`; the normalised weights then by 4 ex relative, their rounding by u_weights, and
    o by U_OUT of itself at the end."""
    wo, wl, av, mag = want
    ex = 2.0 ** -20 * (1.0 + mag) + extra
    tol = U_OUT * wo.abs() + (u_weights + 4 * ex)[:, None] * av * (1 + U_OUT) + 1e-38
    err = (o.double() - wo).abs()
    assert bool((err <= tol).all()), f"o off by {float((err / tol).max())} of its bound"
    if lse is not None:
        fin = torch.isfinite(wl)
        assert torch.equal(torch.isneginf(lse), torch.isneginf(wl))
        el = (lse.double() - wl).abs()[fin]
        tl = (2 * ex + 2.0 ** -22 * wl.abs())[fin]
        assert bool((el <= tl).all()), f"lse off by {float((el / tl).max())} of its bound"
