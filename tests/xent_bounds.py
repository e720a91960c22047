"""The cross entropy's gradients in 64 bits with a bound for each element.

With G = c dl (p - [v = y]) and d = c dl of a token, an element of G is off by

  its arithmetic: p = exp(z - lse) by dz (a logit's sum, D + 8 roundings of its terms' magnitudes), lse's 2^-19 and 2^-22 |lse|, the argument's rounding
  2^-22 |z - lse| and 2^-22 of the exponential, each relative to p, and 2^-22 of G for the factors;
  its rounding: up to 64 tokens the sum of two bfloat16 values, 2^-8 of 2^-8 = 2^-16 of it.  More tokens: 11 bits, 2^-11, and where it is small beside
  its row's largest, 1 - p_y, the spacing of the range's end: the row's largest is brought to 2^13 .. 2^14 (or up to twice beyond, 1 - p_y being known
  to rounding) and numbers end in steps of 2^-24: 2^-38 of 1 - p_y, four times that with room.  (Of what the logit at y may be off by, sqrt(D) roundings of its
  terms' magnitudes, where 1 - p_y is below that.)

For dW of more than 64 tokens the states times c dl and a power of two e (the one that 1 - p_y is brought by) are rounded to 11 bits too, with the same end of range
below the largest of all tokens' states: 2^-36 max |h e| of each, times G / e.  For dH the weights are exact, but for 2^-36 of the largest.  Sums are
off by 2^-24 (their length / 32 + 64) of their terms' magnitudes, bfloat16 outputs by 2^-8 more.
"""
import torch

from vocab_util import BF16, F64, HALF


def formula(h, w, y, dl, c):
    h, w, dl = h.to(F64), w.to(F64), dl.to(F64)
    T, V, D = h.shape[0], w.shape[0], h.shape[1]
    z = c * (h @ w.t())
    dz = c * (D + 8) * 2.0 ** -24 * (h.abs() @ w.abs().t()) + z.abs() * 2.0 ** -24
    lse = torch.logsumexp(z, 1, keepdim=True)
    ok = (y >= 0) & (y < V) & (dl != 0)
    at = torch.where(ok, y, torch.zeros_like(y)).long()[:, None]
    d = torch.where(ok, dl, 0.0)[:, None] * c
    p = (z - lse).exp()
    f = p.clone()
    f.scatter_add_(1, at, torch.full_like(lse, -1.0))
    arith = p * (dz + (p * dz).sum(1, keepdim=True) + 2.0 ** -19 + 2.0 ** -22 * (lse.abs() + (z - lse).abs() + 1)) + 2.0 ** -22 * f.abs()
    noise = 2.0 ** -24 * (D ** 0.5 * c * (h.abs() * w[at[:, 0]].abs()).sum(1, keepdim=True) + lse.abs() + 1)
    left = torch.maximum(-f.gather(1, at), noise)
    g, few = f * d, T <= 64
    rounding = f.abs() * (2.0 ** -16 if few else 2.0 ** -11) + (0.0 if few else 2.0 ** -36 * left)
    g_off = (arith + rounding) * d.abs()
    states, states_off = torch.where(ok[:, None], h, 0.0), torch.zeros_like(h)
    e = d.abs() * left
    if not few:
        most = (states.abs().amax(1, keepdim=True) * e).max()
        states_off = states.abs() * 2.0 ** -11 + torch.where(e > 0, 2.0 ** -36 * most / e.clamp(min=1e-300), 0.0)
    weights_off = 0.0 if few else 2.0 ** -36 * w.abs().max()
    sums = lambda n: 2.0 ** -24 * (n / 32 + 64)  # noqa: E731
    dh, dw = g @ w, g.t() @ states
    return {"dh": (dh, g_off @ (w.abs() + weights_off) + g.abs().sum(1, keepdim=True) * weights_off + (g.abs() @ w.abs()) * sums(V) + dh.abs() * HALF[BF16]),
            "dw": (dw, g_off.t() @ (states.abs() + states_off) + g.abs().t() @ states_off + (g.abs().t() @ states.abs()) * sums(T)), "g": g, "left": left}
