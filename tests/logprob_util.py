"""Plain 64-bit implementations of gk_vocab_logprob and gk_vocab_logprob_grad, and the bounds that the tests hold
the kernels to.

Bounds, from the arithmetic (u = 2^-24; y = z / T; m the row's maximum):
  * a power 2^d of the pass, d = (z - m) log2(e) / T: the difference, the product and log2(e) / T are each rounded,
    3 u |d| log 2 in the exponent, and the power itself is off by 4 u at most: with |d| <= 30 for every power that shows
    (2^-30 and less together are below 2^-13 of the sum for any V here, and off by less than 200 u of themselves),
    a sum is off by at most (3 x 21 + 4) u of itself plus that of adding: a thread adds N <= 100 terms in each half of
    a pair, each addition off by u of the sum so far, which is half of the last one on average: 50 u; the halves, lanes,
    warps and CTAs after: 10 u.  S_TOL = 128 u covers a sum of terms of one sign;
  * lse: log S0 by S_TOL absolute, its own rounding and that of m / T and the sum: 3 u of the larger;
  * logp = (z - m) / T - log S0: the difference rounded once, so 3 u of |(z - m) / T| instead;
  * entropy = log S0 - log 2 S1 / S0: S_TOL + 2 S_TOL |S1 / S0| log 2 <= S_TOL (1 + 2 H), and 4 u (1 + H);
  * a gradient: p from y - lse, where lse is a given fp32 number: y - lse off by 2 u |y - lse| (the product with both
    parts of 1 / T is exact but for its rounding, which is of the result), the exponent's product 2 u more, so p by
    (3 |y - lse| + 4) u; the factor k0 + k1 log p: three roundings of its terms.  The sum with a token's own a:
    two roundings of the result.  Then the output type's half step.
The logits' type shows nowhere: its values are exact in fp32."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
S_TOL = 128 * U


def reference(z, token, T, k):
    """lse, logp, entropy, rank, idx, val of rows z (any type, CPU) in 64 bits; token (n, m) or None."""
    n, V = z.shape
    y = z.double() / T
    top = y.max(1, keepdim=True).values
    nan = torch.isnan(y).any(1)
    none, inf = (top[:, 0] == -math.inf) & ~nan, (top[:, 0] == math.inf) & ~nan
    # relative to the maximum: next to the types' largest and lowest values 64 bits do not hold log V either
    ref = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    log_sum = torch.logsumexp(y - ref, 1)
    lse = log_sum + ref[:, 0]
    lse = torch.where(nan, torch.full_like(lse, math.nan), torch.where(inf, torch.full_like(lse, math.inf), lse))
    logp = y - ref - torch.where(none, torch.zeros_like(lse), torch.where(nan | inf, lse, log_sum))[:, None]
    p = torch.exp(logp)
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    h = torch.where(none, torch.zeros_like(h), torch.where(nan | inf, torch.full_like(h, math.nan), h))
    out = {"lse": lse, "entropy": h, "all": logp}
    key = torch.where(torch.isnan(z), torch.full_like(z, math.inf), z).double()
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    is_nan = torch.isnan(z).gather(1, order)
    order = order.gather(1, torch.sort(is_nan.to(torch.int8), dim=1, descending=True, stable=True).indices)
    place = torch.empty_like(order).scatter_(1, order, torch.arange(V).expand(n, V).contiguous())
    out["idx"], out["val"] = order[:, :k], logp.gather(1, order[:, :k])
    on = torch.ones(n, dtype=torch.bool)
    out["rank"] = torch.full((n,), -1)
    if token is not None:
        ok = (token >= 0) & (token < V)
        on = ok.any(1)
        at = token.clamp(0, V - 1)
        out["logp"] = torch.where(ok, logp.gather(1, at), torch.zeros(()).double())
        out["rank"] = torch.where(ok[:, 0], place.gather(1, at[:, :1])[:, 0], out["rank"])
    out["on"] = on
    for name, gone in (("lse", 0.0), ("entropy", 0.0), ("idx", -1), ("val", 0.0), ("rank", -1)):
        x = out[name]
        out[name] = torch.where(on if x.dim() == 1 else on[:, None], x, torch.full_like(x, gone))
    return out


def close(got, want, tol):
    """Equal where not finite, within tol elsewhere."""
    got, want = got.cpu().double(), want.double()
    fin = torch.isfinite(want)
    same = torch.isnan(got) == torch.isnan(want)
    inf = ~fin & ~torch.isnan(want)
    return bool(same.all()) and bool((got[inf] == want[inf]).all()) and bool(((got - want).abs() <= tol)[fin].all())


def bounds(z, ref, T):
    y = torch.where(torch.isfinite(z), z, torch.zeros_like(z)).double().abs().max(1).values / T
    h = torch.where(torch.isfinite(ref["entropy"]), ref["entropy"], torch.zeros_like(ref["entropy"]))
    return {"lse": S_TOL + 3 * U * (y + math.log(z.shape[1]) + 1), "entropy": (S_TOL + 4 * U) * (1 + 2 * h)}


def logp_tol(logp):
    fin = torch.where(torch.isfinite(logp), logp, torch.zeros_like(logp))
    return S_TOL + 6 * U * (1 + fin.abs())


def grad_reference(z, token, T, lse, entropy, a, b, c):
    """(dz, tolerance before the rounding to the logits' type) in 64 bits, with the given lse and entropy."""
    n, V = z.shape
    y = z.double() / T - lse.double()[:, None]
    p = torch.exp(y)
    on = torch.ones(n, dtype=torch.bool)
    total = torch.zeros(n, 1).double()
    hard = torch.zeros(n, V).double()
    size = torch.zeros(n, V).double()
    if token is not None:
        ok = (token >= 0) & (token < V)
        on = ok.any(1)
        if a is not None:
            g = torch.where(ok, a.double(), torch.zeros(()).double())
            total = g.sum(1, keepdim=True)
            hard.scatter_add_(1, token.clamp(0, V - 1), g)
            size.scatter_add_(1, token.clamp(0, V - 1), g.abs())
            m = token.shape[1]
            spread = g.abs().sum(1, keepdim=True) * (1 + m)
        else:
            spread = total
    else:
        spread = total
    k0, big = -total, spread + total.abs()
    if c is not None:
        k0 = k0 + c.double()[:, None]
        big = big + c.double().abs()[:, None]
    logp = torch.where(p > 0, y, torch.zeros_like(y))
    if b is not None:
        k0 = k0 - b.double()[:, None] * entropy.double()[:, None]
        big = big + (b.double() * entropy.double()).abs()[:, None]
        k1 = -b.double()[:, None]
    else:
        k1 = torch.zeros(n, 1).double()
    dz = (p * (k0 + k1 * logp) + hard) / T
    on = on & ~(lse < -1e30)
    dz = torch.where(on[:, None], dz, torch.zeros_like(dz))
    factor = (k0 + k1 * logp).abs()
    tol = (p * factor * (3 * logp.abs() + 6) * U + p * (big + (k1 * logp).abs()) * 6 * U + size * 6 * U) / T
    return dz, torch.where(on[:, None], tol + dz.abs() * 2 * U, torch.zeros_like(tol))
