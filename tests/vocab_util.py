"""Plain 64-bit implementations of the vocabulary head's operators, and the bounds the GPU tests
hold the kernels to.

Bounds, derived from the arithmetic (u = 2^-8 for bf16 and 2^-11 for fp16, half a unit in the last
place relative to the value; sums of 16-bit products in fp32):
  * a logit: each of the D additions is off by at most 2^-23 of the partial sum, so
    |dz| <= D 2^-23 a with a = max_nv sum_i |h_ni w_vi| / T; the exponent's own arithmetic in
    fp32 adds 2^-22 of the largest |z|, |lse| or |t|;
  * lse is off by no more than the largest logit error, plus the sum's and logarithm's rounding:
    lse_tol = D 2^-23 a + 2^-20 (1 + max |z|, |lse|, |t|); a loss: 2 max(1, Q) lse_tol;
  * a logit gradient is rounded twice to 16 bits (the kept exponential, then the gradient), so it
    is off by 2 u (1 + u) of |g| (Q p + q) / T, plus 4 lse_tol of it from the exponent; fp16 rounds
    below its normal range in absolute steps: 2^-24 of the largest |g| Q / T covers both roundings;
  * dh = dz w inherits these through |w|, adds fp32 sums (V 2^-23, or the number of rows for dw, of
    the sum of magnitudes) and one rounding u of the result (2^-25 absolute at least for fp16).
"""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def head_reference(h, w, idx, q, logq, T, g):
    """loss, lse, dh, dw and the pieces the bounds need, in 64 bits.  idx, q, logq: (n, K) with q = 0
    for pairs that do not count; a row counts when g is not NaN-marked by the caller's `on` mask
    (rows that do not count have q = 0 throughout and are zeroed by the caller)."""
    hd, wd = h.double(), w.double()
    z = hd @ wd.t() / T
    lse = torch.logsumexp(z, 1)
    at = idx.long().clamp(0, w.shape[0] - 1)
    zt = torch.gather(z, 1, at)
    loss = torch.where(q > 0, q * (logq - zt + lse[:, None]), torch.zeros_like(q)).sum(1)
    p = torch.exp(z - lse[:, None])
    Q = q.sum(1, keepdim=True)
    hard = torch.zeros_like(p).scatter_add_(1, at, q)
    unit = (g / T)[:, None]
    dz = unit * (Q * p - hard)
    size = unit.abs() * (Q * p + hard)
    return {"z": z, "lse": lse, "loss": loss, "dz": dz, "size": size, "dh": dz @ wd, "dw": dz.t() @ hd,
            "peak": float((unit.abs() * Q).max()) if g.numel() else 0.0}


def bounds(h, w, ref, q, logq, T, dtype):
    u = U[dtype]
    n, D = h.shape
    V = w.shape[0]
    a = float((h.double().abs() @ w.double().abs().t()).max()) / T if n else 0.0
    big = max([1.0] + [float(x.abs().max()) for x in (ref["z"], ref["lse"], torch.where(q > 0, logq, torch.zeros_like(logq))) if x.numel()])
    lse_tol = D * 2.0 ** -23 * a + 2.0 ** -20 * (1.0 + big)
    Q = float(q.sum(1).max()) if n else 0.0
    dz_tol = (2 * u * (1 + u) + 4 * lse_tol) * ref["size"]
    if dtype == torch.float16:
        dz_tol = dz_tol + 2.0 ** -24 * ref["peak"]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133
    big_dz = ref["size"] + dz_tol
    wa, ha = w.double().abs(), h.double().abs()
    dh_tol = (dz_tol + V * 2.0 ** -23 * big_dz) @ wa
    dw_tol = (dz_tol + n * 2.0 ** -23 * big_dz).t() @ ha
    return {"lse": lse_tol, "loss": 2 * max(1.0, Q) * lse_tol,
            "dh": dh_tol + u * (ref["dh"].abs() + dh_tol) + tiny, "dw": dw_tol + u * (ref["dw"].abs() + dw_tol) + tiny}


def topk_reference(logits, k):
    """Indices (ascending) of the k largest of each row, ties to the lower index, NaN on top."""
    v = logits.double()
    key = torch.where(torch.isnan(v), torch.full_like(v, math.inf), v)
    # NaN above +inf: a second, more significant key
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    nan = torch.isnan(v).gather(1, order)
    order = order.gather(1, torch.sort(nan.to(torch.int8), dim=1, descending=True, stable=True).indices)
    return torch.sort(order[:, :k], dim=1).values
