"""Results of a 4-bit pool against the float64 oracle, within what the kernel's arithmetic can lose.

With x a row's scores in the kernel and x* the exact ones, |x - x*| <= e, e = 2 D 2^-23
max_key sum_d |q_d k_d| / sqrt(D): D products summed in fp32, each step within 2^-23 where the
tensor core cuts off, twice that for the scale and the exponent.  The maximum goes over the
keys that there are, not over the largest magnitude of each dimension, so that at ordinary
values e is 3e-4 and a key that is lost or read twice shows as long as it has a thousandth of
the weight.  The log-sum-exp is within e + 2^-18 (the base-2 exponential and logarithm, sums of
up to 2^17 terms).  O = sum p v: a weight is rounded to f16, 2^-11 of it, and off by e in the
exponent, twice (once in the sum), so |O - O*| <= (2^-11 + 2 e + 2^-15) max |v|, 2^-15 for the
sums, and half a step of bf16 for the result, 2^-8 |O*|.
"""
import numpy as np
import torch

from oracle import kv4


def held(x):
    """bf16 rows as the values that a 4-bit pool holds them as (bf16 has them exactly)."""
    return torch.from_numpy(kv4.hold(x.double().cpu().numpy())).to(torch.bfloat16)


def attend(q, k, v):
    """Queries q [Hq, D] over k, v [n, Hkv, D] in float64: O, the log-sum-exp, e of each head and its largest |v|."""
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    Hq, D = q.shape
    g = Hq // k.shape[1]
    o, lse, e, vmax = np.empty((Hq, D)), np.empty(Hq), np.empty(Hq), np.empty(Hq)
    for kvh in range(k.shape[1]):
        kk, vv, rows = k[:, kvh], v[:, kvh], slice(kvh * g, kvh * g + g)
        x = q[rows] @ kk.T / np.sqrt(D)
        top = x.max(1, keepdims=True)
        w = np.exp(x - top)
        o[rows], lse[rows] = (w @ vv) / w.sum(1, keepdims=True), top[:, 0] + np.log(w.sum(1))
        e[rows] = 2 * D * 2.0 ** -23 / np.sqrt(D) * (np.abs(q[rows]) @ np.abs(kk).T).max(1)
        vmax[rows] = np.abs(vv).max()
    return o, lse, e, vmax


def beyond(o, lse, want):
    """How far o [Hq, D] and lse [Hq] are beyond their tolerances, by head (NaN: not a number)."""
    ro, rl, e, vmax = want
    over = np.abs(o - ro) - (2.0 ** -8 * np.abs(ro) + ((2.0 ** -11 + 2 * e + 2.0 ** -15) * vmax)[:, None])
    return over.max(1), np.abs(lse - rl) - (e + 2.0 ** -18 * np.maximum(1, np.abs(rl)))


def check(o, lse, q, contexts, what=""):
    """o [n, Hq, D], lse [n, Hq] of queries q [n, Hq, D], each over a context (k, v) of [m, Hkv, D]."""
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for i, (k, v) in enumerate(contexts):
        for name, over in zip(("O", "lse"), beyond(o[i], lse[i], attend(q[i], k, v))):
            bad = ~(over <= 0)
            assert not bad.any(), (f"{what} row {i}: {name} of heads {np.flatnonzero(bad).tolist()[:8]} beyond its "
                                   f"tolerance by up to {np.nanmax(over):.3e}")
