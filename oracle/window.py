"""Oracle: causal attention through a sliding window with first tokens that stay
visible, and its error bound for a kernel that rounds its weights to bf16.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Definition: the row at position p sees the keys j <= p with j > p - W or j < n
(W = 0: all j <= p); x_j = scale q.k_j, LSE = ln sum e^{x_j}, O = sum e^{x_j - LSE}
v_j, in float64 from the exact bf16 inputs.  A row that sees no key has O = 0 and
LSE = -inf; keys it does not see have no part in it, whatever they hold.  (The
paper has no window; W = 0 is the attention of its Sec. 2.1.)
"""

from __future__ import annotations

import math

import numpy as np


def attend(q, q_pos, k, v, k_pos, window=0, n_sink=0, scale=None):
    """q [n, Hq, D] at q_pos [n]; k, v [m, Hkv, D] at k_pos [m], float64.  Returns
    (O, LSE, A, S): A = sum e^{x_j - LSE} |v_j| and S = max_j scale sum |q_d k_jd|,
    the scales of the errors that rounded weights and rounded scores make."""
    n, Hq, D = q.shape
    m, Hkv, _ = k.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    o, a = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, s = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    p, j = np.asarray(q_pos)[:, None], np.asarray(k_pos)[None]
    sees = j <= p
    if window:
        sees = sees & ((j > p - window) | (j < n_sink))
    for i in range(n):
        at = np.nonzero(sees[i])[0]
        if not len(at):
            continue
        for h in range(Hq):
            kk, vv = k[at, h // (Hq // Hkv)], v[at, h // (Hq // Hkv)]
            x = scale * (kk @ q[i, h])
            lse[i, h] = x.max() + np.log(np.exp(x - x.max()).sum())
            w = np.exp(x - lse[i, h])
            o[i, h], a[i, h] = w @ vv, w @ np.abs(vv)
            s[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return o, lse, a, s


def bounds(o, lse, a, s, n_keys):
    """(on O, on LSE): how far a kernel may be off that accumulates in fp32, rounds
    each weight to bf16 once and O to bf16 as it stores it.

    A rounding to bf16 is off by at most 2^-8 of the value, to fp32 by 2^-24.
    Scores: 128 products and sums in fp32, 2^-24 each of at most S: delta = 2^-17 S,
    doubled for the exponent's own rounding.  Weights: relative 2^-8 + delta in the
    numerator, and as much in the sum that divides it: 2 (2^-8 + delta) A; O's own
    rounding 2^-8 |O|; 1 % for the second order.  The sum of n weights in fp32:
    relative n 2^-24 (and exp2's own few 2^-24)."""
    delta = 2.0**-16 * s
    on_o = 1.01 * (2 * (2.0**-8 + delta[..., None]) * a + 2.0**-8 * np.abs(o)) + 1e-30
    on_lse = delta + (n_keys + 64) * 2.0**-24 + 2.0**-22 * np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 1e-6
    return on_o, on_lse
