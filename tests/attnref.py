"""Plain 64-bit forms of the attention calls on the CPU, written from their
formulas, and the error bounds that the GPU results have to meet.

Bounds, for D channels, fp32 arithmetic (unit 2^-24) and BF16 roundings (8
significant bits: 1 + 2^-8 lies half way between its neighbours, unit 2^-8):
  * a score is a sum of D products, each exact in fp32 up to its rounding, so
    its error is at most E = D 2^-23 max_j |scale| sum_d |q_d k_jd| (the factor
    2 covers the scaling and the exponent's rounding);
  * a softmax weight carries a relative error of 2 E (its own and the sum's)
    and 2^-8 from its rounding to BF16; with A = sum p |v| / sum p, the output
    is off by at most (2 E + 2^-8) A and its own rounding, 2^-8 of it (at most A);
  * so |out - exact| <= (2^-7 (1 + 2^-6) + 4 E) A, the slack for the second order;
  * |lse - exact| <= 2 E + 2^-20 (1 + |lse|): the exponential and logarithm of
    the hardware are good to a few units;
  * a rotated channel is two products and a sum, then one rounding to BF16:
    2^-8 |exact| (1 + 2^-6) + 2^-21 (|a cos| + |b sin|).
"""
from __future__ import annotations

import math

import torch


def attend(q, K, V, scale, first=None, last=None):
    """q [n, D], K, V [t, D] (any type): query i over keys first[i] <= j <=
    last[i].  Returns out, lse, the bound of out and the bound of lse."""
    q, K, V = q.double(), K.double(), V.double()
    n, D = q.shape
    out = torch.zeros(n, D, dtype=torch.float64)
    lse = torch.full((n,), -math.inf, dtype=torch.float64)
    tol = torch.zeros(n, D, dtype=torch.float64)
    tol_lse = torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        lo = 0 if first is None else int(first[i])
        hi = K.shape[0] if last is None else int(last[i]) + 1
        if hi <= lo:
            continue
        k, v = K[lo:hi], V[lo:hi]
        s = (k @ q[i]) * scale
        p = torch.softmax(s, 0)
        out[i] = p @ v
        lse[i] = torch.logsumexp(s, 0)
        E = D * 2.0 ** -23 * abs(scale) * float((k.abs() @ q[i].abs()).max())
        tol[i] = (2.0 ** -7 * (1 + 2.0 ** -6) + 4 * E) * (p @ v.abs())
        tol_lse[i] = 2 * E + 2.0 ** -20 * (1 + abs(float(lse[i])))
    return out, lse, tol, tol_lse


def assert_close(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    same_inf = torch.isinf(want) & (got == want)
    err = torch.where(same_inf, torch.zeros_like(want), (got - want).abs())
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} off, worst {float((err / tol.clamp_min(1e-300))[bad].max()):.3g} of the bound"


def rotate(x, cos, sin, interleaved):
    """x [heads, D], cos, sin [rot / 2] of one token: the rotated rows and their bound."""
    x, cos, sin = x.double(), cos.double(), sin.double()
    half = cos.numel()
    y, mag = x.clone(), torch.zeros_like(x)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[:, a] = x[:, a] * cos[i] - x[:, b] * sin[i]
        y[:, b] = x[:, b] * cos[i] + x[:, a] * sin[i]
        mag[:, a] = (x[:, a] * cos[i]).abs() + (x[:, b] * sin[i]).abs()
        mag[:, b] = (x[:, b] * cos[i]).abs() + (x[:, a] * sin[i]).abs()
    return y, y.abs() * 2.0 ** -8 * (1 + 2.0 ** -6) + 2.0 ** -21 * mag


def table(max_pos, half, base=1e4):
    a = torch.arange(max_pos, dtype=torch.float64).view(-1, 1) * base ** (-torch.arange(half, dtype=torch.float64) / half)
    return a.cos().float(), a.sin().float()
