"""Orthogonalised updates, the optimizer step around them and AdamW in 64 bits, from their formulas."""
import math

import torch

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonal(u, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    a, b, c = coefficients
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    norm = x.norm() + eps
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * g @ g) @ x
    return x.t() if tall else x


def scale_of(scale, shape):
    return {0: 1.0, 1: math.sqrt(max(1.0, shape[0] / shape[1])), 2: 0.2 * math.sqrt(max(shape))}[scale]


def muon_step(g, m, x, *, lr, wd, mu=0.95, nesterov=True, scale=2, **kw):
    m = mu * m.double() + g.double()
    u = g.double() + mu * m if nesterov else m
    return m, x.double() - lr * (scale_of(scale, x.shape) * orthogonal(u, **kw) + wd * x.double())


def adamw_step(g, m, v, x, t, *, lr, wd, beta1=0.9, beta2=0.95, eps=1e-8):
    g = g.double()
    m = beta1 * m.double() + (1 - beta1) * g
    v = beta2 * v.double() + (1 - beta2) * g * g
    u = (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps)
    return m, v, x.double() - lr * (u + wd * x.double())


# Relative error of O (Frobenius norm) that the kernels' roundings explain.  Operands of the products have 11 bits, off by at most
# r = 2^-11.  Where singular values s have reached 0.7 .. 1.2, the polynomial's off-diagonal part F has |F| <= 1 (b s^2 + c s^4 varies by
# less), so one iteration adds at most r for F, r for X in F X, |b + 2 c d| r <= r for E and 2 c |E| r <= r for E^2: 4 r; the iteration
# before it passes on |p'(s)| <= 1.6 times its own 4 r, those before that grow and shrink to its size: 4 r (1 + 1.6) and half as much.
# Matrices whose smaller side is at most 256 multiply with 22 bits: r is that of fp32 sums then, 2^-24 for each of up to sqrt(K) = 64
# steps of a sum in one direction.
def tolerance(shape):
    return 16 * 2.0 ** -11 if min(shape) > 256 else 16 * 64 * 2.0 ** -24
