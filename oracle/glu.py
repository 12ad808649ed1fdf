"""Oracle gated feed-forward block m = silu(x Wg^T) * (x Wu^T), float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).  The backward is derived
by hand; the tests pin it with central finite differences.
"""
from __future__ import annotations

import numpy as np


def sigmoid(g):
    return 1.0 / (1.0 + np.exp(-g))


def forward(x, wg, wu):
    """(m, g, u)"""
    g, u = x @ wg.T, x @ wu.T
    return g * sigmoid(g) * u, g, u


def backward_act(g, u, dm):
    """(dg, du) of sum(m * dm)"""
    s = sigmoid(g)
    return dm * u * s * (1.0 + g * (1.0 - s)), dm * g * s


def backward(x, wg, wu, g, u, dm):
    """(dx, dwg, dwu) with the gate and up values g and u"""
    dg, du = backward_act(g, u, dm)
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x
