"""Plain float64 NumPy oracle of the operators around the 8-bit products of an MLP (test infrastructure only): activations and their
derivatives, what ends a product, the gradient through it, a router, and a layer of experts. It shares no code with the HIP path or
with ``perf/more_operators.py``.

Definitions
-----------
* relu max(x, 0); gelu x Phi(x), Phi the normal distribution; gelu_tanh x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2; silu
  x / (1 + exp(-x)).
* Forward: z = X W^T + b, y = act(z) mul + residual. Backward, from dh = the gradient of act(u) mul: du = dh mul act'(u), dmul =
  dh act(u), db = the sum of du over the rows.
* Router: the k largest of softmax(X Wr^T) for each row, the lower expert first on equal ones, divided by their sum if asked.
* Experts: y_i = sum_j w_ij down_e(act(gate_e x_i) * (up_e x_i)), e = ids_ij; an index outside 0 .. E - 1 adds nothing.
"""
from __future__ import annotations

import numpy as np
from scipy import special

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_C = np.sqrt(2.0 / np.pi)


def value(act: str, x: np.ndarray) -> np.ndarray:
    if act == "none":
        return x * 1.0
    if act == "relu":
        return np.where(x < 0, 0.0, x)
    if act == "gelu":
        return x * special.ndtr(x)
    if act == "gelu_tanh":
        return x * special.expit(2 * _C * (x + 0.044715 * x ** 3))
    return x * special.expit(x)


def slope(act: str, x: np.ndarray) -> np.ndarray:
    if act == "none":
        return np.ones_like(x, dtype=np.float64)
    if act == "relu":
        return (x > 0) * 1.0
    if act == "gelu":
        return special.ndtr(x) + x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    if act == "gelu_tanh":
        p = special.expit(2 * _C * (x + 0.044715 * x ** 3))
        return p + x * p * (1 - p) * 2 * _C * (1 + 3 * 0.044715 * x * x)
    p = special.expit(x)
    return p + x * p * (1 - p)


def forward(z, act, mul=None, residual=None):
    y = value(act, z)
    y = y if mul is None else y * mul
    return y if residual is None else y + residual


def backward(dh, u, act, mul=None):
    """(du, dmul, db)"""
    du = dh * slope(act, u)
    if mul is not None:
        du = du * mul
    return du, (None if mul is None else dh * value(act, u)), du.sum(axis=0)


def route(x, w, k, renorm):
    """(ids [M, k], weights [M, k]) from rows x [M, D] and the router w [E, D]."""
    logits = x @ w.T
    p = np.exp(logits - logits.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(p, ids, 1)
    return ids, top / top.sum(axis=1, keepdims=True) if renorm else top


def experts(x, gate, up, down, ids, weights, act):
    """y [M, D] from lists of experts' weights gate, up [F, D] (up None: h = act(gate x)) and down [D, F]."""
    y = np.zeros((x.shape[0], down[0].shape[0]))
    for i in range(x.shape[0]):
        for e, w in zip(ids[i], weights[i]):
            if 0 <= e < len(gate):
                h = value(act, gate[e] @ x[i])
                if up is not None:
                    h = h * (up[e] @ x[i])
                y[i] += w * (down[e] @ h)
    return y
