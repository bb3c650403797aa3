"""CPU oracle for what stands around the products (test infrastructure - never on the product path): a product's epilogue and
its gradient, and the gated linear recurrence with its gradient, from their definitions in fp64 NumPy, one column at a time.

Every recurrence also returns how large the numbers behind a result were and how far a 32-bit evaluation in any order may be from
it, so that the tests' tolerances follow from the arithmetic.  With u = 2^-24 (half a step of fp32):
  e = exp(-g) as 2^(-g log2 e): the product rounds by u, the constant by 0.23 u, the power is within 2 ulp = 4 u: x = (1.23 |g| + 4) u of itself;
  sigmoid(g) = a = 1 / (1 + e): the sum's rounding and the reciprocal (1 ulp) are 3 u, and of x it has the share e / (1 + e);
  1 - a = k = e a: one product more, 4 u, and of x, which e and a have the other way round, what is left, 1 / (1 + e).
  So for g >= 0 a is within 3 u + x sigmoid(-|g|) and k within 4 u + x; for g < 0 a is within 3 u + x and k within 4 u + x sigmoid(-|g|).
  (The kernels stop e at 2^115 or e^80, so that a below 2.4e-35 is not told apart; tests that use these bounds keep |g| below 79.)
  tanh(v) is within 8 u, the candidate's factor (1 - a) n within 9 u more than 1 - a;
  a step h = a h + w then adds (off_a + 4 u) |a h| + (off_k + 10 u) |w| to what the state before it was off by, times a: the kernels round a
  column's share of a product of a's once, its sum once when columns are composed and once when the states are worked out.
  Composed as a tree, a term passes two roundings (a product of a's and a sum) on each of five levels of a warp, three of the warps of a
  block and three of the blocks of a cluster, and one when what comes in is applied to block, warp and lane: 25, and no partial
  result is larger than the sum of magnitudes M: 40 u M.  (A round's end rounds once more, behind 256 columns or more.)

Activations, y = act(p): SiLU is p q, q = 1 / (1 + e) with e = exp(-p), which is large where p < 0: q is within (1.23 |p| + 7) u of itself,
and q <= e^-|p|, so y is off by |p| e^-|p| (1.23 |p| + 8) u < 4 u there, and by less than 8 u |p| where p >= 0.  sigmoid is within 8 u, tanh within 8 u.
GELU's tail Q(|p|) = e t P(t), e = 2^(-p^2 / 2 log2 e): square, product and constant round by 2.23 u, so the tail is within
(1.2 p^2 + 10.5) u of itself, Q <= 1/2 and p^2 Q <= 0.17: 5.4 u of 1.  Their products with p stay within 32 u (1 + |p|).
"""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh", "sigmoid", "tanh")
MODES = ("decay", "gate", "gate_tanh")


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def _erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def act(name, p):
    if name == "relu":
        return np.maximum(p, 0.0)
    if name == "silu":
        return p * sigmoid(p)
    if name == "gelu":
        return 0.5 * p * (1.0 + _erf(p / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * p * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (p + 0.044715 * p ** 3)))
    if name == "sigmoid":
        return sigmoid(p)
    return np.tanh(p) if name == "tanh" else p


def act_grad(name, p):
    if name == "relu":
        return (p > 0).astype(np.float64)
    if name == "silu":
        return sigmoid(p) * (1.0 + p * sigmoid(-p))
    if name == "gelu":
        return 0.5 * (1.0 + _erf(p / math.sqrt(2.0))) + p * np.exp(-0.5 * p * p) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (p + 0.044715 * p ** 3))
        return 0.5 * (1.0 + t) + 0.5 * p * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * p * p)
    if name == "sigmoid":
        return sigmoid(p) * sigmoid(-p)
    return 1.0 - np.tanh(p) ** 2 if name == "tanh" else np.ones_like(p)


def gates(mode, G, V):
    """a, 1 - a (the candidate's factor; 1 for decays), the candidate n: h_t = a h_(t-1) + k n."""
    if mode == "decay":
        return G, np.ones_like(G), V
    return sigmoid(G), sigmoid(-G), np.tanh(V) if mode == "gate_tanh" else V


def gates_off(mode, G):
    """Bounds for a and 1 - a, relative."""
    if mode == "decay":
        return np.zeros_like(G), np.zeros_like(G)
    x = 1.23 * np.abs(G) + 4
    share = x * sigmoid(-np.abs(G))
    return np.where(G >= 0, 3 + share, 3 + x) * U, np.where(G >= 0, 4 + x, 4 + share) * U


def glr_seq(mode, G, V, starts=None, h0=None):
    """Y (NaN in columns of no sequence), hT, the states before every column, and (off_Y, off_hT): the bounds of the module's text."""
    H, N = G.shape
    starts = [0, N] if starts is None else list(starts)
    S = len(starts) - 1
    h0 = np.zeros((H, S)) if h0 is None else h0
    a, k, n = gates(mode, G, V)
    w = k * n
    off_a, off_k = gates_off(mode, G)
    Y, before, off = (np.full((H, N), np.nan) for _ in range(3))
    off_before = np.zeros((H, N))
    hT, offT = np.empty((H, S)), np.zeros((H, S))
    mag_before = np.zeros((H, N))
    for s in range(S):
        h, m, e = h0[:, s], np.abs(h0[:, s]), np.zeros(H)
        eo = e
        for t in range(starts[s], starts[s + 1]):
            before[:, t], off_before[:, t], mag_before[:, t] = h, eo, m
            h = a[:, t] * h + w[:, t]
            e = np.abs(a[:, t]) * e + (off_a[:, t] + 4 * U) * np.abs(a[:, t]) * m + (off_k[:, t] + 10 * U) * np.abs(w[:, t])
            m = np.abs(a[:, t]) * m + np.abs(w[:, t])
            eo = e + 40 * U * m
            Y[:, t], off[:, t] = h, eo
        hT[:, s], offT[:, s] = h, eo
    return dict(Y=Y, hT=hT, before=before, mag_before=mag_before, off_before=off_before, off_Y=off, off_hT=offT)


def glr_seq_grad(mode, G, V, dY=None, dhT=None, starts=None, h0=None):
    """dG, dV (NaN in columns of no sequence), dh0, and bounds for a 32-bit evaluation of each."""
    H, N = G.shape
    f = glr_seq(mode, G, V, starts, h0)
    off_a, off_k = gates_off(mode, G)
    starts = [0, N] if starts is None else list(starts)
    S = len(starts) - 1
    dY = np.zeros((H, N)) if dY is None else dY
    dhT = np.zeros((H, S)) if dhT is None else dhT
    a, k, n = gates(mode, G, V)
    delta, mag, off = (np.full((H, N), np.nan) for _ in range(3))
    dh0, off0 = np.empty((H, S)), np.zeros((H, S))
    for s in range(S):
        e, m, x = dhT[:, s], np.abs(dhT[:, s]), np.zeros(H)
        xo = x
        for t in range(starts[s + 1] - 1, starts[s] - 1, -1):
            delta[:, t] = dY[:, t] + e
            x = x + U * (np.abs(dY[:, t]) + m)
            m = np.abs(dY[:, t]) + m
            mag[:, t], off[:, t] = m, x + 40 * U * m
            e = a[:, t] * delta[:, t]
            x = np.abs(a[:, t]) * (x + (off_a[:, t] + 4 * U) * m)
            m = np.abs(a[:, t]) * m
            xo = x + 40 * U * m
        dh0[:, s], off0[:, s] = e, xo
    h = f["before"]
    if mode == "decay":
        dG, dV = delta * h, delta
        off_G = off * np.abs(h) + mag * f["off_before"] + 4 * U * mag * f["mag_before"]
        off_V = off
    else:
        slope = 1.0 - n * n if mode == "gate_tanh" else np.ones_like(n)
        dG, dV = delta * (h - n) * a * k, delta * k * slope
        # h - n: what h is off by, a tanh within 8 u, one rounding; 1 - n^2 within 2 * 8 u and two roundings; then a few products
        off_G = a * k * (off * np.abs(h - n) + mag * (f["off_before"] + 10 * U * (f["mag_before"] + np.abs(n))) +
                         mag * np.abs(h - n) * (off_a + off_k + 4 * U))
        off_V = k * (off + mag * (off_k + 24 * U))
    return dict(dG=dG, dV=dV, dh0=dh0, off_G=off_G, off_V=off_V, off_dh0=off0)
