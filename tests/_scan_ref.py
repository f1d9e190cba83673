"""The gated linear recurrence and its gradients in fp64 numpy, token by token."""
import numpy as np


def sigmoid(v):
    return np.where(v >= 0, 1.0 / (1.0 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1.0 + np.exp(-np.abs(v))))


def forward(x, g, leak, h0=None, lengths=None):
    """y [B][L][D], final state [B][D] and the states before every token [B][L][D]."""
    B, L, D = x.shape
    n = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    h = np.zeros((B, D)) if h0 is None else np.array(h0, np.float64)
    y, before = np.zeros((B, L, D)), np.zeros((B, L, D))
    for t in range(L):
        live = (t < n)[:, None]
        before[:, t] = h
        with np.errstate(invalid="ignore", over="ignore"):
            a, b = sigmoid(g[:, t]), sigmoid(-g[:, t])
            new = a * h + (b * x[:, t] if leak else x[:, t])
        h = np.where(live, new, h)
        y[:, t] = np.where(live, h, 0.0)
    return y, h, before


def backward(dy, x, g, leak, before, dh=None, lengths=None):
    """dx, dg [B][L][D] and the initial state's gradient [B][D]."""
    B, L, D = x.shape
    n = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    c = np.zeros((B, D)) if dh is None else np.array(dh, np.float64)
    dx, dg = np.zeros((B, L, D)), np.zeros((B, L, D))
    for t in range(L - 1, -1, -1):
        live = (t < n)[:, None]
        with np.errstate(invalid="ignore", over="ignore"):
            a, b = sigmoid(g[:, t]), sigmoid(-g[:, t])
            G = dy[:, t] + c
            vx = b * G if leak else G
            vg = a * b * G * (before[:, t] - x[:, t] if leak else before[:, t])
        dx[:, t], dg[:, t] = np.where(live, vx, 0.0), np.where(live, vg, 0.0)
        c = np.where(live, a * G, c)
    return dx, dg, c
