"""Double-precision definitions of the gated recurrence and its vector-Jacobian product in numpy, step by step, on arrays
(batch, channels, steps, inner).  Test infrastructure; shares no code with the CUDA path."""
import numpy as np


def gate(g):
    """f and 1 - f."""
    e = np.exp(-np.abs(g))
    s, t = 1.0 / (1.0 + e), e / (1.0 + e)
    return np.where(g < 0, t, s), np.where(g < 0, s, t)


def order(steps, reverse):
    return range(steps - 1, -1, -1) if reverse else range(steps)


def forward(x, g, state=None, lengths=None, reverse=False):
    """(y, last, before): before holds the state that each step starts from."""
    x, g = x.astype(np.float64), g.astype(np.float64)
    b, c, t, n = x.shape
    h = np.zeros((b, c, n)) if state is None else state.astype(np.float64).copy()
    y, before = np.zeros_like(x), np.zeros_like(x)
    for k in order(t, reverse):
        for i in range(b):
            before[i, :, k] = h[i]
            if lengths is None or k < lengths[i]:
                f, r = gate(g[i, :, k])
                h[i] = f * h[i] + r * x[i, :, k]
                y[i, :, k] = h[i]
    return y, h, before


def vjp(dy, dlast, x, g, before, lengths=None, reverse=False):
    """(grad_x, grad_gate, grad_state)."""
    x, g, dy = x.astype(np.float64), g.astype(np.float64), dy.astype(np.float64)
    b, c, t, n = x.shape
    back = np.zeros((b, c, n)) if dlast is None else dlast.astype(np.float64).copy()
    dx, dg = np.zeros_like(x), np.zeros_like(x)
    for k in order(t, not reverse):
        for i in range(b):
            if lengths is None or k < lengths[i]:
                f, r = gate(g[i, :, k])
                d = dy[i, :, k] + back[i]
                dx[i, :, k] = d * r
                dg[i, :, k] = d * r * f * (before[i, :, k] - x[i, :, k])
                back[i] = d * f
    return dx, dg, back
