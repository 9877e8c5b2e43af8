"""CPU oracle of the Mamba-2 mixer over sequences, with gradients, and of the
embedding.

TEST INFRASTRUCTURE ONLY (see ``oracle/ternary.py``): only ``tests/`` may use
it.  It shares no code with the HIP kernels: the recurrence token by token in
float64, its adjoint by the same recurrence backwards.

The layer is ``oracle/mamba.py``'s, taken over whole sequences: ``conv`` and
``scan`` and ``norm`` give what ``mixer_step`` computes between the projections,
u and y left in float64.  Arrays are those of one sequence, [tokens, ...]; a
batch of packed sequences is a loop over them in the tests.

``absolute=True`` makes every term of every sum positive: the result bounds the
sum of the terms' magnitudes, which is what rounding errors scale with.
"""

from __future__ import annotations

import numpy as np

__all__ = ["conv", "conv_bwd", "scan", "scan_bwd", "norm", "norm_bwd", "embed_bwd"]


def _sigmoid(v):
    return 1.0 / (1.0 + np.exp(-v))


def _softplus(v):
    return np.logaddexp(0.0, v)


def _line(x, past):
    """The inputs with the three before them, [tokens + 3, C]."""
    past = np.zeros((3, x.shape[1])) if past is None else np.asarray(past, np.float64)[-3:]
    return np.concatenate([past, np.asarray(x, np.float64)])


def conv(x, w, b, past=None):
    """x [L, C], w [C, 4] (oldest tap first), b [C], past [>= 3, C] -> SiLU of
    the causal convolution [L, C]."""
    line, n = _line(x, past), len(x)
    a = np.asarray(b, np.float64) + sum(line[j:j + n] * np.asarray(w, np.float64)[:, j]
                                        for j in range(4))
    return a * _sigmoid(a)


def conv_bwd(x, w, b, du, absolute=False):
    """Gradients (dx, dw, db) of conv without a past."""
    x, w, b, du = (np.asarray(v, np.float64) for v in (x, w, b, du))
    line, n = _line(x, None), len(x)
    a = b + sum(line[j:j + n] * w[:, j] for j in range(4))
    s = _sigmoid(a)
    da = du * s * (1.0 + a * (1.0 - s))
    if absolute:
        da, line, w = np.abs(da), np.abs(line), np.abs(w)
    dw = np.stack([(da * line[j:j + n]).sum(0) for j in range(4)], 1)
    dx = np.zeros_like(x)
    for j in range(4):
        k = 3 - j
        if n > k:
            dx[:n - k] += w[:, j] * da[k:]
    return dx, dw, da.sum(0)


def _steps(dt, dt_bias, A_log):
    raw = np.asarray(dt, np.float64) + np.asarray(dt_bias, np.float64)
    step, rate = _softplus(raw), np.exp(np.asarray(A_log, np.float64))
    return raw, step, rate, np.exp(-step * rate)


def scan(x, B, C, dt, dt_bias, A_log, D, state=None):
    """x [L, H, P], B, C [L, N], dt [L, H] -> (y [L, H, P], state [H, P, N])."""
    x, B, C = (np.asarray(v, np.float64) for v in (x, B, C))
    _, step, _, decay = _steps(dt, dt_bias, A_log)
    L, H, P = x.shape
    S = np.zeros((H, P, B.shape[1])) if state is None else np.asarray(state, np.float64).copy()
    y = np.empty_like(x)
    for t in range(L):
        S = S * decay[t][:, None, None] + (x[t] * step[t][:, None])[..., None] * B[t]
        y[t] = S @ C[t]
    return y + np.asarray(D, np.float64)[:, None] * x, S


def scan_bwd(x, B, C, dt, dt_bias, A_log, D, dy, absolute=False):
    """Gradients (dx, dB, dC, ddt, ddt_bias, dA_log, dD) of scan from a zero
    state, of y alone."""
    x, B, C, dy = (np.asarray(v, np.float64) for v in (x, B, C, dy))
    raw, step, rate, decay = _steps(dt, dt_bias, A_log)
    D = np.asarray(D, np.float64)
    if absolute:
        x, B, C, dy, D = (np.abs(v) for v in (x, B, C, dy, D))
    L, H, P = x.shape
    S = [np.zeros((H, P, B.shape[1]))]
    for t in range(L):
        S.append(S[-1] * decay[t][:, None, None] + (x[t] * step[t][:, None])[..., None] * B[t])
    dx, dB, dC = np.empty_like(x), np.empty_like(B), np.empty_like(C)
    dstep, dlog = np.empty_like(step), np.empty_like(step)
    adj = np.zeros_like(S[0])
    for t in range(L - 1, -1, -1):
        adj = adj + dy[t][..., None] * C[t]
        dC[t] = np.einsum("hp,hpn->n", dy[t], S[t + 1])
        dB[t] = np.einsum("hp,hpn->n", x[t] * step[t][:, None], adj)
        dxs = adj @ B[t]
        dx[t] = dxs * step[t][:, None] + D[:, None] * dy[t]
        dstep[t] = (dxs * x[t]).sum(-1)
        adj = adj * decay[t][:, None, None]
        dlog[t] = (adj * S[t]).sum((1, 2))
    sign = 1.0 if absolute else -1.0
    dstep = dstep + sign * rate * dlog
    ddt = dstep * _sigmoid(raw)
    return (dx, dB, dC, ddt, ddt.sum(0), (sign * step * rate * dlog).sum(0),
            (dy * x).sum((0, 2)))


def norm(y, z, w, eps):
    """g = y SiLU(z); g / sqrt(mean(g^2) + eps) w, per row."""
    y, z, w = (np.asarray(v, np.float64) for v in (y, z, w))
    g = y * z * _sigmoid(z)
    return g / np.sqrt((g * g).mean(-1, keepdims=True) + eps) * w


def norm_bwd(y, z, w, eps, dout, absolute=False):
    """Gradients (dy, dz, dw) of norm."""
    y, z, w, dout = (np.asarray(v, np.float64) for v in (y, z, w, dout))
    s = _sigmoid(z)
    si, dsi = z * s, s * (1.0 + z * (1.0 - s))
    if absolute:
        y, w, dout, si, dsi = (np.abs(v) for v in (y, w, dout, si, dsi))
    g = y * si
    r = 1.0 / np.sqrt((g * g).mean(-1, keepdims=True) + eps)
    q = dout * w
    sign = 1.0 if absolute else -1.0
    dg = r * q + sign * g * r ** 3 * (q * g).mean(-1, keepdims=True)
    return dg * si, dg * y * dsi, (dout * g * r).sum(0)


def embed_bwd(ids, dout, vocab, scale):
    """dW [vocab, D]: the sums of dout's rows by their ids, times scale; ids
    outside the vocabulary count nowhere."""
    dW = np.zeros((vocab, dout.shape[1]))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(dW, np.asarray(ids)[ok], np.asarray(dout, np.float64)[ok])
    return dW * scale
