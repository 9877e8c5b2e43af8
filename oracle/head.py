"""Float64 oracle of the head's loss (cross entropy, distillation from a
teacher's top logits) and the block norm, with their gradients (paper Eq. 1)."""

import numpy as np


def _lse(z):
    m = z.max(-1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return m + np.log(np.exp(z - m).sum(-1, keepdims=True))


def _terms(V, labels, ids, top):
    """Which tokens have a cross entropy; which of the teacher's places hold a word."""
    ce = (labels >= 0) & (labels < V)
    if ids is None:
        return ce, None
    return ce, (ids >= 0) & (ids < V) & ~(top == -np.inf)


def teacher(V, ids, top, tau):
    """The teacher's distribution over its places, zeros where no word is kept."""
    kept = (ids >= 0) & (ids < V) & ~(top == -np.inf)
    t = np.where(kept, top, -np.inf)
    some = kept.any(1, keepdims=True)
    t = np.where(some, t, 0.0)
    t = (t - t.max(1, keepdims=True)) / tau
    return np.where(kept, np.exp(t - _lse(t)), 0.0), some[:, 0]


def loss(h, w, labels, ids=None, top=None, alpha=0.5, tau=1.0):
    """Losses [T] of h [T, D], w [V, D]."""
    V = len(w)
    T = len(h)
    ce, kept = _terms(V, labels, ids, top)
    use = ce if kept is None else ce | kept.any(1)
    z = np.zeros((T, V))
    z[use] = h[use] @ w.T
    out = np.zeros(T)
    i = np.nonzero(ce)[0]
    a = 0.0 if kept is None else alpha
    out[i] = (1.0 - a) * (_lse(z[i])[:, 0] - z[i, labels[i]])
    if kept is not None:
        q, some = teacher(V, ids, top, tau)
        logs = z / tau - _lse(z / tau)
        for t in np.nonzero(some)[0]:
            for k in np.nonzero(kept[t] & (q[t] > 0))[0]:
                out[t] += alpha * tau ** 2 * q[t, k] * (np.log(q[t, k]) - logs[t, ids[t, k]])
    return out


def dlogits(h, w, labels, dloss, ids=None, top=None, alpha=0.5, tau=1.0):
    """(dz [T, V], its parts' sizes [T, V]: the shares of the two softmaxes and of
    the label and the teacher added up without their signs)."""
    V = len(w)
    T = len(h)
    ce, kept = _terms(V, labels, ids, top)
    use = (ce if kept is None else ce | kept.any(1)) & (dloss != 0)
    dz, size = np.zeros((T, V)), np.zeros((T, V))
    a = 0.0 if kept is None else alpha
    z = np.zeros((T, V))
    z[use] = h[use] @ w.T
    p = np.exp(z - _lse(z))
    for t in np.nonzero(use & ce)[0]:
        dz[t] += (1.0 - a) * p[t]
        dz[t, labels[t]] -= 1.0 - a
        size[t] += (1.0 - a) * p[t]
        size[t, labels[t]] += 1.0 - a
    if kept is not None:
        q, some = teacher(V, ids, top, tau)
        s = np.exp(z / tau - _lse(z / tau))
        for t in np.nonzero(use & some)[0]:
            dz[t] += alpha * tau * s[t]
            size[t] += alpha * tau * s[t]
            for k in np.nonzero(kept[t])[0]:
                dz[t, ids[t, k]] -= alpha * tau * q[t, k]
                size[t, ids[t, k]] += alpha * tau * q[t, k]
    return dz * dloss[:, None], size * np.abs(dloss)[:, None]


def loss_bwd(h, w, labels, dloss, ids=None, top=None, alpha=0.5, tau=1.0):
    """(dh [T, D], dw [V, D])."""
    dz, _ = dlogits(h, w, labels, dloss, ids, top, alpha, tau)
    use = (dz != 0).any(1)  # rows without a gradient take no part, whatever they hold
    dh = np.zeros(h.shape)
    dh[use] = dz[use] @ w
    return dh, dz[use].T @ h[use]


def norm(residual, y, w, eps):
    """(x, residual + y)."""
    r = residual if y is None else residual + y
    return r / np.sqrt((r * r).mean(-1, keepdims=True) + eps) * w, r


def norm_bwd(r, w, dx, dres, eps):
    """(dr, dw)."""
    rho = 1.0 / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    a = dx * w
    dr = rho * a - r * rho ** 3 * (a * r).mean(-1, keepdims=True)
    return (dr if dres is None else dr + dres), (dx * r * rho).sum(0)
