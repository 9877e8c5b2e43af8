"""The head's loss (cross entropy, distillation) and the block norm against the
float64 oracle, forward and backward.

Tolerances, derived before the first run.  u is half a step of the 16-bit type
(bfloat16 2^-8, float16 2^-11), f = 2^-24.

* A logit is a float32 sum of D exact products: off by at most ez = D f sum_d |h w|,
  for every order of the sum.  Its exponential's argument is rounded at 1.5 |z| + 32 and
  the functions are good to 2^-22: a softmax entry is off by 2 ez / tau +
  (|z| / tau + 40) 2^-22 =: ep of itself.
* A loss is a difference of two logits' sizes: 2 ez + ep for the cross entropy, and
  alpha tau^2 times (2 ez / tau + 2 ep) for the divergence, whose teacher's softmax
  is good to (|t| / tau + 40) 2^-22 of terms ln q - ln s.
* A logit's gradient: size (its parts' magnitudes) times ep, and u of itself
  (float16: or half its smallest number, 2^-25, over 2^13).  dh and dW add up such
  errors times |W|, |h|, their float32 sums V f and T f of the terms'
  magnitudes, and the output's rounding (float16: or 2^-25).
* The norm: some ten float32 roundings and sums of D terms of one sign:
  (D + 16) f, x rounded to bfloat16; dr the same of the magnitudes of its
  terms; dw (T + D + 16) f of the terms' magnitudes.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import head as O  # noqa: E402
from paper_2606_18114_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F = 2.0 ** -24
IGNORE = -100


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Case:
    """Inputs on the GPU and as float64."""

    def __init__(self, T, V, D, dtype, K=0, alpha=0.5, tau=1.0, seed=0, masked=0.0, std=2.0,
                 ids64=True, top_dtype=torch.float32, dloss="mean"):
        g = np.random.default_rng(seed)
        self.T, self.V, self.D, self.dtype, self.K = T, V, D, dtype, K
        self.alpha, self.tau = (alpha, tau) if K else (0.0, 1.0)
        dev = "cuda"
        self.w = torch.from_numpy(g.normal(0, std / np.sqrt(D), (V, D))).to(dtype).to(dev)
        label = g.integers(0, V, T)
        self.h = torch.from_numpy(g.normal(0, 1, (T, D))).to(dtype).to(dev)
        label[g.random(T) < masked] = IGNORE
        it = torch.int64 if ids64 else torch.int32
        self.labels = torch.from_numpy(label).to(it).to(dev)
        self.ids = self.top = None
        if K:
            ids = g.integers(0, V, (T, K))
            ids[:, 0] = np.where(label >= 0, label, 0)
            if K > 2:
                ids[:, 2] = ids[:, 1]  # a word that comes twice
            ids[g.random((T, K)) < masked] = -1
            ids[g.random(T) < 0.5 * masked] = V + 3  # none in the vocabulary
            self.ids = torch.from_numpy(ids).to(it).to(dev)
            self.top = torch.from_numpy(g.normal(0, 3, (T, K))).to(top_dtype).to(dev)
        if dloss == "mean":
            d = np.full(T, 1.0 / T)
        elif dloss == "spread":  # magnitudes over many powers of two, signs, zeros
            d = g.normal(0, 1, T) * 2.0 ** g.integers(-20, 8, T)
            d[g.random(T) < 0.2] = 0.0
        else:
            d = np.full(T, float(dloss))
        self.dloss = torch.from_numpy(d).float().to(dev)

    def run(self, grad=True, **kw):
        teach = dict(teacher_ids=self.ids, alpha=self.alpha, temperature=self.tau) if self.K else {}
        loss, stats = ops.head_loss(self.h, self.w, self.labels, teacher_logits=self.top, **teach)
        if not grad:
            return loss, None, None
        dh, dw = ops.head_loss_bwd(self.h, self.w, self.labels, stats, self.dloss, **teach, **kw)
        return loss, dh, dw

    def args(self):
        lab = self.labels.cpu().numpy()
        a = [_np(self.h), _np(self.w), lab]
        t = dict(ids=None if self.ids is None else self.ids.cpu().numpy(), top=_np(self.top),
                 alpha=self.alpha, tau=self.tau)
        return a, t

    def check(self, loss, dh=None, dw=None, dw0=None):
        (h, w, lab), t = self.args()
        u, D, V, T = U[self.dtype], self.D, self.V, self.T
        z = h @ w.T
        ez = (D * F * (np.abs(h) @ np.abs(w).T)).max(1)
        mag = np.abs(z).max(1)
        ep = 2 * ez / self.tau + (mag / self.tau + 40) * 2.0 ** -22
        if self.tau != 1.0:
            ep = np.maximum(ep, 2 * ez + (mag + 40) * 2.0 ** -22)
        tol = 2 * ez + ep
        ref = O.loss(h, w, lab, **t)
        if self.K:
            tmag = np.where(np.isfinite(t["top"]), np.abs(t["top"]), 0).max(1)
            terms = (2 * mag + 2 * tmag) / self.tau + 2 * np.log(max(V, self.K)) + 40
            tol = tol + self.alpha * self.tau ** 2 * (
                2 * ez / self.tau + 2 * ep + (tmag / self.tau + 40) * 2.0 ** -22 * terms)
        err = np.abs(_np(loss) - ref)
        assert np.all(err <= tol), (err - tol).max()
        if dh is None:
            return
        dl = _np(self.dloss)
        dz, size = O.dlogits(h, w, lab, dl, **t)
        unit = ((1 - self.alpha) + self.alpha * self.tau) * np.abs(dl)[:, None]
        small = unit * 2.0 ** -25 / 2 ** 12 if self.dtype == torch.float16 else 0.0
        edz = size * ep[:, None] + np.abs(dz) * (u + 2 * 2.0 ** -20) + small * (dz != 0)
        rdh, rdw = O.loss_bwd(h, w, lab, dl, **t)
        sub = 2.0 ** -25 if self.dtype == torch.float16 else 0.0
        etol = edz @ np.abs(w) + V * F * (np.abs(dz) @ np.abs(w))
        err = np.abs(_np(dh) - rdh)
        tol = etol * (1 + u) + np.abs(rdh) * u + sub
        assert np.all(err <= tol), ("dh", (err - tol).max(), np.abs(rdh).max())
        # a row of h is scaled by a power of two against the largest gradient: float16 loses
        # what falls under its smallest number there
        hs = 0.0
        if self.dtype == torch.float16:
            big = np.abs(dl[dl != 0]).max() if np.any(dl != 0) else 0.0
            hs = (np.abs(dz) > 0).T.astype(float) @ np.full((T, 1), 2.0 ** -24 * 2 * big)
        etol = edz.T @ np.abs(h) + T * F * (np.abs(dz).T @ np.abs(h)) + hs
        if dw0 is not None:
            rdw = rdw + dw0
        uo = u if dw.dtype == self.dtype else 2 * F
        err = np.abs(_np(dw) - rdw)
        tol = etol * (1 + u) + np.abs(rdw) * uo + (sub if dw.dtype == self.dtype else 0.0)
        assert np.all(err <= tol), ("dw", (err - tol).max(), np.abs(rdw).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D", [(1, 1, 8), (1, 300, 64), (2, 255, 72), (3, 257, 264),
                                   (16, 1000, 128), (33, 100, 2048), (255, 513, 40),
                                   (257, 256, 96), (300, 1201, 200), (600, 700, 768)])
def test_cross_entropy(T, V, D, dtype):
    c = Case(T, V, D, dtype, seed=T + V)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D,K,alpha,tau", [(1, 50, 64, 1, 0.5, 1.0), (1, 400, 128, 64, 0.3, 1.0),
                                               (40, 300, 96, 5, 1.0, 2.0),
                                               (40, 300, 96, 5, 0.0, 3.0),
                                               (270, 600, 200, 17, 0.7, 0.5),
                                               (300, 520, 64, 64, 0.5, 1.0),
                                               (20, 2000, 40, 300, 0.5, 1.5)])
def test_distillation(T, V, D, K, alpha, tau, dtype):
    c = Case(T, V, D, dtype, K=K, alpha=alpha, tau=tau, seed=T + K, masked=0.2 if T > 1 else 0.0)
    c.check(*c.run())


# ---------------------------------------------------------------- the block norm

def _norm_case(T, D, y, dres, seed):
    g = np.random.default_rng(seed)
    f = lambda *s, std=1.0: torch.from_numpy(g.normal(0, std, s)).float().cuda()  # noqa: E731
    return dict(r=f(T, D, std=2.0), y=f(T, D) if y else None, w=1.0 + f(D, std=0.2),
                dx=f(T, D).bfloat16(), dres=f(T, D) if dres else None)


def _check_norm(c, x, r, dr, dw, eps):
    T, D = c["r"].shape
    rx, rr = O.norm(_np(c["r"]), _np(c["y"]), _np(c["w"]), eps)
    assert np.all(np.abs(_np(r) - rr) <= F * np.abs(rr))
    rx, _ = O.norm(_np(r), None, _np(c["w"]), eps)  # (the sum is rounded to float32)
    rel = (D + 16) * F
    assert np.all(np.abs(_np(x) - rx) <= np.abs(rx) * (2.0 ** -8 * (1 + rel) + rel))
    if dr is None:
        return
    s = _np(r)
    rdr, rdw = O.norm_bwd(s, _np(c["w"]), _np(c["dx"]), _np(c["dres"]), eps)
    rho = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    a = np.abs(_np(c["dx"]) * _np(c["w"]))
    mag = rho * a + np.abs(s) * rho ** 3 * (a * np.abs(s)).mean(-1, keepdims=True)
    if c["dres"] is not None:
        mag = mag + np.abs(_np(c["dres"]))
    assert np.all(np.abs(_np(dr) - rdr) <= 2 * rel * mag)
    wmag = (np.abs(_np(c["dx"])) * np.abs(s) * rho).sum(0)
    assert np.all(np.abs(_np(dw) - rdw) <= (T + D + 16) * F * wmag)


@pytest.mark.parametrize("T,D", [(1, 1), (1, 3), (5, 64), (3, 255), (17, 257), (2, 510), (4, 513),
                                 (9, 1023), (1030, 1000), (7, 2048), (3, 2050), (2, 4096),
                                 (3, 5001), (2, 8192), (3, 8195), (1100, 8200)])
@pytest.mark.parametrize("y,dres", [(True, True), (False, False)])
def test_block_norm(T, D, y, dres):
    c = _norm_case(T, D, y, dres, T + D)
    x, r = ops.block_norm(c["r"], c["y"], c["w"], 1e-5)
    if not y:
        assert r is c["r"]
    dr, dw = ops.block_norm_bwd(r, c["w"], c["dx"], c["dres"], 1e-5)
    _check_norm(c, x, r, dr, dw, 1e-5)


def test_block_norm_in_place_and_of_views():
    """The sum over the residual, dr over dresidual, and arrays that begin at any element."""
    T, D = 37, 61
    c = _norm_case(T, D, True, True, 3)
    big = {k: torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda") for k, v in c.items()}
    v = {k: big[k][1:].view(c[k].shape) for k in c}
    for k in c:
        v[k].copy_(c[k])
    x, r = ops.block_norm(v["r"], v["y"], v["w"], 1e-5, residual_out=v["r"])
    assert r is v["r"]
    keep = r.clone()
    dr, dw = ops.block_norm_bwd(r, v["w"], v["dx"], v["dres"], 1e-5, dr=v["dres"])
    assert dr is v["dres"]
    _check_norm(c, x, keep, dr, dw, 1e-5)
    x2, r2 = ops.block_norm(c["r"], None, c["w"], 1e-5, residual_out=torch.empty_like(c["r"]))
    assert torch.equal(r2, c["r"]) and r2 is not c["r"]
