"""The head's loss in every form against float64 on the GPU: pieces of the
vocabulary, cut contractions, few and many tokens, arrays past 2^31 elements,
tokens that count nowhere whatever they hold, teachers with places that hold no
word, infinities; streams, graphs, the modules and a run of them together.

Tolerances as in test_gpu_head.py, derived before the first run: a logit is off by
ez = D f sum |h w|, a softmax entry by ep = 2 ez / tau + (|z| / tau + 40) 2^-22 of
itself, a logit's gradient by u of itself more (bfloat16 2^-8, float16 2^-11), sums by
their length times f = 2^-24 of the terms' magnitudes, an output by u.
"""

import math

import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402
from paper_2606_18114_amd.qat import (BlockNorm, Embedding, Head, Mamba2Mixer,  # noqa: E402
                                      TernaryLinear)

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F = 2.0 ** -24
IGNORE = -100


def _inputs(T, V, D, dtype=torch.bfloat16, K=0, seed=0, masked=0.0, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(V, D, generator=g, device="cuda") * (std / math.sqrt(D))).to(dtype)
    h = torch.randn(T, D, generator=g, device="cuda").to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[torch.rand(T, generator=g, device="cuda") < masked] = IGNORE
    c = dict(h=h, w=w, y=y, ids=None, top=None, alpha=0.0, tau=1.0,
             dloss=(0.5 + torch.rand(T, generator=g, device="cuda")) / T)
    if K:
        c.update(ids=torch.randint(0, V, (T, K), generator=g, device="cuda"),
                 top=3.0 * torch.randn(T, K, generator=g, device="cuda"), alpha=0.5)
        c["ids"][:, 0] = y
    return c


def _run(c, grad=True, **kw):
    t = {}
    if c["ids"] is not None:
        t = dict(teacher_ids=c["ids"], alpha=c["alpha"], temperature=c["tau"])
    loss, stats = ops.head_loss(c["h"], c["w"], c["y"], teacher_logits=c["top"], **t)
    if not grad:
        return loss
    return (loss, *ops.head_loss_bwd(c["h"], c["w"], c["y"], stats, c["dloss"], **t, **kw))


def _reference(c, tokens, words=None):
    """(losses, their tolerance, dz, its tolerance) of the given tokens in float64; dz of the given
    words only."""
    h, w = c["h"][tokens].double(), c["w"].double()
    D, V, u = h.shape[1], len(w), U.get(c["h"].dtype, 0.0)
    z = h @ w.t()
    # sum |h w| by Cauchy's inequality
    ez = D * F * h.norm(dim=1) * w.norm(dim=1).max()
    y, tau, alpha = c["y"][tokens], c["tau"], c["alpha"]
    mag = z.abs().amax(1)
    ep = (2 * ez / min(tau, 1.0) + (mag / min(tau, 1.0) + 40) * 2.0 ** -22)
    logp = torch.log_softmax(z, 1)
    ce = (y >= 0) & (y < V)
    at = y.clamp(0, V - 1)[:, None]
    loss = torch.where(ce, -(1 - alpha) * logp.gather(1, at)[:, 0], 0.0)
    dz = (1 - alpha) * logp.exp() * ce[:, None]
    size = dz.clone()
    hit = torch.where(ce, 1 - alpha, 0.0).double()[:, None]
    dz.scatter_add_(1, at, -hit)
    size.scatter_add_(1, at, hit)
    tol = 2 * ez + ep
    if c["ids"] is not None:
        ids, top = c["ids"][tokens], c["top"][tokens].double() / tau
        kept = (ids >= 0) & (ids < V) & (top > -math.inf)
        some = kept.any(1)
        logq = torch.log_softmax(torch.where(kept, top, -1e300), 1)
        q = torch.where(kept, logq.exp(), 0.0)
        logs = torch.log_softmax(z / tau, 1)
        at = ids.clamp(0, V - 1).long()
        kl = torch.where(q > 0, q * (logq - logs.gather(1, at)), 0.0).sum(1)
        loss = loss + alpha * tau ** 2 * kl
        s = alpha * tau * logs.exp() * some[:, None]
        dz += s
        size += s
        dz.scatter_add_(1, at, -alpha * tau * q)
        size.scatter_add_(1, at, alpha * tau * q)
        tmag = torch.where(kept, top.abs(), 0.0).amax(1)
        tol = tol + alpha * tau ** 2 * (2 * ez / tau + 2 * ep + (tmag + 40) * 2.0 ** -22
                                        * (2 * mag / tau + 2 * tmag + 2 * math.log(V + 1) + 40))
    g = c["dloss"][tokens].double()[:, None]
    unit = ((1 - alpha) + alpha * tau) * g.abs()
    edz = size * g.abs() * ep[:, None] + dz.abs() * g.abs() * (u + 2.0 ** -19)
    if c["h"].dtype == torch.float16:
        edz += unit * 2.0 ** -37
    dz = dz * g
    if words is not None:
        dz, edz = dz[:, words], edz[:, words]
    return loss, tol, dz, edz


def _check(c, loss, dh, dw, tokens=None, words=None, dw0=None):
    """Losses and rows of dh of some tokens, rows of dW of some words (from all tokens)."""
    T, V, u = len(c["h"]), len(c["w"]), U[c["h"].dtype]
    sub = 2.0 ** -25 if c["h"].dtype == torch.float16 else 0.0
    tokens = torch.arange(T, device="cuda") if tokens is None else torch.tensor(tokens, device="cuda")
    words = torch.arange(V, device="cuda") if words is None else torch.tensor(words, device="cuda")
    aw = c["w"].double()
    want, tol, dz, edz = _reference(c, tokens)
    off = (loss[tokens].double() - want).abs()
    assert bool((off <= tol).all()), ("loss", float((off - tol).max()))
    if dh is not None:
        want = dz @ aw
        tol = (edz + V * F * dz.abs()) @ aw.abs()
        tol = tol * (1 + u) + want.abs() * u + sub
        off = (dh[tokens].double() - want).abs()
        assert bool((off <= tol).all()), ("dh", float((off - tol).max()))
    if dw is None:
        return
    want = torch.zeros(len(words), aw.shape[1], dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(want)
    for lo in range(0, T, 4096):
        t = torch.arange(lo, min(T, lo + 4096), device="cuda")
        _, _, dz, edz = _reference(c, t, words)
        h = c["h"][t].double()
        # a token without a loss has no part; one whose gradient is exactly zero (a vocabulary of
        # one word) has a loss, and its logits' roundings edz count
        some = (c["y"][t] >= 0) & (c["y"][t] < V)
        if c["ids"] is not None:
            some |= ((c["ids"][t] >= 0) & (c["ids"][t] < V) & (c["top"][t] > -math.inf)).any(1)
        h = torch.where((some & (c["dloss"][t] != 0))[:, None], h, 0.0)
        want += dz.t() @ h
        tol += (edz + T * F * dz.abs()).t() @ h.abs()
        if c["h"].dtype == torch.float16:  # what falls under the smallest number in h's copy
            tol += (dz != 0).double().sum(0)[:, None] * 2.0 ** -23 * float(c["dloss"].abs().max())
    if dw0 is not None:
        want = want + dw0[words].double()
    uo = u if dw.dtype == c["h"].dtype else 2 * F
    tol = tol * (1 + u) + want.abs() * uo + (sub if dw.dtype == c["h"].dtype else 0.0)
    off = (dw[words].double() - want).abs()
    assert bool((off <= tol).all()), ("dw", float((off - tol).max()))


# ---------------------------------------------------------------- forms

@pytest.mark.parametrize("T,V,D,K,why", [
    (16384, 20001, 264, 0, "two pieces, the last one smaller"),
    (16384, 17000, 2048, 3, "pieces that fill rounds, a last one whose tokens are cut"),
    (70001, 9001, 64, 0, "pieces of 4096 words"),
    (256, 1100000, 64, 0, "two pieces, dh cut along the words, a last piece of fewer parts"),
    (5000, 130, 512, 2, "dW cut along the tokens"),
    (65, 3000, 128, 0, "tiles of 64 tokens"), (129, 3000, 128, 5, "and one token more"),
    (120, 70000, 136, 1, "tiles of 128 tokens"), (64, 70000, 136, 1, "few tokens")])
def test_pieces_and_parts(T, V, D, K, why):
    c = _inputs(T, V, D, K=K, seed=T + V, masked=0.1)
    out = _run(c)
    some = lambda n: sorted({0, 1, n // 2, n - 2, n - 1, *range(0, n, max(1, n // 61))})  # noqa: E731
    words = some(V) + [v for v in (4095, 4096, 8191, 8192, 16383, 16384) if v < V]
    _check(c, *out, tokens=some(T), words=words)


@pytest.mark.parametrize("T,V,D,K,masked", [
    (3001, 5003, 264, 0, 0.6), (1500, 9000, 768, 2, 0.9), (5000, 1000, 72, 0, 0.999),
    (70001, 9001, 64, 0, 0.9), (17000, 17000, 520, 0, 0.97)])  # (the last two: several pieces)
def test_many_tokens_without_a_loss(T, V, D, K, masked):
    """dh's contraction is cut into more parts than for all tokens."""
    c = _inputs(T, V, D, K=K, seed=T + D, masked=masked)
    if K:
        c["ids"][c["y"] == IGNORE] = -1
    c["h"][c["y"] == IGNORE] = math.nan
    out = _run(c)
    some = torch.nonzero(c["y"] != IGNORE)[:, 0].tolist()
    _check(c, *out[:2], None, tokens=some[::max(1, len(some) // 97)] + some[-1:])
    assert bool((out[1][c["y"] == IGNORE] == 0).all())


@pytest.mark.parametrize("T,V,K,tau", [(190, 33000, 2, 1.5), (300, 50000, 0, 1.0),
                                       (384, 50000, 1, 1.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_tiles_of_192_tokens(T, V, K, tau, dtype):
    c = _inputs(T, V, 72, dtype, K=K, seed=T, masked=0.1)
    c["tau"] = tau
    want, tol, _, _ = _reference(c, torch.arange(T, device="cuda"))
    off = (_run(c, grad=False).double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())


@pytest.mark.parametrize("T,V,D,K,tau", [
    (1, 3, 8, 0, 1.0), (1, 5000, 4104, 2, 1.0),     # fewer words than waves; h in two parts
    (16, 70000, 72, 0, 1.0), (17, 70001, 1000, 9, 2.0),  # two blocks of words a wave
    (5, 300, 8200, 0, 1.0), (20, 515, 4160, 40, 0.5),    # three parts of h
    (32, 16383, 64, 0, 1.0), (33, 4097, 2056, 0, 1.0),
    (64, 131073, 1096, 3, 1.5), (64, 2000, 40, 0, 1.0),
    (3, 400, 128, 1024, 1.0), (16, 900, 264, 65, 3.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_tokens(T, V, D, K, tau, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T + V + K, masked=0.2 if T > 2 else 0.0)
    if K:
        c.update(tau=tau)
    if T > 2:
        c["h"][c["y"] == IGNORE] = math.nan if K == 0 else 1.0  # not read
    loss = _run(c, grad=False)
    ok = torch.arange(T, device="cuda") if K else torch.nonzero(c["y"] != IGNORE)[:, 0]
    want, tol, _, _ = _reference(c, ok)
    off = (loss[ok].double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())
    assert K or bool((loss[c["y"] == IGNORE] == 0).all())


@pytest.mark.parametrize("T,V,D,K", [(1, 1, 8, 0), (1, 70, 264, 3), (7, 129, 64, 0),
                                     (16, 1001, 520, 0), (17, 1000, 248, 5), (40, 127, 2056, 0),
                                     (64, 5003, 768, 0), (64, 33001, 72, 2), (33, 263, 4104, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_of_few_tokens(T, V, D, K, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T + V + D, masked=0.3 if T > 6 else 0.0)
    c["dloss"] *= 4.0 ** torch.randint(-3, 4, (T,), device="cuda")
    _check(c, *_run(c))
    dw0 = torch.randn(V, D, device="cuda")
    for kw in ({"dW": torch.full_like(dw0, math.nan)}, {"dW": dw0.clone(), "accumulate": True}):
        loss, dh, dw = _run(c, **kw)
        _check(c, loss, None, dw, dw0=dw0 if "accumulate" in kw else None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_float32_weight_gradient_and_its_sum(dtype):
    c = _inputs(300, 515, 136, dtype, K=4, seed=1, masked=0.2)
    _, dh, dw16 = _run(c)
    dw = torch.full((515, 136), 7.0, device="cuda")
    loss, dh2, out = _run(c, dW=dw)
    assert out is dw and torch.equal(dh, dh2) and torch.equal(dw.to(dtype), dw16)
    _check(c, loss, dh, dw)
    dw0 = torch.randn(515, 136, device="cuda") * 1e-3
    dw = dw0.clone()
    _check(c, *_run(c, dW=dw, accumulate=True), dw0=dw0)
    # few words, many tokens: the parts are added up before they are added
    c = _inputs(3000, 70, 136, dtype, seed=2)
    dw0 = torch.randn(70, 136, device="cuda") * 1e-2
    dw = dw0.clone()
    _check(c, *_run(c, dW=dw, accumulate=True), dw0=dw0)


def test_one_gradient_alone():
    c = _inputs(100, 300, 64, K=2, seed=3)
    loss, dh, dw = _run(c)
    _, dh1, none = _run(c, want_dW=False)
    assert none is None and torch.equal(dh, dh1)
    _, none, dw1 = _run(c, want_dh=False)
    assert none is None and torch.equal(dw, dw1)
    with pytest.raises(ValueError):
        _run(c, want_dh=False, want_dW=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_of_many_sizes(dtype):
    """dloss over many powers of two, with signs and zeros: every row has its own scale in dh."""
    c = _inputs(200, 400, 96, dtype, K=3, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    c["dloss"] = torch.randn(200, generator=g, device="cuda") * torch.exp2(
        torch.randint(-6, 6, (200,), generator=g, device="cuda").float())
    c["dloss"][::7] = 0.0
    loss, dh, dw = _run(c)
    assert not dh[::7].any()
    _check(c, loss, dh, dw)
    # scaling by a power of two scales bfloat16 gradients exactly
    if dtype == torch.bfloat16:
        c["dloss"] *= 2.0 ** -30
        _, dh2, dw2 = _run(c)
        assert torch.equal(dh2, dh * 2.0 ** -30) and torch.equal(dw2, dw * 2.0 ** -30)


def test_results_repeat_bit_for_bit():
    c = _inputs(700, 3001, 264, K=9, seed=6, masked=0.3)
    first = _run(c)
    for _ in range(3):
        for a, b in zip(first, _run(c)):
            assert torch.equal(a, b)


# ---------------------------------------------------------------- tokens that count nowhere

def test_tokens_without_a_loss_may_hold_anything():
    c = _inputs(300, 500, 136, K=3, seed=7)
    out = torch.zeros(300, dtype=torch.bool, device="cuda")
    out[::3] = True
    c["y"][out] = IGNORE
    c["ids"][out] = 2 ** 40
    ref = _run(c)
    c["h"][out] = float("nan")
    c["h"][::6] = float("inf")
    c["dloss"][out] = float("nan")
    got = _run(c)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
    assert not got[0][out].any() and not got[1][out].any()
    # tokens whose gradient is zero
    c = _inputs(300, 500, 136, seed=8)
    c["dloss"][out] = 0.0
    ref = _run(c)
    c["h"][out] = float("nan")
    got = _run(c)
    assert torch.equal(ref[1], got[1]) and torch.equal(ref[2], got[2])
    assert bool(torch.isnan(got[0][out]).all()) and torch.equal(ref[0][~out], got[0][~out])


@pytest.mark.parametrize("T", [1, 70, 3000])
def test_no_token_counts(T):
    c = _inputs(T, 90, 64, K=2, seed=9)
    c["y"].fill_(-1)
    c["ids"].fill_(90)
    c["h"].fill_(float("nan"))
    loss, dh, dw = _run(c)
    assert not loss.any() and not dh.any() and not dw.any()
    keep = torch.randn(90, 64, device="cuda")
    dw = keep.clone()
    _run(c, dW=dw, accumulate=True)
    assert torch.equal(dw, keep)


def test_no_tokens():
    c = _inputs(2, 90, 64, K=2, seed=10)
    c = {k: v[:0].contiguous() if k in ("h", "y", "ids", "top", "dloss") else v
         for k, v in c.items()}
    loss, dh, dw = _run(c)
    assert loss.shape == (0,) and dh.shape == (0, 64) and not dw.any()


@pytest.mark.parametrize("top_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
def test_teachers(top_dtype, ids_dtype):
    """Places without a word, logits of -infinity, rows that keep nothing, words that come twice and
    the label among them, types."""
    c = _inputs(120, 333, 72, K=8, seed=11)
    c["top"] = c["top"].to(top_dtype)
    c["ids"][1::4, 2:5] = -1
    c["top"][2::4, 1:7] = float("-inf")
    c["ids"][3::4] = 333
    c["top"][5] = float("-inf")
    c["ids"][6] = c["ids"][6, :1]
    c["ids"][7] = 5
    c["ids"] = c["ids"].to(ids_dtype)
    c["y"][::5] = IGNORE
    for alpha, tau in ((0.5, 1.0), (1.0, 0.7), (0.0, 1.0), (0.3, 5.0)):
        c.update(alpha=alpha, tau=tau)
        _check(c, *_run(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_that_vanish_beside_large_ones(dtype):
    """A loss's gradient that is zero in float32 once it is taken over the logits' unit (alpha tau
    = 1/4) adds nothing, whatever the others are."""
    c = _inputs(5, 70, 24, dtype, K=3, seed=31)
    c.update(alpha=1.0, tau=0.25)
    c["dloss"] = torch.tensor([8.0, 1e-45, 100.0, -1e-45, 3.0], device="cuda")
    loss, dh, dw = _run(c)
    c["dloss"] = torch.tensor([8.0, 0.0, 100.0, 0.0, 3.0], device="cuda")
    loss0, dh0, dw0 = _run(c)
    assert bool(torch.isfinite(dw.float()).all()) and bool((dh[1::2] == 0).all())
    assert torch.equal(loss, loss0) and torch.equal(dh, dh0) and torch.equal(dw, dw0)


@pytest.mark.parametrize("tau", [2.0 ** -10, 2.0 ** 10])
def test_temperatures_far_from_one(tau):
    """Cold: the softmaxes are single words, the loss stays finite.  Hot: both are uniform."""
    c = _inputs(5, 70, 24, K=3, seed=32)
    c.update(alpha=0.5, tau=tau)
    assert all(bool(torch.isfinite(t.float()).all()) for t in _run(c))


def test_one_word_a_teacher_is_cross_entropy():
    """A teacher that knows one word: the divergence is the cross entropy of it."""
    c = _inputs(50, 200, 64, seed=12)
    ce, dh, dw = _run(c)
    c.update(ids=c["y"][:, None].clone(), top=torch.randn(50, 1, device="cuda"), alpha=1.0, tau=1.0)
    c["y"] = torch.full_like(c["y"], IGNORE)
    kl, dh2, dw2 = _run(c)
    assert torch.allclose(ce, kl, rtol=0, atol=1e-5)
    assert torch.allclose(dh.float(), dh2.float(), rtol=2 ** -7, atol=1e-6)
    assert torch.allclose(dw.float(), dw2.float(), rtol=2 ** -7, atol=1e-6)


def test_infinities_and_nan():
    c = _inputs(300, 500, 64, seed=13)
    ref = _run(c)
    c["h"][7, 3] = float("inf")
    c["h"][290] = float("nan")
    loss, dh, dw = _run(c)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[7, 290]] = True
    assert not torch.isfinite(loss[bad]).any() and torch.equal(loss[~bad], ref[0][~bad])
    assert not torch.isfinite(dh[290]).any() and torch.equal(dh[~bad], ref[1][~bad])
    assert not torch.isfinite(dw).any()
    c = _inputs(300, 500, 64, seed=13)
    c["w"][499, 0] = float("nan")
    assert bool(torch.isnan(_run(c, grad=False)).all())
    # a gradient that is infinite stays with its token in dh
    c = _inputs(300, 500, 64, seed=13)
    c["dloss"][5] = float("inf")
    _, dh, _ = _run(c)
    rest = torch.arange(300, device="cuda") != 5
    assert not torch.isfinite(dh[5]).all() and torch.equal(dh[rest], ref[1][rest])


def test_logits_far_from_zero():
    c = _inputs(64, 300, 128, seed=14, std=60.0)  # logits of some hundreds
    loss = _run(c, grad=False)
    want, tol, _, _ = _reference(c, torch.arange(64, device="cuda"))
    assert bool(((loss.double() - want).abs() <= tol).all())


# ---------------------------------------------------------------- large arrays

def test_hidden_past_2_31_elements():
    T, V, D = 2 ** 20 + 77, 70, 2048
    c = _inputs(T, V, D, seed=15)
    tokens = [0, 1, 255, 256, T // 2, 2 ** 20 - 1, 2 ** 20, T - 2, T - 1]
    loss, dh, dw = _run(c, want_dW=False)
    _check(c, loss, dh, None, tokens=tokens)
    del dh
    c["dloss"][:T - 500] = 0.0  # the last rows alone
    _, _, dw = _run(c, want_dh=False)
    part = {**c, "h": c["h"][T - 500:], "y": c["y"][T - 500:], "dloss": c["dloss"][T - 500:]}
    _check(part, loss[T - 500:], None, dw)


def test_weight_past_2_31_elements():
    T, V, D = 3, 2 ** 20 + 300, 2048
    c = _inputs(T, V, D, seed=16)
    c["y"][:] = torch.tensor([0, 2 ** 20, V - 1], device="cuda")
    loss, dh, dw = _run(c)
    _check(c, loss, dh, dw, words=[0, 1, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, V - 2, V - 1])


# ---------------------------------------------------------------- streams and graphs

def test_two_streams_at_once():
    cases = [_inputs(500, 2000, 264, K=5, seed=s, masked=0.2) for s in (17, 18)]
    want = [_run(c) for c in cases]
    norms = [BlockNorm(264, device="cuda") for _ in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append((_run(c), norms[i](c["h"].float())[0]))
    torch.cuda.synchronize()
    for w, g, c, n in zip(want, got, cases, norms):
        x = n(c["h"].float())[0]
        for out, y in g:
            assert all(torch.equal(a, b) for a, b in zip(w, out)) and torch.equal(x, y)


@pytest.mark.parametrize("T,K", [(333, 4), (9, 4), (40, 3), (64, 0), (1100, 0)])
def test_a_captured_step_and_its_replays(T, K):
    """Forward and backward in a graph, replayed with other inputs, other tokens masked, and eager
    work between the replays."""
    cases = [_inputs(T, 1500, 136, K=K, seed=s, masked=m) for s, m in ((19, 0.0), (20, 0.5),
                                                                       (21, 0.9))]
    c = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in cases[0].items()}
    r = torch.randn(T, 136, device="cuda")
    nw = torch.ones(136, device="cuda")

    def step():
        out = _run(c)
        x, s = ops.block_norm(r, c["h"].float(), nw)
        return (*out, x, *ops.block_norm_bwd(s, nw, out[1], r))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for round in range(2):
        for other in cases:
            for k, v in other.items():
                if isinstance(v, torch.Tensor):
                    c[k].copy_(v)
            graph.replay()
            got = [t.clone() for t in out]
            torch.cuda.synchronize()
            want = step()  # eager, with scratch of its own
            for a, b in zip(want, got):
                assert torch.equal(a, b)


# ---------------------------------------------------------------- modules

@pytest.mark.parametrize("wdtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_head_module(dtype, wdtype):
    c = _inputs(60, 150, 64, dtype, K=3, seed=22)
    head = Head(150, 64, alpha=0.4, temperature=1.5, device="cuda", dtype=wdtype)
    with torch.no_grad():
        head.weight.copy_(c["w"])
    c["w"] = head.weight.detach().to(dtype)
    c.update(alpha=0.4, tau=1.5)
    h = c["h"].view(3, 20, 64).requires_grad_()
    loss = head(h, c["y"].view(3, 20), c["ids"].view(3, 20, 3), c["top"].view(3, 20, 3))
    assert loss.shape == (3, 20) and loss.dtype == torch.float32
    loss.backward(c["dloss"].view(3, 20))
    assert head.weight.grad.dtype == wdtype and h.grad.dtype == dtype
    dw = head.weight.grad
    if wdtype != torch.float32 and wdtype != dtype:  # rounded once more
        dw = None
    _check(c, loss.detach().view(-1), h.grad.view(60, 64), dw)
    plain = {**c, "ids": None, "top": None, "alpha": 0.0, "tau": 1.0}
    _check(plain, head(c["h"], c["y"]).detach(), None, None)
    head.weight.requires_grad_(False)  # a frozen head
    h.grad = None
    head(h, c["y"].view(3, 20)).sum().backward()
    assert h.grad is not None and bool(torch.isfinite(h.grad).all())


def test_block_norm_module():
    norm = BlockNorm(100, device="cuda")
    with torch.no_grad():
        norm.weight.normal_(1.0, 0.1)
    r = torch.randn(2, 5, 100, device="cuda", requires_grad=True)
    y = torch.randn(2, 5, 100, device="cuda").bfloat16().requires_grad_()
    gx, gs = torch.randn(2, 5, 100, device="cuda").bfloat16(), torch.randn(2, 5, 100, device="cuda")
    for two in (True, False):
        x, s = norm(r, y if two else None)
        got = torch.autograd.grad((x, s), (r, y, norm.weight) if two else (r, norm.weight),
                                  (gx, gs))
        r64, y64, w64 = (t.detach().double().requires_grad_() for t in (r, y, norm.weight))
        s64 = r64 + y64 if two else r64 * 1.0
        x64 = s64 / torch.sqrt(s64.pow(2).mean(-1, keepdim=True) + norm.eps) * w64
        want = torch.autograd.grad((x64, s64), (r64, y64, w64) if two else (r64, w64),
                                   (gx.double(), gs.double()))
        assert bool(((x.double() - x64).abs() <= x64.abs() * (2.0 ** -8 + 2.0 ** -16)).all())
        assert bool(((s.double() - s64).abs() <= F * s64.abs()).all())
        for a, b in zip(got, want):
            # float32 sums of 100 terms (y's gradient: bfloat16) of magnitudes of at most 100
            u = 2.0 ** -8 if a.dtype == torch.bfloat16 else 0.0
            assert bool(((a.double() - b).abs() <= u * b.abs() + 200 * F * 100).all())
    with torch.no_grad():
        x, s = norm(r)
        assert s is r
    with pytest.raises(ValueError, match=r"\[..., 100\]"):
        norm(torch.randn(100, 4, device="cuda"))  # 400 values, of another width


def test_gradients_against_differences():
    """Along the gradient's own direction, in float16, where a logit's gradient is good to 2^-11."""
    c = _inputs(40, 64, 64, torch.float16, K=3, seed=23)
    c.update(alpha=0.5, tau=2.0)
    _, dh, dw = _run(c)
    total = lambda d: float((_reference(d, torch.arange(40, device="cuda"))[0]  # noqa: E731
                             * c["dloss"].double()).sum())
    for k, g in (("h", dh), ("w", dw)):
        g = g.double()
        step = 1e-4 / float(g.norm())
        up = total({**c, k: c[k].double() + step * g})
        down = total({**c, k: c[k].double() - step * g})
        want = float(g.pow(2).sum()) * 2 * step
        # third derivatives: the step moves a logit by less than 2e-4; rounding of g: 2^-10
        assert abs((up - down) - want) <= want * 2.0 ** -9


def test_a_training_step_from_ids_to_loss():
    """Embedding, norms, a ternary block and the head, whose weight is the embedding's, in one step:
    the ends against the same step with its norms and loss in float64."""
    V, W, T = 211, 256, 96
    torch.manual_seed(24)
    emb = Embedding(V, W, scale=4.0, device="cuda")
    pre, final = BlockNorm(W, device="cuda"), BlockNorm(W, device="cuda")
    nheads = 8
    Z = 2 * 64 * nheads + 256 + nheads
    inp = TernaryLinear(W, Z, g=64, device="cuda")
    mix = Mamba2Mixer(nheads, device="cuda")
    out = TernaryLinear(64 * nheads, W, g=64, device="cuda")
    head = Head(V, W, weight=emb.weight, alpha=0.5)
    ids = torch.randint(0, V, (T,), device="cuda")
    labels = torch.cat([ids[1:], ids.new_tensor([IGNORE])])
    offsets = torch.tensor([0, 40, T], dtype=torch.int32, device="cuda")
    labels[39] = IGNORE
    tid = torch.randint(0, V, (T, 5), device="cuda")
    top = torch.randn(T, 5, device="cuda")
    params = [emb.weight, pre.weight, final.weight, inp.weight, out.weight, *mix.parameters()]

    e = emb(ids)
    x, r = pre(e)
    r.retain_grad()
    y = out(mix(inp(x), offsets))
    h, s = final(r, y)
    h.retain_grad()
    s.retain_grad()
    losses = head(h, labels, tid, top)
    losses.mean().backward()
    for p in params:
        assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool(p.grad.any())
    # the loss and its gradients, from the h that was there
    c = dict(h=h.detach(), w=emb.weight.detach().to(torch.bfloat16), y=labels, ids=tid, top=top,
             alpha=0.5, tau=1.0, dloss=torch.full((T,), 1.0 / T, device="cuda"))
    _, stats = ops.head_loss(c["h"], c["w"], labels, tid, top, alpha=0.5)
    dh, dw = ops.head_loss_bwd(c["h"], c["w"], labels, stats, c["dloss"], tid, alpha=0.5,
                               dW=torch.zeros(V, W, device="cuda"))
    _check(c, losses.detach(), h.grad, dw)
    # the shared weight: the head's part and the embedding's
    demb = ops.embed_bwd(ids, r.grad + 0.0, V, 4.0)
    r64 = s.detach().double().requires_grad_()
    x64 = r64 / torch.sqrt(r64.pow(2).mean(-1, keepdim=True) + 1e-5) * final.weight.double().detach()
    (want,) = torch.autograd.grad(x64, r64, h.grad.double())
    got = s.grad if s.grad is not None else None
    assert got is None or not got.any()  # nothing reads the sum after the last norm
    rr = ops.block_norm_bwd(s.detach(), final.weight.detach(), h.grad, None)[0]
    a = (h.grad.double() * final.weight.double()).abs()
    rho = 1 / torch.sqrt(r64.detach().pow(2).mean(-1, keepdim=True) + 1e-5)
    mag = rho * a + r64.detach().abs() * rho ** 3 * (a * r64.detach().abs()).mean(-1, keepdim=True)
    assert bool(((rr.double() - want).abs() <= 2 * (W + 16) * F * mag).all())
    assert bool(((emb.weight.grad - (dw + demb)).abs()
                 <= 4 * F * (dw.abs() + demb.abs())).all())
