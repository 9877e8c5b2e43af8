"""The head's loss where numbers come near the ends of their types, and in forms beside those of
test_gpu_head_forms.py, whose inputs, float64 reference and tolerances are used here."""

import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_head_forms import (F, IGNORE, _check, _inputs, _reference,  # noqa: E402
                                 _run)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- teachers

@pytest.mark.parametrize("T,K", [(1, 1), (40, 5), (40, 30), (600, 30)])  # both launch shapes
@pytest.mark.parametrize("top_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [0.5, 2.0 ** -10, 1.0, 3.0])
def test_teachers_of_the_types_ends(T, K, top_dtype, tau):
    """A teacher's softmax does not change when a number is added to all of a token's logits: rows
    of the type's lowest or largest value are uniform, words at the lowest beside others have no
    share, and both are what they are as small numbers, to the last bit."""
    c = _inputs(T, 90, 72, K=K, seed=T + K)
    c.update(alpha=0.5, tau=tau)
    c["top"] = c["top"].to(top_dtype)
    lo, hi = torch.finfo(top_dtype).min, torch.finfo(top_dtype).max
    for value in (lo, hi):
        c["top"][0::3] = 0.0
        want = _run(c)
        _check(c, *want)
        c["top"][0::3] = value
        got = _run(c)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
    if K == 1:
        return
    # some at the lowest value, as places without a word
    c["top"][0::3] = 0.0
    c["top"][1::2, 1:] = -math.inf
    want = _run(c)
    c["top"][1::2, 1:] = lo
    got = _run(c)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # the whole range: the largest alone has a share
    c["top"][1::2, 0] = hi
    got = _run(c)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- gradients of very different sizes

def _check_dw(c, dw, dw0=None):
    """dW float32, row by row within what its own tokens allow.  edz, sums and the output as in
    test_gpu_head_forms.py, but a float16 dlogit that falls under the type's smallest number is off
    by no more than itself.  The float16 copy of h: a value h 2^e of gradient g = m 2^e is off by
    half of float16's smallest step, 2^-25, in units in which the largest has an exponent of 15,
    so by 2^-40 max |g h|; times m < 2 and the unit gradient |dz / g|, which is at most 1."""
    T, V = len(c["h"]), len(c["w"])
    _, _, dz, edz = _reference(c, torch.arange(T, device="cuda"))
    h = c["h"].double()
    hs = torch.zeros_like(edz)
    if c["h"].dtype == torch.float16:
        g = c["dloss"].double().abs()[:, None] * ((1 - c["alpha"]) + c["alpha"] * c["tau"])
        edz = edz - g * 2.0 ** -37 + torch.minimum(dz.abs(), g * 2.0 ** -37)
        reach = (g[:, 0] * h.abs().amax(1)).max()
        hs = torch.where(g > 0, dz.abs() / g, 0.0) * reach * 2.0 ** -39
    want = dz.t() @ h
    tol = (edz + T * F * dz.abs()).t() @ h.abs() + hs.sum(0)[:, None]
    if dw0 is not None:
        want = want + dw0.double()
    tol = tol + want.abs() * 2 * F
    off = (dw.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp(min=1e-300)).max())


def _spread(c, low, high, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = len(c["h"])
    d = torch.randn(T, generator=g, device="cuda") * torch.exp2(
        torch.randint(low, high + 1, (T,), generator=g, device="cuda").float())
    d[torch.rand(T, generator=g, device="cuda") < 0.2] = 0.0
    c["dloss"] = d


@pytest.mark.parametrize("T,K,tau", [(40, 0, 1.0), (40, 3, 2.0), (200, 0, 1.0), (200, 20, 0.5),
                                     (1500, 0, 1.0), (1500, 2, 1.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_small_gradients_beside_large_ones(T, K, tau, dtype):
    """dloss over 2^-20 .. 2^8.  Some words have small tokens only: their logits at the others are
    64 lower, and their rows of dW are as good as if the others were not there."""
    V, D, rare = 300, 96, 40
    c = _inputs(T, V, D, dtype, K=K, seed=T + K)
    c["tau"] = tau
    _spread(c, -20, 8)
    small = torch.arange(T, device="cuda") % 3 == 0
    c["dloss"][small] = c["dloss"][small].sign() * 2.0 ** -20
    c["dloss"][1] = 2.0 ** 8
    c["h"][:, 0] = torch.where(small, 0.0, 8.0).to(dtype)
    c["w"][:, 0] = 0.0
    c["w"][:rare, 0] = -8.0
    n = int(small.sum())
    c["y"] = torch.where(small, torch.arange(T, device="cuda") % rare, c["y"] % (V - rare) + rare)
    if K:
        c["ids"] = torch.where(small[:, None], c["ids"] % rare, c["ids"] % (V - rare) + rare)
    dw = torch.full((V, D), math.nan, device="cuda")
    _run(c, dW=dw)
    _check_dw(c, dw)
    # the same tokens alone
    if n > 1 and dtype == torch.float16:
        _check_dw(c, _run(c, dW=torch.zeros(V, D, device="cuda"), accumulate=True)[2])


@pytest.mark.parametrize("scale", [2.0 ** -24, 2.0 ** -10, 1.0, 2.0 ** 15])
def test_float16_rows_of_any_size(scale):
    """h from float16's smallest numbers to its largest, rows of zeros among them."""
    T, V, D = 70, 200, 64
    for rows in (T, 1100):
        c = _inputs(rows, V, D, torch.float16, seed=rows)
        c["h"] = (c["h"].float().clamp(-1.9, 1.9) * scale).to(torch.float16)
        c["h"][::9] = 0.0
        c["w"] = (c["w"].float() * 2.0 ** -16 if scale > 1 else c["w"].float()).to(torch.float16)
        _spread(c, -6, 6)
        _check_dw(c, _run(c, dW=torch.zeros(V, D, device="cuda"))[2])
        c["h"][:] = 0.0
        assert not _run(c)[2].any()


@pytest.mark.parametrize("T", [5, 1300])
def test_vanishing_and_infinite_gradients_of_float16_rows(T):
    """Gradients of float32's smallest numbers, and of zero once they are taken over the logits'
    unit (alpha tau = 1/4): a gradient of nothing adds nothing."""
    c = _inputs(T, 70, 24, torch.float16, K=3, seed=T)
    c.update(alpha=1.0, tau=0.25)
    c["h"] = (c["h"].float() * 2.0 ** -20).to(torch.float16)
    c["dloss"] = torch.full((T,), 1e-45, device="cuda")
    c["dloss"][0] = 1e-44
    _, dh, dw = _run(c)
    assert bool(torch.isfinite(dh.float()).all()) and bool(torch.isfinite(dw.float()).all())
    c = _inputs(T, 70, 24, torch.float16, seed=T)
    c["dloss"][3] = math.inf
    _, dh, dw = _run(c)
    rest = torch.arange(T, device="cuda") != 3
    assert bool(torch.isfinite(dh[rest].float()).all())
    assert not torch.isfinite(dh[3]).all() and not torch.isfinite(dw).any()


# ---------------------------------------------------------------- forms

def _some(n):
    return sorted({0, 1, n // 2, n - 2, n - 1, *range(0, n, max(1, n // 61))} & set(range(n)))


@pytest.mark.parametrize("T,V,D,K", [(3, 300, 65536, 0), (33, 70, 16392, 2), (70, 515, 32768, 3),
                                     (300, 260, 65536, 0), (1100, 130, 8200, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_wide_heads(T, V, D, K, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T + D, masked=0.1 if T > 3 else 0.0)
    _check(c, *_run(c))


@pytest.mark.parametrize("T,V,D,K,tau", [(16384, 20001, 264, 3, 2.0), (70001, 9001, 64, 1, 0.7),
                                         (256, 1100000, 64, 2, 1.5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_several_pieces_at_a_temperature(T, V, D, K, tau, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T + K, masked=0.1)
    c["tau"] = tau
    words = _some(V) + [v for v in (4095, 4096, 8191, 8192, 16383, 16384) if v < V]
    _check(c, *_run(c), tokens=_some(T), words=words)


@pytest.mark.parametrize("T,V,D,K,tau", [(1, 50000, 264, 64, 2.0), (16, 20001, 1000, 5, 0.5),
                                         (33, 33001, 72, 2, 1.5), (64, 9000, 2056, 17, 3.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_of_few_tokens_at_a_temperature(T, V, D, K, tau, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T + V, masked=0.2 if T > 6 else 0.0)
    c["tau"] = tau
    _check(c, *_run(c))
    dw0 = torch.randn(V, D, device="cuda")
    loss, dh, dw = _run(c, dW=dw0.clone(), accumulate=True)
    _check(c, loss, dh, dw, dw0=dw0)


@pytest.mark.parametrize("T,V,D,K,tau", [(600, 900, 136, 100, 1.0), (513, 2000, 72, 1024, 2.0),
                                         (2000, 300, 64, 257, 0.5), (512, 400, 64, 15, 1.0),
                                         (256, 400, 64, 27, 1.0), (256, 400, 64, 28, 1.0),
                                         (256, 400, 64, 28, 2.0), (257, 400, 64, 28, 1.0),
                                         (40, 900, 136, 75, 1.0), (1, 300, 64, 76, 0.5)])
def test_long_teachers(T, V, D, K, tau):
    c = _inputs(T, V, D, K=K, seed=T + K, masked=0.1)
    c["tau"] = tau
    c["ids"][::7, K // 2:] = -1
    _check(c, *_run(c))


@pytest.mark.parametrize("T,V,D,K,masked", [(3001, 5003, 264, 0, 0.6), (1500, 9000, 768, 2, 0.9),
                                            (5000, 1000, 72, 0, 0.999), (5000, 130, 512, 2, 0.9),
                                            (17000, 17000, 520, 0, 0.97)])
def test_weight_gradients_of_many_tokens_without_a_loss(T, V, D, K, masked):
    """dW's contraction is cut for all tokens: parts that are left without a row."""
    c = _inputs(T, V, D, K=K, seed=T + D, masked=masked)
    if K:
        c["ids"][c["y"] == IGNORE] = -1
    words = _some(V) + [v for v in (4095, 4096, 8191, 8192, 16383, 16384) if v < V]
    c["y"][5] = V - 1
    for kw in ({}, {"dW": torch.full((V, D), math.nan, device="cuda")},
               {"dW": torch.ones(V, D, device="cuda"), "accumulate": True}):
        ones = torch.ones(V, D, device="cuda") if "accumulate" in kw else None
        loss, _, dw = _run(c, want_dh=False, **kw)
        _check(c, loss, None, dw, words=words, dw0=ones)


@pytest.mark.parametrize("T,V,D,K", [(5, 70, 24, 3), (40, 1500, 72, 5), (300, 600, 136, 20)])
@pytest.mark.parametrize("tau", [2.0 ** -10, 2.0 ** -5, 2.0 ** 5, 2.0 ** 10])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_values_at_temperatures_far_from_one(T, V, D, K, tau, dtype):
    c = _inputs(T, V, D, dtype, K=K, seed=T)
    c["tau"] = tau
    _check(c, *_run(c))


@pytest.mark.parametrize("T,K", [(9, 3), (40, 30), (300, 5)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_a_teachers_infinity_or_nan_stays_with_its_token(T, K, value):
    c = _inputs(T, 90, 72, K=K, seed=T)
    want = _run(c)
    c["top"][4, 1] = value
    loss, dh, _ = _run(c)
    rest = torch.arange(T, device="cuda") != 4
    assert bool(torch.isnan(loss[4])) and not torch.isfinite(dh[4]).any()
    assert torch.equal(loss[rest], want[0][rest]) and torch.equal(dh[rest], want[1][rest])
    c["ids"][4, 1] = -1  # no word: nobody looks at it
    assert all(bool(torch.isfinite(t.float()).all()) for t in _run(c))
