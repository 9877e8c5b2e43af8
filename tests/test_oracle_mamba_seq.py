"""Pins of the sequence oracle: its forward is the decode step's oracle taken
token by token, its gradients are central differences of its forward."""

import numpy as np
import pytest

from oracle import mamba as M
from oracle import mamba_seq as O

P, N = 3, 4  # the oracle takes any sizes


def _case(rng, L, H):
    d, cd = H * P, H * P + 2 * N
    return dict(x=rng.standard_normal((L, H, P)), B=rng.standard_normal((L, N)),
                C=rng.standard_normal((L, N)), dt=rng.standard_normal((L, H)),
                dt_bias=rng.standard_normal(H) - 1.0, A_log=0.3 * rng.standard_normal(H),
                D=rng.standard_normal(H)), d, cd


def _numeric(f, args, name, g, eps=1e-6):
    base = {k: np.array(v, np.float64) for k, v in args.items()}
    out = np.zeros_like(base[name])
    for i in np.ndindex(out.shape):
        v = base[name][i]
        base[name][i] = v + eps
        up = (f(**base) * g).sum()
        base[name][i] = v - eps
        dn = (f(**base) * g).sum()
        base[name][i] = v
        out[i] = (up - dn) / (2 * eps)
    return out


def test_forward_is_the_decode_step_token_by_token():
    rng = np.random.default_rng(0)
    L, H = 7, 2
    d, cd = H * P, H * P + 2 * N
    zx = rng.standard_normal((L, 2 * d + 2 * N + H))
    w, b = rng.standard_normal((cd, 4)), rng.standard_normal(cd)
    prm = dict(dt_bias=rng.standard_normal(H), A_log=0.3 * rng.standard_normal(H),
               D=rng.standard_normal(H))
    norm_w = rng.standard_normal(d)
    z, xbc, dt = M.split_in_proj(zx, d, N, H)
    u = O.conv(xbc, w, b)
    y, state = O.scan(u[:, :d].reshape(L, H, P), u[:, d:d + N], u[:, d + N:], dt, **prm)
    out = O.norm(y.reshape(L, d), z, norm_w, 1e-5)
    # the step oracle keeps its states in float16: 2^-11 of them a token
    conv, ssm = np.zeros((1, cd, 4), np.float16), np.zeros((1, H, P, N), np.float16)
    for t in range(L):
        ref, conv, ssm = M.mixer_step(zx[t:t + 1], conv, ssm, w, b, prm["dt_bias"], prm["A_log"],
                                      prm["D"], norm_w, 1e-5, P, N)
        assert np.allclose(out[t], ref[0], rtol=0, atol=2e-2), t
    assert np.allclose(state, ssm[0].astype(np.float64), rtol=0, atol=2e-2)


@pytest.mark.parametrize("L", [1, 2, 5])
def test_conv_gradients_are_differences(L):
    rng = np.random.default_rng(L)
    args = dict(x=rng.standard_normal((L, 6)), w=rng.standard_normal((6, 4)),
                b=rng.standard_normal(6))
    g = rng.standard_normal((L, 6))
    got = O.conv_bwd(args["x"], args["w"], args["b"], g)
    for name, v in zip(("x", "w", "b"), got):
        assert np.allclose(v, _numeric(O.conv, args, name, g), rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("L", [1, 2, 5])
def test_scan_gradients_are_differences(L):
    rng = np.random.default_rng(L + 10)
    args, _, _ = _case(rng, L, 2)
    g = rng.standard_normal((L, 2, P))
    got = O.scan_bwd(args["x"], args["B"], args["C"], args["dt"], args["dt_bias"], args["A_log"],
                     args["D"], g)
    f = lambda **kw: O.scan(**kw)[0]  # noqa: E731
    for name, v in zip(("x", "B", "C", "dt", "dt_bias", "A_log", "D"), got):
        assert np.allclose(v, _numeric(f, args, name, g), rtol=1e-6, atol=1e-7), name


def test_scan_goes_on_from_a_state():
    rng = np.random.default_rng(3)
    args, _, _ = _case(rng, 9, 2)
    par = [args[k] for k in ("dt_bias", "A_log", "D")]
    seq = [args[k] for k in ("x", "B", "C", "dt")]
    y, s = O.scan(*seq, *par)
    y0, s0 = O.scan(*(v[:4] for v in seq), *par)
    y1, s1 = O.scan(*(v[4:] for v in seq), *par, state=s0)
    assert np.allclose(np.concatenate([y0, y1]), y) and np.allclose(s1, s)


def test_norm_gradients_are_differences():
    rng = np.random.default_rng(4)
    args = dict(y=rng.standard_normal((2, 5)), z=rng.standard_normal((2, 5)),
                w=rng.standard_normal(5))
    g = rng.standard_normal((2, 5))
    f = lambda y, z, w: O.norm(y, z, w, 1e-3)  # noqa: E731
    got = O.norm_bwd(args["y"], args["z"], args["w"], 1e-3, g)
    for name, v in zip(("y", "z", "w"), got):
        assert np.allclose(v, _numeric(f, args, name, g), rtol=1e-6, atol=1e-7), name


def test_embed_gradient_is_its_scatter():
    ids = np.array([2, 0, 2, -1, 5])
    dW = O.embed_bwd(ids, np.arange(10.0).reshape(5, 2), 3, 2.0)
    assert np.array_equal(dW, [[4.0, 6.0], [0.0, 0.0], [8.0, 12.0]])
