"""Infinities and NaN in the forward calls: a token's reach its own outputs and
later ones of its sequence, and what depends on it; everything else keeps its
bits, as it does where tokens go one by one."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402
from test_gpu_seq import N, P, _scan_case  # noqa: E402

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _same(a, b):
    return torch.equal(a, b) and bool(b.isfinite().all())


# tokens at the borders of tiles and of their halves; one segment a sequence, and
# segments of 128 tokens; the last token falls into a tile that goes token by token
@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("at", [0, 1, 15, 31, 32, 47, 63, 64, 100, 127, 128, 257])
@pytest.mark.parametrize("offs,dtype", [([0, 5, 263, 300], torch.bfloat16),
                                        ([0, 5, 263, 900], torch.float32)])
@pytest.mark.parametrize("what", ["x", "B", "C", "dt"])
def test_scan_is_causal(what, offs, dtype, at, value):
    H, s, e = 3, offs[1], offs[2]
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, dtype, 5, 0.0)
    t = s + at
    ssm = torch.randn((3, H, P, N), generator=torch.Generator().manual_seed(1)).half().cuda()

    def run(zx, u):
        out = torch.empty_like(ssm)
        y = ops.mixer_scan(u, zx, dev["dt_bias"], dev["A_log"], dev["D"], off, ssm, ssm_out=out)
        return y[:offs[-1]].view(-1, H, P), out

    y0, s0 = run(zx, u)
    zx, u = zx.clone(), u.clone()
    if what == "dt":
        zx[t, zx.shape[1] - H + 1] = value
    else:
        u[t, {"x": P + 7, "B": d + 9, "C": d + N + 9}[what]] = value
    y, st = run(zx, u)
    assert _same(y0[:t], y[:t]) and _same(y0[e:], y[e:]), "tokens before, another sequence"
    assert _same(s0[0], st[0]) and _same(s0[2], st[2])
    if what == "x":
        keep = torch.ones((H, P), dtype=torch.bool, device="cuda")
        keep[1, 7] = False
        assert not y[t:e, 1, 7].isfinite().any() and not st[1, 1, 7].isfinite().any()
        assert _same(y0[:, keep], y[:, keep]) and _same(s0[1][keep], st[1][keep])
    elif what == "B":
        assert not y[t:e].isfinite().any() and not st[1, :, :, 9].isfinite().any()
    elif what == "C":
        assert not y[t].isfinite().any()
        assert _same(y0[t + 1:], y[t + 1:]) and _same(s0, st)
    else:
        if value == -INF:  # a step of zero, which leaves the state as it is
            assert bool(y.isfinite().all()) and bool(st.isfinite().all())
        else:
            assert not y[t:e, 1].isfinite().any() and not st[1, 1].isfinite().any()
        assert _same(y0[:, [0, 2]], y[:, [0, 2]]) and _same(s0[1, [0, 2]], st[1, [0, 2]])


def test_scan_of_many_such_values():
    """In every channel, at tokens of any tile: the first one counts."""
    offs, H = [0, 300], 2
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, torch.bfloat16, 6, 0.0)
    args = (zx, dev["dt_bias"], dev["A_log"], dev["D"], off)
    y0 = ops.mixer_scan(u, *args)[:300]
    first = torch.from_numpy(rng.integers(0, 300, d)).cuda()
    u = u.clone()
    for c, t in enumerate(first.tolist()):
        u[t, c] = NAN
        u[min(t + 1 + c % 70, 299), c] = INF
    y = ops.mixer_scan(u, *args)[:300]
    late = torch.arange(300, device="cuda")[:, None] >= first
    assert _same(y0[~late], y[~late]) and not y[late].isfinite().any()


@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("at", [0, 1, 7, 8, 40])
def test_conv_and_norm_are_causal(at, value):
    offs, H = [0, 5, 60, 90], 2
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, torch.bfloat16, 7, 0.0)
    t, c = offs[1] + at, 9

    def run(zx):
        return (ops.mixer_conv(zx, dev["conv_w"], dev["conv_b"], off)[:90],
                ops.mixer_norm(u[:, :d].contiguous(), zx, dev["norm_w"])[:90])

    u0, n0 = run(zx)
    zx = zx.clone()
    zx[t, d + c] = value
    zx[t, 3] = value
    u1, n1 = run(zx)
    hit = torch.zeros((90, cd), dtype=torch.bool, device="cuda")
    hit[t:min(t + 4, offs[2]), c] = True
    assert _same(u0[~hit], u1[~hit]) and not u1[t, c].isfinite()
    rows = torch.arange(90, device="cuda") != t
    assert _same(n0[rows], n1[rows]) and not n1[t].isfinite().all()
