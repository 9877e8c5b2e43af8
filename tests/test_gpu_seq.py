"""The mixer over packed sequences (convolution, scan, gated norm) and the
embedding against the float64 oracle, forward and backward.

Tolerances: an output rounded to a type is off by half a step of it (bfloat16
2^-8, float16 2^-11, float32 2^-24, of the value), plus the errors of what it
was computed from, relative to the sum of the terms' magnitudes:

* the convolution and the norm compute in float32: some ten roundings and two
  functions good to 2^-22, so 2^-19;
* the scan's y and states come from operands of two bfloat16 terms (2^-17 of
  the operand; the decayed C . B, the state, the state's coefficients), float32
  sums of at most 128 products and exponentials whose arguments are good to
  2^-24 of at most 20 that still matter: 2^-14;
* du's operands are of two or three terms: 2^-14; the float32 gradients come
  from three (2^-25) and float32 sums of at most 128 products, added up over the
  chunks and heads: 2^-17.

Inputs are bfloat16 where the calls take bfloat16, so nothing else is rounded.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mamba_seq as O  # noqa: E402
from paper_2606_18114_amd import ops, synth  # noqa: E402

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
P, N = 64, 128


def _t(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def near(name, got, ref, mag, rel, half=True):
    step = HALF[got.dtype] if half else 0.0
    # below the type's smallest normal number the steps do not shrink further: float16's
    # are 2^-24 there, so its rounding is off by up to 2^-25 whatever the value
    least = step * torch.finfo(got.dtype).smallest_normal
    g = _np(got)
    assert g.shape == ref.shape, name
    tol = step * np.abs(ref) + (1.0 + step) * rel * np.abs(mag) + least
    bad = ~(np.abs(g - ref) <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(g - ref) / tol, 0.0)), bad.shape)
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, worst at {i}: got {g[i]}, "
                             f"expected {ref[i]}, tolerance {tol[i]}")


def _layer(rng, T, H, dtype, dt_shift=0.0):
    d, cd = H * P, H * P + 2 * N
    prm = {k: v for k, v in synth.mixer_params(rng, H).items()}
    prm["D"] = (1.0 + 0.2 * rng.standard_normal(H)).astype(np.float32)
    zx = _t(rng.standard_normal((T, d + cd + H)) + 0.0, dtype)
    if dt_shift:
        zx[:, -H:] += dt_shift
    return prm, {k: _t(v) for k, v in prm.items()}, zx, d, cd


# offsets of the packed sequences: one token; shorter than the taps; ends that
# fall inside, on and right behind tiles of 64 and 128; empty sequences at the
# beginning, in the middle and at the end; tokens behind the last one
PACKS = [
    [0, 1],
    [0, 1, 2, 5, 9],
    [0, 63, 127, 191],
    [0, 64, 128, 256, 385],
    [0, 0, 65, 65, 65, 194, 194],
    [0, 130, 300],
]
TAIL = 7  # tokens behind the last sequence


def _seqs(offs):
    return [(i, a, b) for i, (a, b) in enumerate(zip(offs, offs[1:])) if b > a]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 5, 8])
@pytest.mark.parametrize("offs", PACKS)
def test_conv(offs, H, dtype):
    rng = np.random.default_rng(len(offs) * 100 + H)
    T = offs[-1] + TAIL
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype)
    S, pos = len(offs) - 1, 1 + H % 3
    ring = _t(rng.standard_normal((S, cd, 4)), torch.float16)
    conv_pos = torch.full((1,), pos, dtype=torch.int32, device="cuda")
    off = torch.tensor(offs, dtype=torch.int32, device="cuda")
    u = torch.full((T, cd), 7.0, dtype=torch.bfloat16, device="cuda")
    new = torch.full_like(ring, 9.0)
    ops.mixer_conv(zx, dev["conv_w"], dev["conv_b"], off, ring, conv_pos, conv_out=new, u=u)
    same = ring.clone()
    ops.mixer_conv(zx, dev["conv_w"], dev["conv_b"], off, same, conv_pos, conv_out=same)
    x = _np(zx[:, d:d + cd])
    past = np.roll(_np(ring), -pos, axis=2).transpose(0, 2, 1)  # [S, 4, cd], oldest first
    want_ring = past.copy()
    for i, a, b in _seqs(offs):
        ref = O.conv(x[a:b], prm["conv_w"], prm["conv_b"], past[i])
        mag = np.abs(prm["conv_b"]) + sum(np.abs(v) for v in [np.concatenate(
            [past[i][-3:], x[a:b]])[j:j + b - a] * prm["conv_w"][:, j] for j in range(4)])
        near(f"u of sequence {i}", u[a:b], ref, mag, 2.0 ** -19)
        want_ring[i] = np.concatenate([past[i], x[a:b]])[-4:]
    assert bool((u[offs[-1]:] == 7.0).all()), "rows behind the last sequence were written"
    want = np.roll(want_ring.transpose(0, 2, 1), pos, axis=2).astype(np.float16)
    assert np.array_equal(new.cpu().numpy(), want)
    assert np.array_equal(same.cpu().numpy(), want), "the ring in place"
    assert int(conv_pos.item()) == pos


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 5, 8])
@pytest.mark.parametrize("offs", PACKS)
def test_conv_bwd(offs, H, dtype):
    rng = np.random.default_rng(len(offs) * 100 + H + 50)
    T = offs[-1] + TAIL
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype)
    du = _t(0.1 * rng.standard_normal((T, cd)), torch.bfloat16)
    off = torch.tensor(offs, dtype=torch.int32, device="cuda")
    dzx = torch.full_like(zx, 3.0)
    dw, db = ops.mixer_conv_bwd(zx, dev["conv_w"], dev["conv_b"], du, dzx, off)
    x, g = _np(zx[:, d:d + cd]), _np(du)
    tw, tb, mw, mb = 0.0, 0.0, 0.0, 0.0
    for i, a, b in _seqs(offs):
        r = O.conv_bwd(x[a:b], prm["conv_w"], prm["conv_b"], g[a:b])
        m = O.conv_bwd(x[a:b], prm["conv_w"], prm["conv_b"], g[a:b], absolute=True)
        # SiLU' loses relative accuracy around its zero: the magnitude of du itself counts
        mx = m[0] + sum(np.abs(prm["conv_w"][:, j]) for j in range(4)) * np.abs(g[a:b]).max()
        near(f"dx of sequence {i}", dzx[a:b, d:d + cd], r[0], mx, 2.0 ** -19)
        tw, tb = tw + r[1], tb + r[2]
        mw, mb = mw + m[1], mb + m[2]
    scale = np.abs(g).sum(0)
    near("dconv_w", dw, tw, mw + scale[:, None] * np.abs(x).max(), 2.0 ** -19)
    near("dconv_b", db, tb, mb + scale, 2.0 ** -19)
    assert bool((dzx[:, :d] == 3.0).all()) and bool((dzx[:, d + cd:] == 3.0).all())
    assert bool((dzx[offs[-1]:] == 3.0).all())


def _scan_case(offs, H, dtype, seed, dt_shift):
    rng = np.random.default_rng(seed)
    T = offs[-1] + TAIL
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype, dt_shift)
    v = rng.standard_normal((T, cd))
    u = _t(v / (1.0 + np.exp(-v)), torch.bfloat16)
    off = torch.tensor(offs, dtype=torch.int32, device="cuda")
    un = _np(u)
    parts = (un[:, :d].reshape(T, H, P), un[:, d:d + N], un[:, d + N:], _np(zx[:, -H:]))
    return rng, T, prm, dev, zx, u, off, parts, d, cd


# dt_shift 4: decays that forget within a few tokens (exponents in the hundreds)
@pytest.mark.parametrize("dt_shift", [0.0, 4.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 5])
@pytest.mark.parametrize("offs", PACKS)
def test_scan(offs, H, dtype, dt_shift):
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(
        offs, H, dtype, len(offs) * 100 + H, dt_shift)
    S = len(offs) - 1
    ssm = _t(0.5 * rng.standard_normal((S, H, P, N)), torch.float16)
    y = torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    new = torch.full_like(ssm, 9.0)
    args = (u, zx, dev["dt_bias"], dev["A_log"], dev["D"], off)
    ops.mixer_scan(*args, ssm, ssm_out=new, y=y)
    same = ssm.clone()
    ops.mixer_scan(*args, same, ssm_out=same)
    zero = ops.mixer_scan(*args)
    s0 = _np(ssm)
    for i, a, b in _seqs(offs):
        seq = (x[a:b], B[a:b], C[a:b], dt[a:b], prm["dt_bias"], prm["A_log"])
        mags = (np.abs(x[a:b]), np.abs(B[a:b]), np.abs(C[a:b]), dt[a:b], prm["dt_bias"],
                prm["A_log"])
        ry, rs = O.scan(*seq, prm["D"], s0[i])
        my, ms = O.scan(*mags, np.abs(prm["D"]), np.abs(s0[i]))
        near(f"y of sequence {i}", y[a:b].reshape(-1, H, P), ry, my, 2.0 ** -14)
        near(f"state of sequence {i}", new[i], rs, ms, 2.0 ** -14)
        ry, _ = O.scan(*seq, prm["D"])
        my, _ = O.scan(*mags, np.abs(prm["D"]))
        near(f"y of sequence {i} from zero", zero[a:b].reshape(-1, H, P), ry, my, 2.0 ** -14)
    for i in range(S):
        if offs[i] == offs[i + 1]:
            assert torch.equal(new[i], ssm[i]), "an empty sequence's state"
    assert torch.equal(same, new), "the state in place"
    assert bool((y[offs[-1]:] == 7.0).all()), "rows behind the last sequence were written"


# long enough for sequences to be cut into segments whose states meet: in the
# workgroups themselves (32 heads) and by a launch in between (2 heads)
@pytest.mark.parametrize("H,offs", [(32, [0, 700, 700, 703, 1100]), (2, [0, 2300, 2600])])
def test_scan_segments(H, offs):
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(offs, H, torch.bfloat16, H, 0.0)
    S = len(offs) - 1
    ssm = _t(0.5 * rng.standard_normal((S, H, P, N)), torch.float16)
    args = (u, zx, dev["dt_bias"], dev["A_log"], dev["D"], off)
    new, same = torch.empty_like(ssm), ssm.clone()
    outs = [(ops.mixer_scan(*args, ssm, ssm_out=new), new),
            (ops.mixer_scan(*args, same, ssm_out=same), same),
            (ops.mixer_scan(*args, ssm), None)]
    s0 = _np(ssm)
    for i, a, b in _seqs(offs):
        ry, rs = O.scan(x[a:b], B[a:b], C[a:b], dt[a:b], prm["dt_bias"], prm["A_log"], prm["D"],
                        s0[i])
        my, ms = O.scan(np.abs(x[a:b]), np.abs(B[a:b]), np.abs(C[a:b]), dt[a:b], prm["dt_bias"],
                        prm["A_log"], np.abs(prm["D"]), np.abs(s0[i]))
        for y, st in outs:
            near(f"y of sequence {i}", y[a:b].reshape(-1, H, P), ry, my, 2.0 ** -14)
            if st is not None:
                near(f"state of sequence {i}", st[i], rs, ms, 2.0 ** -14)


def test_scan_in_place_at_length():
    """Many segments of many heads, more than the chip takes at once: the states
    in place are those out of place (to the rounding of the two ways they meet)."""
    T, H = 9000, 64
    rng = np.random.default_rng(3)
    g = torch.Generator(device="cuda").manual_seed(3)
    prm = {k: _t(v) for k, v in synth.mixer_params(rng, H).items()}
    zx = torch.randn(T, 2 * H * P + 256 + H, generator=g, device="cuda").to(torch.bfloat16)
    u = torch.randn(T, H * P + 256, generator=g, device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, 8000, T], dtype=torch.int32, device="cuda")
    ssm = torch.randn(2, H, P, N, generator=g, device="cuda").to(torch.float16)
    args = (u, zx, prm["dt_bias"], prm["A_log"], prm["D"], off)
    new, same = torch.empty_like(ssm), ssm.clone()
    a = ops.mixer_scan(*args, ssm, ssm_out=new)
    b = ops.mixer_scan(*args, same, ssm_out=same)
    # both round once; before that they differ by float32 sums in another order
    for x, y, step in ((a, b, 2.0 ** -7), (new, same, 2.0 ** -10)):
        x, y = x.double(), y.double()
        assert bool(((x - y).abs() <= step * y.abs() + 2.0 ** -14 * y.abs().max()).all())


@pytest.mark.parametrize("dt_shift", [0.0, 4.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [1, 5])
@pytest.mark.parametrize("offs", PACKS)
def test_scan_bwd(offs, H, dtype, dt_shift):
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(
        offs, H, dtype, len(offs) * 100 + H + 50, dt_shift)
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    dzx = torch.full_like(zx, 3.0)
    du = torch.full((T, cd), 7.0, dtype=torch.bfloat16, device="cuda")
    _, dbias, dalog, dd = ops.mixer_scan_bwd(u, zx, dev["dt_bias"], dev["A_log"], dev["D"], dy,
                                             dzx, off, du=du)
    g = _np(dy).reshape(T, H, P)
    total, mag = 0.0, 0.0
    for i, a, b in _seqs(offs):
        seq = (x[a:b], B[a:b], C[a:b], dt[a:b], prm["dt_bias"], prm["A_log"], prm["D"], g[a:b])
        r, m = O.scan_bwd(*seq), O.scan_bwd(*seq, absolute=True)
        near(f"dx of sequence {i}", du[a:b, :d].reshape(-1, H, P), r[0], m[0], 2.0 ** -14)
        near(f"dB of sequence {i}", du[a:b, d:d + N], r[1], m[1], 2.0 ** -14)
        near(f"dC of sequence {i}", du[a:b, d + N:], r[2], m[2], 2.0 ** -14)
        near(f"ddt of sequence {i}", dzx[a:b, -H:], r[3], m[3], 2.0 ** -17)
        total = total + np.stack(r[4:])
        mag = mag + np.stack(m[4:])
    near("ddt_bias", dbias, total[0], mag[0], 2.0 ** -17)
    near("dA_log", dalog, total[1], mag[1], 2.0 ** -17)
    near("dD", dd, total[2], mag[2], 2.0 ** -17)
    assert bool((dzx[:, :-H] == 3.0).all()) and bool((dzx[offs[-1]:] == 3.0).all())
    assert bool((du[offs[-1]:] == 7.0).all())


@pytest.mark.parametrize("T", [1, 100, 128])
def test_scan_bwd_of_one_chunk(T):
    """Up to 128 tokens there are no states between chunks; the same tokens in a
    longer batch give the same bits."""
    rng, n, prm, dev, zx, u, off, _, d, cd = _scan_case([0, T, T + 130], 1, torch.float32, T, 0.0)
    dy = _t(0.1 * rng.standard_normal((n, d)), torch.bfloat16)
    par = (dev["dt_bias"], dev["A_log"], dev["D"])
    dzx, short = torch.zeros_like(zx), torch.zeros_like(zx[:T])
    du, *_ = ops.mixer_scan_bwd(u, zx, *par, dy, dzx, off)
    got, *heads = ops.mixer_scan_bwd(u[:T], zx[:T], *par, dy[:T], short)
    assert torch.equal(got, du[:T]) and torch.equal(short, dzx[:T])
    alone = torch.tensor([0, T, T], dtype=torch.int32, device="cuda")
    _, *same = ops.mixer_scan_bwd(u, zx, *par, dy, dzx, alone)
    assert all(torch.equal(a, b) for a, b in zip(heads, same))


def test_scan_outlier_steps():
    """Single tokens whose step is so long that the state before them is gone
    (exponents of millions): the decays among the tokens behind them keep their
    accuracy, forward and backward."""
    offs, H = [0, 130, 300], 2
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, torch.float32, 77, 0.0)
    for t in (20, 64, 150, 299):
        zx[t, -H:] = 3.0e5
    un = _np(u)
    x, B, C, dt = (un[:, :d].reshape(T, H, P), un[:, d:d + N], un[:, d + N:], _np(zx[:, -H:]))
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    args = (u, zx, dev["dt_bias"], dev["A_log"], dev["D"])
    y = ops.mixer_scan(*args, off)
    dzx = torch.empty_like(zx)
    du, *heads = ops.mixer_scan_bwd(*args, dy, dzx, off)
    g = _np(dy).reshape(T, H, P)
    total, mag = 0.0, 0.0
    for i, a, b in _seqs(offs):
        seq = (x[a:b], B[a:b], C[a:b], dt[a:b], prm["dt_bias"], prm["A_log"], prm["D"])
        ry, _ = O.scan(*seq)
        my, _ = O.scan(*(np.abs(v) for v in seq[:3]), *seq[3:6], np.abs(prm["D"]))
        near(f"y of sequence {i}", y[a:b].reshape(-1, H, P), ry, my, 2.0 ** -14)
        r, m = O.scan_bwd(*seq, g[a:b]), O.scan_bwd(*seq, g[a:b], absolute=True)
        near(f"dx of sequence {i}", du[a:b, :d].reshape(-1, H, P), r[0], m[0], 2.0 ** -14)
        near(f"dB of sequence {i}", du[a:b, d:d + N], r[1], m[1], 2.0 ** -14)
        near(f"dC of sequence {i}", du[a:b, d + N:], r[2], m[2], 2.0 ** -14)
        near(f"ddt of sequence {i}", dzx[a:b, -H:], r[3], m[3], 2.0 ** -17)
        total, mag = total + np.stack(r[4:]), mag + np.stack(m[4:])
    for k, name in enumerate(("ddt_bias", "dA_log", "dD")):
        near(name, heads[k], total[k], mag[k], 2.0 ** -17)


def test_scan_steps_that_end_every_state():
    """A_log beyond what float32's e^A_log holds, and steps of 2^-4096 and less:
    every token stands alone, with no gradient through the state."""
    offs, H = [0, 130, 131, 300], 2
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, torch.float32, 78, 0.0)
    prm["A_log"] = np.array([100.0, 20.0], np.float32)
    dev["A_log"] = _t(prm["A_log"])
    un, dtn = _np(u), _np(zx[:, -H:])
    x, B, C = un[:, :d].reshape(T, H, P), un[:, d:d + N], un[:, d + N:]
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    args = (u, zx, dev["dt_bias"], dev["A_log"], dev["D"])
    y = ops.mixer_scan(*args, off)
    dzx = torch.empty_like(zx)
    du, *heads = ops.mixer_scan_bwd(*args, dy, dzx, off)
    g = _np(dy).reshape(T, H, P)
    for i, a, b in _seqs(offs):
        seq = (x[a:b], B[a:b], C[a:b], dtn[a:b], prm["dt_bias"], prm["A_log"], prm["D"])
        ry, _ = O.scan(*seq)
        my, _ = O.scan(*(np.abs(v) for v in seq[:3]), *seq[3:6], np.abs(prm["D"]))
        near(f"y of sequence {i}", y[a:b].reshape(-1, H, P), ry, my, 2.0 ** -14)
        r, m = O.scan_bwd(*seq, g[a:b]), O.scan_bwd(*seq, g[a:b], absolute=True)
        near(f"dx of sequence {i}", du[a:b, :d].reshape(-1, H, P), r[0], m[0], 2.0 ** -14)
        near(f"dB of sequence {i}", du[a:b, d:d + N], r[1], m[1], 2.0 ** -14)
        near(f"dC of sequence {i}", du[a:b, d + N:], r[2], m[2], 2.0 ** -14)
    assert all(bool(v.isfinite().all()) for v in heads)


@pytest.mark.parametrize("H", [2, 300])
@pytest.mark.parametrize("where", ["behind", "sequence"])
def test_what_is_not_a_sequences_own_stays_out(where, H):
    """NaN in the tokens behind the last sequence reaches nothing; NaN in all of
    one sequence reaches no output of the others' tokens."""
    offs = [0, 65, 130, 194]
    rng, T, prm, dev, zx, u, off, _, d, cd = _scan_case(offs, H, torch.bfloat16, 79, 0.0)
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    du = _t(0.1 * rng.standard_normal((T, cd)), torch.bfloat16)
    bad = slice(offs[-1], T) if where == "behind" else slice(offs[1], offs[2])
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[offs[-1]:] = False
    keep[bad] = False

    def run(spoil):
        v = [t.clone() for t in (zx, u, dy, du)]
        if spoil:
            for t in v:
                t[bad] = float("nan")
        z, uu, g, gu = v
        rows, sums = [torch.zeros_like(z)], []
        rows.append(ops.mixer_conv(z, dev["conv_w"], dev["conv_b"], off))
        rows.append(ops.mixer_scan(uu, z, dev["dt_bias"], dev["A_log"], dev["D"], off))
        rows.append(torch.full_like(g, 5.0))
        ops.mixer_norm(g, z, dev["norm_w"], 0.0, rows[-1], off)
        a, w = ops.mixer_norm_bwd(g, z, dev["norm_w"], gu[:, :d].contiguous(), rows[0], 0.0, off)
        rows.append(a)
        sums.append(w)
        a, *w = ops.mixer_scan_bwd(uu, z, dev["dt_bias"], dev["A_log"], dev["D"], g, rows[0], off)
        rows.append(a)
        sums += w
        sums += ops.mixer_conv_bwd(z, dev["conv_w"], dev["conv_b"], gu, rows[0], off)
        assert bool((rows[3][offs[-1]:] == 5.0).all()) and bool((rows[0][offs[-1]:] == 0.0).all())
        return [r[keep] for r in rows] + (sums if where == "behind" else [])

    for i, (a, b) in enumerate(zip(run(False), run(True))):
        assert bool(a.isfinite().all()) and torch.equal(a, b), i


@pytest.mark.parametrize("H", [1, 300])
def test_norm_of_no_rows(H):
    """All rows behind the last sequence: nothing is written, the sums are zero."""
    T, d = 5, 64 * H
    rng = np.random.default_rng(H)
    prm, dev, zx, d, cd = _layer(rng, T, H, torch.bfloat16)
    y = _t(rng.standard_normal((T, d)), torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, dzx = torch.full_like(y, 5.0), torch.full_like(zx, 3.0)
    ops.mixer_norm(y, zx, dev["norm_w"], 1e-5, out, off)
    _, dw = ops.mixer_norm_bwd(y, zx, dev["norm_w"], y, dzx, 1e-5, off)
    assert bool((out == 5.0).all()) and bool((dzx == 3.0).all()) and bool((dw == 0.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1, 1), (3, 5), (5, 12), (4, 24), (2, 64), (2, 100), (2, 200),
                                 (3, 300)])
def test_norm(T, H, dtype):
    rng = np.random.default_rng(T * 1000 + H)
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype)
    y = _t(rng.standard_normal((T, d)), torch.bfloat16)
    dout = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    if T > 1:
        y[0] = 0  # a row without anything: only eps under the root
    out = ops.mixer_norm(y, zx, dev["norm_w"], 1e-5)
    dzx = torch.full_like(zx, 3.0)
    dy, dw = ops.mixer_norm_bwd(y, zx, dev["norm_w"], dout, dzx, 1e-5)
    a = (_np(y), _np(zx[:, :d]), prm["norm_w"], float(np.float32(1e-5)))
    ref = O.norm(*a)
    near("out", out, ref, ref, 2.0 ** -19)
    r = O.norm_bwd(*a, _np(dout))
    m = O.norm_bwd(*a, _np(dout), absolute=True)
    near("dy", dy, r[0], m[0], 2.0 ** -19)
    # SiLU' around its zero: its terms' magnitudes, at most |dg y|
    sig = 1.0 / (1.0 + np.exp(-a[1]))
    flat = m[1] / np.maximum(np.abs(sig * (1 + a[1] * (1 - sig))), 1e-9)
    near("dz", dzx[:, :d], r[1], flat, 2.0 ** -19)
    near("dnorm_w", dw, r[2], m[2], 2.0 ** -19)
    assert bool((dzx[:, d:] == 3.0).all())


def test_norm_many_rows():
    """More rows than the backward has row groups."""
    T, H = 2500, 1
    rng = np.random.default_rng(9)
    prm, dev, zx, d, cd = _layer(rng, T, H, torch.float32)
    y = _t(rng.standard_normal((T, d)), torch.bfloat16)
    dout = _t(rng.standard_normal((T, d)), torch.bfloat16)
    dzx = torch.empty_like(zx)
    _, dw = ops.mixer_norm_bwd(y, zx, dev["norm_w"], dout, dzx, 1e-5)
    a = (_np(y), _np(zx[:, :d]), prm["norm_w"], float(np.float32(1e-5)), _np(dout))
    near("dnorm_w", dw, O.norm_bwd(*a)[2], O.norm_bwd(*a, absolute=True)[2], 2.0 ** -17)


@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (3, 7, 5), (70, 11, 67), (300, 1000, 256)])
def test_embed(T, V, D, w_dtype, ids_dtype):
    rng = np.random.default_rng(T + V)
    ids = rng.integers(-1, V + 1, T)  # some outside: padding
    if ids_dtype == torch.int64 and T > 1:
        ids[1] = 2 ** 40
    w = _t(rng.standard_normal((V, D)), w_dtype)
    out = ops.embed(torch.from_numpy(ids).to(ids_dtype).cuda(), w, 1.5)
    ok = (ids >= 0) & (ids < V)
    ref = np.where(ok[:, None], _np(w)[np.clip(ids, 0, V - 1)] * 1.5, 0.0)
    near("rows", out, ref, ref, 0.0)


# one id for all tokens (in pieces), exactly 64 and 65 of one, all different; few
# enough tokens for a row's workgroup to find its own (up to 256), for a token's
# (up to 4096), and more, sorted
@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("D", [1, 67, 256])
@pytest.mark.parametrize("kind", ["one", "same", "edge", "apart", "mixed", "few", "few_same", "few_wide", "odd",
                                  "most", "long", "long_same", "long_wide"])
def test_embed_bwd(kind, D, ids_dtype):
    rng = np.random.default_rng(D)
    V = {"odd": 301, "long_wide": 74001, "few_wide": 16500}.get(kind, 300)
    ids = {"one": np.array([3]), "same": np.full(1000, 17),
           "edge": np.repeat([5, 299, 0], [64, 65, 129]),
           "apart": rng.permutation(V), "mixed": np.minimum(rng.geometric(0.02, 3000) - 2, V),
           "few": rng.integers(-1, V + 1, 256), "few_same": np.full(200, 299),
           "few_wide": rng.integers(-1, V + 1, 200),
           "odd": rng.integers(-1, V + 1, 500),
           "most": np.minimum(rng.geometric(0.02, 4096) - 2, V),
           "long": np.minimum(rng.geometric(0.02, 9000) - 2, V),
           "long_same": np.repeat([5, 299, 0, 7], [64, 65, 129, 4097]),
           "long_wide": np.minimum(rng.geometric(0.001, 5000) * 7, V)}[kind]
    rng.shuffle(ids)
    T = len(ids)
    de = _t(rng.standard_normal((T, D)))
    t = torch.from_numpy(ids).to(ids_dtype).cuda()
    dW = ops.embed_bwd(t, de, V, 0.5)
    ref = O.embed_bwd(ids, _np(de), V, 0.5)
    mag = O.embed_bwd(ids, np.abs(_np(de)), V, 0.5)
    near("dW", dW, ref, mag, 2.0 ** -17)
    assert torch.equal(dW, ops.embed_bwd(t, de, V, 0.5)), "repeated calls differ"
    base = torch.ones_like(dW)
    ops.embed_bwd(t, de, V, 0.5, dW=base, accumulate=True)
    near("dW accumulated", base, ref + 1.0, mag + 1.0, 2.0 ** -17)
