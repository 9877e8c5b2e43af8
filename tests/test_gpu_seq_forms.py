"""The forms of the sequence kernels that the sizes of ``test_gpu_seq.py`` do not
reach, against the same float64 oracle: backward workgroups of several heads,
convolution runs longer than a token, embedding rows wider than a workgroup's
step, steps that end every state.  Tolerances as derived there; a sum over many
tokens adds 2^-24 of its terms' magnitudes for every link of its longest chain
of float32 additions.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mamba_seq as O  # noqa: E402
from paper_2606_18114_amd import ops  # noqa: E402
from test_gpu_seq import N, P, TAIL, _layer, _np, _scan_case, _seqs, _t, near  # noqa: E402

pytestmark = pytest.mark.gpu


def _off(offs):
    return torch.tensor(offs, dtype=torch.int32, device="cuda")


def _packed(lengths):
    return [0, *np.cumsum(lengths).tolist()]


def _scan_bwd_ref(seqs, T, H, d, cd, x, B, C, dt, prm, g):
    """Gradients of the packed sequences and their terms' magnitudes:
    [(du, ddt, [ddt_bias, dA_log, dD]), the same]."""
    out = []
    for absolute in (False, True):
        du, ddt, heads = np.zeros((T, cd)), np.zeros((T, H)), np.zeros((3, H))
        for _, a, b in seqs:
            r = O.scan_bwd(x[a:b], B[a:b], C[a:b], dt[a:b], prm["dt_bias"], prm["A_log"],
                           prm["D"], g[a:b], absolute=absolute)
            du[a:b] = np.concatenate([r[0].reshape(-1, d), r[1], r[2]], 1)
            ddt[a:b] = r[3]
            heads += np.stack(r[4:])
        out.append((du, ddt, heads))
    return out


# 406 chunks and ends: two groups, of three and two heads a workgroup; 900: one
# group of all five.  The long sequences lie before, between and behind the short
# ones, so that states enter and gradients reach chunks beside those without any
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [[300] + [1] * 400, [1] * 350 + [300, 0, 130] + [2] * 500 + [257]])
def test_scan_bwd_of_several_heads_a_workgroup(lengths, dtype):
    offs, H = _packed(lengths), 5
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(
        offs, H, dtype, len(lengths), 0.0)
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    dzx = torch.full_like(zx, 3.0)
    du = torch.full((T, cd), 7.0, dtype=torch.bfloat16, device="cuda")
    _, *heads = ops.mixer_scan_bwd(u, zx, dev["dt_bias"], dev["A_log"], dev["D"], dy, dzx, off,
                                   du=du)
    (rdu, rdt, rh), (mdu, mdt, mh) = _scan_bwd_ref(_seqs(offs), T, H, d, cd, x, B, C, dt, prm,
                                                   _np(dy).reshape(T, H, P))
    e = offs[-1]
    for name, sl in (("dx", slice(0, d)), ("dB", slice(d, d + N)), ("dC", slice(d + N, cd))):
        near(name, du[:e, sl], rdu[:e, sl], mdu[:e, sl], 2.0 ** -14)
    near("ddt", dzx[:e, -H:], rdt[:e], mdt[:e], 2.0 ** -17)
    for k, name in enumerate(("ddt_bias", "dA_log", "dD")):
        near(name, heads[k], rh[k], mh[k], 2.0 ** -17)
    assert bool((dzx[:, :-H] == 3.0).all()) and bool((dzx[e:] == 3.0).all())
    assert bool((du[e:] == 7.0).all())


# sequences of several segments beside many of one: their states meet in the
# workgroups themselves (H = 2: segments of 128 tokens, 12 of them) and in a launch
# in between (24 of them; and always in place)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [[1] * 100 + [300, 0, 700] + [2] * 60 + [259],
                                     [900] + [3] * 200 + [128, 256, 0, 1000] + [1] * 50])
def test_scan_of_many_sequences(lengths, dtype):
    offs, H = _packed(lengths), 2
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(
        offs, H, dtype, len(lengths), 0.0)
    S = len(offs) - 1
    ssm = _t(0.5 * rng.standard_normal((S, H, P, N)), torch.float16)
    args = (u, zx, dev["dt_bias"], dev["A_log"], dev["D"], off)
    new, same, from0 = torch.full_like(ssm, 9.0), ssm.clone(), torch.full_like(ssm, 9.0)
    got = [(ops.mixer_scan(*args, ssm, ssm_out=new), new),
           (ops.mixer_scan(*args, same, ssm_out=same), same),
           (ops.mixer_scan(*args, ssm_out=from0), from0)]
    s0 = _np(ssm)
    for (y, st), start in zip(got, (s0, s0, 0.0 * s0)):
        ry, my, rs, ms = np.zeros((T, H, P)), np.zeros((T, H, P)), start.copy(), np.abs(start)
        for i, a, b in _seqs(offs):
            seq = (dt[a:b], prm["dt_bias"], prm["A_log"])
            ry[a:b], rs[i] = O.scan(x[a:b], B[a:b], C[a:b], *seq, prm["D"], start[i])
            my[a:b], ms[i] = O.scan(np.abs(x[a:b]), np.abs(B[a:b]), np.abs(C[a:b]), *seq,
                                    np.abs(prm["D"]), np.abs(start[i]))
        e = offs[-1]
        near("y", y[:e].reshape(-1, H, P), ry[:e], my[:e], 2.0 ** -14)
        near("states", st, rs, ms, 2.0 ** -14)


def _conv_lengths(rng, T):
    """Ragged lengths that add up to T: empty ones, single tokens, less than the
    taps, ends anywhere in a run and on its border."""
    out = []
    while sum(out) < T:
        out.append(int(rng.choice([0, 1, 2, 3, 4, 5, 16, 17, 31, 64, 100, 333])))
    out[-1] -= sum(out) - T
    return out


# one head (320 channels): 11000 tokens are walked in runs of 5, 33000 of 16
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [11000, 33000])
def test_conv_in_runs(T, dtype):
    rng = np.random.default_rng(T)
    offs = _packed(_conv_lengths(rng, T - TAIL))
    prm, dev, zx, d, cd = _layer(rng, T, 1, dtype)
    S, pos = len(offs) - 1, 2
    ring = _t(rng.standard_normal((S, cd, 4)), torch.float16)
    conv_pos = torch.full((1,), pos, dtype=torch.int32, device="cuda")
    off = _off(offs)
    u = torch.full((T, cd), 7.0, dtype=torch.bfloat16, device="cuda")
    new = torch.full_like(ring, 9.0)
    ops.mixer_conv(zx, dev["conv_w"], dev["conv_b"], off, ring, conv_pos, conv_out=new, u=u)
    same = ring.clone()
    ops.mixer_conv(zx, dev["conv_w"], dev["conv_b"], off, same, conv_pos, conv_out=same)
    x = _np(zx[:, d:d + cd])
    w, b = prm["conv_w"].astype(np.float64), prm["conv_b"].astype(np.float64)
    past = np.roll(_np(ring), -pos, axis=2).transpose(0, 2, 1)
    ref, mag, want = np.zeros((T, cd)), np.zeros((T, cd)), past.copy()
    for i, s, e in _seqs(offs):
        ref[s:e] = O.conv(x[s:e], w, b, past[i])
        line = np.abs(np.concatenate([past[i][-3:], x[s:e]]))
        mag[s:e] = np.abs(b) + sum(line[j:j + e - s] * np.abs(w[:, j]) for j in range(4))
        want[i] = np.concatenate([past[i], x[s:e]])[-4:]
    n = offs[-1]
    near("u", u[:n], ref[:n], mag[:n], 2.0 ** -19)
    assert bool((u[n:] == 7.0).all())
    want = np.roll(want.transpose(0, 2, 1), pos, axis=2).astype(np.float16)
    assert np.array_equal(new.cpu().numpy(), want)
    assert np.array_equal(same.cpu().numpy(), want), "the ring in place"


# 48 heads: the parameters' sums take 64 columns a workgroup.  Their longest chain: a
# run's tokens (16), a chain's rows (33 of 2063), the chains (64): 113 x 2^-24 and the
# terms' own 2^-19 are below 2^-16
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(11000, 1), (33000, 1), (700, 48)])
def test_conv_bwd_in_runs(T, H, dtype):
    rng = np.random.default_rng(T + H)
    offs = _packed(_conv_lengths(rng, T - TAIL))
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype)
    du = _t(0.1 * rng.standard_normal((T, cd)), torch.bfloat16)
    dzx = torch.full_like(zx, 3.0)
    dw, db = ops.mixer_conv_bwd(zx, dev["conv_w"], dev["conv_b"], du, dzx, _off(offs))
    x, g = _np(zx[:, d:d + cd]), _np(du)
    ref, mag = np.zeros((T, cd)), np.zeros((T, cd))
    sums = [[np.zeros((cd, 4)), np.zeros(cd)] for _ in range(2)]
    for _, s, e in _seqs(offs):
        for k, absolute in enumerate((False, True)):
            r = O.conv_bwd(x[s:e], prm["conv_w"], prm["conv_b"], g[s:e], absolute=absolute)
            (ref, mag)[k][s:e] = r[0]
            sums[k][0] += r[1]
            sums[k][1] += r[2]
    n = offs[-1]
    # SiLU' loses relative accuracy around its zero: du's own magnitude counts
    mag += np.abs(prm["conv_w"]).sum(1) * np.abs(g).max()
    near("dx", dzx[:n, d:d + cd], ref[:n], mag[:n], 2.0 ** -19)
    scale = np.abs(g[:n]).sum(0)
    near("dconv_w", dw, sums[0][0], sums[1][0] + scale[:, None] * np.abs(x[:n]).max(), 2.0 ** -16)
    near("dconv_b", db, sums[0][1], sums[1][1] + scale, 2.0 ** -16)
    assert bool((dzx[:, :d] == 3.0).all()) and bool((dzx[:, d + cd:] == 3.0).all())
    assert bool((dzx[n:] == 3.0).all())


# the backward's row forms at their borders, with more rows than it has groups of
# them (the sums of dnorm_w go on from row to row)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [8, 9, 16, 17, 33, 64, 65, 97, 128, 129, 193, 256, 257])
def test_norm_bwd_forms(H, dtype):
    T = 1030
    rng = np.random.default_rng(H)
    prm, dev, zx, d, cd = _layer(rng, T, H, dtype)
    y = _t(rng.standard_normal((T, d)), torch.bfloat16)
    dout = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    dzx = torch.full_like(zx, 3.0)
    dy, dw = ops.mixer_norm_bwd(y, zx, dev["norm_w"], dout, dzx, 1e-5)
    a = (_np(y), _np(zx[:, :d]), prm["norm_w"], float(np.float32(1e-5)), _np(dout))
    r, m = O.norm_bwd(*a), O.norm_bwd(*a, absolute=True)
    near("dy", dy, r[0], m[0], 2.0 ** -19)
    sig = 1.0 / (1.0 + np.exp(-a[1]))
    flat = m[1] / np.maximum(np.abs(sig * (1 + a[1] * (1 - sig))), 1e-9)
    near("dz", dzx[:, :d], r[1], flat, 2.0 ** -19)
    # (two rows a group, 16 or 64 chains of up to 64: 2^-24 of 82 links and 2^-19)
    near("dnorm_w", dw, r[2], m[2], 2.0 ** -17)
    assert bool((dzx[:, d:] == 3.0).all())


# rows of more columns than any workgroup takes in one step, and no multiple of 8
@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_embed_wide(w_dtype):
    rng = np.random.default_rng(4)
    T, V, D = 50, 31, 2051
    ids = rng.integers(-1, V + 1, T)
    w = _t(rng.standard_normal((V, D)), w_dtype)
    out = ops.embed(torch.from_numpy(ids).cuda(), w, 1.5)
    ok = (ids >= 0) & (ids < V)
    ref = np.where(ok[:, None], _np(w)[np.clip(ids, 0, V - 1)] * 1.5, 0.0)
    near("rows", out, ref, ref, 0.0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("D", [1025, 2051, 4100])
@pytest.mark.parametrize("kind", ["few", "same", "mixed", "long"])
def test_embed_bwd_wide(kind, D, accumulate):
    rng = np.random.default_rng(D)
    V = 120
    ids = {"few": rng.integers(-1, V + 1, 200), "same": np.full(1000, 17),
           "mixed": np.minimum(rng.geometric(0.05, 2000) - 2, V),
           "long": np.minimum(rng.geometric(0.05, 4500) - 2, V)}[kind]
    de = _t(rng.standard_normal((len(ids), D)))
    t = torch.from_numpy(ids).cuda()
    base = torch.ones((V, D), device="cuda") if accumulate else None
    dW = ops.embed_bwd(t, de, V, 0.5, dW=base, accumulate=accumulate)
    add = 1.0 if accumulate else 0.0
    ref = O.embed_bwd(ids, _np(de), V, 0.5) + add
    near("dW", dW, ref, O.embed_bwd(ids, np.abs(_np(de)), V, 0.5) + add, 2.0 ** -17)


# more tokens than pieces search through: sorted by one, two and three digits of the
# id, at the digits' borders; pieces that are folded.  Equal rows make the roundings
# of a chain of additions add up: the longest one, 64 tokens, with the roundings of
# the sums that are added in float64, the scale and the first value is below 2^-17
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("kind", ["one id", "uniform", "text", "wide", 255, 256, 65535, 65536])
def test_embed_bwd_of_many_tokens(kind, ids_dtype, accumulate):
    rng = np.random.default_rng(6)
    T, V, D = {"one id": ((1 << 20) + 37, 5, 4), "uniform": (200003, 3000, 6),
               "text": (98305, 20000, 33), "wide": (99001, 300000, 1)}.get(kind, (100000, kind, 3))
    if kind == "one id":
        ids, de = np.full(T, 2), torch.full((T, D), 0.1, device="cuda")
    else:
        ids = (rng.integers(-1, V + 1, T) if kind != "text"
               else np.minimum(np.exp(rng.uniform(0, np.log(V), T)).astype(np.int64), V))
        ids[:2] = 0, V - 1
        de = _t(rng.standard_normal((T, D)))
    t = torch.from_numpy(ids).to(ids_dtype).cuda()

    def run():
        base = torch.ones((V, D), device="cuda") if accumulate else None
        return ops.embed_bwd(t, de, V, 0.5, dW=base, accumulate=accumulate)

    dW, add = run(), 1.0 if accumulate else 0.0
    near("dW", dW, O.embed_bwd(ids, _np(de), V, 0.5) + add,
         O.embed_bwd(ids, np.abs(_np(de)), V, 0.5) + add, 2.0 ** -17)
    assert torch.equal(dW, run()), "repeated calls differ"


def test_gradients_of_steps_that_end_every_state():
    """No gradient reaches a step through a state that is over: dt's is that of
    the token's own input, A_log's is zero, whatever the rate."""
    offs, H = [0, 130, 131, 300], 2
    rng, T, prm, dev, zx, u, off, (x, B, C, dt), d, cd = _scan_case(
        offs, H, torch.float32, 78, 0.0)
    prm["A_log"] = np.array([100.0, 20.0], np.float32)
    dev["A_log"] = _t(prm["A_log"])
    dy = _t(0.1 * rng.standard_normal((T, d)), torch.bfloat16)
    dzx = torch.empty_like(zx)
    _, *heads = ops.mixer_scan_bwd(u, zx, dev["dt_bias"], dev["A_log"], dev["D"], dy, dzx, off)
    (_, rdt, rh), (_, mdt, mh) = _scan_bwd_ref(_seqs(offs), T, H, d, cd, x, B, C, dt, prm,
                                               _np(dy).reshape(T, H, P))
    e = offs[-1]
    near("ddt", dzx[:e, -H:], rdt[:e], mdt[:e], 2.0 ** -17)
    for k, name in enumerate(("ddt_bias", "dA_log", "dD")):
        near(name, heads[k], rh[k], mh[k], 2.0 ** -17)
    assert not _np(heads[1]).any()
