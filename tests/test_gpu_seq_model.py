"""The sequence operators as a model uses them: the training modules, a whole
block's step, prompts through Mamba2Decoder and the tokens behind them, side
streams and captured graphs."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mamba_seq as O  # noqa: E402
from oracle import ternary as OT  # noqa: E402
from paper_2606_18114_amd import ops, synth  # noqa: E402
from paper_2606_18114_amd.qat import Embedding, Mamba2Mixer, TernaryLinear  # noqa: E402
from paper_2606_18114_amd.stack import Mamba2Decoder  # noqa: E402

pytestmark = pytest.mark.gpu

P, N = 64, 128
BF = torch.bfloat16


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf(a):
    """Rounded to bfloat16, in float64."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32).to(BF).double().numpy()


def _rel(got, ref):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    return np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300)


def _mixer(H, seed):
    torch.manual_seed(seed)
    m = Mamba2Mixer(H, device="cuda")
    rng = np.random.default_rng(seed)
    with torch.no_grad():
        for k, v in synth.mixer_params(rng, H).items():
            getattr(m, k).copy_(torch.from_numpy(v))
    return m, rng


def _mixer_ref(m, zx, seqs, dout):
    """Outputs and gradients in float64 with u, y, and their gradients rounded
    to bfloat16 where the calls store them so."""
    H = m.nheads
    d, cd = H * P, H * P + 2 * N
    p = {k: _np(getattr(m, k)) for k in m.PARAMS}
    out = np.zeros((len(zx), d))
    dzx = np.zeros_like(zx)
    g = {k: np.zeros_like(v) for k, v in p.items()}
    for a, b in seqs:
        z, x, dt = zx[a:b, :d], zx[a:b, d:d + cd], zx[a:b, d + cd:]
        u = _bf(O.conv(x, p["conv_w"], p["conv_b"]))
        parts = (u[:, :d].reshape(-1, H, P), u[:, d:d + N], u[:, d + N:], dt, p["dt_bias"],
                 p["A_log"], p["D"])
        y = _bf(O.scan(*parts)[0].reshape(-1, d))
        out[a:b] = O.norm(y, z, p["norm_w"], m.eps)
        dy, dz, dnw = O.norm_bwd(y, z, p["norm_w"], m.eps, dout[a:b])
        dx, dB, dC, ddt, db, da, dD = O.scan_bwd(*parts, _bf(dy).reshape(-1, H, P))
        du = _bf(np.concatenate([dx.reshape(-1, d), dB, dC], 1))
        dxx, dw, dcb = O.conv_bwd(x, p["conv_w"], p["conv_b"], du)
        dzx[a:b] = np.concatenate([dz, dxx, ddt], 1)
        for k, v in zip(m.PARAMS, (dw, dcb, db, da, dD, dnw)):
            g[k] += v
    return out, dzx, g


# relative 2-norms: a bfloat16 rounding is 2^-9 in the mean square at most (half
# a step of 2^-8 at worst), and values next to a rounding border of u, y, dy or du
# that fall the other way move single elements by a step, which a float32
# gradient then shows; 2^-7 and 2^-8 bound both with room for neither
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("shape", ["rows", "packed", "single"])
def test_mixer_module(shape, dtype):
    m, rng = _mixer(3, 5)
    H = 3
    Z = 2 * H * P + 2 * N + H
    T = 2 * 150
    zx = torch.from_numpy(rng.standard_normal((T, Z))).to(dtype).cuda()
    offsets, seqs = None, [(0, 150), (150, 300)]
    inp = zx.view(2, 150, Z)
    if shape == "packed":
        offs = [0, 1, 1, 200, 280]
        offsets = torch.tensor(offs, dtype=torch.int32, device="cuda")
        seqs, inp = [(a, b) for a, b in zip(offs, offs[1:]) if b > a], zx
    elif shape == "single":
        seqs, inp = [(0, T)], zx
    inp = inp.clone().requires_grad_(True)
    out = m(inp, offsets)
    dout = torch.from_numpy(0.1 * rng.standard_normal((T, H * P))).to(BF).cuda()
    out.backward(dout.view(out.shape))
    ref, dzx, g = _mixer_ref(m, _np(zx), seqs, _np(dout))
    assert _rel(out.reshape(T, -1), ref) < 2.0 ** -8
    end = seqs[-1][1]
    got = _np(inp.grad.reshape(T, Z))
    d = H * P
    for name, sl in (("z", slice(0, d)), ("xBC", slice(d, Z - H)), ("dt", slice(Z - H, Z))):
        assert _rel(got[:end, sl], dzx[:end, sl]) < 2.0 ** -7, name
    assert not got[end:].any() and not _np(out.reshape(T, -1))[end:].any()
    for k in m.PARAMS:
        assert _rel(getattr(m, k).grad, g[k]) < 2.0 ** -8, k


def test_mixer_module_repeats_its_bits_and_skips_unneeded_gradients():
    m, rng = _mixer(2, 6)
    zx = torch.from_numpy(rng.standard_normal((140, 2 * 128 + 256 + 2))).to(BF).cuda()
    m.D.requires_grad_(False)

    def step():
        m.zero_grad()
        m(zx).float().square().sum().backward()
        return {k: getattr(m, k).grad for k in m.PARAMS}

    a, b = step(), step()
    assert a["D"] is None
    for k in m.PARAMS:
        if k != "D":
            assert torch.equal(a[k], b[k]), k


def test_a_second_derivative_is_refused():
    m, e = Mamba2Mixer(1, device="cuda"), Embedding(5, 8, device="cuda")
    zx = torch.randn((3, 385), device="cuda", requires_grad=True)
    ids = torch.tensor([1, 7, 1], device="cuda")
    for f, leaf in ((lambda: m(zx).float(), zx), (lambda: e(ids), e.weight)):
        out = f()
        w = torch.ones_like(out, requires_grad=True)
        (g,) = torch.autograd.grad((out * w).sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()


@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_embedding_module(dtype):
    torch.manual_seed(1)
    e = Embedding(40, 24, scale=2.0, device="cuda", dtype=dtype)
    ids = torch.tensor([[3, 39, 3], [-1, 0, 40]], device="cuda")
    out = e(ids)
    assert out.shape == (2, 3, 24) and out.dtype == torch.float32
    w = _np(e.weight)
    ref = np.where(((_np(ids) >= 0) & (_np(ids) < 40))[..., None],
                   2.0 * w[np.clip(ids.cpu().numpy(), 0, 39)], 0.0)
    assert np.array_equal(_np(out), ref)
    g = torch.randn(out.shape, device="cuda")
    out.backward(g)
    dw = O.embed_bwd(ids.cpu().numpy().reshape(-1), _np(g).reshape(-1, 24), 40, 2.0)
    assert e.weight.grad.dtype == dtype
    assert _rel(e.weight.grad, dw) < (2.0 ** -23 if dtype == torch.float32 else 2.0 ** -8)


def test_block_step():
    """Embedding, in_proj, mixer, out_proj and back: every gradient against the
    float64 chain with the layers' own codes and scales."""
    rng = np.random.default_rng(8)
    H, dm, g, T = 8, 128, 64, 130  # (in_proj has 1288 outputs: its backward takes multiples of 8)
    d, Z = H * P, 2 * H * P + 2 * N + H
    m, _ = _mixer(H, 9)
    emb = Embedding(30, dm, scale=4.0, device="cuda")
    lin = TernaryLinear.from_weight(torch.from_numpy(synth.weights(rng, Z, dm)).cuda() * 20, g=g,
                                    out_dtype=BF)
    lout = TernaryLinear.from_weight(torch.from_numpy(synth.weights(rng, dm, d)).cuda(), g=g)
    with torch.no_grad():
        emb.weight.mul_(30.0)
    ids = torch.from_numpy(rng.integers(0, 30, T)).cuda()
    x = emb(ids).to(BF)
    zx = lin(x)
    y = lout(m(zx))
    go = torch.from_numpy(0.01 * rng.standard_normal((T, dm))).to(BF).cuda().float()
    y.backward(go)

    def what(l):
        codes, s, _, _ = ops.ternarize_pack(l.weight.detach(), g, l.eps)
        q = OT.unpack(codes.cpu().numpy(), l.in_features).astype(np.float64)
        return q * np.repeat(_np(s), g, axis=1)

    wi, wo = what(lin), what(lout)
    xr = _bf(4.0 * _np(emb.weight)[ids.cpu().numpy()])
    zr = _bf(xr @ wi.T)
    dm_ = _bf(_np(go) @ wo)             # the gradient of the mixer's output
    out, dzx, grads = _mixer_ref(m, zr, [(0, T)], dm_)
    assert _rel(y, _bf(out) @ wo.T) < 2.0 ** -6
    # (two products, whose operands are rounded to bfloat16, around the mixer's own)
    for k in m.PARAMS:
        assert _rel(getattr(m, k).grad, grads[k]) < 2.0 ** -6, k
    dzx = _bf(dzx)
    assert _rel(lin.weight.grad, dzx.T @ xr) < 2.0 ** -6
    assert _rel(lout.weight.grad, _bf(_np(go)).T @ _bf(out)) < 2.0 ** -6
    dx = _bf(dzx @ wi)
    assert _rel(emb.weight.grad, O.embed_bwd(ids.cpu().numpy(), dx, 30, 4.0)) < 2.0 ** -6


# ---------------------------------------------------------------- prompts

def _decoder(L=2, dm=128, H=2, g=64, B=1, keep=(), seed=3, embedding=None):
    rng = np.random.default_rng(seed)
    d, Z = H * P, 2 * H * P + 2 * N + H
    w = {("in", l): torch.from_numpy(synth.weights(rng, Z, dm) * 4).cuda() for l in range(L)}
    w |= {("out", l): torch.from_numpy(synth.weights(rng, dm, d) * 4).cuda() for l in range(L)}
    mix = [synth.mixer_params(rng, H) for _ in range(L)]
    pre = [torch.from_numpy((1 + 0.1 * rng.standard_normal(dm)).astype(np.float32))
           for _ in range(L)]
    return Mamba2Decoder(lambda k, l: w[(k, l)], lambda l: mix[l], lambda l: pre[l], L, dm, H,
                         keep=keep, g=g, batch=B, embedding=embedding), mix, pre, w


def _prefill_ref(dec, mix, pre, w, emb, states):
    """One row's prompt in float64, rounded to bfloat16 where the calls store
    so; states: per layer (inputs before, state before); returns the final
    norm behind the last token and the states after."""
    H, d = dec.nheads, dec.d_inner
    res, after = emb.astype(np.float64), []

    def mat(kind, l, p):
        if p[0] == "dense":
            return _np(p[1][0])
        q = OT.unpack(p[1][0].cpu().numpy(), w[(kind, l)].shape[1]).astype(np.float64)
        return q * np.repeat(_np(p[2][0]), dec.g, axis=1)

    def rms(v, wt):
        return v / np.sqrt((v * v).mean(-1, keepdims=True) + dec.eps) * wt

    for l, lay in enumerate(dec.layers):
        p = {k: v.astype(np.float64) for k, v in mix[l].items()}
        x = _bf(rms(res, _np(pre[l])))
        zx = _bf(x @ mat("in", l, lay["in"]).T)
        z, xbc, dt = zx[:, :d], zx[:, d:-H], zx[:, -H:]
        past, state = states[l]
        u = _bf(O.conv(xbc, p["conv_w"], p["conv_b"], past))
        y, state = O.scan(u[:, :d].reshape(-1, H, P), u[:, d:d + N], u[:, d + N:], dt, p["dt_bias"],
                          p["A_log"], p["D"], state)
        m = _bf(O.norm(_bf(y.reshape(-1, d)), z, p["norm_w"], dec.eps))
        res = res + m @ mat("out", l, lay["out"]).T
        after.append((np.concatenate([past, xbc])[-4:], state))
    return rms(res[-1], 1.0), after


def _states(dec, l, b):
    lay = dec.layers[l]
    pos = int(lay["pos"].item())
    return (np.roll(_np(lay["conv"][b]), -pos, axis=1).T.copy(), _np(lay["ssm"][b]))


@pytest.mark.parametrize("keep", [(), (1,)])
@pytest.mark.parametrize("offs", [[0, 9, 9, 140], [0, 1, 70, 134]])
def test_prefill(offs, keep):
    B = len(offs) - 1
    dec, mix, pre, w = _decoder(B=B, keep=keep)
    rng = np.random.default_rng(11)
    emb = rng.standard_normal((offs[-1] + 2, 128)).astype(np.float32)
    off = torch.tensor(offs, dtype=torch.int32, device="cuda")
    start = []
    for l in range(dec.L):
        conv, ssm = synth.mixer_states(rng, B, dec.nheads)
        dec.set_states(l, torch.from_numpy(conv).cuda(), torch.from_numpy(ssm).cuda(), pos=1 + l)
        start.append([_states(dec, l, b) for b in range(B)])
    out = dec.prefill(torch.from_numpy(emb).cuda(), off)
    for b, (s, e) in enumerate(zip(offs, offs[1:])):
        if e == s:
            for l in range(dec.L):
                conv, ssm = _states(dec, l, b)
                assert np.array_equal(conv, start[l][b][0]) and np.array_equal(ssm, start[l][b][1])
            assert not _np(out[b]).any()
            continue
        ref, after = _prefill_ref(dec, mix, pre, w, emb[s:e], [start[l][b] for l in range(dec.L)])
        # two blocks of some six bfloat16 roundings each: 2^-9 apiece in the mean square
        assert _rel(out[b], ref) < 2.0 ** -6, b
        for l in range(dec.L):
            conv, ssm = _states(dec, l, b)
            assert _rel(conv, after[l][0]) < 2.0 ** -7, (b, l)
            assert _rel(ssm, after[l][1]) < 2.0 ** -7, (b, l)
            assert int(dec.layers[l]["pos"].item()) == 1 + l


def test_prefill_in_pieces_and_the_tokens_behind_it():
    """A prompt at once, in two pieces, and a token at a time agree (the last
    rounds the states at every token and keeps float32 projections), and so do
    the tokens decoded behind it."""
    table = torch.randn((50, 128), generator=torch.Generator().manual_seed(0)).cuda()
    ids = torch.from_numpy(np.random.default_rng(2).integers(0, 50, 90)).cuda()
    whole, _, _, _ = _decoder(embedding=table)
    parts, _, _, _ = _decoder(embedding=table)
    steps, _, _, _ = _decoder(embedding=table)
    a = whole.prefill(ids).clone()
    parts.prefill(ids[:37])
    b = parts.prefill(ids[37:]).clone()
    for t in range(90):
        steps.set_ids(ids[t:t + 1])
        c = steps.token()
    # the state in float16 between the pieces moves them by 2^-11 of a state
    assert _rel(a, _np(b)) < 2.0 ** -7
    assert _rel(a, _np(c)) < 2.0 ** -5  # 90 roundings of the state, bfloat16 projections
    for dec in (whole, parts, steps):
        dec.set_ids(ids[:1])
    outs = [_np(dec.token()) for dec in (whole, parts, steps)]
    assert _rel(outs[0], outs[1]) < 2.0 ** -7 and _rel(outs[0], outs[2]) < 2.0 ** -5


def test_prefill_refusals():
    dec, _, _, _ = _decoder(B=2)
    x = torch.zeros((4, 128), device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        dec.prefill(x)                       # a batch needs offsets
    with pytest.raises(ValueError):
        dec.prefill(x, off[:2])
    with pytest.raises(ValueError):
        dec.prefill(x[:, :64].contiguous(), off)
    with pytest.raises(TypeError):
        dec.prefill(x.to(BF), off)
    with pytest.raises(TypeError):
        dec.prefill(x, off.long())
    with pytest.raises(RuntimeError):
        dec.prefill(torch.zeros(4, dtype=torch.int64, device="cuda"), off)
    with pytest.raises(RuntimeError):
        dec.set_ids(torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        _decoder(embedding=torch.zeros((5, 64), device="cuda"))


# ---------------------------------------------------------------- streams and graphs

class _Chain:
    """All calls of a training step and a prompt on fixed inputs."""

    def __init__(self, seed, T=700, H=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        d, cd = H * P, H * P + 2 * N
        self.zx = r(T, d + cd + H).to(BF)
        self.par = [0.3 * r(cd, 4), 0.3 * r(cd), r(H) - 3.0, r(H).abs(), r(H), 1 + 0.1 * r(d)]
        self.dout = r(T, d).to(BF)
        self.off = torch.tensor([0, 3, 3, 130, T], dtype=torch.int32, device="cuda")
        self.ring = r(4, cd, 4).to(torch.float16)
        self.ssm = r(4, H, P, N).to(torch.float16)
        self.pos = torch.ones(1, dtype=torch.int32, device="cuda")
        self.ids = torch.randint(0, 90, (T,), generator=g, device="cuda")
        self.table, self.de = r(90, 96), r(T, 96)

    def run(self):
        cw, cb, bias, alog, D, nw = self.par
        ring, ssm = torch.empty_like(self.ring), torch.empty_like(self.ssm)
        u = ops.mixer_conv(self.zx, cw, cb, self.off, self.ring, self.pos, conv_out=ring)
        y = ops.mixer_scan(u, self.zx, bias, alog, D, self.off, self.ssm, ssm_out=ssm)
        out = ops.mixer_norm(y, self.zx, nw)
        dzx = torch.empty_like(self.zx)
        dy, dnw = ops.mixer_norm_bwd(y, self.zx, nw, self.dout, dzx)
        du, *dh = ops.mixer_scan_bwd(u, self.zx, bias, alog, D, dy, dzx, self.off)
        dcw, dcb = ops.mixer_conv_bwd(self.zx, cw, cb, du, dzx, self.off)
        e = ops.embed(self.ids, self.table, 2.0)
        dw = ops.embed_bwd(self.ids, self.de, 90, 2.0)
        return [u, y, out, ring, ssm, dzx, dy, dnw, du, *dh, dcw, dcb, e, dw]


def test_side_stream():
    c = _Chain(1)
    ref = [t.clone() for t in c.run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)


def test_captured_and_replayed():
    """Two graphs of the same calls, replayed in turn with new inputs and eager
    work between: every replay equals the eager result bit for bit."""
    chains = [_Chain(1), _Chain(2)]
    graphs = []
    for c in chains:
        c.run()  # sizes are asked, the library is loaded
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = c.run()
        graphs.append((gr, out))
    for step in range(4):
        for c, (gr, out) in zip(chains, graphs):
            new = _Chain(10 * step + 3)
            for name in ("zx", "dout", "ring", "ssm", "ids", "table", "de"):
                getattr(c, name).copy_(getattr(new, name))
            gr.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            for a, b in zip(c.run(), got):
                assert torch.equal(a, b)
