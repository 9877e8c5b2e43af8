"""Arrays of more than 2^31 elements, and the embedding gradient's long form in
captured graphs and on two streams."""

import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

P, N = 64, 128
BF = torch.bfloat16


def _near(a, b, step):
    """Both round once (half a step of the type each); before that they differ by
    float32 sums in another order (2^-14 of the largest at most)."""
    a, b = a.double(), b.double()
    return bool(((a - b).abs() <= step * b.abs() + 2.0 ** -14 * b.abs().max()).all())


def test_rows_beyond_32_bits():
    """The last sequence of a long batch is what it is by itself, forward and
    backward: in_proj's output has 2.3e9 elements."""
    H, L = 64, 700
    d, cd = H * P, H * P + 2 * N
    Z = d + cd + H
    T = 270000
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731

    def rows(width, scale=1.0):  # blocks of 4500 rows again and again, the last L their own
        t = (scale * r(4500, width)).to(BF).repeat(T // 4500, 1)
        t[-L:] = (scale * r(L, width)).to(BF)
        return t

    zx, dout = rows(Z), rows(d, 0.1)
    assert zx.numel() > 2 ** 31
    par = [0.3 * r(cd, 4), 0.3 * r(cd), r(H) - 4.0, r(H).abs(), r(H), 1 + 0.1 * r(d)]
    cw, cb, bias, alog, D, nw = par

    def run(zx, dout, off):
        u = ops.mixer_conv(zx, cw, cb, off)
        y = ops.mixer_scan(u, zx, bias, alog, D, off)
        out = ops.mixer_norm(y, zx, nw)
        dzx = torch.empty_like(zx)
        dy, _ = ops.mixer_norm_bwd(y, zx, nw, dout, dzx)
        du, *_ = ops.mixer_scan_bwd(u, zx, bias, alog, D, dy, dzx, off)
        ops.mixer_conv_bwd(zx, cw, cb, du, dzx, off)
        return [t[-L:].clone() for t in (u, y, out, dy, du, dzx)]

    off = torch.tensor([0, 1000, T - L, T], dtype=torch.int32, device="cuda")
    long = run(zx, dout, off)
    short = run(zx[-L:].clone(), dout[-L:].clone(), None)
    assert torch.equal(long[0], short[0])
    for name, a, b in zip(("y", "out", "dy", "du"), long[1:], short[1:]):
        # a value that falls to the other side of a border in y or dy shows in what follows
        assert _near(a, b, 2.0 ** -6), name
    assert _near(long[5], short[5], 2.0 ** -5), "dzxbcdt"


@pytest.mark.parametrize("T", [3, 300, 5000, 100000])
def test_embedding_rows_beyond_32_bits(T):
    V, D = 1060000, 2048
    w = torch.zeros((V, D), dtype=BF, device="cuda")
    w[-3:] = torch.arange(1, 4, device="cuda")[:, None]
    ids = torch.arange(T, device="cuda") % 3 + V - 3
    out = ops.embed(ids[:300], w, 2.0)
    assert torch.equal(out, (2.0 * (ids[:300] - (V - 4))).float()[:, None].expand(-1, D))
    del w
    dW = ops.embed_bwd(ids, torch.ones((T, D), device="cuda"), V)
    n = torch.bincount(ids - (V - 3), minlength=3).float()
    assert torch.equal(dW[-3:], n[:, None].expand(3, D))
    assert not dW[:-3].any()


def test_long_embedding_gradient_captured_and_on_two_streams():
    T, V, D = 110000, 3000, 8
    g = torch.Generator(device="cuda").manual_seed(3)

    def fresh():
        return (torch.randint(-1, V, (T,), generator=g, device="cuda"),
                torch.randn((T, D), generator=g, device="cuda"))

    calls = [fresh(), fresh()]
    graphs = []
    for ids, de in calls:
        ops.embed_bwd(ids, de, V, 0.5)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = ops.embed_bwd(ids, de, V, 0.5)
        graphs.append((gr, out))
    for _ in range(4):
        for (ids, de), (gr, out) in zip(calls, graphs):
            a, b = fresh()
            ids.copy_(a)
            de.copy_(b)
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ops.embed_bwd(ids, de, V, 0.5))
    want = [ops.embed_bwd(ids, de, V, 0.5) for ids, de in calls]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s, (ids, de) in zip(streams, calls):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(ops.embed_bwd(ids, de, V, 0.5))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
