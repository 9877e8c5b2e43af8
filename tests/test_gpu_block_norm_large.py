"""The block norm at its largest sizes."""

import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


def _room(gib):
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    if free < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of GPU memory are needed")


def _rows(t, rows):
    return (t if rows is None else torch.stack([t[i] for i in rows])).double()


def _check_rows(rows, r, w, x, eps=1e-5):
    """x of some rows: float32 sums of D terms of one sign, then a rounding to bfloat16."""
    s = _rows(r, rows)
    want = s / torch.sqrt(s.pow(2).mean(-1, keepdim=True) + eps) * w.double()
    rel = (s.shape[1] + 16) * F
    off = (_rows(x, rows) - want).abs()
    assert bool((off <= want.abs() * (2.0 ** -8 * (1 + rel) + rel)).all())


def test_the_most_rows_of_wide_workgroups():
    """2^23 rows of 4097 columns, for which a row has 512 threads: 128 GiB and 64 GiB."""
    T, D = 2 ** 23, 4097
    _room(210)
    block = torch.randn(4096, D, device="cuda")
    r = torch.empty((T, D), device="cuda")
    r.view(-1, 4096, D).copy_(block.expand(T // 4096, 4096, D))
    w = 1 + 0.1 * torch.randn(D, device="cuda")
    some = [0, 1, 4095, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, T - 2, T - 1]
    for i in some:
        r[i].normal_()
    x, s = ops.block_norm(r, None, w)
    assert s is r
    _check_rows(some, r, w, x)
    part = x.view(-1, 4096, D)  # the other rows: the same in every block
    first = torch.ones(4096, dtype=torch.bool, device="cuda")
    first[[i % 4096 for i in some]] = False
    for i in range(0, T // 4096, 97):
        assert torch.equal(part[i][first], part[1024][first])
    del x, s, r, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,D", [(2 ** 22, 3), (2 ** 22 + 1, 3), (2 ** 22 + 4097, 2), (2 ** 23, 1)])
def test_many_short_rows(T, D):
    """Rows of the launch's second dimension; what lies behind the last one stays."""
    r, y = torch.randn(T, D, device="cuda"), torch.randn(T, D, device="cuda")
    w = 1 + 0.1 * torch.randn(D, device="cuda")
    keep = torch.full(((T + 8) * D,), 7.0, device="cuda").bfloat16()
    x, s = ops.block_norm(r, y, w, x=keep[:T * D].view(T, D))
    assert torch.equal(s, r + y) and bool((keep[T * D:] == 7.0).all())
    _check_rows(None, s, w, x)


def test_past_2_31_elements_with_gradients():
    T, D = 2 ** 20 + 500, 2048
    _room(60)
    g = torch.Generator(device="cuda").manual_seed(1)
    r, y = (torch.randn(T, D, generator=g, device="cuda") for _ in range(2))
    w = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    some = [0, 1, 1023, 1024, 2 ** 20 - 1, 2 ** 20, T - 1]
    x, s = ops.block_norm(r, y, w, residual_out=r)
    assert s is r
    _check_rows(some, s, w, x)
    del y, x
    dx = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    dx[T - 300:] *= 100.0
    dres = torch.randn(T, D, generator=g, device="cuda")
    keep = _rows(dres, some)
    dr, dw = ops.block_norm_bwd(s, w, dx, dres, dr=dres)
    assert dr is dres
    s64, a = _rows(s, some), _rows(dx, some) * w.double()
    rho = 1 / torch.sqrt(s64.pow(2).mean(-1, keepdim=True) + 1e-5)
    mean = (a * s64).mean(-1, keepdim=True)
    want = keep + rho * a - s64 * rho ** 3 * mean
    mag = keep.abs() + rho * a.abs() + s64.abs() * rho ** 3 * (a * s64).abs().mean(-1, keepdim=True)
    assert bool(((_rows(dr, some) - want).abs() <= 2 * (D + 16) * F * mag).all())
    want, mag = (torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(2))
    for lo in range(0, T, 2 ** 16):
        s64, d64 = s[lo:lo + 2 ** 16].double(), dx[lo:lo + 2 ** 16].double()
        t = d64 * s64 / torch.sqrt(s64.pow(2).mean(-1, keepdim=True) + 1e-5)
        want += t.sum(0)
        mag += t.abs().sum(0)
    # 1024 groups of 1025 rows, added up one by one, then the groups
    assert bool(((dw.double() - want).abs() <= (1025 + 1024 + D + 16) * F * mag).all())


@pytest.mark.parametrize("T,D,y,dres", [(3, 2 ** 20, True, True), (1100, 20001, False, True),
                                        (1030, 16384, True, False), (2, 65537, False, False)])
def test_wide_rows(T, D, y, dres):
    """Rows that are read twice, their weight's gradient added up in memory over two rows a group."""
    g = torch.Generator(device="cuda").manual_seed(D)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    r0, y0, w = 2 * rnd(T, D), rnd(T, D) if y else None, 1 + 0.2 * rnd(D)
    dx, dr0 = rnd(T, D).bfloat16(), rnd(T, D) if dres else None
    x, r = ops.block_norm(r0, y0, w)
    assert torch.equal(r, r0 + y0 if y else r0)
    _check_rows(None, r, w, x)
    dr, dw = ops.block_norm_bwd(r, w, dx, dr0)
    s, a = r.double(), dx.double() * w.double()
    rho = 1 / torch.sqrt(s.pow(2).mean(-1, keepdim=True) + 1e-5)
    want = rho * a - s * rho ** 3 * (a * s).mean(-1, keepdim=True)
    mag = rho * a.abs() + s.abs() * rho ** 3 * (a * s).abs().mean(-1, keepdim=True)
    if dres:
        want, mag = want + dr0.double(), mag + dr0.double().abs()
    assert bool(((dr.double() - want).abs() <= 2 * (D + 16) * F * mag).all())
    t = dx.double() * s * rho
    assert bool(((dw.double() - t.sum(0)).abs() <= (T + D + 16) * F * t.abs().sum(0)).all())
