"""The head's loss where numbers come near the ends of their types, and in forms beside those of
test_gpu_head_forms.py, whose inputs, float64 reference and tolerances are used here."""

import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_head_forms import IGNORE, _check, _inputs, _run  # noqa: E402

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- teachers

@pytest.mark.parametrize("T,K", [(1, 1), (40, 5), (40, 20), (600, 20)])  # both launch shapes
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
