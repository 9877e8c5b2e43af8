"""Calls of ``Mamba2Decoder.prefill`` and ``set_ids`` that a program makes beside
those of ``test_gpu_seq_model.py``: strided prompts and ids, a decoder on another
device than the current one, projections kept in float32."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mamba_seq as O  # noqa: E402
from oracle import ternary as OT  # noqa: E402
from test_gpu_seq_model import BF, N, P, _bf, _decoder, _np, _rel, _states  # noqa: E402

pytestmark = pytest.mark.gpu


def _table():
    return torch.randn((50, 128), generator=torch.Generator().manual_seed(0)).cuda()


def test_strided_prompts_and_ids():
    """A transposed prompt, every second id, a column of a batch's ids."""
    table = _table()
    ids = torch.from_numpy(np.random.default_rng(2).integers(0, 50, (40, 2))).cuda()
    emb = table[ids[:, 1]]
    outs = []
    for prompt in (emb, emb.t().contiguous().t(), torch.stack([emb, emb], 1)[:, 0], ids[:, 1],
                   ids[:, 1].contiguous()):
        dec, _, _, _ = _decoder(embedding=table)
        outs.append(dec.prefill(prompt).clone())
        assert torch.equal(outs[0], outs[-1])
    assert torch.equal(emb, table[ids[:, 1]]), "the prompt was written"
    dec, _, _, _ = _decoder(B=2, embedding=table)
    turned = ids[:2].t().contiguous()  # [sequence, token]
    assert torch.equal(dec.set_ids(turned[:, 1]), table[ids[1]])


def test_prefill_runs_on_the_decoders_device(monkeypatch):
    """Its calls take the current device's stream, so that device is made current."""
    dec, _, _, _ = _decoder()
    seen = []

    class Device(torch.cuda.device):
        def __init__(self, device):
            seen.append(torch.device(device))
            super().__init__(device)

    monkeypatch.setattr(torch.cuda, "device", Device)
    dec.prefill(torch.zeros((3, 128), device="cuda"))
    assert dec.emb.device in seen


# the inputs of layer 0's states, rounded only where the calls do: x to bfloat16, u to
# bfloat16 (2^-9 in the mean square, averaged over tokens in the state; the oracle's
# alike but for values next to a border), the state to float16: 2^-12 in the mean
# square at most; 2^-10 with bfloat16's rounding of B or x falling the other way for
# one value in a hundred
def test_float32_projections():
    """zx_dtype float32: the states are those of unrounded projections."""
    rng = np.random.default_rng(5)
    emb = rng.standard_normal((140, 128)).astype(np.float32)
    dec, mix, pre, w = _decoder()
    dec.prefill(torch.from_numpy(emb).cuda(), zx_dtype=torch.float32)
    H, d = dec.nheads, dec.d_inner
    lay, p = dec.layers[0], {k: v.astype(np.float64) for k, v in mix[0].items()}
    q = OT.unpack(lay["in"][1][0].cpu().numpy(), 128).astype(np.float64)
    wi = q * np.repeat(_np(lay["in"][2][0]), dec.g, axis=1)
    res = emb.astype(np.float64)
    x = _bf(res / np.sqrt((res * res).mean(-1, keepdims=True) + dec.eps) * _np(pre[0]))
    zx = x @ wi.T
    xbc = zx[:, d:-H]
    u = _bf(O.conv(xbc, p["conv_w"], p["conv_b"]))
    _, state = O.scan(u[:, :d].reshape(-1, H, P), u[:, d:d + N], u[:, d + N:], zx[:, -H:],
                      p["dt_bias"], p["A_log"], p["D"])
    conv, ssm = _states(dec, 0, 0)
    assert _rel(conv, xbc[-4:]) < 2.0 ** -11  # float16 alone
    assert _rel(ssm, state) < 2.0 ** -10
    with pytest.raises(TypeError, match="zx_dtype"):
        dec.prefill(torch.from_numpy(emb).cuda(), zx_dtype=torch.float16)
    dec, _, _, _ = _decoder()
    a = dec.prefill(torch.from_numpy(emb).cuda()).clone()
    dec, _, _, _ = _decoder()
    assert torch.equal(a, dec.prefill(torch.from_numpy(emb).cuda(), zx_dtype=BF))
