"""Calls of ``Mamba2Decoder.prefill`` and ``set_ids`` that a program makes beside
those of ``test_gpu_seq_model.py``: strided prompts and ids, a decoder on another
device than the current one."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_seq_model import _decoder  # noqa: E402

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
