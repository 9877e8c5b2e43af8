"""A workspace's size may depend on the device (the head's products are cut for its number of
compute units): the binding asks with the tensors' device current, and once for each."""

import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402


def test_sizes_are_asked_for_on_the_calls_device(monkeypatch):
    units, current, asked = {0: 256, 1: 32}, [0], []

    class Lib:
        @staticmethod
        def tm_some_workspace(T, V):
            asked.append((current[-1], T, V))
            return 1000 * T + V + units[current[-1]] if T < 100 else -1

    @contextlib.contextmanager
    def device(d):
        current.append(d if isinstance(d, int) else d.index)
        yield
        current.pop()

    monkeypatch.setattr(ops, "lib", lambda: Lib)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(ops.torch, "empty", lambda shape, dtype, device:
                        torch.zeros(shape, dtype=dtype))
    a, b = torch.device("cuda", 0), torch.device("cuda", 1)
    for _ in range(2):
        for dev in (a, b, a):
            ws, ptr, n = ops._seq_ws("tm_some_workspace", dev, 3, 5)
            assert n == 3005 + units[dev.index] == ws.numel() and ptr == ws.data_ptr()
    assert sorted(asked) == [(0, 3, 5), (1, 3, 5)] and current == [0]
    with pytest.raises(ValueError, match="out of range"):
        ops._seq_ws("tm_some_workspace", a, 100, 5)
