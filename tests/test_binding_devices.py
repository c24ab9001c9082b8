"""Where the binding's launches go (CPU): the library launches on the current device, so that a call for tensors of another device makes that
one current for every launch it asks for."""
import contextlib

import pytest
import torch

from paper_2510_26692_amd import kda as binding


class Elsewhere:
    """As much of a tensor on device 1 as marshalling looks at."""
    device = torch.device("cuda", 1)

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return 2

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def current(monkeypatch):
    """The current device, as a list of one, with torch's switch in front of it; streams are named after their device."""
    at = [0]

    @contextlib.contextmanager
    def device(dev):
        before, at[0] = at[0], torch.device(dev).index
        try:
            yield
        finally:
            at[0] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 100 + index)
    return at


def test_rows_of_nobody_are_cleared_on_the_tensors_device(monkeypatch, current):
    seen = []

    class Library:
        @staticmethod
        def kda_clear_unowned_rows(cu, num_seqs, tokens, n, arrays, rows, stream):
            seen.append((current[0], stream.value, num_seqs, tokens, list(rows)))
            return 0

    monkeypatch.setattr(binding, "load_library", lambda: Library)
    for index in (0, 1):
        current[0] = index
        binding._clear_unowned(Elsewhere(4), [Elsewhere(1, 50, 2, 64), Elsewhere(1, 50, 8)])
        assert current[0] == index
    assert seen == [(1, 101, 3, 50, [256, 16])] * 2
