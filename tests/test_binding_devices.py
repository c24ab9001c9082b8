"""Where the binding's launches go (CPU): the library launches on the current device, so that a call for tensors of another device makes that
one current for every launch it asks for."""
import contextlib

import pytest
import torch

from paper_2510_26692_amd import kda as binding


class Elsewhere:
    """As much of a tensor on device 1 as marshalling looks at."""
    device, is_cuda = torch.device("cuda", 1), True

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (0,) * len(self.shape)                        # (looked at where a tensor is not contiguous)

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

    monkeypatch.setattr(binding, "_current_device", lambda: at[0])
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


def test_kda_calls_launch_on_the_tensors_device(monkeypatch, current):
    seen = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                seen.append((name, current[0], args[-1].value))
                return 0
            return entry

    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "_native", None)
    x, g, f32 = Elsewhere(1, 70, 2, 64), Elsewhere(1, 70, 2), torch.float32
    state, ws = Elsewhere(1, 2, 64, 64, dtype=f32), Elsewhere(1 << 20, dtype=torch.uint8)
    grads = {n: Elsewhere(1, 70, 2, 64, dtype=f32) for n in ("dq", "dk", "dv", "dlog_alpha")}
    grads.update(dbeta=Elsewhere(1, 70, 2, dtype=f32), dh0=state)
    binding.kda_chunk_fwd(x, x, x, x, g, o=x, hT=state, workspace=ws, check=True)
    binding.kda_chunk_fwd_scalar_gate(x, x, x, g, g, o=x, hT=state, workspace=ws)
    binding.kda_chunk_fwd_fused(x, x, x, x, g, o=x, hT=state, workspace=ws)
    binding.kda_chunk_fwd_static_scratch(x, x, x, x, g, x, hT=state)
    binding.kda_chunk_bwd(x, x, x, x, g, x, workspace=ws, out=grads)
    one, four = Elsewhere(1, 2, 64), Elsewhere(1, 4, 2, 64)
    binding.kda_recurrent_step(one, one, one, one, Elsewhere(1, 2), state, o=one)
    binding.kda_recurrent_steps_pooled(four, four, four, four, Elsewhere(1, 4, 2), state, o=four)
    assert [s[0] for s in seen] == ["kda_chunk_fwd", "kda_chunk_fwd_check", "kda_chunk_fwd_scalar_gate", "kda_chunk_fwd_fused",
                                    "kda_chunk_fwd_static_scratch", "kda_chunk_bwd", "kda_recurrent_step", "kda_recurrent_steps"]
    assert all(s[1:] == (1, 101) for s in seen) and current[0] == 0


def test_packed_attention_calls_launch_everything_on_the_tensors_device(monkeypatch, current):
    """What the calls allocate themselves is cleared behind them: two launches each, on one device and stream."""
    from paper_2510_26692_amd import attn
    seen = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                if name.endswith("_size"):
                    return 1024
                seen.append((name, current[0], args[-1].value))
                return 0
            return entry

    fresh = lambda *shape, dtype, device: Elsewhere(*(shape[0] if isinstance(shape[0], torch.Size) else shape), dtype=dtype)
    for module in (binding, attn):
        monkeypatch.setattr(module, "load_library", Library)
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(torch, "empty", fresh)
    monkeypatch.setattr(torch, "zeros", fresh)
    q, k, cu = Elsewhere(1, 70, 4, 64), Elsewhere(1, 70, 2, 64), Elsewhere(4, dtype=torch.int32)
    o, lse = attn.kda_window_attn_fwd(q, k, k, cu_seqlens=cu, out_dtype=torch.bfloat16)
    attn.kda_window_attn_bwd(q, k, k, o, lse, q, cu_seqlens=cu)
    assert [s[0] for s in seen] == ["kda_window_attn_fwd", "kda_clear_unowned_rows", "kda_window_attn_bwd", "kda_clear_unowned_rows"]
    assert all(s[1:] == (1, 101) for s in seen) and current[0] == 0
