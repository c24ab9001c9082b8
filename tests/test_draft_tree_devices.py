"""Where the launches of the calls for draft trees and shared pages go (CPU): to the tensors' device and its stream, whichever is current."""
import torch

from test_binding_devices import Elsewhere, binding, current  # noqa: F401  (a fixture)


def test_calls_launch_on_the_tensors_device(monkeypatch, current):  # noqa: F811
    from paper_2510_26692_amd import tree
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
    for module in (binding, tree):
        monkeypatch.setattr(module, "load_library", Library)
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(torch, "empty", fresh)
    i32, f32 = torch.int32, torch.float32
    ints = lambda *shape: Elsewhere(*shape, dtype=i32)
    q, k = Elsewhere(3, 5, 4, 64), Elsewhere(3, 5, 2, 64)
    codes, scale = Elsewhere(9, 2, 16, 64, dtype=torch.float8_e4m3fn), Elsewhere(9, 2, dtype=f32)
    beta, states = Elsewhere(3, 5, 2), Elsewhere(3, 2, 64, 64, dtype=f32)
    tree.kda_rotate(q, k, ints(3, 5), Elsewhere(32, dtype=f32), axes=[0] * 32)
    tree.kda_cache_tree_attn(q, codes, codes, scale, scale, ints(3, 4), ints(3), ints(3, 5))
    tree.kda_cache_keep(codes, codes, scale, scale, ints(3, 4), ints(3), ints(3, 5))
    tree.kda_cache_copy_pages(codes, codes, scale, scale, ints(7, 2))
    tree.kda_pages_fork(ints(3, 4), ints(9), ints(3))
    tree.kda_pages_reserve(ints(3, 4), ints(3), ints(3), ints(9), 16)
    tree.kda_pages_compact(ints(3, 4), ints(9))
    tree.kda_tree_steps(k, k, k, k, beta, states, ints(3, 5))
    tree.kda_tree_commit(k, k, k, beta, states, ints(3, 5))
    assert [s[0] for s in seen] == ["kda_rotate", "kda_cache_tree_attn", "kda_cache_keep", "kda_cache_copy_pages", "kda_pages_fork", "kda_pages_reserve",
                                    "kda_pages_compact", "kda_tree_steps", "kda_tree_commit"]
    assert all(s[1:] == (1, 101) for s in seen) and current[0] == 0
