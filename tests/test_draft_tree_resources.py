"""What the compiler reported for the kernels of draft trees and shared pages: the waves that their launches count on, and no spills."""
from test_kernel_resources import _kernels, resources  # noqa: F401  (a fixture)


def test_tree_kernels_keep_their_waves(resources):  # noqa: F811
    # (scratch of the attention kernel: of the call that repeats a walk with care)
    attend, steps, commit = (_kernels(resources, n) for n in ("kda_cache_tree_kernel", "kda_tree_steps_kernel", "kda_tree_commit_kernel"))
    assert len(attend) == 4 and len(steps) == 12 and len(commit) == 4
    for name, r in attend.items():
        assert r["Occupancy [waves/SIMD]"] >= 2 and r["VGPRs Spill"] == 0, (name, r)
    for name, r in (steps | commit).items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)
        assert r["Occupancy [waves/SIMD]"] >= (3 if "Li16E" in name or "commit" in name else 2), (name, r)


def test_kernels_of_few_rows_are_the_cache_attention_s(resources):  # noqa: F811
    few = _kernels(resources, "kda_cache_few_kernel")
    assert len(few) == 3                                     # heads of 64 with 16 and 32 rows, of 128 with 16
    for name, r in few.items():
        assert r["Occupancy [waves/SIMD]"] >= 2 and r["VGPRs Spill"] == 0, (name, r)


def test_moving_and_turning_kernels_use_no_scratch(resources):  # noqa: F811
    some = {}
    for n in ("kda_rotate_kernel", "kda_cache_copy_kernel", "kda_cache_keep_kernel", "kda_pages_"):
        found = _kernels(resources, n)
        assert found, n
        some |= found
    assert len(some) == 8 + 1 + 2 + 4
    for name, r in some.items():
        assert r["ScratchSize [bytes/lane]"] == 0 and r["VGPRs Spill"] == 0, (name, r)
