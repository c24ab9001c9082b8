"""What the compiler reported for the kernels of draft trees, against the waves that their launches count on."""
from test_kernel_resources import _kernels, resources  # noqa: F401  (a fixture)


def test_kernels_of_fp32_results_keep_their_waves(resources):  # noqa: F811
    fine = _kernels(resources, "kda_cache_tree_fine_kernel")
    assert len(fine) == 4                                    # heads of 64 and 128, 64 and 128 rows
    few = _kernels(resources, "kda_cache_few_fine_kernel")
    assert len(few) == 2                                     # heads of 64 with 16 and 32 rows
    for name, r in (fine | few).items():
        assert r["Occupancy [waves/SIMD]"] >= 2 and r["VGPRs Spill"] == 0, (name, r)
