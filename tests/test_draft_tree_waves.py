"""What the compiler reported for the kernels of draft trees, against the waves that their launches count on."""
from test_kernel_resources import _kernels, resources  # noqa: F401  (a fixture)


def test_kernels_of_fp32_results_keep_their_waves(resources):  # noqa: F811
    fine = _kernels(resources, "kda_cache_tree_fine_kernel")
    assert len(fine) == 4                                    # heads of 64 and 128, 64 and 128 rows
    few = _kernels(resources, "kda_cache_few_fine_kernel")
    assert len(few) == 2                                     # heads of 64 with 16 and 32 rows
    for name, r in (fine | few).items():
        assert r["Occupancy [waves/SIMD]"] >= 2 and r["VGPRs Spill"] == 0, (name, r)


def test_workgroups_on_a_compute_unit(resources):  # noqa: F811
    """Three of the tree attention's for heads of 64, as its parts are counted, two for heads of 128; four of KDA's for trees of up to 16 tokens and 128 channels (a
    workgroup is a wave a SIMD; of 64 channels, half of one), two for larger ones, three of the commit's."""
    attend, steps, commit = (_kernels(resources, n) for n in ("kda_cache_tree_kernel", "kda_tree_steps_kernel", "kda_tree_commit_kernel"))
    assert len(attend) == 4 and len(steps) == 12 and len(commit) == 4
    for name, r in attend.items():
        assert r["Occupancy [waves/SIMD]"] >= (3 if "ILi64E" in name else 2), (name, r)
    for name, r in steps.items():
        assert r["Occupancy [waves/SIMD]"] >= (4 if "ELi16EE" in name else 2), (name, r)
    for name, r in commit.items():
        assert r["Occupancy [waves/SIMD]"] >= 3, (name, r)
