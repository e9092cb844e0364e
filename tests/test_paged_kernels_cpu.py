"""What the compiler made of the paged cache's kernels: their launches count on registers and LDS that a change elsewhere can tip over."""
from test_kernels_cpu import kernels  # noqa: F401  (mangled name -> bytes of code, of scratch per lane, of LDS)


def test_no_paged_kernel_spills(kernels):  # noqa: F811
    """Three (two) workgroups of the attention on a CU leave a lane 168 (256) registers; what does not fit would go to memory in the inner loop."""
    seen = {k: v for k, v in kernels.items() if "swa_paged" in k}
    assert sum("swa_paged_decode_kernel" in k for k in seen) == 60 and sum("swa_paged_append_kernel" in k for k in seen) == 40
    for k, (_, scratch, _) in seen.items():
        assert scratch == 0, k


def test_the_sums_of_all_sequences_fit_beside_the_joins_lds(kernels):  # noqa: F811
    from paper_2403_17312_amd import binding as B
    for k, (_, _, lds) in kernels.items():
        if "swa_paged_decode_kernel" in k:
            assert lds + 4 * (B.SWA_MAX_PAGED_SEQS + 1) <= 64 * 1024, k
        if "swa_paged_plan_kernel" in k:
            assert lds + 16 * B.SWA_MAX_PAGED_SEQS <= 64 * 1024, k
