"""Where the paged cache's kernels put things in LDS: by the library's own rules."""
import ctypes

from test_paged_cpu import B  # noqa: F401


def test_the_plans_lists_are_aligned(B):  # noqa: F811
    """Four lists of int32; the sums of up to sixteen waves, pairs of them, lie where the fourth begins."""
    rule = getattr(ctypes.CDLL(B.LIB_PATH), "_ZN3swa14paged_plan_ldsEi")
    rule.restype = ctypes.c_size_t
    for b in range(1, B.SWA_MAX_PAGED_SEQS + 1):
        room, rest = divmod(rule(b), 4 * 4)
        assert rest == 0 and room >= max(b, 2 * 16) and 3 * room * 4 % 8 == 0, b
    assert rule(B.SWA_MAX_PAGED_SEQS) <= 64 * 1024
