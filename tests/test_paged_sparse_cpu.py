"""What the paged cache's sparse attention and its attention behind shared prefixes refuse, and rules of theirs that no result shows; no GPU is needed."""
import ctypes

import pytest
import torch

from test_kernels_cpu import kernels  # noqa: F401
from test_paged_cpu import B, ok, params  # noqa: F401


def call(B, name, p, names, ints=(), q=None, n=4, **bad):  # noqa: F811
    """names: the pointers, in order; an integer in its place is passed as it is."""
    a = {m: ok for m in names if isinstance(m, str)}
    a.update(bad)
    lead = () if q is None else (q, n)
    args = [a[m] if isinstance(m, str) else m for m in names]
    return getattr(B.lib(), name)(ctypes.byref(p) if p is not None else None, *lead, *ints, *args, None)


def bounds(B, p, n=4, **bad):  # noqa: F811
    return call(B, "swa_paged_bounds", p, ["slot", "k_pages", "k_scale", "bounds", "workspace"], (n,), **bad)


def score(B, p, n=4, q=None, **bad):  # noqa: F811
    return call(B, "swa_paged_score", p, ["row_start", "slot", "bounds", "block_table", "cache_len", "score", "workspace"], q=q or B.SwaRows(ok, 256), n=n, **bad)


def select(B, p, n_sel=3, first=1, last=1, **bad):  # noqa: F811
    return call(B, "swa_paged_select", p, ["score", "cache_len", n_sel, first, last, "sel", "sel_cnt", "workspace"], **bad)


CACHE = ["row_start", "slot", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "cache_len"]


def selected(B, p, n=4, q=None, n_sel=3, **bad):  # noqa: F811
    return call(B, "swa_paged_decode_selected", p, CACHE + ["sel", "sel_cnt", n_sel, "out", "lse", "workspace"], q=q or B.SwaRows(ok, 256), n=n, **bad)


def shared(B, p, n=4, q=None, **bad):  # noqa: F811
    return call(B, "swa_paged_decode_shared", p, CACHE + ["prefix_of", "out", "lse", "workspace"], q=q or B.SwaRows(ok, 256), n=n, **bad)


NEEDED = {bounds: ("slot", "k_pages", "bounds", "workspace"), score: ("bounds", "block_table", "cache_len", "score", "workspace"),
          select: ("score", "cache_len", "sel", "sel_cnt", "workspace"),
          selected: ("k_pages", "v_pages", "block_table", "cache_len", "sel", "sel_cnt", "out", "workspace"),
          shared: ("k_pages", "v_pages", "block_table", "cache_len", "prefix_of", "out", "workspace")}
SCALES = {bounds: ("k_scale",), selected: ("k_scale", "v_scale"), shared: ("k_scale", "v_scale")}
ALIGNED = {bounds: ("k_pages", "bounds", "workspace"), score: ("bounds", "workspace"), select: ("workspace",),
           selected: ("k_pages", "v_pages", "out", "workspace"), shared: ("k_pages", "v_pages", "out", "workspace")}


@pytest.mark.parametrize("fn", list(NEEDED), ids=lambda f: f.__name__)
def test_missing_and_misplaced_tensors(B, fn):  # noqa: F811
    p, q8 = params(B), params(B, flags=B.SWA_KV_INT8)
    assert fn(B, None) == B.SWA_ERR_NULL
    for n in NEEDED[fn]:
        assert fn(B, p, **{n: None}) == B.SWA_ERR_NULL, n
    for n in SCALES.get(fn, ()):
        assert fn(B, q8, **{n: None}) == B.SWA_ERR_NULL, n
        assert fn(B, q8, **{n: ok + 4}) == B.SWA_ERR_ALIGNMENT, n
    for n in ALIGNED[fn]:
        assert fn(B, p, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT, n
    assert fn(B, params(B, d=96)) == B.SWA_ERR_UNSUPPORTED_D
    assert fn(B, params(B, dtype=3)) == B.SWA_ERR_UNSUPPORTED_DTYPE
    assert fn(B, params(B, h_q=3)) == B.SWA_ERR_BAD_SHAPE


@pytest.mark.parametrize("fn", [bounds, score, selected, shared], ids=lambda f: f.__name__)
def test_numbers_of_rows(B, fn):  # noqa: F811
    for n in (0, -1, (1 << 24) + 1):
        assert fn(B, params(B), n=n) == B.SWA_ERR_BAD_SHAPE


@pytest.mark.parametrize("fn", [score, selected, shared], ids=lambda f: f.__name__)
def test_rows_of_queries(B, fn):  # noqa: F811
    p = params(B)
    assert fn(B, p, row_start=None) == B.SWA_ERR_NULL                        # slots without the rows they are of
    assert fn(B, p, n=1, row_start=None, slot=None) == B.SWA_ERR_BAD_SHAPE   # fewer rows than sequences
    assert fn(B, p, q=B.SwaRows(ok, 248)) == B.SWA_ERR_BAD_SHAPE
    assert fn(B, p, q=B.SwaRows(None, 256)) == B.SWA_ERR_NULL
    assert fn(B, p, q=B.SwaRows(ok + 8, 256)) == B.SWA_ERR_ALIGNMENT
    assert fn(B, p, q=B.SwaRows(ok, 260)) == B.SWA_ERR_ALIGNMENT


@pytest.mark.parametrize("fn", [score, select, selected, shared], ids=lambda f: f.__name__)
def test_windows_are_refused(B, fn):  # noqa: F811
    assert fn(B, params(B, window=5)) == B.SWA_ERR_BAD_SHAPE


def test_selections_that_do_not_fit(B):  # noqa: F811
    p = params(B)                                            # four pages to a sequence
    for n_sel, first, last in ((0, 0, 0), (-1, 0, 0), (5, 0, 0), (3, -1, 0), (3, 0, -1), (3, 2, 2), (3, 4, 0), (3, 2 ** 31 - 1, 1), (3, 1, 2 ** 31 - 1)):
        assert select(B, p, n_sel, first, last) == B.SWA_ERR_BAD_SHAPE, (n_sel, first, last)
    for n_sel in (0, -1, 5):
        assert selected(B, p, n_sel=n_sel) == B.SWA_ERR_BAD_SHAPE


def test_more_than_a_launch_holds(B):  # noqa: F811
    p = params(B, b=4096, h_q=16384, h_kv=16384, n_pages=1, max_pages=1)
    q = B.SwaRows(ok, 16384 * p.d)
    assert selected(B, p, n=4096, q=q, n_sel=1) == B.SWA_ERR_CAPACITY
    assert shared(B, p, n=4096, q=q) == B.SWA_ERR_CAPACITY
    assert select(B, p, 1, 0, 0) == B.SWA_ERR_CAPACITY
    p = params(B, b=64, h_q=8, h_kv=8, n_pages=1, max_pages=1 << 26)         # 2^30 tokens a sequence
    assert shared(B, p, n=64, q=B.SwaRows(ok, 512)) == B.SWA_ERR_CAPACITY
    assert score(B, p, n=64, q=B.SwaRows(ok, 512)) == B.SWA_ERR_CAPACITY


@pytest.mark.parametrize("general", [False, True])
def test_tensors_elsewhere(B, monkeypatch, general):  # noqa: F811
    if general:
        monkeypatch.setattr(B, "_native", B._General())
    p, t, rows = params(B), torch.zeros(64, dtype=torch.int32), torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    calls = [lambda q: B.swa_paged_bounds(p, 4, t, t, None, t, t, 0), lambda q: B.swa_paged_score(p, q, 4, t, t, t, t, t, t, t, 0),
             lambda q: B.swa_paged_select(p, t, t, 3, 1, 1, t, t, t, 0),
             lambda q: B.swa_paged_decode_selected(p, q, 4, t, t, t, t, None, None, t, t, t, t, 3, t, None, t, 0),
             lambda q: B.swa_paged_decode_shared(p, q, 4, t, t, t, t, None, None, t, t, t, t, None, t, 0)]
    for i, c in enumerate(calls):
        with pytest.raises(ValueError, match="current GPU"):
            c(rows)
        if i in (1, 3, 4):
            with pytest.raises(ValueError, match="dense"):
                c(rows[..., ::2])


def test_the_lists_of_all_sequences_fit_in_lds(B, kernels):  # noqa: F811
    """Beside the kernel's own, of which the launch takes 36 KiB for the most."""
    seen = 0
    for k, (_, _, lds) in kernels.items():
        if "swa_paged_shared_kernel" in k:
            seen += 1
            assert lds <= 36 * 1024 and lds + 4 * (2 * B.SWA_MAX_PAGED_SEQS + 1) + 2 * (2 * B.SWA_MAX_PAGED_SEQS + 2) <= 160 * 1024, k
    assert seen


# (a call that is not refused goes to the device: only where there is none)
@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors are none")
@pytest.mark.parametrize("b,h_q,h_kv,tokens,more", [
    (2048, 128, 8, 1 << 22, {}), (256, 136, 8, 1 << 24, {}), (64, 1024, 8, 1 << 26, {}), (1, 4096, 32, 1 << 30, {}),
    (2, 40, 5, 1 << 30, {}), (4, 5, 1, 1 << 30, {}), (16, 64, 4, 1 << 29, dict(dtype=0)), (4096, 4095, 1, 1 << 18, {}), (17, 8, 8, 1 << 30, dict(len_bound=1 << 29)),
])
def test_sizes_that_a_launch_holds(B, b, h_q, h_kv, tokens, more):  # noqa: F811
    """Just below the limit that the header states, which a call twice as long (or wide) passes."""
    p = params(B, b=b, h_q=h_q, h_kv=h_kv, page_size=4096, n_pages=1, max_pages=tokens // 4096, **more)
    assert shared(B, p, n=b, q=B.SwaRows(ok, h_q * p.d)) not in (B.SWA_ERR_CAPACITY, B.SWA_OK)


@pytest.mark.parametrize("b,h_q,h_kv,page,tokens,more", [
    (2048, 128, 8, 4096, 1 << 24, {}), (256, 136, 8, 4096, 1 << 27, {}), (256, 136, 8, 4092, 1023 * 4092 * 60, {}), (64, 1024, 8, 4096, 1 << 29, {}), (256, 8, 8, 4096, 1 << 30, {}),
    (2, 1 << 15, 128, 4096, 1 << 30, dict(dtype=0)), (4096, 4096, 1, 4096, 4096, {}), (1, 65535, 65535, 4096, 1 << 30, {}),
])
def test_sizes_that_no_launch_holds(B, b, h_q, h_kv, page, tokens, more):  # noqa: F811
    """Just beyond it."""
    p = params(B, b=b, h_q=h_q, h_kv=h_kv, page_size=page, n_pages=1, max_pages=tokens // page, **more)
    assert shared(B, p, n=b, q=B.SwaRows(ok, h_q * p.d)) == B.SWA_ERR_CAPACITY


def test_a_single_sequence_needs_no_room_for_prefixes(B):  # noqa: F811
    """It has the decode's workspace: at most two pieces for each of 1024 shares, of 16 heads' sums and outputs."""
    for h_q, h_kv, d, dtype in ((1, 1, 64, 1), (32, 8, 128, 2), (16, 16, 128, 0), (64, 8, 64, 1)):
        n = B.swa_paged_workspace_bytes(params(B, b=1, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype))
        assert 256 < n <= 2 * 1024 * 16 * (d + 2) * 4 + 512
        assert B.swa_paged_workspace_bytes(params(B, b=2, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype)) > n


@pytest.mark.parametrize("t", ["3F16", "4BF16"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_lists_fit_beside_the_tiles_of_many_columns(B, kernels, t, d):  # noqa: F811
    """Of which the launch takes 1 KiB for the kernel's own LDS, and twelve tiles of 32 rows or the results of 128 columns; and its loop spills nothing."""
    seen = [k for k in kernels if "swa_paged_shared_wide_kernel" in k and f"INS_{t}ELi{d}EE" in k]
    assert len(seen) == 1
    tiles = max(12 * 32 * d * 2, 128 * (d + 6) * 4)
    _, scratch, lds = kernels[seen[0]]
    assert scratch == 0 and lds <= 1024 and lds + tiles + 4 * (2 * B.SWA_MAX_PAGED_SEQS + 2) + 2 * (2 * B.SWA_MAX_PAGED_SEQS + 1) + 15 <= 160 * 1024
