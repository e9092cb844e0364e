"""swa_paged_decode_planned refuses what swa_paged_decode refuses, and a call without a plan's lists; no GPU is needed."""
import ctypes

import pytest
import torch

from test_paged_cpu import B, ok, params  # noqa: F401


def planned(B, p, n=4, q=None, **bad):  # noqa: F811
    names = ["row_start", "slot", "k_pages", "v_pages", "k_scale", "v_scale", "block_table", "cache_len", "out", "lse", "workspace"]
    a = {m: ok for m in names}
    a.update(bad)
    return B.lib().swa_paged_decode_planned(ctypes.byref(p) if p is not None else None, q or B.SwaRows(ok, 256), n, *[a[m] for m in names], None)


def test_what_it_refuses(B):  # noqa: F811
    p, q8 = params(B), params(B, flags=B.SWA_KV_INT8)
    assert planned(B, None) == B.SWA_ERR_NULL
    for n in ("row_start", "slot", "k_pages", "v_pages", "block_table", "cache_len", "out", "workspace"):
        assert planned(B, p, **{n: None}) == B.SWA_ERR_NULL, n
    for n in ("k_scale", "v_scale"):
        assert planned(B, q8, **{n: None}) == B.SWA_ERR_NULL, n
    for n in ("k_pages", "v_pages", "out", "workspace"):
        assert planned(B, p, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT, n
    for n in (0, -1, (1 << 24) + 1):
        assert planned(B, p, n=n) == B.SWA_ERR_BAD_SHAPE
    assert planned(B, p, q=B.SwaRows(ok, 248)) == B.SWA_ERR_BAD_SHAPE
    assert planned(B, params(B, d=96)) == B.SWA_ERR_UNSUPPORTED_D


@pytest.mark.parametrize("general", [False, True])
def test_tensors_elsewhere(B, monkeypatch, general):  # noqa: F811
    if general:
        monkeypatch.setattr(B, "_native", B._General())
    p, t, rows = params(B), torch.zeros(64, dtype=torch.int32), torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current GPU"):
        B.swa_paged_decode_planned(p, rows, 4, t, t, t, t, None, None, t, t, t, None, t, 0)
    with pytest.raises(ValueError, match="dense"):
        B.swa_paged_decode_planned(p, rows[..., ::2], 4, t, t, t, t, None, None, t, t, t, None, t, 0)
