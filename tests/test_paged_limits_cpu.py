"""Calls that no launch holds are refused as such, before the device is touched."""
import pytest

from test_paged_cpu import B, decode, params  # noqa: F401


@pytest.mark.parametrize("h_q,h_kv,span", [
    (4096, 4096, dict(max_pages=20)),                        # 2^24 workgroups of 256 threads, 320 tokens
    (65535, 21845, dict(max_pages=60, window=900)),          # three query heads on each key head
    (65535, 65535, dict(max_pages=60)),
    (16384, 16384, dict(max_pages=1)),                       # 2^26 workgroups of one wave, 16 tokens
    (32768, 32768, dict(max_pages=64, len_bound=200)),
    (4096, 4096, dict(max_pages=1 << 26)),                   # 2^24 pairs of 2^30 tokens
])
def test_more_than_a_launch_holds(B, h_q, h_kv, span):  # noqa: F811
    p = params(B, b=4096, h_q=h_q, h_kv=h_kv, n_pages=1, **span)
    assert decode(B, p, n=4096, q=B.SwaRows(0x1000, h_q * p.d)) == B.SWA_ERR_CAPACITY
