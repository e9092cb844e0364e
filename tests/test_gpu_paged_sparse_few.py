"""PagedCache.decode_sparse with few selected pages, and with first and last ones that do not fit."""
import pytest
import torch

import test_gpu_paged_sparse as S
from test_gpu_paged_sparse_run import B, Step, check_row, make  # noqa: F401

pytestmark = pytest.mark.gpu


def filled(B, select, n=100):  # noqa: F811
    cache = make(B, 2, torch.bfloat16, 16, 40, 20, select=select)
    step = Step(cache, n + 40, torch.Generator().manual_seed(3))
    step.put(torch.tensor([n, 40], dtype=torch.int32, device="cuda"))
    return cache, step


@pytest.mark.parametrize("select,first,last", [(1, 0, 1), (2, 0, 2), (3, 1, 2), (4, 1, 2)])
def test_what_is_always_selected(B, select, first, last):  # noqa: F811
    """Unless said otherwise: the last two pages and the first one, as far as they go."""
    cache, step = filled(B, select)
    cache.decode_sparse(0, step.q, step.out, lse=step.lse, by_rows=True)
    assert cache.check_status() == B.SWA_OK
    for s, n, row in ((0, 100, 99), (1, 40, 139)):
        for head in range(2):
            want = S.selection(cache.score[s, head].tolist(), -(-n // 16), select, first, last)
            assert cache.sel[s, head].tolist() == want + [-1] * (select - len(want))
        check_row(B, cache, 0, step, row, s, lambda head: [(s, [t for e in cache.sel[s, head].tolist() if e >= 0 for t in range(e * 16, min(n, e * 16 + 16))])])


@pytest.mark.parametrize("said,first,last", [(dict(first=2), 2, 0), (dict(first=1), 1, 1), (dict(last=0), 1, 0), (dict(last=2), 0, 2), (dict(first=0, last=0), 0, 0)])
def test_one_of_the_two_is_said(B, said, first, last):  # noqa: F811
    cache, step = filled(B, 2)
    cache.decode_sparse(0, step.q, step.out, by_rows=True, **said)
    for s, n in ((0, 100), (1, 40)):
        for head in range(2):
            assert cache.sel[s, head].tolist() == S.selection(cache.score[s, head].tolist(), -(-n // 16), 2, first, last)


@pytest.mark.parametrize("said", [dict(first=1, last=2), dict(first=3), dict(last=3), dict(first=-1), dict(last=-1), dict(first=2, last=1), dict(first=-1, last=3)])
def test_first_and_last_ones_that_do_not_fit(B, said):  # noqa: F811
    """Refused before anything is written."""
    cache, step = filled(B, 2)
    cache.score.fill_(5)
    with pytest.raises(ValueError, match="first and last"):
        cache.decode_sparse(0, step.q, step.out, by_rows=True, **said)
    torch.cuda.synchronize()
    assert (cache.score == 5).all() and (cache.sel == -1).all() and (step.out == 7).all()
