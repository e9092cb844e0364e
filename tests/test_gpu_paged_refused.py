"""Sequences that a plan refuses take no part in the attention over its rows: nobody has written their queries."""
import math

import pytest
import torch

import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("first,width,scale_up", [(40, 60, 1), (1300, 200, 1), (1300, 200, 20), (3, 8, 40)])
@pytest.mark.parametrize("why", ["pages", "rows", "table", "bad page"])
def test_refused_sequences_are_left_out(B, first, width, scale_up, why):
    """Four kinds of sequence, `scale_up` of each: two that get their tokens, one that is refused, one that brings none.  One workgroup a sequence, chunks
    that are joined, shares, and single waves."""
    h_q, h_kv, d, page, dt = 4, 2, 64, 16, torch.bfloat16
    b = 4 * scale_up
    lens = [first, first + 5, 0, 7] * scale_up
    new = [1, 3, 0, 2] * scale_up
    need = [-(-m // page) for m in lens]
    ask = [-(-(m + c) // page) for m, c in zip(lens, new)]
    rows = sum(new)
    # those that are refused: the last of the four kinds, from some place on
    if why == "pages":
        for i in range(3, b, 4):
            new[i] = 40 if i == b - 1 else new[i]
        ask = [-(-(m + c) // page) for m, c in zip(lens, new)]
        rows, refused = sum(new), {b - 1}
    elif why == "rows":
        rows, refused = rows - 1, {b - 1}
    elif why == "table":
        lens[b - 1], refused = width * page - 1, {b - 1}
        need[b - 1] = ask[b - 1] = width
    else:
        refused = {b - 1}
    spare = sum(a - n for a, n in zip(ask, need)) - (1 if why == "pages" else 0)
    n_pages = sum(need) + spare
    p = B.make_paged_params(b, h_q, h_kv, d, page, n_pages, width, dt)
    cache = B.PagedCache(p)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(b)).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [-1] * (width - n))
        at += n
    if why == "bad page":
        table[b - 1][0] = n_pages + 3                          # 7 tokens, so that the new ones would go there
    cache.block_table.copy_(ints(table))
    cache.cache_len.copy_(ints(lens))
    cache.free_ring.copy_(ints(order[at:] + [-1] * at))
    cache.free_state.copy_(ints([0, n_pages - at]))
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (cache.k_pages[0], cache.v_pages[0]):
        x.normal_(generator=g)
    total = sum(new)
    slot, pos = ints([5] * rows), ints([5] * rows)
    cache.plan(ints(new), slot, pos)
    assert cache.check_status() == (B.SWA_ERR_BAD_REQUEST if why == "bad page" else B.SWA_ERR_CAPACITY)
    start = cache.row_start.tolist()
    assert start[-1] == total
    for s in range(b):
        for r in range(start[s], min(start[s + 1], rows)):
            assert (slot[r].item() < 0) == (s in refused), (s, r)
    # rows that nobody writes are no numbers
    q = torch.randn((total, h_q, d), generator=g, device="cuda").to(dt)
    for s in refused:
        q[start[s]:start[s + 1]] = math.nan
    k = v = torch.zeros((rows, h_kv, d), dtype=dt, device="cuda")
    before = [x.clone() for x in (cache.k_pages[0], cache.v_pages[0])]
    q_out = torch.full((rows, h_q, d), math.nan, dtype=dt, device="cuda")
    cache.append(0, q[:rows], k, v, slot, pos, None, q_out)
    for by_class in (True, False):
        out = torch.full((total, h_q, d), 7.0, dtype=dt, device="cuda")
        lse = torch.full((total, h_q), 7.0, device="cuda")
        if by_class:
            cache.decode(0, q, out, lse, by_rows=True)          # (more rows than the plan had room for)
        else:
            B.swa_paged_decode_planned(p, q_out, rows, cache.row_start, slot, cache.k_pages[0], cache.v_pages[0], None, None, cache.block_table,
                                       cache.cache_len, out, lse, cache.workspace)
        assert cache.check_status() == B.SWA_OK
        said = set()
        table_now, len_now = cache.block_table.tolist(), cache.cache_len.tolist()
        for s in range(b):
            if s in refused or start[s] == start[s + 1]:
                continue
            r = start[s + 1] - 1
            said.add(r)
            kk, vv = (R.gather(x.cpu(), None, torch.tensor(table_now[s]), page, 0, len_now[s]) for x in (cache.k_pages[0], cache.v_pages[0]))
            want, want_lse, tol, lse_tol = R.attention(q[r].cpu().double(), kk, vv, d ** -0.5, dt, R.half_step(dt))
            assert ((out[r].cpu().double() - want).abs() <= tol).all() and ((lse[r].cpu().double() - want_lse).abs() <= lse_tol).all(), s
        rest = [r for r in range(total) if r not in said]
        assert (out[rest] == 7).all() and (lse[rest] == 7).all()
    del before


def test_a_plan_that_refuses_inside_a_graph(B):
    """A captured step of the class, replayed with counts that change: what is refused in one replay is left as it was, and served in another."""
    b, h, d, page, dt, rows = 3, 2, 64, 4, torch.float16, 12
    p = B.make_paged_params(b, h, h, d, page, 6, 6, dt)
    cache = B.PagedCache(p)
    new, slot, pos = ints([1] * b), ints([0] * rows), ints([0] * rows)
    x = torch.randn((rows, h, d), device="cuda").to(dt)
    out = torch.zeros_like(x)
    lengths, state = cache.cache_len, cache.free_state
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            cache.plan(new, slot, pos)
            cache.append(0, x, x, x, slot, pos, None, x)
            cache.decode(0, x, out, by_rows=True)
    torch.cuda.current_stream().wait_stream(side)
    for counts, free, served in (([4, 4, 4], 6, {0, 1, 2}), ([4, 9, 5], 6, {0}), ([4, 4, 4], 2, {0, 1}), ([1, 5, 1], 2, {0}), ([1, 1, 1], 6, {0, 1, 2}),
                                 ([13, 1, 1], 6, set())):
        new.copy_(ints(counts))
        lengths.zero_()                                         # (every replay plans from an empty cache)
        state.copy_(ints([0, free]))
        out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").sum()
        ends = [sum(counts[:i + 1]) for i in range(b)]
        *_, want_slot, _, _ = R.plan(counts, [0] * b, [[-1] * 6] * b, list(range(6)), state.tolist(), page, rows)
        assert slot.tolist() == want_slot
        assert {r for r in range(rows) if (out[r] != 7).any()} == {ends[i] - 1 for i in served}, counts
