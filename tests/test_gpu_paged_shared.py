"""Attention behind shared prefixes on the GPU, against float64."""
import math
import random

import pytest
import torch

import paged_reference as R
import test_gpu_paged as T

pytestmark = pytest.mark.gpu
TYPES = T.TYPES


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def check_shared(B, lens, prefix_of, h_q, h_kv, d, dtype, page, int8=False, scale=0.0, row_start=None, slot=None, n_rows=None, strided=False, bad=(), lse=True, loud=1.3,
                 skipped=(), refused=(), len_bound=0, wider=0, edit=None):
    """skipped: sequences that are too long, or whose prefix is; refused: those whose prefix is none."""
    b = len(lens)
    held = [-(-max(m, 0) // page) for m in lens]
    n_pages, width = sum(held) + 2, max(max(held), 1) + wider
    table, _ = T.make_tables(lens, page, width, n_pages, 11)
    k, v, ks, vs = T.make_pool(n_pages, h_kv, page, d, dtype, int8, 7)
    live = torch.zeros(n_pages, page, dtype=torch.bool)
    for s, m in enumerate(lens):
        t = torch.arange(max(m, 0))
        live[table[s].long()[t // page], t % page] = True
    for x in (ks, vs) if int8 else (k, v):
        x[(~live)[:, None, :].expand(-1, h_kv, -1).cuda()] = math.nan
    n_rows = n_rows or b
    q = (loud * torch.randn((n_rows, h_q, d), generator=torch.Generator().manual_seed(13))).to(dtype)
    if edit:
        edit(k, v, q, table)
    for s, j, x in bad:
        table[s, j] = x
    p = B.make_paged_params(b, h_q, h_kv, d, page, n_pages, width, dtype, scale=scale, len_bound=len_bound, flags=8 if int8 else 0)
    nbytes = B.swa_paged_workspace_bytes(p)
    ws = torch.full((nbytes + (1 << 16),), 0xFF, dtype=torch.uint8, device="cuda")    # of NaN, with a guard behind it
    B.swa_paged_workspace_init(p, ws)
    qd = q.cuda()
    if strided:
        wide = torch.full((n_rows, h_q + 3, d), math.nan, dtype=dtype, device="cuda")
        wide[:, :h_q] = qd
        qd = wide[:, :h_q]
    out = torch.full((n_rows, h_q, d), 7.0, dtype=dtype, device="cuda")
    sums = torch.full((n_rows, h_q), 7.0, device="cuda") if lse else None
    args = (p, qd, n_rows, T.ints(row_start) if row_start else None, T.ints(slot) if slot else None, k, v, ks, vs, table.cuda(), T.ints(lens), T.ints(prefix_of), out,
            sums, ws)
    B.swa_paged_decode_shared(*args)
    first = out.clone()
    assert B.swa_paged_check_status(p, ws) == (B.SWA_ERR_CAPACITY if skipped else B.SWA_ERR_BAD_REQUEST if bad or refused else B.SWA_OK)
    B.swa_paged_decode_shared(*args)
    assert torch.equal(first.view(torch.uint8), out.view(torch.uint8)) and (ws[nbytes:] == 0xFF).all()
    kc, vc, ksc, vsc = (t.cpu() if t is not None else None for t in (k, v, ks, vs))
    got, got_lse = out.cpu().double(), sums.cpu().double() if lse else None
    seen, gathered = set(), {}

    def tokens(s):
        if s not in gathered:
            gathered[s] = [R.gather(x, y, table[s], page, 0, lens[s]) for x, y in ((kc, ksc), (vc, vsc))]
        return gathered[s]
    for s, m in enumerate(lens):
        row = row_start[s + 1] - 1 if row_start else s
        if m < 0 or s in skipped or s in refused or (row_start and row < row_start[s]) or not 0 <= row < n_rows or (slot and slot[row] < 0):
            continue
        seen.add(row)
        kr, vr = tokens(s)
        if prefix_of[s] >= 0:
            kr, vr = (torch.cat([a, z]) for a, z in zip(tokens(prefix_of[s]), (kr, vr)))
        steps = (R.half_step(dtype) if dtype != torch.float32 else 0.0, 0.0)
        if int8:
            steps = (2.0 ** -16, 0.0)                        # (codes are exact in either type, and queries are multiplied as they are)
        want, want_lse, tol, lse_tol = R.attention(q[row].double(), kr, vr, scale or d ** -0.5, dtype, *steps)
        nothing = want_lse == -math.inf                      # every logit is -inf: out = 0
        want[nothing], tol[nothing], lse_tol[nothing] = 0, 0, 0
        for name, x, y, z in (("out", got[row], want, tol),) + ((("lse", got_lse[row], want_lse, lse_tol),) if lse else ()):
            fine = torch.isfinite(y)
            assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x[~fine & ~torch.isnan(y)], y[~fine & ~torch.isnan(y)]), (name, s)
            over = ((x - y).abs() - z)[fine]
            assert not over.numel() or over.max() <= 0, (name, s, m, float(over.max()))
    for row in set(range(n_rows)) - seen:
        assert (got[row] == 7).all() and (not lse or (got_lse[row] == 7).all()), row


def behind(m, own):
    """prefix_of for sequences with these prefixes behind m sequences that have none."""
    return [-1] * m + own


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 16, 20, 64])
def test_prefixes_of_every_type(B, dtype, int8, d, page):
    t = TYPES[dtype]
    check_shared(B, [300, 1, 0, 16, 33, 200, 128], behind(1, [0] * 6), 8, 2, d, t, page, int8=int8)
    check_shared(B, [129, 40, 64, 5, 17, 0, 90, 31], behind(2, [0, 1, 1, -1, 0, 1]), 4, 4, d, t, page, int8=int8)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (12, 12), (5, 1), (14, 2), (17, 1), (32, 1), (40, 1), (66, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_heads_that_share_keys(B, h_q, h_kv, dtype):
    for d in (64, 128):
        check_shared(B, [400, 7, 200, 1, 77], behind(1, [0, 0, 0, 0]), h_q, h_kv, d, TYPES[dtype], 16)
        check_shared(B, [130, 33], behind(1, [0]), h_q, h_kv, d, TYPES[dtype], 16, scale=0.4, lse=False)


@pytest.mark.parametrize("members", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 33, 70])
def test_numbers_of_sequences_behind_a_prefix(B, members):
    check_shared(B, [700] + [(i * 19) % 50 for i in range(members)], behind(1, [0] * members), 8, 2, 64, torch.bfloat16, 16)
    check_shared(B, [260] + [3] * members, behind(1, [0] * members), 6, 2, 128, torch.float16, 16)


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True)])
def test_long_prefixes_are_split_and_joined(B, dtype, int8):
    t = TYPES[dtype]
    check_shared(B, [20011, 5, 300, 2000], behind(1, [0, 0, 0]), 4, 1, 128, t, 16, int8=int8)
    check_shared(B, [9000, 3001, 5, 0, 300, 2000], behind(2, [0, 1, 0, 1]), 8, 2, 64, t, 64, int8=int8, len_bound=9000)
    check_shared(B, [5000] + [20] * 40, behind(1, [0] * 40), 16, 2, 64, t, 16, int8=int8)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 24, 256])
def test_many_columns(B, dtype, d, page):
    """More than 32 query heads behind a prefix: whole and part tiles of columns, of tokens and of rounds."""
    t = TYPES[dtype]
    for n in (1, 31, 32, 33, 64, 65, 100, 127, 128, 129, 192, 193, 255, 257, 320, 450, 1000):
        check_shared(B, [n] + [5, 0, 40, 17, 1] * 2, behind(1, [0] * 10), 8, 2, d, t, page)
    for members, h_q, h_kv in ((33, 1, 1), (11, 12, 4), (9, 16, 1), (8, 20, 1), (33, 8, 2), (3, 40, 1), (2, 33, 1), (3, 66, 2)):
        check_shared(B, [500, 129] + [i % 19 for i in range(2 * members)], behind(2, [0, 1] * members), h_q, h_kv, d, t, page)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_columns_over_long_prefixes(B, dtype):
    t = TYPES[dtype]
    check_shared(B, [30011] + [30] * 20, behind(1, [0] * 20), 8, 1, 128, t, 16, len_bound=30011)
    check_shared(B, [9001, 2500] + [30] * 40, behind(2, [0, 1] * 20), 8, 2, 64, t, 64)
    for loud in (0.1, 5.0, 20.0):
        check_shared(B, [3000] + [30] * 20, behind(1, [0] * 20), 8, 1, 128, t, 16, loud=loud)


def test_many_columns_and_what_is_reported_or_not_finite(B):
    lens, own = [300] + [i * 7 % 40 for i in range(24)], behind(1, [0] * 24)
    for t in (torch.float16, torch.bfloat16):
        for d in (64, 128):
            check_shared(B, lens, own, 4, 2, d, t, 16, bad=[(0, 3, -1), (0, 9, 10 ** 6), (3, 0, 2 ** 31 - 1)])

        def edit(k, v, q, table):
            v[table[0, 2], 0, 3, 5], v[table[0, 18], 1, 11, 7] = math.inf, -math.inf
            q[7, 3, 1], k[table[5, 0], 0, 0, 2] = math.nan, math.nan
        check_shared(B, lens, own, 4, 2, 64, t, 16, edit=edit)

        def cold(k, v, q, table):
            q[:] = 0
            k[:, :, :, 0] = -math.inf                        # every logit is -inf
            q[:, :, 0] = 1
        check_shared(B, [300] + [0] * 24, own, 4, 2, 64, t, 16, edit=cold)
        starts = [0, 0] + list(range(1, 25))
        check_shared(B, lens, own, 4, 2, 128, t, 16, row_start=starts, n_rows=24, slot=[i % 5 - 1 for i in range(24)], strided=True)


def test_many_prefixes_and_many_sequences(B):
    rng = random.Random(5)
    lens = [rng.randrange(0, 300) for _ in range(300)]
    check_shared(B, lens, [rng.choice((-1, rng.randrange(20), rng.randrange(20))) if i >= 20 else -1 for i in range(300)], 4, 2, 64, torch.bfloat16, 16)
    check_shared(B, lens[:200], [-1 if i < 100 else 199 - i for i in range(200)], 2, 1, 64, torch.float32, 16)     # a prefix for each
    check_shared(B, [40] * 100 + [900], [100] * 100 + [-1], 4, 1, 128, torch.float16, 16)                             # the last one is the prefix


@pytest.mark.parametrize("b", [1024, 4096])
def test_as_many_sequences_as_there_may_be(B, b):
    lens = [500] + [i % 23 for i in range(b - 1)]
    check_shared(B, lens, behind(1, [0 if i % 3 else -1 for i in range(b - 1)]), 2, 1, 64, torch.bfloat16, 16)


def test_without_prefixes(B):
    check_shared(B, [0], [-1], 8, 2, 64, torch.float16, 16)
    check_shared(B, [5000], [-1], 8, 2, 64, torch.float16, 16)
    check_shared(B, [0, 0, 0], [-1, 0, 0], 8, 2, 64, torch.float32, 16)
    check_shared(B, [1, 1000, 0, 20], [-1] * 4, 8, 2, 128, torch.bfloat16, 16)
    check_shared(B, [0, 40, 0, 20], behind(1, [0] * 3), 8, 2, 128, torch.bfloat16, 16)        # an empty one


def test_prefixes_that_have_prefixes(B):
    """One counts: a prefix's own is not looked at."""
    check_shared(B, [100, 50, 30, 20], [-1, 0, 1, 2], 4, 2, 64, torch.float32, 16)
    check_shared(B, [100, 50], [1, 0], 4, 2, 64, torch.float32, 16)


def test_whose_rows(B):
    """Prefixes that are kept have no rows."""
    starts, lens = [0, 0, 0, 1, 4, 4, 6], [300, 129, 40, 260, 33, 90]
    own = behind(2, [0, 1, 1, 0])
    for t in (torch.bfloat16, torch.float32):
        check_shared(B, lens, own, 4, 2, 64, t, 16, row_start=starts, n_rows=6, strided=True)
        check_shared(B, lens, own, 4, 2, 64, t, 16, row_start=starts, n_rows=5)
        check_shared(B, lens, own, 4, 2, 64, t, 16, row_start=starts, n_rows=6, slot=[5, 1, 2, -1, 3, 9])
        check_shared(B, lens[:5] + [-1], own, 4, 2, 64, t, 16, row_start=starts, n_rows=6)


def test_what_is_reported(B):
    lens = [300, 100, 40, 90, 10, -1, 20]
    check_shared(B, lens, [-1, 0, 7, -2, 4, 0, 5], 4, 2, 64, torch.bfloat16, 16, refused=(2, 3, 4, 6))
    check_shared(B, lens, [-1, 0, 2 ** 31 - 1, 0, -2 ** 31, 0, 0], 4, 2, 64, torch.bfloat16, 16, refused=(2, 4))
    check_shared(B, lens, [-1, 0, 1, -1, 3, 0, 1], 4, 2, 64, torch.bfloat16, 16, len_bound=100, skipped=(0, 1))
    check_shared(B, lens, [-1, 0, 1, -1, 0, 0, 1], 4, 2, 64, torch.float32, 16, bad=[(0, 3, -1), (0, 9, 10 ** 6), (3, 5, 2 ** 31 - 1)])


def test_what_is_not_finite(B):
    """An infinite value behind a prefix stays in the sequences that see it; logits of -inf weigh nothing."""
    def edit(k, v, q, table):
        v[table[0, 2], 0, 3, 5] = math.inf
        k[table[3, 0], 1, 0, 0] = math.nan
    for t in TYPES.values():
        check_shared(B, [90, 70, 5, 20, 30, 8], behind(2, [0, 1, 1, 0]), 4, 2, 64, t, 16, edit=edit)


def test_loud_tokens_on_either_side(B):
    for loud in (0.1, 5.0, 20.0):
        check_shared(B, [700, 130, 3, 500], behind(1, [0, 0, 0]), 4, 2, 128, torch.float16, 16, loud=loud)
        check_shared(B, [700, 130, 3, 500], behind(1, [0, 0, 0]), 4, 2, 64, torch.bfloat16, 16, int8=True, loud=loud)


def test_the_same_as_a_table_that_names_the_prefixs_pages(B):
    """Whole pages in front of a sequence's own are the same tokens: within what the order of sums changes."""
    page, h_q, h_kv, d = 16, 8, 2, 128
    lens, full = [640, 100, 17, 300], [640, 740, 657, 940]
    held = [-(-m // page) for m in lens]
    table, _ = T.make_tables(lens, page, 60, sum(held), 4)
    k, v, _, _ = T.make_pool(sum(held), h_kv, page, d, torch.float32, False, 3)
    q = torch.randn((4, h_q, d), generator=torch.Generator().manual_seed(1)).cuda()
    p = B.make_paged_params(4, h_q, h_kv, d, page, sum(held), 60, torch.float32)
    ws = T.workspace(B, p)
    a, b, x, y = (torch.zeros(shape, device="cuda") for shape in (q.shape, q.shape, (4, h_q), (4, h_q)))
    B.swa_paged_decode_shared(p, q, 4, None, None, k, v, None, None, table.cuda(), T.ints(lens), T.ints([-1, 0, 0, 0]), a, x, ws)
    for s in (1, 2, 3):
        table[s, 40:60] = table[s, :20].clone()
        table[s, :40] = table[0, :40]
    B.swa_paged_decode(p, q, 4, None, k, v, None, None, table.cuda(), T.ints(full), b, y, ws)
    assert (a - b).abs().max() <= 1e-5 and (x - y).abs().max() <= 1e-5
