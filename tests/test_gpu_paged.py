"""The paged cache on the GPU: its plan against lists, rows and attention against float64."""
import math
import random

import pytest
import torch

import paged_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def workspace(B, p):
    ws = torch.full((B.swa_paged_workspace_bytes(p),), 0xA5, dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    return ws


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- plan --------------------------------------------------------------------------------------------------------------------------

def run_plan(B, p, new_cnt, lens, table, ring, state, max_rows, ws):
    out = dict(new_len=ints([-7] * p.b), table=ints(table), ring=ints(ring), state=ints([-7, -7]), row_start=ints([-7] * (p.b + 1)),
               slot=ints([-7] * max_rows), pos=ints([-7] * max_rows))
    args = (ints(new_cnt), ints(lens), out["new_len"], out["table"], out["ring"], ints(state), out["state"], max_rows, out["row_start"],
            out["slot"], out["pos"], ws)
    first = None
    for _ in range(2):                                   # the same call again gives the same lists
        B.swa_paged_plan(p, *args)
        got = [out[n].tolist() for n in ("new_len", "table", "ring", "state", "row_start", "slot", "pos")]
        assert first is None or got == first
        first = got
    return got


def check_plan(B, p, new_cnt, lens, table, ring, state, max_rows, ws):
    got = run_plan(B, p, new_cnt, lens, table, ring, state, max_rows, ws)
    *want, bits = R.plan(new_cnt, lens, table, ring, state, p.page_size, max_rows)
    for name, g, w in zip(("new_len", "table", "ring", "state", "row_start", "slot", "pos"), got, want):
        assert g == w, name
    code = B.SWA_ERR_CAPACITY if "capacity" in bits else B.SWA_ERR_BAD_REQUEST if "request" in bits else B.SWA_OK
    assert B.swa_paged_check_status(p, ws) == code
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK
    return got, bits


@pytest.mark.parametrize("b,page,width,spare,max_rows", [(1, 16, 4, 8, 20), (3, 1, 40, 30, 64), (64, 16, 8, 20, 300), (65, 24, 5, 400, 4000),
                                                         (257, 7, 12, 90, 700), (1000, 16, 9, 3000, 30000), (4096, 16, 3, 500, 5000),
                                                         (4096, 128, 2, 10000, 70000)])
def test_plan_follows_the_lists(B, b, page, width, spare, max_rows):
    rng = random.Random(b * 1000 + page)
    lens = [rng.choice((0, rng.randrange(width * page + 1), -1)) for _ in range(b)]
    new_cnt = [rng.choice((0, 1, 1, -1, rng.randrange(1, 2 * page + 2))) for _ in range(b)]
    pages = list(range(sum(-(-max(m, 0) // page) for m in lens) + spare))
    rng.shuffle(pages)
    n = len(pages)
    table = [[pages.pop() for _ in range(-(-max(m, 0) // page))] for m in lens]
    table = [r + [-1] * (width - len(r)) for r in table]
    head = rng.randrange(n)
    ring = [-1] * n
    for i, x in enumerate(pages):
        ring[(head + i) % n] = x
    p = B.make_paged_params(b, 1, 1, 64, page, n, width, torch.float16)
    check_plan(B, p, new_cnt, lens, table, ring, [head, len(pages)], max_rows, workspace(B, p))


@pytest.mark.parametrize("case", ["none", "no pages", "no rows", "table full", "all finished", "long cache_len", "bad ring", "bad page", "huge count"])
def test_plan_at_its_edges(B, case):
    new_cnt, lens, table = [2, 0, 3, 1], [3, 4, 7, 0], [[0, -1, -1], [1, -1, -1], [2, 3, -1], [-1, -1, -1]]
    ring, state, rows = [4, 5, 6, 7, 0, 0, 0, 0], [0, 4], 16
    if case == "none":
        new_cnt = [0] * 4
    elif case == "no pages":
        state = [0, 1]
    elif case == "no rows":
        rows = 3
    elif case == "table full":
        new_cnt = [9, 8, 6, 13]
    elif case == "all finished":
        new_cnt = [-1] * 4
    elif case == "long cache_len":
        lens[1] = 13
        new_cnt[1] = 1
    elif case == "bad ring":
        ring[1] = 8
    elif case == "bad page":
        table[0][0] = -3
    elif case == "huge count":
        new_cnt = [2, 2 ** 31 - 1, 2 ** 31 - 1, 1]
    p = B.make_paged_params(4, 1, 1, 64, 4, 8, 3, torch.float16)
    check_plan(B, p, new_cnt, lens, table, ring, state, rows, workspace(B, p))


# ---- rows --------------------------------------------------------------------------------------------------------------------------

def make_rows(n, h_q, h_kv, d, dtype, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    x = (1.5 * torch.randn((n, h_q + 2 * h_kv, d), generator=g)).to(dtype)
    if fused:
        x = x.cuda()
        return x[:, :h_q], x[:, h_q:h_q + h_kv], x[:, h_q + h_kv:]
    return tuple(t.contiguous().cuda() for t in x.split([h_q, h_kv, h_kv], 1))


def make_pool(n_pages, h_kv, page, d, dtype, int8, seed):
    g = torch.Generator().manual_seed(seed)
    shape = (n_pages, h_kv, page, d)
    if int8:
        k, v = (torch.randint(-127, 128, shape, generator=g, dtype=torch.int8).cuda() for _ in "kv")
        ks, vs = (torch.rand(shape[:3], generator=g).mul_(0.02).add_(0.001).cuda() for _ in "kv")
        return k, v, ks, vs
    k, v = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in "kv")
    return k, v, None, None


def check_append(B, n, h_q, h_kv, d, dtype, page, rot, sections=None, neighbours=False, norms=(True, True), int8=False, fused=True, far=1000,
                 in_place=False, slots=None, extra=3, eps=1e-5):
    sections = sections or [rot // 2]
    q, k, v = make_rows(n, h_q, h_kv, d, dtype, n + d, fused)
    n_pages = -(-n // page) + extra
    pool = make_pool(n_pages, h_kv, page, d, dtype, int8, 5)
    old = [t.clone() if t is not None else None for t in pool]
    g = torch.Generator().manual_seed(9)
    if slots is None:
        slots = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
        if n > 2:
            slots[n // 2] = -1
            slots[-1] = n_pages * page                          # outside the pool
    pos = torch.randint(0, far, (len(sections), n), generator=g, dtype=torch.int32)
    inv_freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) * 2 / max(rot, 1))
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(dtype) if on else None for on in norms]
    used = (slots >= 0) & (slots < n_pages * page)
    q0, k0, v0 = (t.cpu().double() for t in (q, k, v))
    for t in (q, k, v):
        t[~used.cuda()] = math.nan                              # rows without a slot are not looked at
    q_out = q if in_place else torch.full((n, h_q, d), 7.0, dtype=dtype, device="cuda")
    p = B.make_paged_params(1, h_q, h_kv, d, page, n_pages, n_pages, dtype, flags=(8 if int8 else 0) | (32 if neighbours else 0), rot_dim=rot,
                            sections=sections, eps=eps)
    ws = workspace(B, p)
    B.swa_paged_append(p, q, k, v, n, pos.cuda() if rot else None, slots.cuda(), inv_freq.cuda() if rot else None,
                       *[x.cuda() if x is not None else None for x in w], q_out, *pool, ws)
    assert B.swa_paged_check_status(p, ws) == (B.SWA_ERR_BAD_REQUEST if (slots >= n_pages * page).any() else B.SWA_OK)
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    wide = [x.double() if x is not None else None for x in w]

    def turned(x, weight):
        x = R.norm(x, weight, eps)
        return R.turn(x, pos, inv_freq, axis, rot, neighbours) if rot else (x, x.abs())
    y, size = turned(q0, wide[0])
    got = q_out.cpu().double()
    off = (got - y).abs() - R.row_tolerance(y, size, dtype, d)
    assert (off[used] <= 0).all(), float(off[used].max())
    assert (torch.isnan(got[~used]).all() if in_place else (got[~used] == 7).all())
    at, rest = slots[used].long(), torch.ones(n_pages * page, dtype=torch.bool)
    rest[at] = False
    for i, (x, (y, size)) in enumerate((("k", turned(k0, wide[1])), ("v", (v0, v0.abs())))):
        new, was = pool[i].cpu(), old[i].cpu()
        rows, rows0 = (t.transpose(1, 2).reshape(n_pages * page, h_kv, d) for t in (new, was))
        assert torch.equal(rows[rest], rows0[rest]), f"{x}: other slots"
        y, size = y[used], size[used]
        if int8:
            s, s0 = (t[2 + i].cpu().transpose(1, 2).reshape(n_pages * page, h_kv) for t in (pool, old))
            assert torch.equal(s[rest], s0[rest])
            step = y.abs().amax(-1) / 127
            err = R.row_tolerance(y, size, torch.float32, d)
            assert ((s[at].double() - step).abs() <= err.amax(-1) / 127 + 2.0 ** -22 * step).all()
            # half a step, and what moves a value over the border between two codes
            tol = step[..., None] * (0.5 + 2.0 ** -15) + 2 * err.amax(-1, keepdim=True)
            assert ((rows[at].double() * s[at].double()[..., None] - y).abs() <= tol).all()
            assert (rows[at].abs().amax(-1) == 127).all()
        elif x == "v":
            assert torch.equal(rows[at].double(), y)
        else:
            off = (rows[at].double() - y).abs() - R.row_tolerance(y, size, dtype, d)
            assert (off <= 0).all(), float(off.max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rows_of_every_type(B, dtype, d, neighbours):
    for h_q, h_kv, n in ((4, 2, 37), (5, 5, 1), (7, 1, 3)):
        check_append(B, n, h_q, h_kv, d, TYPES[dtype], 16, d, neighbours=neighbours)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_as_codes(B, dtype, d):
    check_append(B, 41, 8, 2, d, TYPES[dtype], 16, d, int8=True)
    check_append(B, 5, 3, 3, d, TYPES[dtype], 1, d // 2, int8=True, neighbours=True, norms=(True, False))
    check_append(B, 1, 1, 1, d, TYPES[dtype], 7, 0, int8=True, norms=(False, False))


@pytest.mark.parametrize("d,rot", [(64, 0), (64, 16), (64, 48), (128, 16), (128, 64), (128, 80), (128, 112)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_parts_of_a_row_are_rotated(B, d, rot, neighbours):
    check_append(B, 19, 6, 3, d, torch.float32, 8, rot, neighbours=neighbours)
    check_append(B, 19, 6, 3, d, torch.bfloat16, 8, rot, neighbours=neighbours, norms=(False, True))


@pytest.mark.parametrize("sections", [[32, 32], [16, 24, 24], [1, 62, 1], [0, 64], [64, 0, 0], [5, 6, 7, 46]])
def test_position_axes(B, sections):
    check_append(B, 23, 4, 2, 128, torch.float32, 16, 128, sections=sections)
    check_append(B, 23, 4, 2, 128, torch.float16, 16, 128, sections=sections, neighbours=True)


def test_far_positions_and_single_norms(B):
    for norms in ((True, False), (False, True), (False, False)):
        check_append(B, 33, 4, 4, 128, torch.float32, 16, 128, far=2 ** 31 - 1, norms=norms)
    check_append(B, 33, 4, 4, 64, torch.float32, 16, 64, far=2 ** 31 - 1, neighbours=True, eps=0.0)


def test_many_rows_share_waves_otherwise(B):
    check_append(B, 2500, 32, 8, 64, torch.bfloat16, 16, 64)
    check_append(B, 6000, 3, 1, 128, torch.float16, 32, 128, int8=True)


def test_rows_in_place_and_from_tensors_of_their_own(B):
    check_append(B, 50, 8, 2, 128, torch.bfloat16, 16, 128, fused=False, in_place=True)
    check_append(B, 50, 8, 2, 64, torch.float32, 16, 32, fused=False, in_place=True, neighbours=True)


def test_rows_that_are_not_finite_stay_in_their_rows(B):
    """A NaN or an infinity in one row's head; every other head as without it.  8-bit codes: the row reads back as NaN."""
    for int8 in (False, True):
        q, k, v = make_rows(4, 2, 2, 64, torch.float16, 3)
        k[1, 0, 5], v[2, 1, 7], q[3, 0, 63] = math.nan, math.inf, math.inf
        slots = torch.arange(4, dtype=torch.int32, device="cuda")
        k_pages, v_pages, ks, vs = make_pool(1, 2, 4, 64, torch.float16, int8, 1)
        p = B.make_paged_params(1, 2, 2, 64, 4, 1, 1, torch.float16, flags=8 if int8 else 0, rot_dim=32)
        ws = workspace(B, p)
        q_out = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
        inv = torch.ones(16, device="cuda")
        B.swa_paged_append(p, q, k, v, 4, slots, slots, inv, None, None, q_out, k_pages, v_pages, ks, vs, ws)
        kk, vv = (x.float() * s[..., None] if int8 else x.float() for x, s in ((k_pages, ks), (v_pages, vs)))
        bad = torch.zeros(2, 4, dtype=torch.bool, device="cuda")
        bad[0, 1] = True
        assert torch.equal(~torch.isfinite(kk[0]).all(-1), bad) and torch.isfinite(kk[0][~bad]).all()
        if int8:
            assert torch.isnan(kk[0, 0, 1]).all() and torch.isnan(vv[0, 1, 2]).all()
        else:
            assert int((~torch.isfinite(kk)).sum()) == 2       # the channel and its pair
            assert int((~torch.isfinite(vv)).sum()) == 1 and int((~torch.isfinite(q_out)).sum()) == 1
        assert torch.isfinite(vv[0, 0]).all()


def test_rows_of_zeros_and_tiny_values_as_codes(B):
    q, k, v = make_rows(3, 1, 1, 64, torch.bfloat16, 3)
    k[0], v[0] = 0, 0
    k[1], v[1] = 2.0 ** -130, 1e-30
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    pool = make_pool(1, 1, 4, 64, torch.bfloat16, True, 1)
    p = B.make_paged_params(1, 1, 1, 64, 4, 1, 1, torch.bfloat16, flags=8)
    B.swa_paged_append(p, q, k, v, 3, None, slots, None, None, None, torch.zeros_like(q), *pool, workspace(B, p))
    assert (pool[0][0, 0, :2] == 0).all() and (pool[2][0, 0, :2] == 0).all()
    assert (pool[1][0, 0, 0] == 0).all() and (pool[1][0, 0, 1] == 127).all()


# ---- attention ---------------------------------------------------------------------------------------------------------------------

def make_tables(lens, page, width, n_pages, seed):
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.full((len(lens), width), -5, dtype=torch.int32), 0
    for s, m in enumerate(lens):
        held = -(-max(m, 0) // page)
        table[s, :held] = order[at:at + held]
        at += held
    return table, order[at:]


def check_decode(B, lens, h_q, h_kv, d, dtype, page, window=0, int8=False, scale=0.0, len_bound=0, row_start=None, n_rows=None, strided=False,
                 spare=2, edit=None, bad=None, lse=True, loud=1.3, skipped=(), wider=0):
    """loud: how large queries are (softmaxes that are nearly flat, or nearly one key's)."""
    b = len(lens)
    held = [-(-max(m, 0) // page) for m in lens]
    n_pages, width = sum(held) + spare, max(max(held), 1) + wider
    table, free = make_tables(lens, page, width, n_pages, 11)
    k, v, ks, vs = make_pool(n_pages, h_kv, page, d, dtype, int8, 7)
    n_rows = n_rows or b
    g = torch.Generator().manual_seed(13)
    q = (loud * torch.randn((n_rows, h_q, d), generator=g)).to(dtype)
    # what lies outside the sequences is not a number
    live = torch.zeros(n_pages, page, dtype=torch.bool)
    for s, m in enumerate(lens):
        t = torch.arange(max(0, m - window) if window else 0, max(m, 0))
        live[table[s].long()[t // page], t % page] = True
    dead = (~live)[:, None, :].expand(-1, h_kv, -1).cuda()
    for x in (ks, vs) if int8 else (k, v):
        x[dead] = math.nan
    if edit:
        edit(k, v, q, table)
    if bad:
        for s, j, x in bad:
            table[s, j] = x
    p = B.make_paged_params(b, h_q, h_kv, d, page, n_pages, width, dtype, scale=scale, window=window, len_bound=len_bound, flags=8 if int8 else 0)
    ws = workspace(B, p)
    qd = q.cuda()
    if strided:
        wide = torch.full((n_rows, h_q + 3, d), math.nan, dtype=dtype, device="cuda")
        wide[:, :h_q] = qd
        qd = wide[:, :h_q]
    out = torch.full((n_rows, h_q, d), 7.0, dtype=dtype, device="cuda")
    sums = torch.full((n_rows, h_q), 7.0, device="cuda") if lse else None
    args = (p, qd, n_rows, ints(row_start) if row_start else None, k, v, ks, vs, table.cuda(), ints(lens), out, sums, ws)
    B.swa_paged_decode(*args)
    first = out.clone()
    code = B.SWA_ERR_CAPACITY if skipped else B.SWA_ERR_BAD_REQUEST if bad else B.SWA_OK
    assert B.swa_paged_check_status(p, ws) == code
    B.swa_paged_decode(*args)                              # the same bits again, whatever the first call left in the workspace
    assert torch.equal(first.view(torch.uint8), out.view(torch.uint8))
    B.swa_paged_check_status(p, ws)
    kc, vc, ksc, vsc = (t.cpu() if t is not None else None for t in (k, v, ks, vs))
    got, got_lse = out.cpu().double(), sums.cpu().double() if lse else None
    seen = set()
    for s, m in enumerate(lens):
        row = row_start[s + 1] - 1 if row_start else s
        if m < 0 or s in skipped or (row_start and row < row_start[s]) or not 0 <= row < n_rows:
            continue
        seen.add(row)
        lo = max(0, m - window) if window else 0
        kr, vr = (R.gather(x, y, table[s], page, lo, m) for x, y in ((kc, ksc), (vc, vsc)))
        steps = (R.half_step(dtype) if dtype != torch.float32 else 0.0, 0.0)
        if int8:                                           # 16-bit mantissas: of the weights, and of fp16 queries
            steps = (2.0 ** -16, 2.0 ** -16 if dtype == torch.float16 else 0.0)
        want, want_lse, tol, lse_tol = R.attention(q[row].double(), kr, vr, scale or d ** -0.5, dtype, *steps)
        for name, x, y, t in (("out", got[row], want, tol),) + ((("lse", got_lse[row], want_lse, lse_tol),) if lse else ()):
            fine = torch.isfinite(y)
            assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x[~fine & ~torch.isnan(y)], y[~fine & ~torch.isnan(y)]), (name, s)
            over = ((x - y).abs() - t)[fine]
            assert not over.numel() or over.max() <= 0, (name, s, m, float(over.max()), float(t[fine].max()))
    for row in set(range(n_rows)) - seen:
        assert (got[row] == 7).all() and (not lse or (got_lse[row] == 7).all()), row


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 300, 511, 513, 1000]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 20, 64])
def test_attention_of_every_type(B, dtype, d, page):
    check_decode(B, LENS, 8, 2, d, TYPES[dtype], page)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 32])
def test_attention_over_codes(B, dtype, d, page):
    check_decode(B, LENS, 8, 2, d, TYPES[dtype], page, int8=True)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (12, 12), (5, 1), (14, 2), (16, 1), (17, 1), (32, 1), (40, 1), (66, 2), (128, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_heads_that_share_keys(B, h_q, h_kv, dtype):
    check_decode(B, [7, 200, 1, 77], h_q, h_kv, 64, TYPES[dtype], 16)
    check_decode(B, [130, 33], h_q, h_kv, 128, TYPES[dtype], 16)
    if dtype == "bf16":
        check_decode(B, [130, 33, 1], h_q, h_kv, 128, torch.float16, 16, int8=True)
        check_decode(B, [130, 33, 1], h_q, h_kv, 64, torch.float16, 5)


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", True)])
def test_many_heads_over_long_caches(B, dtype, int8):
    """More query heads than a workgroup has, in chunks and in shares."""
    for d in (64, 128):
        check_decode(B, [3000, 77, 0, 1500], 71, 1, d, TYPES[dtype], 16, int8=int8)
        check_decode(B, [2000, 7, 0, 1100] * 8, 80, 2, d, TYPES[dtype], 16, int8=int8, len_bound=2000)


@pytest.mark.parametrize("page", [1, 3, 16, 48, 128, 1024])
@pytest.mark.parametrize("window", [0, 1, 31, 33, 200])
def test_pages_and_windows(B, page, window):
    check_decode(B, [1, 40, 250, 777], 4, 2, 64, torch.bfloat16, page, window=window)
    check_decode(B, [1, 40, 250, 777], 4, 4, 64, torch.float32, page, window=window)


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True)])
def test_long_caches_are_split_and_joined(B, dtype, int8):
    check_decode(B, [5000], 4, 1, 128, TYPES[dtype], 16, int8=int8, len_bound=5000)
    check_decode(B, [9000, 3, 0, 1025], 8, 2, 64, TYPES[dtype], 16, int8=int8)
    check_decode(B, [20011, 129], 3, 3, 64, TYPES[dtype], 64, int8=int8, window=7001)


@pytest.mark.parametrize("len_bound", [0, 100000])
def test_tables_far_wider_than_the_lengths(B, len_bound):
    check_decode(B, [5000, 0, 700], 4, 1, 128, torch.bfloat16, 16, wider=7000, len_bound=len_bound)
    check_decode(B, [3, 260], 4, 4, 64, torch.float16, 16, wider=130000, len_bound=len_bound)
    check_decode(B, [3000, 260] * 16, 8, 2, 64, torch.float32, 16, wider=9000, len_bound=len_bound, window=900)
    check_decode(B, [3000, 260] * 16, 8, 2, 64, torch.bfloat16, 16, wider=9000, len_bound=len_bound)


def test_many_sequences(B):
    rng = random.Random(3)
    check_decode(B, [rng.randrange(0, 400) for _ in range(300)], 8, 2, 128, torch.bfloat16, 16)
    check_decode(B, [rng.randrange(0, 60) for _ in range(1500)], 2, 1, 64, torch.float16, 16, len_bound=60)


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("bf16", False), ("f16", True)])
def test_short_sequences_by_one_wave(B, dtype, int8):
    """Up to 32 tokens, and up to 128 and 256 of many sequences and heads; the same with more query heads than a wave's threads join at once."""
    rng = random.Random(4)
    for d in (64, 128):
        check_decode(B, [0, 1, 31, 32, 17, -1], 7, 7, d, TYPES[dtype], 16, int8=int8)
        check_decode(B, [0, 1, 31, 32, 17], 32, 2, d, TYPES[dtype], 3, int8=int8)
        check_decode(B, [0, 1, 31, 32, 17], 37, 1, d, TYPES[dtype], 16, int8=int8)
    check_decode(B, [rng.randrange(0, 129) for _ in range(64)], 32, 16, 64, TYPES[dtype], 16, int8=int8)
    check_decode(B, [rng.randrange(0, 257) for _ in range(128)], 16, 16, 64, TYPES[dtype], 16, int8=int8)
    check_decode(B, [rng.randrange(0, 500) for _ in range(64)], 16, 16, 64, TYPES[dtype], 16, int8=int8, window=90)


@pytest.mark.parametrize("dtype,int8", [("bf16", False), ("f16", True)])
def test_few_long_sequences_in_shares(B, dtype, int8):
    check_decode(B, [70000, 3, 20001], 16, 8, 128, TYPES[dtype], 64, int8=int8)


def test_queries_sharp_and_scales(B):
    for dtype in (torch.float32, torch.bfloat16):
        check_decode(B, [300, 64], 4, 2, 128, dtype, 16, loud=20.0)
        check_decode(B, [300, 64], 4, 2, 128, dtype, 16, scale=0.01)
    check_decode(B, [300, 64], 4, 2, 128, torch.float16, 16, int8=True, loud=20.0)


def test_strided_queries_and_no_lse(B):
    check_decode(B, [33, 90, 12], 4, 2, 128, torch.bfloat16, 16, strided=True, lse=False)
    check_decode(B, [33, 90, 12], 4, 2, 64, torch.float32, 16, strided=True)


def test_padded_batches_and_rows_of_a_plan(B):
    check_decode(B, [33, -1, 90, 0, -1], 4, 2, 64, torch.bfloat16, 16)
    # sequence 1 has no new rows, sequence 2 three, sequence 4's row lies beyond the call's
    check_decode(B, [33, 50, 90, 12, 8], 4, 2, 64, torch.bfloat16, 16, row_start=[0, 1, 1, 4, 5, 6], n_rows=5)
    # rows that no plan gives
    check_decode(B, [33, 50, 90], 4, 2, 64, torch.bfloat16, 16, row_start=[-5, -1, 1, 2 ** 30], n_rows=3)
    check_decode(B, [1500, 50, 90] * 12, 4, 2, 64, torch.bfloat16, 16, row_start=[-5, -1, 1] + [2 ** 30] * 34, n_rows=3)


def test_sequences_beyond_the_bound_are_skipped(B):
    check_decode(B, [33, 100, 64, 65], 4, 2, 64, torch.bfloat16, 16, len_bound=64, skipped=(1, 3))
    check_decode(B, [33, 1300, 1200, 1201] * 10, 4, 2, 64, torch.bfloat16, 16, len_bound=1200, skipped=tuple(range(1, 40, 2)))


def test_pages_outside_the_pool_are_left_out(B):
    check_decode(B, [33, 100, 16], 4, 2, 64, torch.bfloat16, 16, bad=[(0, 1, -1), (1, 3, 12345678), (1, 6, -2 ** 31), (2, 0, 2 ** 31 - 1)])
    check_decode(B, [33, 100, 16], 4, 2, 128, torch.float16, 5, int8=True, bad=[(0, 1, -1), (1, 3, 12345678)])
    check_decode(B, [700, 100], 4, 2, 64, torch.float32, 16, bad=[(0, j, -1) for j in range(8, 40)])


def test_values_that_are_not_finite(B):
    """Infinite values of tokens that are seen reach the output as the formula says, in their head and channel only; keys that give
    a logit of -inf count nothing, also where a whole sequence has no other."""
    def no_key(k, v, q, table):
        k[table[0, 0].item(), 1, 3, 5] = math.nan            # its head's two query heads, nothing else
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        check_decode(B, [20, 4000], 4, 2, 64, dtype, 16, edit=no_key)
        check_decode(B, [20, 4000] * 20, 4, 2, 64, dtype, 16, edit=no_key)

    def infinite_value(k, v, q, table):
        v[table[0, 0].item(), 0, 3, 5] = math.inf
        v[table[1, 1].item(), 1, 2, 9] = math.nan
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        check_decode(B, [20, 40], 4, 2, 64, dtype, 16, edit=infinite_value)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_logits_of_minus_infinity(B, dtype):
    t = TYPES[dtype]
    k = torch.randn(40, 2, 16, 64).to(t).cuda()
    v = torch.randn(40, 2, 16, 64).to(t).cuda()
    q = torch.randn(2, 4, 64).to(t).cuda()
    q[..., 0] = q[..., 0].abs() + 1
    k[:20, :, :, 0] = -math.inf                          # sequence 0's first half, all of sequence 1's head 0
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    table[0, :10], table[0, 10:] = torch.arange(10), torch.arange(20, 30)
    table[1] = torch.arange(20)
    k[:20, 1] = torch.randn(20, 16, 64).to(t).cuda()
    p = B.make_paged_params(2, 4, 2, 64, 16, 40, 20, t)
    out, lse = torch.full((2, 4, 64), 7.0, dtype=t, device="cuda"), torch.zeros(2, 4, device="cuda")
    B.swa_paged_decode(p, q, 2, None, k, v, None, None, table, ints([320, 320]), out, lse, workspace(B, p))
    assert (out[1, :2] == 0).all() and (lse[1, :2] == -math.inf).all()
    assert torch.isfinite(out[0]).all() and torch.isfinite(lse[0]).all() and torch.isfinite(out[1, 2:]).all()
    half = torch.cat([k[20:30], v[20:30]]).cpu()
    want, want_lse, tol, lse_tol = R.attention(q[0, :2].cpu().double(), half[:10, 0].reshape(160, 1, 64).double(), half[10:, 0].reshape(160, 1, 64).double(),
                                               0.125, t, R.half_step(t))
    assert ((out[0, :2].cpu().double() - want).abs() <= tol).all() and ((lse[0, :2].cpu().double() - want_lse).abs() <= lse_tol).all()


def test_a_million_tokens_and_the_most_sequences(B):
    check_decode(B, [1 << 20], 1, 1, 64, torch.bfloat16, 16, len_bound=1 << 20)
    check_decode(B, [1] * 4095 + [40], 2, 1, 64, torch.bfloat16, 16)
    check_decode(B, [3] * 4094 + [2000, 40], 2, 1, 64, torch.float16, 16)


def test_offsets_beyond_32_bits(B):
    """A pool of 2^25 rows of 256 bytes: the last pages begin 2^33 bytes and 2^32 elements in."""
    n_pages, page, d = (1 << 25) // 16 + 40, 16, 128
    k, v = (torch.empty((n_pages, 1, page, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    p = B.make_paged_params(1, 2, 1, d, page, n_pages, 40, torch.bfloat16, rot_dim=d)
    ws = workspace(B, p)
    last = torch.arange(n_pages - 40, n_pages, dtype=torch.int32)
    for x in (k, v):
        x[n_pages - 40:] = math.nan
        x[:40] = math.nan
    q, kn, vn = make_rows(600, 2, 1, d, torch.bfloat16, 4)
    pos = torch.arange(600, dtype=torch.int32)
    slot = last[pos // 16] * 16 + pos % 16
    inv = 10000.0 ** (-torch.arange(64, dtype=torch.float32) / 64)
    q_out = torch.zeros_like(q).contiguous()
    B.swa_paged_append(p, q, kn, vn, 600, pos.cuda(), slot.cuda(), inv.cuda(), None, None, q_out, k, v, None, None, ws)
    out, lse = torch.zeros((1, 2, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 2), device="cuda")
    B.swa_paged_decode(p, q_out[-1:], 1, None, k, v, None, None, last[None].cuda(), ints([600]), out, lse, ws)
    rows = [R.gather(x[n_pages - 40:].cpu(), None, torch.arange(40), page, 0, 600) for x in (k, v)]
    want, want_lse, tol, lse_tol = R.attention(q_out[-1].cpu().double(), *rows, d ** -0.5, torch.bfloat16, 2.0 ** -8)
    assert ((out[0].cpu().double() - want).abs() <= tol).all() and ((lse[0].cpu().double() - want_lse).abs() <= lse_tol).all()
    assert torch.equal(rows[1][:, 0], vn[:, 0].cpu().double())
    del k, v
    torch.cuda.empty_cache()
