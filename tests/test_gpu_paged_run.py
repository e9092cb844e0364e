"""The paged cache's operators together, as a server uses them: plan, append and decode over many steps, in captured graphs, on other
streams, and with the calls over the contiguous cache."""
import random

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


class Model:
    """One layer's projections of tokens that are known beforehand, and its cache in float64 on the CPU."""

    def __init__(self, h_q, h_kv, d, dtype, rot, seed):
        g = torch.Generator().manual_seed(seed)
        self.h_q, self.h_kv, self.d, self.dtype, self.rot, self.g = h_q, h_kv, d, dtype, rot, g
        self.inv_freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) * 2 / rot)
        self.weights = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype) for _ in "qk"]
        self.axis = torch.zeros(rot // 2, dtype=torch.int64)

    def project(self, n):
        return torch.randn((n, self.h_q + 2 * self.h_kv, self.d), generator=self.g).to(self.dtype)

    def rotated(self, x, which, pos):
        x = R.norm(x.double(), self.weights[which], 1e-6)
        return R.turn(x, torch.tensor([pos]), self.inv_freq, self.axis, self.rot, False)[0]


def check_rows(got, want, tol, what):
    over = (got.double().cpu() - want).abs() - tol
    assert over.max() <= 0, (what, float(over.max()))


@pytest.mark.parametrize("dtype,int8,page,window", [(torch.bfloat16, False, 16, 0), (torch.float32, False, 5, 40), (torch.float16, True, 16, 0)])
def test_a_server_of_many_requests(B, dtype, int8, page, window):
    """Requests arrive with prompts, grow token by token, finish, and hand their pages on; the pool is small enough that some wait.  Rows
    of a step are packed; sequences without a new token take part in no attention."""
    h_q, h_kv, d, b, rows = 6, 2, 64, 9, 150
    m = Model(h_q, h_kv, d, dtype, 32, 4)
    p = B.make_paged_params(b, h_q, h_kv, d, page, 420 // page, 200 // page, dtype, rot_dim=32, eps=1e-6, window=window,
                            flags=B.SWA_KV_INT8 if int8 else 0)
    cache, rng = B.PagedCache(p, layers=2), random.Random(7)
    inv, wq, wk = m.inv_freq.cuda(), m.weights[0].cuda(), m.weights[1].cuda()
    slot, pos = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    live = [dict(k=[], v=[]) for _ in range(b)]
    refused = finished = 0
    for step in range(30):
        new = []
        for s in range(b):
            n = len(live[s]["k"])
            new.append(rng.choice((0, rng.randrange(1, 60))) if n == 0 else -1 if n > 90 or rng.random() < 0.05 else rng.choice((0, 1, 1, 1, 2)))
        lens = [len(x["k"]) for x in live]
        table = cache.block_table.tolist()
        want = R.plan(new, lens, table, cache.free_ring.tolist(), cache.free_state.tolist(), page, rows)
        cache.plan(torch.tensor(new, dtype=torch.int32, device="cuda"), slot, pos)
        assert cache.cache_len.tolist() == want[0] and slot.tolist() == want[5] and pos.tolist() == want[6]
        assert cache.check_status() == (B.SWA_ERR_CAPACITY if "capacity" in want[7] else B.SWA_OK)
        # every page is in one place
        held = [x for s in range(b) for x in want[1][s][:-(-want[0][s] // page)]]
        head, count = want[3]
        assert sorted(held + [want[2][(head + i) % p.n_pages] for i in range(count)]) == list(range(p.n_pages))
        qkv = m.project(rows)
        x = qkv.cuda()
        q_out, out = (torch.zeros((rows, h_q, d), dtype=dtype, device="cuda") for _ in range(2))
        lse = torch.zeros((rows, h_q), device="cuda")
        layer = step % 2                                   # (both layers hold the same tokens)
        for i in range(2):
            cache.append(i, x[:, :h_q], x[:, h_q:h_q + h_kv], x[:, h_q + h_kv:], slot, pos, inv, q_out, wq, wk)
        cache.decode(layer, q_out, out, lse, by_rows=True)
        assert cache.check_status() == B.SWA_OK
        for s in range(b):
            if new[s] < 0:
                live[s] = dict(k=[], v=[])
                finished += 1
                continue
            if new[s] and want[0][s] == lens[s]:
                refused += 1
                continue
            for i in range(new[s]):
                r = want[4][s] + i
                live[s]["k"].append(qkv[r, h_q:h_q + h_kv])
                live[s]["v"].append(qkv[r, h_q + h_kv:])
            n = want[0][s]
            if not new[s]:
                continue
            row = want[4][s + 1] - 1
            q = m.rotated(qkv[row:row + 1, :h_q], 0, [n - 1])[0]
            k, v = m.rotated(torch.stack(live[s]["k"]), 1, list(range(n))), torch.stack(live[s]["v"]).double()
            lo = max(0, n - window) if window else 0
            k, v = k[lo:], v[lo:]
            u = R.half_step(dtype)
            o, l, tol, lse_tol = R.attention(q, k, v, d ** -0.5, dtype, u if dtype != torch.float32 else 0)
            # queries and keys were rounded on their way, codes to half of max / 127; a logit moves by that, a weight by as much of itself
            key = k.abs().amax(-1, keepdim=True) / 254 + 2.0 ** -20 * k.abs() if int8 else u * k.abs() + 2.0 ** -20 * k.abs()
            val = v.abs().amax(-1, keepdim=True) / 254 if int8 else torch.zeros_like(v)
            g = h_q // h_kv
            kk, dk, vv, dv = (t.repeat_interleave(g, 1).permute(1, 0, 2).expand(h_q, -1, d) for t in (k, key, v, val))
            move = (((u + 2.0 ** -20) * q[:, None].abs() * kk.abs() + (1 + u) * q[:, None].abs() * dk).sum(-1) * d ** -0.5).amax(-1)
            w = torch.softmax((kk * q[:, None]).sum(-1) * d ** -0.5, -1)[..., None]
            tol = tol + 2 * torch.expm1(2 * move)[:, None] * (w * (vv.abs() + dv)).sum(1) + (w * dv).sum(1)
            check_rows(out[row], o, tol, (step, s, n))
            check_rows(lse[row], l, lse_tol + move, (step, s, n, "lse"))
    assert refused and finished                            # (the run has seen both)


def test_steps_in_captured_graphs(B):
    """Two graphs, one for each way round of the swapped lists, replayed with eager work between, against the same steps made eagerly."""
    b, h_q, h_kv, d, page = 5, 8, 2, 128, 16
    p = B.make_paged_params(b, h_q, h_kv, d, page, 200, 40, torch.bfloat16, rot_dim=d, eps=1e-6, len_bound=640)
    m = Model(h_q, h_kv, d, torch.bfloat16, d, 5)
    inv, wq, wk = m.inv_freq.cuda(), m.weights[0].cuda(), m.weights[1].cuda()
    lens = [0, 17, 300, 31, 64]
    new = torch.ones(b, dtype=torch.int32, device="cuda")
    steps = [m.project(b).cuda() for _ in range(9)]

    def start():
        c = B.PagedCache(p)
        s, q = (torch.zeros(sum(lens), dtype=torch.int32, device="cuda") for _ in range(2))
        c.plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), s, q)
        x = first.cuda()
        c.append(0, x[:, :h_q], x[:, h_q:h_q + h_kv], x[:, h_q + h_kv:], s, q, inv, torch.zeros_like(x[:, :h_q]).contiguous(), wq, wk)
        return c, torch.zeros(b, dtype=torch.int32, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")
    first = m.project(sum(lens))

    def step(c, slot, pos, x, q_out, out, lse):
        c.plan(new, slot, pos)
        c.append(0, x[:, :h_q], x[:, h_q:h_q + h_kv], x[:, h_q + h_kv:], slot, pos, inv, q_out, wq, wk)
        c.decode(0, q_out, out, lse)

    def buffers():
        return [torch.zeros((b, h_q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.zeros((b, h_q), device="cuda")]
    eager, eb = start(), buffers()
    want = []
    for x in steps:
        step(*eager, x, *eb)
        want.append([t.clone() for t in eb[1:]])
    state, gb = start(), buffers()
    x = torch.zeros_like(steps[0])
    lengths, frees, ring, table = state[0].cache_len.clone(), state[0].free_state.clone(), state[0].free_ring.clone(), state[0].block_table.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):
            step(*state, x, *gb)                           # (each way round once before it is captured)
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step(*state, x, *gb)
            graphs.append(g)
    torch.cuda.current_stream().wait_stream(side)
    # back to the prompts' end
    state[0].cache_len.copy_(lengths)
    state[0].free_state.copy_(frees)
    state[0].free_ring.copy_(ring)
    state[0].block_table.copy_(table)
    for i, y in enumerate(steps):
        x.copy_(y)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").sum()              # eager work between replays
        for got, w in zip(gb[1:], want[i]):
            assert torch.equal(got, w), i
    assert state[0].check_status() == B.SWA_OK and eager[0].check_status() == B.SWA_OK


def test_another_stream_and_two_calls_at_once(B):
    """Calls on streams of their own, with workspaces of their own, over one pool."""
    b, h_q, h_kv, d, page, n = 4, 8, 2, 64, 16, 2000
    p = B.make_paged_params(b, h_q, h_kv, d, page, b * 125, 125, torch.float16)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((b * 125, h_kv, page, d), generator=g, device="cuda").half() for _ in "kv")
    table = torch.randperm(b * 125, generator=g, device="cuda").view(b, 125).int()
    lens = torch.tensor([n, 3, 1111, 64], dtype=torch.int32, device="cuda")
    qs = [torch.randn((b, h_q, d), generator=g, device="cuda").half() for _ in range(2)]

    def call(q, out, ws):
        B.swa_paged_decode(p, q, b, None, k, v, None, None, table, lens, out, None, ws)

    def fresh():
        ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
        B.swa_paged_workspace_init(p, ws)
        return torch.zeros((b, h_q, d), dtype=torch.float16, device="cuda"), ws
    want = []
    for q in qs:
        out, ws = fresh()
        call(q, out, ws)
        want.append(out)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in qs], [fresh() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, q, (out, ws) in zip(streams, qs, got):
            with torch.cuda.stream(st):
                call(q, out, ws)
    torch.cuda.synchronize()
    for (out, _), w in zip(got, want):
        assert torch.equal(out, w)
    # a stream handed in as an object
    out, ws = fresh()
    torch.cuda.synchronize()
    B.swa_paged_decode(p, qs[0], b, None, k, v, None, None, table, lens, out, None, ws, streams[0])
    streams[0].synchronize()
    assert torch.equal(out, want[0])


def test_the_contiguous_cache_is_a_pool_of_one_page_each(B):
    """append into a cache [b, h, cap, d], prefill attention over it, then decode steps of both kinds: with everything kept, the sparse
    step and the dense one attend over the same tokens."""
    b, h, d, cap, n = 3, 4, 128, 96, 60
    dt = torch.float16
    m = Model(h, h, d, dt, d, 8)
    inv, wq, wk = m.inv_freq.cuda(), m.weights[0].cuda(), m.weights[1].cuda()
    p = B.make_paged_params(b, h, h, d, cap, b, 1, dt, rot_dim=d, eps=1e-6)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    sp = B.make_params(b, h, d, cap, 8, 0, dt)
    st = B.DecodeState(sp)
    # prompts of n tokens: row s * n + t into slot s * cap + t
    x = m.project(b * n).cuda()
    t = torch.arange(n, dtype=torch.int32, device="cuda")
    slot = (torch.arange(b, dtype=torch.int32, device="cuda")[:, None] * cap + t).flatten()
    q = torch.zeros((b * n, h, d), dtype=dt, device="cuda")
    B.swa_paged_append(p, x[:, :h], x[:, h:2 * h], x[:, 2 * h:], b * n, t.repeat(b), slot, inv, wq, wk, q, st.K, st.V, None, None, ws)
    qc = torch.zeros((b, h, cap, d), dtype=dt, device="cuda")
    qc[:, :, :n] = q.view(b, n, h, d).transpose(1, 2)
    st.cache_len.fill_(n)
    st.pos[:, :, :n] = t
    out = torch.zeros_like(qc)
    B.swa_prefill_attention(sp, qc, st.K, st.V, st.cache_len, out, 0, None, st.workspace)
    # the prompt's last token by the paged call
    table = torch.arange(b, dtype=torch.int32, device="cuda").view(b, 1)
    last, lse = torch.zeros((b, h, d), dtype=dt, device="cuda"), torch.zeros((b, h), device="cuda")
    B.swa_paged_decode(p, qc[:, :, n - 1].contiguous(), b, None, st.K, st.V, None, None, table, st.cache_len, last, lse, ws)
    for s in range(b):
        k, v = (y[s, :, :n].transpose(0, 1).cpu().double() for y in (st.K, st.V))
        want, want_lse, tol, lse_tol = R.attention(qc[s, :, n - 1].cpu().double(), k, v, d ** -0.5, dt, R.half_step(dt))
        check_rows(last[s], want, tol, s)
        check_rows(lse[s], want_lse, lse_tol, s)
        check_rows(out[s, :, n - 1], want, tol, s)
    # a new token: rows of one token a page for the sparse step, which appends them itself
    rows = B.make_paged_params(b, h, h, d, 1, b, 1, dt, rot_dim=d, eps=1e-6)
    x = m.project(b).cuda()
    k_new, v_new, q_new, o = (torch.zeros((b, h, d), dtype=dt, device="cuda") for _ in range(4))
    B.swa_paged_append(rows, x[:, :h], x[:, h:2 * h], x[:, 2 * h:], b, torch.full((b,), n, dtype=torch.int32, device="cuda"),
                       torch.arange(b, dtype=torch.int32, device="cuda"), inv, wq, wk, q_new, k_new, v_new, None, None, ws)
    st.seq_len.fill_(n + 1)
    st.decode_step(q_new, k_new, v_new)
    B.swa_paged_decode(p, q_new, b, None, st.K, st.V, None, None, table, st.cache_len, o, lse, ws)
    assert (st.cache_len == n + 1).all() and torch.equal(st.K[:, :, n], k_new)
    for s in range(b):
        k, v = (y[s, :, :n + 1].transpose(0, 1).cpu().double() for y in (st.K, st.V))
        want, _, tol, _ = R.attention(q_new[s].cpu().double(), k, v, d ** -0.5, dt, R.half_step(dt))
        check_rows(o[s], want, tol, s)
        check_rows(st.out[s], want, tol, s)
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK


def test_the_class_refuses_what_does_not_fit(B):
    p = B.make_paged_params(2, 4, 2, 64, 16, 8, 4, torch.bfloat16, rot_dim=64)
    c = B.PagedCache(p)
    i32 = dict(dtype=torch.int32, device="cuda")
    rows, q, kv = torch.zeros(3, **i32), torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    inv = torch.ones(32, device="cuda")
    with pytest.raises(ValueError, match="new_cnt"):
        c.plan(torch.zeros(3, **i32), rows, rows)
    with pytest.raises(ValueError, match="slot"):
        c.plan(torch.zeros(2, **i32), rows.long(), rows)
    with pytest.raises(ValueError, match="k must"):
        c.append(0, q, q, kv, rows, rows, inv, q)
    with pytest.raises(ValueError, match="q must"):
        c.append(0, q.float(), kv, kv, rows, rows, inv, q)
    with pytest.raises(ValueError, match="inv_freq"):
        c.append(0, q, kv, kv, rows, rows, inv[:16], q)
    with pytest.raises(ValueError, match="out"):
        c.decode(0, q, q[:2])
    with pytest.raises(B.SwaError):
        c.decode(0, q[:1], q[:1])                          # two sequences, one row
    with pytest.raises(ValueError):
        B.PagedCache(B.make_paged_params(2, 3, 2, 64, 16, 8, 4, torch.bfloat16))
