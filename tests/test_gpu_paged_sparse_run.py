"""Sparse attention and shared prefixes as a server uses them: plan, append, bounds, scores, selection and attention over many steps, in captured graphs and
on other streams."""
import math
import random

import pytest
import torch

import paged_reference as R
import test_gpu_paged_sparse as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def make(B, b, dtype, page, pages, width, select=0, int8=False, h_q=6, h_kv=2, d=64, layers=2, **more):
    p = B.make_paged_params(b, h_q, h_kv, d, page, pages, width, dtype, rot_dim=32, eps=1e-6, flags=B.SWA_KV_INT8 if int8 else 0, **more)
    return B.PagedCache(p, layers=layers, select=select)


class Step:
    """One step's rows, and the calls that put them into a cache."""

    def __init__(self, cache, rows, g):
        p = cache.params
        self.cache, self.rows = cache, rows
        self.x = torch.randn((rows, p.h_q + 2 * p.h_kv, p.d), generator=g).to(cache.dtype).cuda()
        self.slot, self.pos = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        self.inv = 10000.0 ** (-torch.arange(16, dtype=torch.float32, device="cuda") / 16)
        self.q, self.out = (torch.full((rows, p.h_q, p.d), 7.0, dtype=cache.dtype, device="cuda") for _ in range(2))
        self.lse = torch.full((rows, p.h_q), 7.0, device="cuda")

    def put(self, new, stream=None):
        c, p = self.cache, self.cache.params
        c.plan(new, self.slot, self.pos, stream)
        for layer in range(len(c.k_pages)):
            c.append(layer, self.x[:, :p.h_q], self.x[:, p.h_q:p.h_q + p.h_kv], self.x[:, p.h_q + p.h_kv:], self.slot, self.pos, self.inv, self.q, stream=stream)


def stored(cache, layer, s, head, tokens):
    """Keys and values that the cache holds of a sequence's tokens, for a key head, in float64."""
    page, table = cache.params.page_size, cache.block_table[s].cpu().long()
    t = torch.as_tensor(tokens, dtype=torch.long)
    at, off = table[t // page], t % page

    def rows(x, scale):
        x = x[layer].cpu()[at, head, off].double()
        return (x * scale[layer].cpu()[at, head, off].double()[:, None] if scale[layer] is not None else x)[:, None]
    return rows(cache.k_pages, cache.k_scale), rows(cache.v_pages, cache.v_scale)


def check_row(B, cache, layer, step, row, s, tokens_of):
    """The output of a row against the stored tokens tokens_of(head): (sequence, tokens) pieces."""
    p = cache.params
    g, dtype = p.h_q // p.h_kv, cache.dtype
    for head in range(p.h_kv):
        pieces = [stored(cache, layer, of, head, t) for of, t in tokens_of(head) if len(t)]
        k, v = (torch.cat(x) for x in zip(*pieces))
        steps = 2.0 ** -16 if p.flags & B.SWA_KV_INT8 else R.half_step(dtype) if dtype != torch.float32 else 0.0
        heads = slice(head * g, head * g + g)
        want, want_lse, tol, lse_tol = R.attention(step.q[row, heads].cpu().double(), k, v, p.d ** -0.5, dtype, steps)
        for name, x, y, z in (("out", step.out[row, heads], want, tol), ("lse", step.lse[row, heads], want_lse, lse_tol)):
            over = ((x.cpu().double() - y).abs() - z).max()
            assert over <= 0, (name, s, head, float(over))


@pytest.mark.parametrize("dtype,int8,page", [(torch.bfloat16, False, 16), (torch.float32, False, 5), (torch.float16, True, 8)])
def test_a_server_with_sparse_layers(B, dtype, int8, page):
    """Pages are handed on from finished sequences to others, whose bounds begin anew; refused sequences are left out."""
    b, rows = 8, 160
    cache = make(B, b, dtype, page, 700 // page, 200 // page, select=5, int8=int8)
    rng, g, refused = random.Random(3), torch.Generator().manual_seed(2), 0
    for turn in range(14):
        lens = cache.cache_len.tolist()
        new = [rng.choice((0, rng.randrange(1, 120))) if n == 0 else -1 if n > 170 or rng.random() < 0.08 else rng.choice((0, 1, 1, rng.randrange(1, 30))) for n in lens]
        step, layer = Step(cache, rows, g), turn % 2
        step.put(torch.tensor(new, dtype=torch.int32, device="cuda"))
        assert cache.check_status() in (B.SWA_OK, B.SWA_ERR_CAPACITY)
        cache.decode_sparse(layer, step.q, step.out, first=1, last=2, lse=step.lse, by_rows=True)
        assert cache.check_status() == B.SWA_OK
        now, start, slot = cache.cache_len.tolist(), cache.row_start.tolist(), step.slot.tolist()
        bounds, seen = cache.bounds[layer].cpu().float(), set()
        for s, n in enumerate(now):
            held = -(-n // page)
            for j in range(held):                            # of every page that holds tokens
                for head in range(2):
                    k = stored(cache, layer, s, head, range(j * page, min(n, j * page + page)))[0][:, 0].float().to(dtype).float()
                    box = bounds[int(cache.block_table[s, j]), head]
                    assert torch.equal(box[0], k.amin(0)) and torch.equal(box[1], k.amax(0)), (s, j)
            if new[s] <= 0 or start[s + 1] > rows or slot[start[s]] < 0:
                refused += new[s] > 0
                continue
            row = start[s + 1] - 1
            seen.add(row)
            for head in range(2):
                want = S.selection(cache.score[s, head].tolist(), held, 5, 1, 2)
                assert cache.sel[s, head].tolist() == want + [-1] * (5 - len(want)) and int(cache.sel_cnt[s, head]) == len(want)
            check_row(B, cache, layer, step, row, s,
                      lambda head: [(s, [t for e in cache.sel[s, head].tolist() if e >= 0 for t in range(e * page, min(n, e * page + page))])])
        for row in set(range(rows)) - seen:
            assert (step.out[row] == 7).all() and (step.lse[row] == 7).all()
    assert refused


@pytest.mark.parametrize("dtype,int8,page", [(torch.bfloat16, False, 16), (torch.float32, False, 5), (torch.float16, True, 8)])
def test_a_server_with_prefixes(B, dtype, int8, page):
    """Two instructions are written once; sequences behind either come and go."""
    b, rows, g, rng = 14, 700, torch.Generator().manual_seed(2), random.Random(8)
    cache = make(B, b, dtype, page, 2400 // page, 400 // page, int8=int8, h_q=12)
    step = Step(cache, rows, g)
    step.put(torch.tensor([390, 211] + [0] * 12, dtype=torch.int32, device="cuda"))
    of = [-1, -1] + [i % 3 - 1 for i in range(12)]           # behind the first, the second or none
    prefix_of = torch.tensor(of, dtype=torch.int32, device="cuda")
    for turn in range(8):
        lens = cache.cache_len.tolist()
        new = [0, 0] + [rng.choice((0, rng.randrange(1, 60))) if n == 0 else -1 if n > 90 or rng.random() < 0.08 else rng.choice((0, 1, 1, 3)) for n in lens[2:]]
        step, layer = Step(cache, rows, g), turn % 2
        step.put(torch.tensor(new, dtype=torch.int32, device="cuda"))
        cache.decode_shared(layer, step.q, step.out, prefix_of, step.lse, by_rows=True)
        assert cache.check_status() == B.SWA_OK
        now, start, seen = cache.cache_len.tolist(), cache.row_start.tolist(), set()
        for s, n in enumerate(now):
            if new[s] > 0:
                seen.add(start[s + 1] - 1)
                check_row(B, cache, layer, step, start[s + 1] - 1, s, lambda head: ([(of[s], range(now[of[s]]))] if of[s] >= 0 else []) + [(s, range(n))])
        for row in set(range(rows)) - seen:
            assert (step.out[row] == 7).all() and (step.lse[row] == 7).all()


def test_steps_in_captured_graphs(B):
    """Two graphs that share a workspace, one for each way round of the swapped lists, replayed with eager work between, against the same steps made eagerly."""
    b, g = 12, torch.Generator().manual_seed(4)
    caches = [make(B, b, torch.bfloat16, 16, 400, 40, select=6, h_q=16, h_kv=4, d=128, len_bound=640) for _ in range(2)]
    prefix_of = torch.tensor([-1] + [0] * 11, dtype=torch.int32, device="cuda")
    first, ones = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([400] + [30 + 7 * i for i in range(11)], [0] + [1] * 11))
    prompt = torch.randn((1000, 24, 128), generator=g).to(torch.bfloat16).cuda()
    for c in caches:
        s = Step(c, 1000, torch.Generator().manual_seed(0))
        s.x = prompt
        s.put(first)
        assert c.check_status() == B.SWA_ERR_CAPACITY        # (the rows of the last two end beyond the call's: they begin with the next step)
    tokens = [torch.randn((11, 24, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(8)]
    steps = [[Step(c, 11, torch.Generator().manual_seed(0)) for _ in range(2)] for c in caches]
    more = [[(torch.zeros_like(s.out), torch.zeros_like(s.lse)) for s in two] for two in steps]

    def one(i, k):
        c, s, (out, lse) = caches[i], steps[i][k], more[i][k]
        s.put(ones)
        c.decode_sparse(1, s.q, s.out, lse=s.lse, by_rows=True)
        c.decode_shared(0, s.q, out, prefix_of, lse, by_rows=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        for k in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                one(0, k)
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(stream)
    for i, t in enumerate(tokens):
        k = i % 2
        for j in range(2):
            steps[j][k].x.copy_(t)
        graphs[k].replay()
        torch.cuda.synchronize()
        one(1, k)
        for x, y in ((steps[0][k].out, steps[1][k].out), (steps[0][k].lse, steps[1][k].lse), (more[0][k][0], more[1][k][0]), (more[0][k][1], more[1][k][1]),
                     (caches[0].sel, caches[1].sel), (caches[0].score, caches[1].score), (caches[0].bounds[1], caches[1].bounds[1])):
            assert torch.equal(x, y), i
        junk = torch.randn((1 << 20,), device="cuda")        # eager work of the program's own
        assert math.isfinite(float(junk.sum()))
    assert caches[0].check_status() == B.SWA_OK and caches[1].check_status() == B.SWA_OK


def test_on_streams_at_once(B):
    """Two caches, each on a stream of its own and with its own workspace, make the steps that one makes on the default stream."""
    g = torch.Generator().manual_seed(4)
    caches = [make(B, 20, torch.float16, 16, 500, 60, select=4, h_q=8, h_kv=2, d=128) for _ in range(3)]
    prefix_of = torch.tensor([-1] + [0] * 19, dtype=torch.int32, device="cuda")
    new = torch.tensor([700] + [20 + 9 * i for i in range(19)], dtype=torch.int32, device="cuda")
    steps = [Step(c, 3000, torch.Generator().manual_seed(1)) for c in caches]
    x = torch.randn((3000, 12, 128), generator=g).to(torch.float16).cuda()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), None]
    shared = [torch.full_like(s.out, 7.0) for s in steps]
    for s in steps:
        s.x = x
    torch.cuda.synchronize()
    for s, c, st, o in zip(steps, caches, streams, shared):
        s.put(new, st)
        for _ in range(3):
            c.decode_sparse(0, s.q, s.out, lse=s.lse, by_rows=True, stream=st)
            c.decode_shared(1, s.q, o, prefix_of, by_rows=True, stream=st)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(steps[i].out, steps[2].out) and torch.equal(steps[i].lse, steps[2].lse) and torch.equal(shared[i], shared[2])


def test_what_a_cache_refuses(B):
    with pytest.raises(ValueError, match="select"):
        make(B, 2, torch.float16, 16, 20, 8, select=9)
    with pytest.raises(ValueError, match="select"):
        make(B, 2, torch.float16, 16, 20, 8, select=4, window=30)
    cache = make(B, 2, torch.float16, 16, 20, 8)
    q = torch.zeros((2, 6, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError, match="bounds"):
        cache.decode_sparse(0, q, q.clone())
    with pytest.raises(ValueError, match="prefix_of"):
        cache.decode_shared(0, q, q.clone(), torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="out"):
        cache.decode_shared(0, q, q[:1].clone(), torch.zeros(2, dtype=torch.int32, device="cuda"))
    cache = make(B, 2, torch.float16, 16, 20, 8, window=30)
    with pytest.raises(B.SwaError) as e:
        cache.decode_shared(0, q, q.clone(), torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert e.value.code == B.SWA_ERR_BAD_SHAPE
