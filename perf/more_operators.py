"""Cases of the paged cache's sparse attention and of its attention behind shared prefixes.

Five operators, each also in a plain form of elementary torch operations:

  bounds   swa_paged_bounds: smallest and largest key values of every page that new rows went into.
  score    swa_paged_score: for each sequence, key head and page an upper bound of its logits, from the bounds alone.
  select   swa_paged_select: the pages of highest score for each sequence and key head, with the first and the last ones.
  attend   swa_paged_decode_selected: attention of each sequence's newest token over the selected pages.
  shared   swa_paged_decode_shared: attention of each sequence's newest token over a prefix that many share, and its own pages.

Lengths are spread evenly over lo..hi (the same for every seed, so that the work is), in a mixed order; values, pages and
their order come from the seed.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    def bounds(name, b, h_kv, d, dtype, page, lo, hi, least, most, int8):
        # b sequences of lo..hi tokens bring least..most more
        return dict(name=name, op="bounds", b=b, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi, least=least, most=most, int8=int8)

    def score(name, b, h_q, h_kv, d, dtype, page, lo, hi):
        return dict(name=name, op="score", b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi)

    def select(name, b, h_kv, page, lo, hi, n_sel, first, last):
        return dict(name=name, op="select", b=b, h_kv=h_kv, page=page, lo=lo, hi=hi, n_sel=n_sel, first=first, last=last)

    def attend(name, b, h_q, h_kv, d, dtype, page, lo, hi, n_sel, int8):
        return dict(name=name, op="attend", b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi, n_sel=n_sel, int8=int8)

    def shared(name, b, prefixes, h_q, h_kv, d, dtype, page, plo, phi, lo, hi, int8):
        # b sequences of lo..hi tokens behind `prefixes` prefixes of plo..phi tokens
        return dict(name=name, op="shared", b=b, prefixes=prefixes, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, plo=plo, phi=phi,
                    lo=lo, hi=hi, int8=int8)

    return [
        # one step of a serving batch: latency counts
        bounds("bounds_step", 64, 8, 128, "bf16", 16, 100, 1500, 1, 1, False),
        # pieces of prompts into the compressed cache, beginning and ending inside pages
        bounds("bounds_prompts_int8", 13, 8, 128, "f16", 64, 1, 900, 77, 1207, True),
        # a few chats with some thousand tokens each: latency counts
        score("score_step", 8, 32, 8, 128, "bf16", 16, 1000, 8003),
        # a batch far into its contexts
        score("score_batch", 32, 32, 8, 128, "bf16", 16, 1000, 65536),
        # the same chats
        select("select_step", 8, 8, 16, 1000, 8003, 64, 1, 2),
        # 131071 tokens in pages of 16, and shorter ones beside them
        select("select_long", 16, 8, 16, 4001, 131071, 256, 4, 16),
        # one chat with a long context: latency counts
        attend("attend_one", 1, 32, 8, 128, "bf16", 16, 16001, 16001, 64, False),
        # a full serving batch that reads 2048 tokens of up to 32768 each
        attend("attend_batch", 64, 32, 8, 128, "bf16", 16, 2048, 32768, 128, False),
        # the compressed cache, large pages, sequences shorter than what may be selected among them
        attend("attend_int8", 48, 28, 4, 128, "f16", 64, 100, 20011, 32, True),
        # a few requests with one system prompt, 32 heads of their own in fp32
        shared("shared_chat_f32", 8, 1, 32, 32, 64, "f32", 20, 1001, 1001, 1, 300, False),
        # a full serving batch behind three instructions
        shared("shared_batch", 128, 3, 32, 8, 128, "bf16", 16, 2049, 8191, 16, 1500, False),
        # many questions about one long document: the matrix cores are the bound
        shared("shared_document", 64, 1, 64, 8, 128, "f16", 64, 32768, 32768, 1, 300, False),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("bounds", "score", "select", "attend", "attend", "shared", "shared"))
    d, dtype = rng.choice((64, 128, 128)), rng.choice(("f32", "f16", "bf16", "bf16"))
    h_q, h_kv = rng.choice(((32, 32), (40, 40), (12, 12), (32, 8), (28, 4), (64, 8), (16, 1), (25, 5)))
    int8, page = dtype != "f32" and rng.random() < 0.25, rng.choice((1, 8, 16, 16, 20, 32, 64, 128))
    width = h_kv * d * (1 if int8 else BYTES[dtype])
    if op == "bounds":
        b, hi, most = spread(1, 256), spread(1, 4000), rng.choice((1, spread(1, 2000)))
        while b > 1 and b * (hi + most) * width > 1 << 28:
            b = b * 2 // 3
        return dict(op=op, b=b, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=rng.choice((0, 1, hi // 3)), hi=hi,
                    least=rng.choice((1, most)), most=most, int8=int8)
    if op in ("score", "select"):
        page, hi, b = rng.choice((8, 16, 16, 32, 64, 128)), spread(16, 131072), spread(1, 256)
        while b > 1 and b * (hi / page) * h_kv * d * BYTES[dtype] > 1 << 27:
            b = b * 2 // 3
        lo = rng.choice((hi, max(1, hi // 4), 1))
        if op == "score":
            return dict(op=op, b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi)
        n_sel = min(spread(2, 1024), 131072 // (3 * page))
        hi = max(hi, 3 * n_sel * page)                       # (some pages are left out)
        lo = rng.choice((hi, hi // 4, 1))
        first, last = rng.choice((0, 1, 4)), rng.choice((1, 2, 16))
        first, last = min(first, n_sel // 4), min(last, n_sel // 4)
        return dict(op=op, b=b, h_kv=h_kv, page=page, lo=lo, hi=hi, n_sel=n_sel, first=first, last=last)
    if op == "attend":
        hi, b = spread(1, 131072), spread(1, 256)
        while b > 1 and b * hi * width > 1 << 31:
            b = b * 2 // 3
        n_sel = min(-(-hi // page), spread(1, 8192 // page + 1))
        while n_sel > 1 and b * n_sel * page * width > 1 << 28:
            n_sel = n_sel * 2 // 3
        return dict(op=op, b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=rng.choice((hi, max(1, hi // 4), 1)), hi=hi,
                    n_sel=n_sel, int8=int8)
    b, phi, hi, prefixes = spread(2, 256), spread(16, 32768), spread(1, 2000), rng.choice((1, 1, 2, 4))
    while prefixes * phi * width > 1 << 28:
        phi = phi * 2 // 3
    while b > 2 and (b * h_q * phi * d * 4 / 50 > 1 << 30 or b * hi * width > 1 << 29 or prefixes * b * h_q * phi > 1 << 29):
        b = b * 2 // 3
    return dict(op=op, b=b, prefixes=prefixes, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, plo=rng.choice((phi, max(1, phi // 4))),
                phi=phi, lo=rng.choice((0, 1, hi)), hi=hi, int8=int8)


def _lengths(lo, hi, n):
    """n lengths, evenly over lo..hi, in a mixed order."""
    even = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    step = next(k for k in (61, 67, 71, 73) if n % k)
    return [even[i * step % n] for i in range(n)]


def _all_lengths(c):
    """Of every row of the block table: the prefixes' first."""
    lens = _lengths(c["lo"], c["hi"], c["b"])
    return _lengths(c["plo"], c["phi"], c["prefixes"]) + lens if c["op"] == "shared" else lens


def _read(c):
    """Tokens that an attention reads of each sequence, for one key head."""
    lens = _lengths(c["lo"], c["hi"], c["b"])
    # the last page is among the selected ones
    return [n if -(-n // c["page"]) <= c["n_sel"] else (c["n_sel"] - 1) * c["page"] + (n - 1) % c["page"] + 1 for n in lens]


def _lib(int8=False, **more):
    from paper_2403_17312_amd import binding as B
    p = B.make_paged_params(**more, flags=B.SWA_KV_INT8 if int8 else 0)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    return B, p, ws


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    made = {"bounds": _prepare_bounds, "score": _prepare_score, "select": _prepare_select, "attend": _prepare_attend, "shared": _prepare_shared}
    return made[case["op"]](case, g)


def _tables(lens, page, g):
    """(block table, pages of the pool) of sequences of these lengths, whose pages lie anywhere in it."""
    held = [-(-m // page) for m in lens]
    n_pages, table = sum(held) + 2, max(1, max(held))
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    h = _int(held)
    first = torch.cumsum(h, 0) - h
    j = torch.arange(table, device="cuda")
    return torch.where(j < h[:, None], order[(first[:, None] + j).clamp(max=n_pages - 1)], -1).to(torch.int32), n_pages


def _pool(c, n_pages, g, which):
    """Pages (and scales) of keys or values."""
    shape = (n_pages, c["h_kv"], c["page"], c["d"])
    if c["int8"]:
        return {which + "_pages": torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8),
                which + "_scale": torch.rand(shape[:3], generator=g, device="cuda").mul_(0.02).add_(0.005)}
    return {which + "_pages": torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g), which + "_scale": None}


def _prepare_bounds(c, g):
    t, page, b = DTYPES[c["dtype"]], c["page"], c["b"]
    lens, new = _int(_lengths(c["lo"], c["hi"], b)), _int(_lengths(c["least"], c["most"], b))
    grown = [m + n for m, n in zip(_lengths(c["lo"], c["hi"], b), _lengths(c["least"], c["most"], b))]
    table, n_pages = _tables(grown, page, g)
    rows = sum(_lengths(c["least"], c["most"], b))
    # packed rows, and one behind the last
    of = torch.repeat_interleave(torch.arange(b, device="cuda"), new.long(), output_size=rows)
    at = lens.long()[of] + torch.arange(rows, device="cuda") - (torch.cumsum(new, 0) - new).long()[of]
    slot = torch.cat([table.long()[of, at // page] * page + at % page, torch.full((1,), -1, device="cuda")]).to(torch.int32)
    mid = torch.empty((n_pages, c["h_kv"], 2, c["d"]), device="cuda").normal_(generator=g)
    mid += torch.tensor([-1.7, 1.7], device="cuda")[:, None]
    s = dict(case=c, slot=slot, rows=rows + 1, bounds=torch.sort(mid, 2).values.to(t), **_pool(c, n_pages, g, "k"))
    if own:
        s["lib"] = _lib(b=b, h_q=c["h_kv"], h_kv=c["h_kv"], d=c["d"], page_size=page, n_pages=n_pages, max_pages=table.shape[1], dtype=t,
                        int8=c["int8"])
    return s


def _prepare_score(c, g):
    t, b, page = DTYPES[c["dtype"]], c["b"], c["page"]
    lens = _lengths(c["lo"], c["hi"], b)
    table, n_pages = _tables(lens, page, g)
    bounds = torch.empty((n_pages, c["h_kv"], 2, c["d"]), dtype=t, device="cuda").normal_(generator=g).mul_(0.4)
    bounds += torch.tensor([-1.7, 1.7], dtype=t, device="cuda")[:, None]      # of about sixteen normal keys
    s = dict(case=c, q=torch.randn((b, c["h_q"], c["d"]), generator=g, device="cuda").mul_(1.3).to(t), bounds=bounds, block_table=table,
             cache_len=_int(lens), score=torch.zeros((b, c["h_kv"], table.shape[1]), device="cuda"))
    if own:
        s["lib"] = _lib(b=b, h_q=c["h_q"], h_kv=c["h_kv"], d=c["d"], page_size=page, n_pages=n_pages, max_pages=table.shape[1], dtype=t,
                        len_bound=c["hi"])
    return s


def _prepare_select(c, g):
    b, h_kv, page = c["b"], c["h_kv"], c["page"]
    table = -(-c["hi"] // page)
    # scores of pages lie close together, and some are equal
    score = torch.randn((b, h_kv, table), generator=g, device="cuda").mul_(2).add_(20).mul_(256).round_().div_(256)
    s = dict(case=c, score=score, cache_len=_int(_lengths(c["lo"], c["hi"], b)), sel=_int([0]).expand(b, h_kv, c["n_sel"]).contiguous(),
             sel_cnt=_int([0]).expand(b, h_kv).contiguous())
    if own:
        s["lib"] = _lib(b=b, h_q=h_kv, h_kv=h_kv, d=64, page_size=page, n_pages=1, max_pages=table, dtype=torch.bfloat16, len_bound=c["hi"])
    return s


def _prepare_attend(c, g):
    t, b, h_kv, page = DTYPES[c["dtype"]], c["b"], c["h_kv"], c["page"]
    lens = _lengths(c["lo"], c["hi"], b)
    table, n_pages = _tables(lens, page, g)
    # the selected pages: the first, the last, and others anywhere
    n = ((_int(lens) + page - 1) // page)[:, None, None]
    j = torch.arange(table.shape[1], device="cuda")
    chance = torch.rand((b, h_kv, table.shape[1]), generator=g, device="cuda")
    chance = torch.where(j < n, chance + 2.0 * (j == n - 1) + 1.0 * (j == 0), -1)
    sel = torch.topk(chance, c["n_sel"], -1).indices
    sel = torch.sort(torch.where(sel < n, sel, table.shape[1]), dim=-1).values
    s = dict(case=c, q=torch.randn((b, c["h_q"], c["d"]), generator=g, device="cuda").mul_(1.3).to(t), block_table=table,
             cache_len=_int(lens), sel=torch.where(sel < n, sel, -1).to(torch.int32),
             sel_cnt=n.clamp(max=c["n_sel"])[:, :, 0].expand(b, h_kv).to(torch.int32).contiguous(),
             out=torch.zeros((b, c["h_q"], c["d"]), dtype=t, device="cuda"), lse=torch.zeros((b, c["h_q"]), device="cuda"),
             **_pool(c, n_pages, g, "k"), **_pool(c, n_pages, g, "v"))
    if own:
        s["lib"] = _lib(b=b, h_q=c["h_q"], h_kv=h_kv, d=c["d"], page_size=page, n_pages=n_pages, max_pages=table.shape[1], dtype=t,
                        len_bound=c["hi"], int8=c["int8"])
    return s


def _prepare_shared(c, g):
    t, b, m, page = DTYPES[c["dtype"]], c["b"], c["prefixes"], c["page"]
    lens = _all_lengths(c)
    table, n_pages = _tables(lens, page, g)
    of = [i * 7 % 11 % m for i in range(b)]
    s = dict(case=c, q=torch.randn((b, c["h_q"], c["d"]), generator=g, device="cuda").mul_(1.3).to(t), block_table=table, cache_len=_int(lens),
             prefix_of=_int([-1] * m + of), row_start=_int([0] * m + list(range(b + 1))),
             out=torch.zeros((b, c["h_q"], c["d"]), dtype=t, device="cuda"), lse=torch.zeros((b, c["h_q"]), device="cuda"),
             **_pool(c, n_pages, g, "k"), **_pool(c, n_pages, g, "v"))
    if own:
        s["lib"] = _lib(b=m + b, h_q=c["h_q"], h_kv=c["h_kv"], d=c["d"], page_size=page, n_pages=n_pages, max_pages=table.shape[1], dtype=t,
                        len_bound=max(lens), int8=c["int8"])
    return s


def run(state):
    return {"bounds": _run_bounds, "score": _run_score, "select": _run_select, "attend": _run_attend, "shared": _run_shared}[state["case"]["op"]](state)


def _run_bounds(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_bounds(p, s["rows"], s["slot"], s["k_pages"], s["k_scale"], s["bounds"], ws)
        return s["bounds"]
    n, page = s["bounds"].shape[0], c["page"]
    slot = s["slot"].long()
    at = torch.where(slot >= 0, slot, n * page)              # rows that have no slot count for a page behind the pool
    of, off = at // page, at % page
    inside = of.clamp(max=n - 1)
    key = s["k_pages"][inside, :, off].float()               # [rows, h_kv, d]
    if c["int8"]:
        key = key * s["k_scale"][inside, :, off][..., None]
    old = torch.cat([s["bounds"], s["bounds"][:1]]).float()
    fresh = torch.where(off == 0, of, n)
    low = old[:, :, 0].index_fill(0, fresh, math.inf).index_reduce(0, of, key, "amin")
    high = old[:, :, 1].index_fill(0, fresh, -math.inf).index_reduce(0, of, key, "amax")
    s["bounds"].copy_(torch.stack([low, high], 2)[:n])
    return s["bounds"]


def _run_score(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_score(p, s["q"], c["b"], None, None, s["bounds"], s["block_table"], s["cache_len"], s["score"], ws)
        return s["score"]
    b, h_kv, d = c["b"], c["h_kv"], c["d"]
    got = s["bounds"][s["block_table"].clamp(min=0).long()].float().transpose(1, 2)     # [b, h_kv, pages, 2, d]
    q = s["q"].float().view(b, h_kv, -1, d)
    both = torch.cat([q.clamp(max=0), q.clamp(min=0)], -1)
    bound = torch.matmul(got.reshape(b, h_kv, -1, 2 * d), both.transpose(2, 3)) * d ** -0.5
    j = torch.arange(bound.shape[2], device=bound.device)
    held = (s["cache_len"] + c["page"] - 1) // c["page"]
    s["score"].copy_(torch.where(j < held[:, None, None], bound.amax(-1), s["score"]))
    return s["score"]


def _run_select(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_select(p, s["score"], s["cache_len"], c["n_sel"], c["first"], c["last"], s["sel"], s["sel_cnt"], ws)
        return [s["sel"], s["sel_cnt"]]
    score, n_sel = s["score"], c["n_sel"]
    n = ((s["cache_len"] + c["page"] - 1) // c["page"])[:, None, None]
    j = torch.arange(score.shape[2], device=score.device)
    always = (j < c["first"]) | (j >= n - c["last"])
    rank = torch.where(j < n, torch.where(always, math.inf, score), -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :n_sel]
    best = torch.sort(torch.where(best < n, best, score.shape[2]), dim=-1).values
    sel = torch.where(best < n, best, -1).to(torch.int32)
    return [sel, n.clamp(max=n_sel)[:, :, 0].expand(-1, score.shape[1]).to(torch.int32)]


def _attention(q, keys, values, live):
    """(sum of weighted values, top logit, sum of weights) of q [.., rows, d] over keys [.., n, d], where live."""
    logits = torch.where(live, torch.matmul(q, keys.transpose(-1, -2)), -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(logits - top)
    return torch.matmul(p, values), top, p.sum(-1, keepdim=True)


def _run_attend(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_decode_selected(p, s["q"], c["b"], None, None, s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["block_table"],
                                    s["cache_len"], s["sel"], s["sel_cnt"], c["n_sel"], s["out"], s["lse"], ws)
        return [s["out"], s["lse"]]
    b, h_kv, d, page = c["b"], c["h_kv"], c["d"], c["page"]
    sel = s["sel"].clamp(min=0).long()
    where = s["block_table"].long()[torch.arange(b, device=sel.device)[:, None, None], sel].clamp(min=0)
    head = torch.arange(h_kv, device=sel.device)[:, None]

    def rows(x):                                             # [b, h_kv, tokens, d]
        got = s[x + "_pages"][where, head].float()
        if c["int8"]:
            got = got * s[x + "_scale"][where, head][..., None]
        return got.reshape(b, h_kv, -1, d)
    t = sel[..., None] * page + torch.arange(page, device=sel.device)
    live = (t < s["cache_len"][:, None, None, None]) & (s["sel"] >= 0)[..., None]
    q = s["q"].float().view(b, h_kv, -1, d) * d ** -0.5
    out, top, total = _attention(q, rows("k"), rows("v"), live.reshape(b, h_kv, 1, -1))
    return [(out / total).reshape(b, -1, d).to(s["q"].dtype), (top + torch.log(total)).reshape(b, -1)]


def _run_shared(s):
    c = s["case"]
    b, m, h_kv, d, page = c["b"], c["prefixes"], c["h_kv"], c["d"], c["page"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_decode_shared(p, s["q"], b, s["row_start"], None, s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["block_table"],
                                  s["cache_len"], s["prefix_of"], s["out"], s["lse"], ws)
        return [s["out"], s["lse"]]

    def rows(x, table):                                      # [sequences, h_kv, tokens, d]
        got = s[x + "_pages"][table].float()
        if c["int8"]:
            got = got * s[x + "_scale"][table][..., None]
        return got.transpose(1, 2).reshape(table.shape[0], h_kv, -1, d)

    def live(lens, width):
        return (torch.arange(width, device=lens.device) < lens[:, None])[:, None, None]
    # every query against every prefix, of which each takes its own
    q = s["q"].float().view(b, h_kv, -1, d) * d ** -0.5
    g = q.shape[2]
    wide = -(-c["phi"] // page)
    table = s["block_table"][:m, :wide].clamp(min=0).long()
    everyone = q.transpose(0, 1).reshape(1, h_kv, b * g, d)
    mine = s["prefix_of"][m:].long(), slice(None), torch.arange(b, device=q.device)
    theirs = [x.reshape(m, h_kv, b, g, -1)[mine] for x in
              _attention(everyone, rows("k", table), rows("v", table), live(s["cache_len"][:m], wide * page))]
    table = s["block_table"][m:, :max(1, -(-c["hi"] // page))].clamp(min=0).long()
    out, top, total = _attention(q, rows("k", table), rows("v", table), live(s["cache_len"][m:], table.shape[1] * page))
    most = torch.maximum(top, theirs[1])
    a, z = torch.exp(theirs[1] - most), torch.exp(top - most)
    total = a * theirs[2] + z * total
    out = (a * theirs[0] + z * out) / total
    return [out.reshape(b, -1, d).to(s["q"].dtype), (most + torch.log(total)).reshape(b, -1)]


def work(case):
    c = case
    page, b = c["page"], c["b"]
    if c["op"] == "select":
        pages = sum(-(-n // page) for n in _lengths(c["lo"], c["hi"], b))
        return {"bytes": 4 * c["h_kv"] * (pages + b * (c["n_sel"] + 1)) + 4 * b, "flops": 0}
    w, h_kv, d = BYTES[c["dtype"]], c["h_kv"], c["d"]
    row = d + 4 if c.get("int8") else d * w
    if c["op"] == "bounds":
        old, new = _lengths(c["lo"], c["hi"], b), _lengths(c["least"], c["most"], b)
        rows = sum(new)
        pages = sum(-(-(m + n) // page) - m // page for m, n in zip(old, new))
        begun = sum(m % page > 0 for m in old)               # whose bounds are read, too
        return {"bytes": h_kv * (rows * row + (pages + begun) * 2 * d * w) + 4 * rows, "flops": 2 * rows * h_kv * d}
    if c["op"] == "score":
        pages = sum(-(-n // page) for n in _lengths(c["lo"], c["hi"], b))
        return {"bytes": pages * (h_kv * (2 * d * w + 4) + 4) + b * (c["h_q"] * d * w + 4), "flops": 4 * pages * c["h_q"] * d}
    ends = b * c["h_q"] * (2 * d * w + 4)
    if c["op"] == "attend":
        keys = sum(_read(c))
        return {"bytes": h_kv * (2 * keys * row + 4 * b * (c["n_sel"] + 1) + 4 * (keys // page)) + ends, "flops": 4 * keys * c["h_q"] * d}
    lens, m = _all_lengths(c), c["prefixes"]
    behind = sum(lens[i * 7 % 11 % m] for i in range(b))     # prefix tokens that each sequence sees
    used = sum(lens[m:]) + sum(lens[i] for i in {i * 7 % 11 % m for i in range(b)})
    return {"bytes": 2 * used * h_kv * row + 4 * (used // page) + ends, "flops": 4 * (behind + sum(lens[m:])) * c["h_q"] * d}


def exact(case, seed):
    c = case
    if c["op"] == "select":
        return None                                          # whole numbers only
    s = prepare(case, seed)
    h_kv, d, page = c["h_kv"], c["d"], c["page"]
    if c["op"] == "bounds":
        got = s["bounds"].double()
        key = s["k_pages"].double()
        if c["int8"]:
            key = key * s["k_scale"].double()[..., None]
        seen = torch.zeros(key.shape[0] * page, dtype=torch.bool, device="cuda")
        seen[s["slot"][s["slot"] >= 0].long()] = True
        seen = seen.view(-1, page)
        low = torch.where(seen[:, None, :, None], key, math.inf).amin(2)
        high = torch.where(seen[:, None, :, None], key, -math.inf).amax(2)
        keep = (seen.any(1) & ~seen[:, 0])[:, None, None]    # pages that had tokens before
        low, high = (torch.where(keep, torch.minimum(low, got[:, :, 0]), low), torch.where(keep, torch.maximum(high, got[:, :, 1]), high))
        touched = seen.any(1)[:, None, None]
        return torch.stack([torch.where(touched, low, got[:, :, 0]), torch.where(touched, high, got[:, :, 1])], 2)
    lens = _all_lengths(c)
    if c["op"] == "score":
        out = s["score"].double()
        for i, n in enumerate(lens):
            pages = s["block_table"][i, :-(-n // page)].long()
            q = s["q"][i].double().view(h_kv, -1, d)
            for lo in range(0, len(pages), 512):
                box = s["bounds"][pages[lo:lo + 512]].double()                # [pages, h_kv, 2, d]
                ends = box[:, :, None] * q[None, :, :, None]                  # [pages, h_kv, heads, 2, d]
                out[i, :, lo:lo + len(box)] = (torch.maximum(ends[..., 0, :], ends[..., 1, :]).sum(-1) / math.sqrt(d)).amax(-1).t()
        return out
    m = c.get("prefixes", 0)
    if sum(lens[m:]) * h_kv * d > 1 << 32 or (m and sum(lens[i * 7 % 11 % m] for i in range(c["b"])) * h_kv * d > 1 << 33):
        return None

    def tokens(i, at):                                       # [h_kv, tokens, d] of keys and of values; at [h_kv, tokens]
        page_no = s["block_table"][i].long()[at // page]
        head = torch.arange(h_kv, device="cuda")[:, None]
        got = [s[x + "_pages"][page_no, head, at % page].double() for x in "kv"]
        return [r * s[x + "_scale"][page_no, head, at % page].double()[..., None] for x, r in zip("kv", got)] if c["int8"] else got
    outs, sums = [], []
    for i, n in enumerate(lens[m:]):
        if c["op"] == "attend":
            at = s["sel"][i][:, :int(s["sel_cnt"][i, 0])].long()[..., None] * page + torch.arange(page, device="cuda")
            at = at.flatten(1)
            k, v = tokens(i, at[at < n].view(h_kv, -1))
        else:
            k, v = [torch.cat(two, 1) for two in zip(*[tokens(of, torch.arange(have, device="cuda").expand(h_kv, have)) for of, have in
                                                       ((int(s["prefix_of"][m + i]), lens[int(s["prefix_of"][m + i])]), (m + i, n))])]
        q = s["q"][i].double().view(h_kv, -1, d)
        logits = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        sums.append(torch.logsumexp(logits, -1).flatten())
        outs.append(torch.bmm(torch.softmax(logits, -1), v.contiguous()).reshape(-1, d))
    return [torch.stack(outs), torch.stack(sums)]
