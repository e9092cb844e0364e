"""Cases of the paged cache: its plan, the rows that are appended to it, and the attention of new tokens over it.

Three operators, each also in a plain form of elementary torch operations:

  plan     swa_paged_plan: block tables, slots and positions of a call's packed rows, from request lengths.
  append   swa_paged_append: norm of queries and keys, rotation by position, keys and values into their slots.
  decode   swa_paged_decode: attention of each sequence's newest token over its pages.

Lengths are spread evenly over lo..hi (the same for every seed, so that the work is), in a mixed order; values, pages and
their order come from the seed.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    def plan(name, b, page, table, lo, hi, new, least, most, gone):
        # b sequences of lo..hi tokens; every `new`-th gets least..most tokens; every `gone`-th (0: none) has finished
        return dict(name=name, op="plan", b=b, page=page, table=table, lo=lo, hi=hi, new=new, least=least, most=most, gone=gone)

    def append(name, rows, pad, h_q, h_kv, d, dtype, page, far, rot, axes, interleaved, norm, int8):
        return dict(name=name, op="append", rows=rows, pad=pad, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, far=far,
                    rot=rot, axes=axes, interleaved=interleaved, norm=norm, int8=int8)

    def decode(name, b, h_q, h_kv, d, dtype, page, lo, hi, window, int8):
        return dict(name=name, op="decode", b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi, window=window,
                    int8=int8)

    return [
        # the steady state of a server: one new token for every sequence of a full batch
        plan("plan_step", 256, 16, 512, 40, 8000, 1, 1, 1, 0),
        # a thousand sequences, a quarter of them with a prompt's piece, one in twenty finished
        plan("plan_mixed", 1024, 16, 1024, 1, 9000, 4, 1, 600, 20),
        # one step of a batch far into its contexts: latency counts
        append("append_step", 64, 0, 32, 8, 128, "bf16", 16, 500000, 128, 1, False, True, False),
        # several prompts packed into one call, with the unused rows of a fixed-size batch behind them
        append("append_prompts", 8192, 64, 32, 8, 128, "bf16", 16, 4000, 128, 1, False, True, False),
        # a video's tokens: time, height and width have their own positions
        append("append_video", 4097, 0, 28, 4, 128, "f16", 32, 20000, 128, 3, False, False, False),
        # a 32-head model in fp32 that rotates half of its channels, neighbours in pairs
        append("append_partial_f32", 1001, 7, 32, 32, 64, "f32", 24, 2000, 32, 1, True, False, False),
        # a long prompt into the compressed cache
        append("append_int8", 8191, 0, 64, 8, 128, "f16", 64, 9000, 128, 1, False, True, True),
        # one chat turn: latency counts
        decode("decode_one", 1, 32, 8, 128, "bf16", 16, 1031, 1031, 0, False),
        # a full serving batch of mixed lengths
        decode("decode_batch", 128, 32, 8, 128, "bf16", 16, 512, 8192, 0, False),
        # one long context with many query heads to a key head
        decode("decode_long", 1, 64, 4, 128, "f16", 64, 131071, 131071, 0, False),
        # the compressed cache
        decode("decode_int8", 64, 32, 8, 128, "f16", 32, 100, 8001, 0, True),
        # 32 heads of their own in fp32, a local window, pages of an odd size
        decode("decode_window_f32", 16, 32, 32, 64, "f32", 20, 1, 1090, 512, False),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("plan", "append", "append", "decode", "decode", "decode"))
    if op == "plan":
        page, hi = rng.choice((1, 16, 16, 24, 64, 128)), spread(16, 16000)
        most = rng.choice((1, spread(1, 800)))
        return dict(op=op, b=spread(1, 1024), page=page, table=-(-(hi + most) // page) + rng.randrange(3), lo=rng.choice((0, 1, hi // 3)),
                    hi=hi, new=rng.randrange(1, 6), least=1, most=most, gone=rng.choice((0, 0, 7, 30)))
    d, dtype = rng.choice((64, 128, 128)), rng.choice(("f32", "f16", "bf16", "bf16"))
    h_q, h_kv = rng.choice(((32, 32), (40, 40), (12, 12), (32, 8), (28, 4), (64, 8), (16, 1), (25, 5)))
    int8 = dtype != "f32" and rng.random() < 0.25
    if op == "append":
        rows = spread(1, 8192)
        while rows * (h_q + 2 * h_kv) * d * BYTES[dtype] > 8192 * 80 * 128 * 2:
            rows = rows * 2 // 3
        axes = rng.choice((1, 1, 2, 3))
        return dict(op=op, rows=rows, pad=rng.choice((0, rng.randrange(1, 65))), h_q=h_q, h_kv=h_kv, d=d, dtype=dtype,
                    page=rng.choice((1, 16, 24, 32, 64)), far=spread(1000, 1000000), rot=rng.choice((d, d, d // 2)), axes=axes,
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.5, int8=int8)
    hi = spread(1, 131072)
    lo = rng.choice((hi, max(1, hi // 4), 1))
    b = spread(1, 256)
    while (b > 1 or hi > 1) and b * (lo + hi) / 2 * h_kv * d * (1 if int8 else BYTES[dtype]) > 128 * 4352 * 8 * 128 * 2:
        if b > 1:
            b = b * 2 // 3
        else:
            hi = hi * 2 // 3
            lo = min(lo, hi)
    page = rng.choice((1, 16, 16, 20, 32, 64, 128))
    return dict(op=op, b=b, h_q=h_q, h_kv=h_kv, d=d, dtype=dtype, page=page, lo=lo, hi=hi,
                window=rng.choice((0, 0, 0, spread(1, hi))), int8=int8)


def _lengths(lo, hi, n):
    """n lengths, evenly over lo..hi, in a mixed order."""
    even = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    step = next(k for k in (61, 67, 71, 73) if n % k)
    return [even[i * step % n] for i in range(n)]


def _counts(c):
    """Tokens that each sequence of a plan brings: -1 where it has finished."""
    most = _lengths(c["least"], c["most"], c["b"])
    return [-1 if c["gone"] and i % c["gone"] == 2 else most[i] if i % c["new"] == 0 else 0 for i in range(c["b"])]


def _sections(c):
    """Rotated pairs of each axis."""
    pairs = c["rot"] // 2
    return {1: [pairs], 2: [pairs // 2, pairs - pairs // 2], 3: [pairs // 4, 3 * pairs // 8, pairs - pairs // 4 - 3 * pairs // 8]}[c["axes"]]


def _params(c, **more):
    from paper_2403_17312_amd import binding as B
    p = B.make_paged_params(**more)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    return B, p, ws


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"plan": _prepare_plan, "append": _prepare_append, "decode": _prepare_decode}[case["op"]](case, g)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_plan(c, g):
    b, page, table = c["b"], c["page"], c["table"]
    lens, counts = _lengths(c["lo"], c["hi"], b), _counts(c)
    held = [-(-m // page) for m in lens]
    fresh = sum(-(-(m + n) // page) - h for m, n, h in zip(lens, counts, held) if n > 0)
    n_pages = sum(held) + fresh + 8
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    h = _int(held)
    first = torch.cumsum(h, 0) - h
    j = torch.arange(table, device="cuda")
    at = (first[:, None] + j).clamp(max=n_pages - 1)
    tables = torch.where(j < h[:, None], order[at], -1).to(torch.int32)
    head = int(torch.randint(n_pages, (1,), generator=g, device="cuda"))
    ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free = order[sum(held):]
    ring[(head + torch.arange(free.numel(), device="cuda")) % n_pages] = free
    rows = sum(n for n in counts if n > 0)
    new = dict(new_len=_int([0] * b), free_state_out=_int([0, 0]), row_start=_int([0] * (b + 1)), slot=_int([0] * (rows + 5)),
               pos=_int([0] * (rows + 5)))
    s = dict(case=c, new_cnt=_int(counts), cache_len=_int(lens), block_table=tables, free_ring=ring, free_state=_int([head, free.numel()]),
             rows=rows + 5, n_pages=n_pages, **new)
    if own:
        s["lib"] = _params(c, b=b, h_q=1, h_kv=1, d=64, page_size=page, n_pages=n_pages, max_pages=table, dtype=torch.bfloat16)
    return s


def _prepare_append(c, g):
    t, n, d, page = DTYPES[c["dtype"]], c["rows"] + c["pad"], c["d"], c["page"]
    h_q, h_kv = c["h_q"], c["h_kv"]
    n_pages = -(-c["rows"] // page) + 3

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    # one projection holds a row's queries, keys and values
    qkv = normal(n, h_q + 2 * h_kv, d).mul_(1.5).to(t)
    pages = torch.randperm(n_pages, generator=g, device="cuda")
    r = torch.arange(n, device="cuda")
    slot = torch.where(r < c["rows"], pages[(r // page).clamp(max=n_pages - 1)] * page + r % page, -1).to(torch.int32)
    first = torch.randint(0, c["far"], (c["axes"], 1), generator=g, device="cuda")
    pos = first + torch.stack([r, r // 7 % 31, r % 43])[:c["axes"]]
    s = dict(case=c, q=qkv[:, :h_q], k=qkv[:, h_q:h_q + h_kv], v=qkv[:, h_q + h_kv:], n=n, pos=pos.to(torch.int32), slot=slot,
             inv_freq=10000.0 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float32) * 2 / c["rot"]),
             axis=torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda")),
             q_out=torch.zeros((n, h_q, d), dtype=t, device="cuda"), q_weight=None, k_weight=None, k_scale=None, v_scale=None)
    if c["norm"]:
        s["q_weight"], s["k_weight"] = (1 + 0.2 * normal(d)).to(t), (1 + 0.2 * normal(d)).to(t)
    shape = (n_pages, h_kv, page, d)
    if c["int8"]:
        for x in "kv":
            s[x + "_pages"] = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
            s[x + "_scale"] = normal(*shape[:3]).abs_().mul_(0.02)
            s[x + "_values"] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    else:
        s["k_pages"], s["v_pages"] = normal(*shape).to(t), normal(*shape).to(t)
    if own:
        from paper_2403_17312_amd import binding as B
        s["lib"] = _params(c, b=1, h_q=h_q, h_kv=h_kv, d=d, page_size=page, n_pages=n_pages, max_pages=n_pages, dtype=t, eps=1e-6,
                           flags=(B.SWA_KV_INT8 if c["int8"] else 0) | (B.SWA_ROPE_INTERLEAVED if c["interleaved"] else 0),
                           rot_dim=c["rot"], sections=_sections(c))
    return s


def _prepare_decode(c, g):
    t, b, d, page = DTYPES[c["dtype"]], c["b"], c["d"], c["page"]
    h_q, h_kv = c["h_q"], c["h_kv"]
    lens = _lengths(c["lo"], c["hi"], b)
    held = [-(-m // page) for m in lens]
    n_pages, table = sum(held) + 2, max(held)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    h = _int(held)
    first = torch.cumsum(h, 0) - h
    j = torch.arange(table, device="cuda")
    tables = torch.where(j < h[:, None], order[(first[:, None] + j).clamp(max=n_pages - 1)], -1).to(torch.int32)
    shape = (n_pages, h_kv, page, d)
    s = dict(case=c, q=torch.randn((b, h_q, d), generator=g, device="cuda").mul_(1.3).to(t), block_table=tables, cache_len=_int(lens),
             k_scale=None, v_scale=None, out=torch.zeros((b, h_q, d), dtype=t, device="cuda"),
             lse=torch.zeros((b, h_q), device="cuda"))
    for x in "kv":
        if c["int8"]:
            s[x + "_pages"] = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
            s[x + "_scale"] = torch.rand(shape[:3], generator=g, device="cuda").mul_(0.02).add_(0.005)
        else:
            s[x + "_pages"] = torch.empty(shape, dtype=t, device="cuda").normal_(generator=g)
    if own:
        from paper_2403_17312_amd import binding as B
        s["lib"] = _params(c, b=b, h_q=h_q, h_kv=h_kv, d=d, page_size=page, n_pages=n_pages, max_pages=table, dtype=t,
                           window=c["window"], len_bound=c["hi"], flags=B.SWA_KV_INT8 if c["int8"] else 0)
    return s


def run(state):
    return {"plan": _run_plan, "append": _run_append, "decode": _run_decode}[state["case"]["op"]](state)


def _run_plan(s):
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_plan(p, s["new_cnt"], s["cache_len"], s["new_len"], s["block_table"], s["free_ring"], s["free_state"],
                         s["free_state_out"], s["rows"], s["row_start"], s["slot"], s["pos"], ws)
        return [s[x] for x in ("new_len", "block_table", "free_ring", "free_state_out", "row_start", "slot", "pos")]
    page, table, ring, n = s["case"]["page"], s["block_table"], s["free_ring"], s["n_pages"]
    c, m = s["new_cnt"].long(), s["cache_len"].long()
    head, free = s["free_state"].long()
    rows = c.clamp(min=0)
    end = torch.cumsum(rows, 0)
    held = (m + page - 1) // page
    fits = (c >= 0) & (m + rows <= table.shape[1] * page) & (end <= s["rows"])
    need = torch.where(fits, (m + rows + page - 1) // page - held, 0)
    taken = torch.cumsum(need, 0)
    ok = fits & ((need == 0) | (taken <= free))
    got = torch.where(ok, need, 0)
    new_len = torch.where(c < 0, 0, torch.where(ok, m + rows, m))
    j = torch.arange(table.shape[1], device=table.device)
    fresh = (j >= held[:, None]) & (j < (held + got)[:, None])
    new_table = torch.where(fresh, ring[(head + (taken - need)[:, None] + j - held[:, None]) % n], table)
    back = torch.where(c < 0, held, 0)
    first = torch.cumsum(back, 0) - back
    put = torch.where(j < back[:, None], (head + free + first[:, None] + j) % n, n)
    new_ring = torch.cat([ring, ring[:1]]).scatter(0, put.flatten(), table.flatten())[:n]
    state = torch.stack([(head + got.sum()) % n, free - got.sum() + back.sum()])
    r = torch.arange(s["rows"], device=table.device)
    of = torch.searchsorted(end, r, right=True).clamp(max=len(c) - 1)
    at = m[of] + r - (end - rows)[of]
    used = (r < end[-1]) & ok[of]
    at = torch.where(used, at, 0)
    slot = torch.where(used, new_table[of, at // page] * page + at % page, -1)
    row_start = torch.cat([torch.zeros_like(end[:1]), end])
    return [x.to(torch.int32) for x in (new_len, new_table, new_ring, state, row_start, slot, at)]


def _rotated(x, weight, s, cos, sin):
    """Norm and rotation of [rows, heads, d], in the type of cos."""
    c = s["case"]
    x = x.to(cos.dtype)
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.to(cos.dtype)
    turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    if c["interleaved"]:
        a, z = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - z * sin, z * cos + a * sin], -1).flatten(-2)
    else:
        a, z = turned.chunk(2, -1)
        turned = torch.cat([a * cos - z * sin, z * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _run_append(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_append(p, s["q"], s["k"], s["v"], s["n"], s["pos"], s["slot"], s["inv_freq"], s["q_weight"], s["k_weight"], s["q_out"],
                           s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], ws)
    else:
        angle = s["pos"][s["axis"]].t().double() * s["inv_freq"].double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        used = s["slot"] >= 0
        q = _rotated(s["q"], s["q_weight"], s, cos, sin).to(s["q_out"].dtype)
        torch.where(used[:, None, None], q, s["q_out"], out=s["q_out"])
        at = s["slot"][used].long()
        page, off = at // c["page"], at % c["page"]
        for x, new in (("k", _rotated(s["k"], s["k_weight"], s, cos, sin)), ("v", s["v"].float())):
            new = new[used]
            if c["int8"]:
                scale = new.abs().amax(-1) / 127
                s[x + "_scale"][page, :, off] = scale
                new = torch.where(scale[..., None] > 0, torch.round(new / scale[..., None]), 0)
            s[x + "_pages"][page, :, off] = new.to(s[x + "_pages"].dtype)
    if not c["int8"]:
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    # 8-bit codes: the values that they stand for
    for x in "kv":
        torch.mul(s[x + "_pages"], s[x + "_scale"][..., None], out=s[x + "_values"])
    return [s["q_out"], s["k_values"], s["v_values"]]


def _run_decode(s):
    c = s["case"]
    if own:
        B, p, ws = s["lib"]
        B.swa_paged_decode(p, s["q"], c["b"], None, s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["block_table"], s["cache_len"],
                           s["out"], s["lse"], ws)
        return [s["out"], s["lse"]]
    b, h_kv, d = c["b"], c["h_kv"], c["d"]
    table = s["block_table"].clamp(min=0).long()

    def rows(x):                                             # [b, h_kv, keys, d]
        got = s[x + "_pages"][table].float()
        if c["int8"]:
            got = got * s[x + "_scale"][table][..., None]
        return got.transpose(1, 2).reshape(b, h_kv, -1, d)
    q = s["q"].float().view(b, h_kv, -1, d) * d ** -0.5
    logits = torch.matmul(q, rows("k").transpose(2, 3))
    i = torch.arange(logits.shape[-1], device=table.device)
    n = s["cache_len"][:, None]
    live = (i < n) & (i >= (n - c["window"] if c["window"] else torch.zeros_like(n)))
    logits = torch.where(live[:, None, None], logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, rows("v")) / total
    lse = top + torch.log(total)
    return [out.reshape(b, -1, d).to(s["q"].dtype), lse.reshape(b, -1)]


def work(case):
    c = case
    if c["op"] == "plan":
        lens, counts = _lengths(c["lo"], c["hi"], c["b"]), _counts(c)
        rows = sum(n for n in counts if n > 0)
        pages = sum(-(-(m + n) // c["page"]) - -(-m // c["page"]) if n > 0 else -(-m // c["page"]) if n < 0 else 0 for m, n in zip(lens, counts))
        return {"bytes": 4 * (4 * c["b"] + 2 * (rows + 5) + 2 * pages), "flops": 0}
    w = BYTES[c["dtype"]]
    if c["op"] == "append":
        n, h_q, h_kv, d = c["rows"], c["h_q"], c["h_kv"], c["d"]
        kv = 2 * h_kv * (d + 4) if c["int8"] else 2 * h_kv * d * w
        values = 2 * (-(-n // c["page"]) + 3) * c["page"] * h_kv * (3 * d + 4) if c["int8"] else 0    # the codes' values, as returned
        return {"bytes": n * ((2 * h_q + 2 * h_kv) * d * w + kv + 4 * (1 + c["axes"])) + values, "flops": n * (h_q + h_kv) * d * (7 if c["norm"] else 3)}
    keys = sum(min(m, c["window"] or m) for m in _lengths(c["lo"], c["hi"], c["b"]))
    row = c["h_kv"] * (c["d"] + 4 if c["int8"] else c["d"] * w)
    return {"bytes": 2 * keys * row + 2 * c["b"] * c["h_q"] * c["d"] * w + 4 * c["b"] * c["h_q"] + 4 * (keys // c["page"]),
            "flops": 4 * keys * c["h_q"] * c["d"]}


def exact(case, seed):
    c = case
    if c["op"] == "plan":
        return None                                          # whole numbers only
    s = prepare(case, seed)
    if c["op"] == "append":
        # a pair of channels is a complex number, and the rotation a product with exp(i angle)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[s["axis"]].t() * s["inv_freq"].double())[:, None]

        def rotated(x, weight):
            x = x.double()
            if weight is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + 1e-6).sqrt() * weight.double()
            y, half = x.clone(), c["rot"] // 2
            first = slice(0, c["rot"], 2) if c["interleaved"] else slice(0, half)
            second = slice(1, c["rot"], 2) if c["interleaved"] else slice(half, c["rot"])
            z = torch.complex(x[..., first], x[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y
        used = s["slot"] >= 0
        at = s["slot"][used].long()
        q = s["q_out"].double()
        q[used] = rotated(s["q"], s["q_weight"])[used]
        out = [q]
        for x, new in (("k", rotated(s["k"], s["k_weight"])), ("v", s["v"].double())):
            old = s[x + "_pages"].double()
            if c["int8"]:
                old = old * s[x + "_scale"].double()[..., None]
                step = new.abs().amax(-1, keepdim=True) / 127
                new = torch.round(new / step) * step         # (no row of these inputs is all zero)
            old[at // c["page"], :, at % c["page"]] = new[used]
            out.append(old)
        return out
    b, h_kv, d, g = c["b"], c["h_kv"], c["d"], c["h_q"] // c["h_kv"]
    if b * c["hi"] * h_kv * d > 1 << 32:
        return None
    outs, sums = [], []
    for i, n in enumerate(_lengths(c["lo"], c["hi"], b)):
        at = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device="cuda")
        page, off = s["block_table"][i].long()[at // c["page"]], at % c["page"]
        k, v = (s[x + "_pages"][page, :, off].double() for x in "kv")     # [keys, h_kv, d]
        if c["int8"]:
            k, v = (r * s[x + "_scale"][page, :, off].double()[..., None] for x, r in (("k", k), ("v", v)))
        q = s["q"][i].double().view(h_kv, g, d)
        logits = torch.bmm(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(d)
        sums.append(torch.logsumexp(logits, -1).flatten())
        outs.append(torch.bmm(torch.softmax(logits, -1), v.transpose(0, 1).contiguous()).reshape(-1, d))
    return [torch.stack(outs), torch.stack(sums)]
