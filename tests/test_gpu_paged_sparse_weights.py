"""The weights of the attentions over lists of pages and behind shared prefixes: in every form no rounding of theirs shows in an output that is small beside its values,
and tokens that one token drowns out reach the output."""
import pytest
import torch

import paged_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# A weight goes as two numbers of the type: its leading bits, cut off, and the rest, rounded.  bf16 has 8 bits, so the rest is below 2^-7 of the weight and half a step of it
# 2^-8 of that; fp16 11, 2^-10 and 2^-11.
STEP = {torch.bfloat16: 2.0 ** -15, torch.float16: 2.0 ** -21}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """Sequences of these lengths with normal queries, keys and values, on the CPU."""

    def __init__(self, lens, h_q, h_kv, d, dtype, page, seed=0):
        g, held = torch.Generator().manual_seed(seed), [-(-m // page) for m in lens]
        order, at = torch.randperm(sum(held), generator=g).int(), 0
        self.lens, self.held, self.page, self.dtype = lens, held, page, dtype
        self.table = torch.zeros((len(lens), max(held)), dtype=torch.int32)
        for s, n in enumerate(held):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.k, self.v = (torch.randn((sum(held), h_kv, page, d), generator=g).to(dtype) for _ in "kv")
        self.q = torch.randn((len(lens), h_q, d), generator=g).to(dtype)

    def put(self, x, s, rows):
        """Rows [tokens, h_kv, d] of a sequence into a pool."""
        t = torch.arange(rows.shape[0])
        x[self.table[s].long()[t // self.page], :, t % self.page] = rows.to(self.dtype)

    def rows(self, x, s):
        return R.gather(x, None, self.table[s], self.page, 0, self.lens[s])

    def run(self, B, prefix_of):
        """Behind prefixes, or (prefix_of None) over lists of all pages: outputs and logarithms, in float64."""
        b, (n_pages, h_kv, page, d), h_q = len(self.lens), self.k.shape, self.q.shape[1]
        p = B.make_paged_params(b, h_q, h_kv, d, page, n_pages, self.table.shape[1], self.dtype)
        ws = torch.full((B.swa_paged_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
        B.swa_paged_workspace_init(p, ws)
        out, lse = torch.zeros((b, h_q, d), dtype=self.dtype, device="cuda"), torch.zeros((b, h_q), device="cuda")
        args = (p, self.q.cuda(), b, None, None, self.k.cuda(), self.v.cuda(), None, None, self.table.cuda(), ints(self.lens))
        if prefix_of is None:
            n_sel = self.table.shape[1]
            sel = ints([[list(range(n)) + [-1] * (n_sel - n)] * h_kv for n in self.held])
            B.swa_paged_decode_selected(*args, sel, ints([[n] * h_kv for n in self.held]), n_sel, out, lse, ws)
        else:
            B.swa_paged_decode_shared(*args, ints(prefix_of), out, lse, ws)
        assert B.swa_paged_check_status(p, ws) == B.SWA_OK
        return out.cpu().double(), lse.cpu().double()

    def check(self, B, prefix_of, which=None):
        out, lse = self.run(B, prefix_of)
        h_q, h_kv, d = self.q.shape[1], self.k.shape[1], self.q.shape[2]
        for s in which or range(len(self.lens)):
            of = prefix_of[s] if prefix_of else -1
            kk, vv = (torch.cat([self.rows(x, of), self.rows(x, s)]) if of >= 0 else self.rows(x, s) for x in (self.k, self.v))
            want, want_lse, tol, lse_tol = R.attention(self.q[s].double(), kk, vv, d ** -0.5, torch.float32, STEP[self.dtype])
            tol = tol + R.half_step(self.dtype) * want.abs()
            if self.dtype == torch.float16:
                # (the output's smallest numbers; and a rest of less than 2^-24 counts as that, 2^-39 of the largest weight)
                tol = tol + 2.0 ** -25 + 2.0 ** -39 * vv.abs().sum(0).repeat_interleave(h_q // h_kv, 0)
            over = float(((out[s] - want).abs() / tol).max())
            assert over <= 1, (s, self.lens[s], over)
            assert ((lse[s] - want_lse).abs() <= lse_tol).all(), s


OWN = [5, 40, 17, 1, 33]
# lengths, query and key heads, page, and the prefix of all but the first (None: lists)
FORMS = {"lists": ([300, 1, 17, 999, 5000], 8, 2, 16, None), "lists, 32 heads": ([400, 33], 24, 1, 16, None), "lists, short": ([30, 9, 100] * 90, 4, 4, 8, None),
         "16 columns": ([700, 5, 40], 8, 2, 16, 0), "32 columns": ([2000] + OWN + [300, 2, 3], 8, 2, 16, 0), "one head": ([900, 5, 1], 1, 1, 5, 0),
         "many columns": ([3000] + OWN * 4, 8, 2, 16, 0), "a few more than 32": ([130] + OWN + [20] * 4, 8, 2, 8, 0), "many columns, odd pages": ([1000] + OWN * 4, 8, 2, 20, 0)}


def make(form, d, dtype, seed=0):
    lens, h_q, h_kv, page, of = FORMS[form]
    return Cache(lens, h_q, h_kv, d, dtype, page, seed), None if of is None else [-1] + [of] * (len(lens) - 1)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_outputs_are_rounded_once(B, form, dtype, d):
    cache, prefix_of = make(form, d, TYPES[dtype])
    cache.check(B, prefix_of)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_others_of_the_cache_change_no_rounding(B, dtype):
    """The same requests with room for many more beside them: both results within what weights of two numbers leave."""
    lens, h_q, h_kv, d = [1500, 30, 7], 8, 2, 64
    for more in (0, 40):
        cache = Cache(lens + [0] * more, h_q, h_kv, d, TYPES[dtype], 16)
        cache.check(B, [-1, 0, 0] + [-1] * more, range(3))


@pytest.mark.parametrize("form", ["lists", "16 columns", "32 columns", "many columns", "many columns, odd pages"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("gap", [12.0, 17.4, 24.0])
@pytest.mark.parametrize("at", [0, 19999])
def test_quiet_tokens_beside_a_loud_one_without_value(B, form, dtype, gap, at):
    """Token `at` of the first sequence, a prefix where there are any, is `gap` louder than its others, for all query heads but the last, and its value is 0."""
    _, h_q, h_kv, page, of = FORMS[form]
    d, n, dt = 64, 20000, TYPES[dtype]
    lens = [n] + FORMS[form][0][1:]
    cache = Cache(lens, h_q, h_kv, d, dt, page, 3)
    g, scale = torch.Generator().manual_seed(9), d ** -0.5
    one = torch.randn(d, generator=g)
    cache.q[:, :-1] = (one + 0.05 * torch.randn((len(lens), h_q - 1, d), generator=g)).to(dt)
    k, v = 0.02 * torch.randn((n, h_kv, d), generator=g), 1 + 0.1 * torch.randn((n, h_kv, d), generator=g)
    k[at], v[at] = one * (gap / (one.square().sum() * scale)), 0
    cache.put(cache.k, 0, k)
    cache.put(cache.v, 0, v)
    for s in range(1, len(lens)):
        cache.put(cache.k, s, 0.02 * torch.randn((lens[s], h_kv, d), generator=g))
    cache.check(B, None if of is None else [-1] + [0] * (len(lens) - 1), range(3))
