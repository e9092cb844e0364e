"""The attention's weights over 16-bit pages: no rounding of theirs shows in an output that is small beside its values, and infinite values stay what
they are."""
import math

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


def call(B, lens, h_q, h_kv, d, dtype, page, edit=None, len_bound=0, seed=0):
    b, held = len(lens), [-(-m // page) for m in lens]
    g = torch.Generator().manual_seed(seed)
    order, table, at = torch.randperm(sum(held), generator=g).int(), torch.zeros((b, max(held)), dtype=torch.int32), 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((sum(held), h_kv, page, d), generator=g).to(dtype) for _ in "kv")
    q = torch.randn((b, h_q, d), generator=g).to(dtype)
    if edit:
        edit(q, k, v, table)
    p = B.make_paged_params(b, h_q, h_kv, d, page, sum(held), max(held), dtype, len_bound=len_bound)
    ws = torch.full((B.swa_paged_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    out, lse = torch.zeros((b, h_q, d), dtype=dtype, device="cuda"), torch.zeros((b, h_q), device="cuda")
    B.swa_paged_decode(p, q.cuda(), b, None, k.cuda(), v.cuda(), None, None, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, ws)
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK
    return q, k, v, table, out.cpu().double(), lse.cpu().double()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,h_q,h_kv,page", [([300, 1, 17, 999], 8, 2, 16), ([5000], 4, 1, 16), ([200, 31], 4, 4, 5), ([1200, 40, 3000] * 12, 8, 2, 16), ([400, 33], 24, 1, 16),
                                                ([30, 9], 3, 3, 16), ([2000, 1100] * 8, 40, 1, 16)])
def test_outputs_are_rounded_once(B, dtype, d, lens, h_q, h_kv, page):
    dt = TYPES[dtype]
    q, k, v, table, out, lse = call(B, lens, h_q, h_kv, d, dt, page)
    for s, m in enumerate(lens):
        kk, vv = (R.gather(x, None, table[s], page, 0, m) for x in (k, v))
        want, want_lse, tol, lse_tol = R.attention(q[s].double(), kk, vv, d ** -0.5, torch.float32, STEP[dt])
        tol = tol + R.half_step(dt) * want.abs()
        if dt == torch.float16:
            # (the output's smallest numbers; and a rest of less than 2^-24 counts as that, 2^-39 of the largest weight)
            tol = tol + 2.0 ** -25 + 2.0 ** -39 * vv.abs().sum(0).repeat_interleave(h_q // h_kv, 0)
        assert ((out[s] - want).abs() / tol).max() <= 1, (s, m, float(((out[s] - want).abs() / tol).max()))
        assert ((lse[s] - want_lse).abs() <= lse_tol).all(), (s, m)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("lens", [[40], [700, 40], [1500, 700] * 16])
def test_infinite_values(B, dtype, page, lens):
    """In the loudest token, whose weight is a power of two, in others with weights of all kinds, and of both signs: infinite with its sign in its
    channel where all are of one sign, no number where both are, finite in all others."""
    dt, d, h_q, h_kv = TYPES[dtype], 64, 4, 2

    def edit(q, k, v, table):
        for s, m in enumerate(lens):
            def at(x, t):
                return x[table[s, t // page].item(), :, t % page]
            at(k, 3)[:] = (q[s].view(h_kv, -1, d).double().mean(1) * 1.5).to(dt)   # (the loudest, for most heads)
            at(v, 3)[:, 7] = math.inf
            for t in range(m):
                at(v, t)[:, 11] = -math.inf
            for t in range(0, m, 3):
                at(v, t)[:, 20] = math.inf
            for i in range(21, 41):
                at(v, (17 * i) % m)[:, i] = math.inf if i % 2 else -math.inf
            at(v, 0)[:, 50], at(v, m - 1)[:, 50] = math.inf, -math.inf
    q, k, v, table, out, lse = call(B, lens, h_q, h_kv, d, dt, page, edit)
    assert torch.isfinite(lse).all()
    signs = torch.zeros(d)
    signs[7], signs[11], signs[20] = 1, -1, 1
    for i in range(21, 41):
        signs[i] = 1 if i % 2 else -1
    inf = signs != 0
    assert torch.equal(out[..., inf], (signs[inf] * math.inf).double().expand(out[..., inf].shape))
    assert torch.isnan(out[..., 50]).all()
    rest = ~inf
    rest[50] = False
    assert torch.isfinite(out[..., rest]).all()
