"""Attention over a paged cache in which one token drowns the others out: what the quiet ones add up to has to reach the output."""
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


def tolerance(q, k, v, scale, dtype):
    """want, lse and how far they may be off: what fp32 arithmetic and rounding each weight to dtype leave (paged_reference.attention without the term
    of fp16's smallest numbers), one rounding of the output, and what fp16 leaves of a weight.  Weights are at most 2^15 there, so that half a step
    of the smallest, 2^-25, is 2^-40 of the largest weight seen, and the sum of all is at least that."""
    step = 0.0 if dtype == torch.float32 else R.half_step(dtype)
    want, lse, tol, lse_tol = R.attention(q, k, v, scale, torch.float32, step)
    tol = tol + R.half_step(dtype) * want.abs()
    if dtype == torch.float16:
        g = q.shape[0] // k.shape[1]
        tol = tol + 2.0 ** -25 + 2.0 ** -40 * v.abs().sum(0).repeat_interleave(g, 0)
    return want, lse, tol, lse_tol


def check(B, b, h_q, h_kv, d, dtype, n, gap, page=16, window=0, len_bound=0, at=0):
    """b sequences over the same pages; token `at` is `gap` louder than the others, for all query heads but the last, and its value is a hundredth."""
    g = torch.Generator().manual_seed(n + h_q)
    scale, lo = d ** -0.5, max(0, n - window) if window else 0
    q = torch.randn((h_q, d), generator=g).to(dtype)
    one = torch.randn(d, generator=g)
    q[:-1] = (one + 0.05 * torch.randn((h_q - 1, d), generator=g)).to(dtype)
    k = 0.02 * torch.randn((n, h_kv, d), generator=g)
    k[at] = one * (gap / (one.square().sum() * scale))
    v = 1 + 0.1 * torch.randn((n, h_kv, d), generator=g)
    v[at] = 0.01
    k, v = k.to(dtype), v.to(dtype)
    held = -(-n // page)
    order = torch.randperm(held, generator=g)
    pools = []
    for x in (k, v):
        rows = torch.zeros((held * page, h_kv, d), dtype=dtype)
        rows[:n] = x
        pool = torch.zeros((held, h_kv, page, d), dtype=dtype)
        pool[order] = rows.view(held, page, h_kv, d).transpose(1, 2)
        pools.append(pool.cuda())
    p = B.make_paged_params(b, h_q, h_kv, d, page, held, held, dtype, window=window, len_bound=len_bound)
    ws = torch.full((B.swa_paged_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    out, lse = torch.zeros((b, h_q, d), dtype=dtype, device="cuda"), torch.zeros((b, h_q), device="cuda")
    B.swa_paged_decode(p, q.expand(b, -1, -1).contiguous().cuda(), b, None, *pools, None, None,
                       order.int().expand(b, -1).contiguous().cuda(), torch.full((b,), n, dtype=torch.int32, device="cuda"), out, lse, ws)
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK
    want, want_lse, tol, lse_tol = tolerance(q.double(), k[lo:].double(), v[lo:].double(), scale, dtype)
    over = ((out.double().cpu() - want).abs() / tol).amax()
    assert over <= 1, ("out", float(over))
    over = ((lse.double().cpu() - want_lse).abs() / lse_tol).amax()
    assert over <= 1, ("lse", float(over))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,b", [(16384, 1024), (131072, 1024), (131072, 1), (1000, 3)])
def test_quiet_tokens_beside_a_loud_one_of_small_value(B, dtype, n, b):
    """Whole sequences in one workgroup, pieces of one that are joined, and a short one in one piece."""
    check(B, b, 2, 1, 64, TYPES[dtype], n, 17.4)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("gap", [12.0, 20.0, 26.0])
def test_quiet_tokens_at_several_distances(B, dtype, gap):
    check(B, 768, 3, 1, 128, TYPES[dtype], 20000, gap, at=19999)
    check(B, 512, 20, 1, 128, TYPES[dtype], 9001, gap, page=24, at=4000)   # 32 heads to a workgroup, pages that tiles cross
    check(B, 768, 4, 2, 64, TYPES[dtype], 30000, gap, window=20000, at=10100)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_quiet_tokens_of_one_wave(B, dtype):
    check(B, 2048, 2, 1, 64, TYPES[dtype], 250, 17.4)
    check(B, 1, 2, 1, 64, TYPES[dtype], 31, 17.4)
