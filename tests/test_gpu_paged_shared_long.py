"""Attention behind shared prefixes in caches whose tables name so many tokens that a sequence's own go in longer steps."""
import pytest
import torch

import paged_reference as R
import test_gpu_paged as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("b,h_q,h_kv,width", [(256, 136, 8, 1024), (64, 1024, 8, 4096), (17, 8, 8, 32768)])
def test_long_tables(B, b, h_q, h_kv, width):
    """Pages of 16384 tokens, of which all sequences read the same six: two the prefix, one each other sequence.  Own steps of 64, 256 and 64 tokens."""
    page, d, t = 16384, 64, torch.float16
    k, v, _, _ = T.make_pool(6, h_kv, page, d, t, False, 3)
    lens = [20000] + [(i * 211) % 3000 for i in range(b - 1)]
    table = torch.full((b, width), -1, dtype=torch.int32)
    table[0, :2] = torch.tensor([3, 0])
    for s in range(1, b):
        table[s, 0] = (1, 2, 4, 5)[s % 4]
    q = torch.randn((b, h_q, d), generator=torch.Generator().manual_seed(1)).to(t)
    p = B.make_paged_params(b, h_q, h_kv, d, page, 6, width, t)
    nbytes = B.swa_paged_workspace_bytes(p)
    ws = torch.full((nbytes + (1 << 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    out, lse = torch.full((b, h_q, d), 7.0, dtype=t, device="cuda"), torch.zeros((b, h_q), device="cuda")
    prefix_of = [-1] + [0 if s % 5 else -1 for s in range(1, b)]
    B.swa_paged_decode_shared(p, q.cuda(), b, None, None, k, v, None, None, table.cuda(), T.ints(lens), T.ints(prefix_of), out, lse, ws)
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK and (ws[nbytes:] == 0xFF).all()
    kc, vc = k.cpu(), v.cpu()
    for s in (0, 1, 5, 14, b // 2, b - 1):
        kk, vv = (torch.cat([R.gather(x, None, table[of], page, 0, lens[of]) for of in ([0] if prefix_of[s] == 0 else []) + [s]]) for x in (kc, vc))
        heads = slice(0, 3 * (h_q // h_kv))                  # (of three key heads)
        want, want_lse, tol, lse_tol = R.attention(q[s, heads].double(), kk[:, :3], vv[:, :3], d ** -0.5, t, R.half_step(t))
        assert ((out[s, heads].cpu().double() - want).abs() <= tol).all() and ((lse[s, heads].cpu().double() - want_lse).abs() <= lse_tol).all(), s
        last = slice(h_q - h_q // h_kv, h_q)
        want, _, tol, _ = R.attention(q[s, last].double(), kk[:, -1:], vv[:, -1:], d ** -0.5, t, R.half_step(t))
        assert ((out[s, last].cpu().double() - want).abs() <= tol).all(), s
