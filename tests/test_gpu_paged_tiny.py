"""Rows whose squares leave fp32's normal numbers: the norm without an eps is that of the row all the same."""
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** -55, 2.0 ** -62, 2.0 ** -63, 2.0 ** -64, 2.0 ** -65])
def test_the_norm_of_tiny_rows(B, dtype, d, size):
    """x = size (1 + u), 0 <= u < 1: every square is at least size^2 and, from 2^-149 on in steps of that, off by 2^-150 at most, relative 2^-150 / size^2 (2^-20 for the
    smallest).  The mean is off by that and the norm by half of it."""
    n, h = 5, 3
    g = torch.Generator().manual_seed(d)
    x = (size * (1 + torch.rand((n, 3 * h, d), generator=g)) * (1 - 2 * torch.randint(0, 2, (n, 3 * h, d), generator=g))).to(dtype)
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(dtype)
    pos = torch.arange(n, dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float32) * 2 / d)
    p = B.make_paged_params(1, h, h, d, n, 1, 1, dtype, rot_dim=d)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    q, k, v = (t.contiguous().cuda() for t in x.split(h, 1))
    k_pages, v_pages = (torch.zeros((1, h, n, d), dtype=dtype, device="cuda") for _ in "kv")
    q_out = torch.zeros_like(q)
    B.swa_paged_append(p, q, k, v, n, pos.cuda(), pos.cuda(), inv.cuda(), w.cuda(), w.cuda(), q_out, k_pages, v_pages, None, None, ws)
    squares = 2.0 ** -150 / size ** 2
    for got, raw in ((q_out, q), (k_pages[0].transpose(0, 1), k)):
        y, mag = R.turn(R.norm(raw.cpu().double(), w, 0.0), pos[None], inv, torch.zeros(d // 2, dtype=torch.int64), d, False)
        tol = R.row_tolerance(y, mag, dtype, d) + squares * mag
        assert ((got.cpu().double() - y).abs() <= tol).all(), float(((got.cpu().double() - y).abs() / tol).max())
    assert torch.equal(v_pages[0].transpose(0, 1), v)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_rows_of_zeros(B, dtype):
    """0 with an eps, 0 / 0 without one: in their own heads only."""
    x = torch.randn((2, 2, 64)).to(dtype).cuda()
    x[0, 1] = 0
    slot = torch.arange(2, dtype=torch.int32, device="cuda")
    w = torch.ones(64, dtype=dtype, device="cuda")
    for eps in (0.0, 1e-6):
        p = B.make_paged_params(1, 2, 2, 64, 2, 1, 1, dtype, eps=eps)
        ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
        B.swa_paged_workspace_init(p, ws)
        k_pages, v_pages = (torch.zeros((1, 2, 2, 64), dtype=dtype, device="cuda") for _ in "kv")
        q_out = torch.zeros_like(x)
        B.swa_paged_append(p, x, x, x, 2, None, slot, None, w, w, q_out, k_pages, v_pages, None, None, ws)
        for got in (q_out, k_pages[0].transpose(0, 1)):
            if eps:
                assert (got[0, 1] == 0).all()
            else:
                assert torch.isnan(got[0, 1]).all()
            assert torch.isfinite(got[1]).all() and torch.isfinite(got[0, 0]).all()
