"""Rotated fp32 rows are as near to the exact ones as fp32's own operations leave them."""
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


def rotated(B, x, pos, inv, neighbours):
    n, h, d = x.shape
    p = B.make_paged_params(1, h, h, d, 16, -(-n // 16), 1, torch.float32, flags=32 if neighbours else 0, rot_dim=d)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    k, v = (torch.zeros((p.n_pages, h, 16, d), device="cuda") for _ in "kv")
    q = x.cuda()
    q_out, slot = torch.zeros_like(q), torch.arange(n, dtype=torch.int32, device="cuda")
    B.swa_paged_append(p, q, q, q, n, pos.cuda(), slot, inv.cuda(), None, None, q_out, k, v, None, None, ws)
    assert torch.equal(k.transpose(1, 2).reshape(-1, h, d)[:n], q_out)
    return q_out.cpu()


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("far", [300, 2 ** 31 - 1])
def test_rms_error_of_a_rotation(B, neighbours, far):
    """Against x cos - y sin in fp32 with sine and cosine rounded once: there a sine, a cosine, a product and a sum are rounded, each by 2^-24 / sqrt(3) rms of its
    binade's end.  The kernel's sine and cosine are off by up to two further roundings each, of numbers half as large at most (x in quarter turns, the
    series' last step): (4 + 4 / 4) / 4 of the variance, 1.12 times the rms; a quarter more leaves room for the sample."""
    g = torch.Generator().manual_seed(3)
    n, h, d = 500, 4, 128
    x = torch.randn((n, h, d), generator=g)
    pos = torch.randint(0, far, (n,), generator=g, dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float32) * 2 / d)
    axis = torch.zeros(d // 2, dtype=torch.int64)
    want, _ = R.turn(x.double(), pos[None], inv, axis, d, neighbours)
    angle = pos.double()[:, None] * inv.double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, z = (slice(0, d, 2), slice(1, d, 2)) if neighbours else (slice(0, d // 2), slice(d // 2, d))
    plain = x.clone()
    plain[..., a], plain[..., z] = x[..., a] * c - x[..., z] * s, x[..., z] * c + x[..., a] * s
    got = rotated(B, x, pos, inv, neighbours)
    off, ours = ((t.double() - want).square().mean().sqrt().item() for t in (plain, got))
    assert ours <= 1.4 * off, (ours / off, off)
    assert (got.double() - want).abs().max() <= 8 * 2.0 ** -24 * x.abs().max()


@pytest.mark.parametrize("neighbours", [False, True])
def test_quarter_turns(B, neighbours):
    """Angles of whole quarter turns (inv_freq pi / 2 rounded, times 0 .. 9): (x, y) goes to (x, y), (-y, x), (-x, -y), (y, -x), but for what the rounded frequency is off."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn((10, 2, 64), generator=g)
    pos, inv = torch.arange(10, dtype=torch.int32), torch.full((32,), 1.5707963267948966, dtype=torch.float32)
    got = rotated(B, x, pos, inv, neighbours).double()
    want, size = R.turn(x.double(), pos[None], inv, torch.zeros(32, dtype=torch.int64), 64, neighbours)
    assert ((got - want).abs() <= 4 * 2.0 ** -24 * size).all()
    assert torch.equal(got[0], x[0].double())
