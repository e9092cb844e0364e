"""Values as codes: scale = max |x| / 127 and round(x / scale) to the last bit and the last tie, as IEEE divisions in fp32 give them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


def append(B, x, dtype):
    n, h, d = x.shape
    p = B.make_paged_params(1, h, h, d, 16, -(-n // 16), 1, dtype, flags=B.SWA_KV_INT8)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    pages = [torch.zeros((p.n_pages, h, 16, d), dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.zeros((p.n_pages, h, 16), device="cuda") for _ in "kv"]
    v, slot = x.cuda(), torch.arange(n, dtype=torch.int32, device="cuda")
    B.swa_paged_append(p, v, v, v, n, None, slot, None, None, None, torch.zeros_like(v), *pages, *scales, ws)
    got = [(c.transpose(1, 2).reshape(-1, h, d)[:n].cpu(), s.transpose(1, 2).reshape(-1, h)[:n].cpu()) for c, s in zip(pages, scales)]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])     # (keys without norm and rotation are values)
    return got[1]


def check(B, x, dtype):
    codes, scale = append(B, x, dtype)
    want_scale = x.float().abs().amax(-1) / 127
    assert torch.equal(scale, want_scale)
    want = torch.round(torch.where(want_scale[..., None] > 0, x.float() / want_scale[..., None], torch.zeros(())))
    assert torch.equal(codes.float(), want), int((codes.float() != want).sum())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_values(B, dtype, d):
    g = torch.Generator().manual_seed(d)
    check(B, torch.randn((4000, 8, d), generator=g).to(dtype), dtype)
    # rows of few different values, whose quotients often lie half way between codes
    check(B, torch.randint(-100, 101, (4000, 8, d), generator=g).to(dtype), dtype)
    check(B, (torch.randint(-127, 128, (2000, 8, d), generator=g).float() * 2.0 ** torch.randint(-8, 1, (2000, 8, d), generator=g).float()).to(dtype), dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_codes_of_rows_of_every_size(B, dtype):
    """Largest values from the type's smallest normal number (bf16: 2^-90, far from where a remainder leaves fp32's numbers) to its largest."""
    low, high = (-14, 15) if dtype == torch.float16 else (-90, 127)
    g = torch.Generator().manual_seed(1)
    size = 2.0 ** torch.linspace(low, high, 600, dtype=torch.float64)
    x = (torch.rand((600, 4, 64), generator=g, dtype=torch.float64) * 2 - 1) * size[:, None, None]
    check(B, x.to(dtype), dtype)


def test_zeros(B):
    x = torch.zeros((20, 2, 64), dtype=torch.float16)
    x[3, 1, 7] = 1
    check(B, x, torch.float16)
