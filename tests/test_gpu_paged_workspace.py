"""The attention's workspace: nothing in it counts that the same call has not written, and nothing behind it is touched."""
import pytest
import torch

import paged_reference as R
import test_gpu_paged as T

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on CPU-only hosts)")
    from paper_2403_17312_amd import binding
    binding.lib()
    return binding


class Spy:
    """The binding, with a workspace of NaN before every attention and 64 KiB of the same behind it."""

    def __init__(self, B):
        self.B, self.calls = B, 0

    def __getattr__(self, name):
        return getattr(self.B, name)

    def swa_paged_decode(self, p, *args):
        ws = args[-1]
        n = self.B.swa_paged_workspace_bytes(p)
        assert ws.numel() == n
        whole = torch.full((n + GUARD,), 0xFF, dtype=torch.uint8, device="cuda")
        self.B.swa_paged_workspace_init(p, whole)
        self.B.swa_paged_decode(p, *args[:-1], whole)
        assert (whole[n:] == 0xFF).all(), "written behind the workspace"
        ws[:256] = whole[:256]                               # (the status)
        self.calls += 1


@pytest.fixture(autouse=True)
def exact_queries(monkeypatch):
    """Codes are exact in fp16 and its queries are multiplied as they are: no rounding of queries to allow for."""
    attention = R.attention
    monkeypatch.setattr(R, "attention", lambda q, k, v, scale, dtype, weight_step, query_step=0.0: attention(q, k, v, scale, dtype, weight_step))


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128])
def test_every_form_of_the_call(B, dtype, int8, d):
    t, spy = T.TYPES[dtype], Spy(B)
    for lens, h_q, h_kv, more in (
            ([5000], 4, 1, dict(len_bound=5000)), ([131], 1, 1, {}), ([9000, 3, 0, 1025], 8, 2, {}), ([900, 40], 4, 4, dict(wider=3000)),   # chunks
            ([1500, 7, 0, 1100] * 16, 16, 4, {}), ([2500, 300] * 20, 8, 2, dict(window=1200)), ([70, 3000, 20001], 16, 8, {}),           # shares
            ([3000, 77, 0, 1500], 71, 1, {}), ([2000, 7, 0, 1100] * 8, 80, 2, {}), ([1100] * 5, 400, 1, {}), ([40, 1300], 24, 1, {}),       # tiles of heads
            ([0, 1, 31, 32, 17, -1], 7, 7, {}), ([3] * 300 + [2000], 2, 1, {})):
        T.check_decode(spy, lens, h_q, h_kv, d, t, 16, int8=int8, **more)
    T.check_decode(spy, [1000, 260, 3], 6, 3, d, t, 5, int8=int8)
    assert spy.calls == 28


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_codes_and_loud_queries(B, dtype):
    spy = Spy(B)
    for loud in (0.1, 5.0, 20.0):
        for d in (64, 128):
            T.check_decode(spy, [300, 64, 2000], 4, 2, d, T.TYPES[dtype], 16, int8=True, loud=loud)


def test_stated_sizes_hold_for_every_length_and_window(B):
    """One size for all bounds and windows of a pool."""
    for b, h_q, h_kv, d, dt in ((1, 8, 8, 128, torch.float16), (40, 32, 8, 128, torch.bfloat16), (3, 71, 1, 64, torch.float32), (512, 4, 4, 64, torch.float16)):
        sizes = {B.swa_paged_workspace_bytes(B.make_paged_params(b, h_q, h_kv, d, 16, 9000, width, dt, window=w, len_bound=n))
                 for width in (1, 70, 9000) for w in (0, 5, 3000) for n in (0, 10, 2000, 100000)}
        assert len(sizes) == 1
