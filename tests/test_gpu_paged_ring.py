"""A ring of free pages whose state is none hands nothing out, and says so."""
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


@pytest.mark.parametrize("state", [[-1, 4], [8, 4], [2 ** 31 - 1, 1], [-2 ** 31, 8], [0, 9], [3, -1], [0, 2 ** 31 - 1], [0, -2 ** 31]])
@pytest.mark.parametrize("new", [[0, 1, 0], [2, 0, 0], [3, 1, 1], [0, 0, 0], [0, -1, 1]])
def test_a_state_outside_the_ring(B, state, new):
    """Sequence 0 has room for two tokens in its page, the others for none."""
    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    lens, table, ring = [2, 8, 4], [[0, -1, -1], [1, 2, -1], [3, -1, -1]], [4, 5, 6, 7, 9, 9, 9, 9]
    p = B.make_paged_params(3, 1, 1, 64, 4, 8, 3, torch.float16)
    ws = torch.zeros((B.swa_paged_workspace_bytes(p),), dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    new_len, t, r, out, start, slot, pos = ints([0] * 3), ints(table), ints(ring), ints([-7, -7]), ints([0] * 4), ints([0] * 6), ints([0] * 6)
    B.swa_paged_plan(p, ints(new), ints(lens), new_len, t, r, ints(state), out, 6, start, slot, pos, ws)
    want = R.plan(new, lens, table, ring, [0, 0], 4, 6)
    got = [x.tolist() for x in (new_len, t, r, out, start, slot, pos)]
    assert got == [list(x) for x in want[:7]]
    assert B.swa_paged_check_status(p, ws) == (B.SWA_ERR_CAPACITY if "capacity" in want[7] else B.SWA_ERR_BAD_REQUEST)
