"""The attention behind shared prefixes for a single sequence, which can have none: the decode's workspace, and what it reports."""
import pytest
import torch

import test_gpu_paged as T
import test_gpu_paged_shared as S
from test_gpu_paged_shared import B  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,int8", [("f32", False), ("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("n", [0, 1, 31, 300, 5000, 40011])
def test_one_sequence(B, dtype, int8, n):  # noqa: F811
    t = T.TYPES[dtype]
    for h_q, h_kv, d, page in ((1, 1, 64, 16), (8, 2, 128, 16), (40, 1, 64, 20)):
        S.check_shared(B, [n], [-1], h_q, h_kv, d, t, page, int8=int8)
    S.check_shared(B, [n], [-1], 4, 2, 64, t, 16, int8=int8, len_bound=n + 5, lse=False, scale=0.3, strided=True)


def test_what_one_sequence_reports(B):  # noqa: F811
    for t in (torch.bfloat16, torch.float32):
        for of in (0, 1, -2, 2 ** 31 - 1, -2 ** 31):
            S.check_shared(B, [300], [of], 4, 2, 64, t, 16, refused=(0,))
            S.check_shared(B, [-1], [of], 4, 2, 64, t, 16)                                   # (an unused row reports nothing)
            S.check_shared(B, [300], [of], 4, 2, 64, t, 16, row_start=[2, 2], n_rows=3)      # nor one without rows
            S.check_shared(B, [300], [of], 4, 2, 64, t, 16, row_start=[0, 2], n_rows=3, slot=[3, -1, 5])
            S.check_shared(B, [300], [of], 4, 2, 64, t, 16, len_bound=100, skipped=(0,))
        S.check_shared(B, [300], [-1], 4, 2, 64, t, 16, row_start=[0, 2], n_rows=3, slot=[3, 4, 5])
        S.check_shared(B, [300], [-1], 4, 2, 64, t, 16, bad=[(0, 3, -1), (0, 9, 10 ** 6)])


def test_one_sequence_in_a_graph(B):  # noqa: F811
    """Replays follow the lengths and the prefix that they find."""
    d, page = 64, 16
    k, v, _, _ = T.make_pool(100, 2, page, d, torch.float16, False, 3)
    p = B.make_paged_params(1, 8, 2, d, page, 100, 100, torch.float16)
    ws, table = T.workspace(B, p), torch.arange(100, dtype=torch.int32, device="cuda")[None].contiguous()
    q = torch.randn((1, 8, d), generator=torch.Generator().manual_seed(1)).to(torch.float16).cuda()
    n, of, out, want = T.ints([1]), T.ints([-1]), torch.zeros_like(q), torch.zeros_like(q)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        B.swa_paged_decode_shared(p, q, 1, None, None, k, v, None, None, table, n, of, out, None, ws)
    torch.cuda.current_stream().wait_stream(stream)
    for m, prefix in ((700, -1), (3, -1), (1600, 0), (1599, -1), (0, -1), (40, 3)):
        n.fill_(m)
        of.fill_(prefix)
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert B.swa_paged_check_status(p, ws) == (B.SWA_OK if prefix == -1 else B.SWA_ERR_BAD_REQUEST)
        B.swa_paged_decode(p, q, 1, None, k, v, None, None, table, n, want, None, ws)
        assert torch.equal(out, want) if prefix == -1 else (out == 7).all(), m
