"""Infinite values of tokens that a louder one drowns out stay infinite, in every form of the paged attention."""
import math

import pytest
import torch

import test_gpu_paged_sparse_weights as W
from test_gpu_paged_sparse_weights import B  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, **W.TYPES}


def decode(B, cache):  # noqa: F811
    b, (n_pages, h_kv, page, d), h_q = len(cache.lens), cache.k.shape, cache.q.shape[1]
    p = B.make_paged_params(b, h_q, h_kv, d, page, n_pages, cache.table.shape[1], cache.dtype)
    ws = torch.full((B.swa_paged_workspace_bytes(p),), 0xFF, dtype=torch.uint8, device="cuda")
    B.swa_paged_workspace_init(p, ws)
    out, lse = torch.zeros((b, h_q, d), dtype=cache.dtype, device="cuda"), torch.zeros((b, h_q), device="cuda")
    B.swa_paged_decode(p, cache.q.cuda(), b, None, cache.k.cuda(), cache.v.cuda(), None, None, cache.table.cuda(), W.ints(cache.lens), out, lse, ws)
    assert B.swa_paged_check_status(p, ws) == B.SWA_OK
    return out.cpu().double(), lse.cpu().double()


@pytest.mark.parametrize("form", ["decode", "lists", "16 columns", "32 columns", "many columns", "many columns, odd pages"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [10.0, 26.0, 28.5, 40.0, 60.0, 80.0])
def test_infinite_values_of_quiet_tokens(B, form, dtype, gap):  # noqa: F811
    """The loud token comes before them, behind them, and in another part of a sequence.  (2^-126 of the largest weight, 87 nats, are a number still.)"""
    lens, h_q, h_kv, page, of = W.FORMS["lists" if form == "decode" else form]
    d, n, dt = 64, 1500, TYPES[dtype]
    lens = [n] + lens[1:]
    one = torch.randn(d, generator=torch.Generator().manual_seed(5)).to(dt).double()
    for loud in (0, 20, n - 1):
        cache = W.Cache(lens, h_q, h_kv, d, dt, page)
        cache.q[:] = one.to(dt)
        cache.k[:] = 0
        k, v = torch.zeros((n, h_kv, d)), torch.randn((n, h_kv, d), generator=torch.Generator().manual_seed(6))
        k[loud] = (one * (gap / (one.square().sum() * d ** -0.5))).float()
        signs = torch.zeros(d)
        for i, (t, sign) in enumerate([(1, 1), (17, -1), (40, 1), (64, -1), (700, 1), (1203, -1), (n - 2, 1)]):
            v[t, :, 3 + 5 * i], signs[3 + 5 * i] = sign * math.inf, sign
        v[30, :, 50], v[999, :, 50] = math.inf, -math.inf
        cache.put(cache.k, 0, k)
        cache.put(cache.v, 0, v)
        prefix_of = None if of is None else [-1] + [0] * (len(lens) - 1)
        out, lse = decode(B, cache) if form == "decode" else cache.run(B, prefix_of)
        inf, none = signs != 0, torch.arange(d) == 50
        assert torch.isfinite(lse).all()
        for s in range(len(lens) if prefix_of else 1):
            assert torch.equal(out[s][:, inf], (signs[inf] * math.inf).double().expand(h_q, -1)), (loud, s)
            assert torch.isnan(out[s][:, none]).all() and torch.isfinite(out[s][:, ~(inf | none)]).all(), (loud, s)
