"""The paged cache's refusals, which need no GPU: every call here is refused before the device is touched."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    from paper_2403_17312_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2403_17312_amd import build
        build.build()
    binding.lib()
    return binding


BASE = dict(b=2, h_q=4, h_kv=2, d=64, page_size=16, n_pages=8, max_pages=4, dtype=2, scale=0.0, window=0, len_bound=0, flags=0, rot_dim=64,
            eps=1e-6)
ok = 0x1000


def params(B, sections=None, **kw):
    return B.make_paged_params(**{**BASE, **kw}, sections=sections)


def plan(B, p, max_rows=4, **bad):
    names = ["new_cnt", "cache_len", "new_len", "block_table", "free_ring", "free_state", "free_state_out", "row_start", "slot", "pos",
             "workspace"]
    a = {n: ok + 0x1000 * i for i, n in enumerate(names)}
    a.update(bad)
    a = [a[n] for n in names]
    return B.lib().swa_paged_plan(ctypes.byref(p) if p is not None else None, *a[:7], max_rows, *a[7:], None)


def append(B, p, n=4, rows=None, **bad):
    h = (4, 2, 2)
    r = rows or [B.SwaRows(ok, k * 64) for k in h]
    names = ["pos", "slot", "inv_freq", "q_weight", "k_weight", "q_out", "k_pages", "v_pages", "k_scale", "v_scale", "workspace"]
    a = {m: ok + 0x1000 * (1 + i) for i, m in enumerate(names)}
    a.update(bad)
    return B.lib().swa_paged_append(ctypes.byref(p) if p is not None else None, *r, n, *[a[m] for m in names], None)


def decode(B, p, n=4, q=None, row_start=None, **bad):
    names = ["k_pages", "v_pages", "k_scale", "v_scale", "block_table", "cache_len", "out", "lse", "workspace"]
    a = {m: ok for m in names}
    a.update(bad)
    return B.lib().swa_paged_decode(ctypes.byref(p) if p is not None else None, q or B.SwaRows(ok, 256), n, row_start, *[a[m] for m in names],
                                    None)


def test_params_struct_matches_header(B):
    text = open(os.path.join(ROOT, "include", "swa.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.findall(r"typedef struct \{([^}]*)\} swa_paged_params;", text)[0]
    fields = [f for f in re.findall(r"(?:int32_t|float)\s+(\w+)", body)]
    assert fields == [f[0] for f in B.SwaPagedParams._fields_]
    assert ctypes.sizeof(B.SwaPagedParams) == 76 and ctypes.sizeof(B.SwaRows) == 16
    for name in ("SWA_MAX_PAGED_SEQS", "SWA_MAX_ROPE_AXES", "SWA_ROPE_INTERLEAVED"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(B, name)


@pytest.mark.parametrize("kw,code", [
    (dict(d=96), "SWA_ERR_UNSUPPORTED_D"),
    (dict(dtype=3), "SWA_ERR_UNSUPPORTED_DTYPE"),
    (dict(b=0), "SWA_ERR_BAD_SHAPE"),
    (dict(b=4097), "SWA_ERR_BAD_SHAPE"),
    (dict(h_q=5), "SWA_ERR_BAD_SHAPE"),              # not a multiple of h_kv
    (dict(h_q=0), "SWA_ERR_BAD_SHAPE"),
    (dict(h_kv=0), "SWA_ERR_BAD_SHAPE"),
    (dict(page_size=0), "SWA_ERR_BAD_SHAPE"),
    (dict(n_pages=0), "SWA_ERR_BAD_SHAPE"),
    (dict(max_pages=0), "SWA_ERR_BAD_SHAPE"),
    (dict(page_size=16385), "SWA_ERR_CAPACITY"),
    (dict(n_pages=1 << 26), "SWA_ERR_CAPACITY"),     # 2^26 pages of 16 tokens and 2 heads: 2^31 rows
    (dict(max_pages=(1 << 26) + 1), "SWA_ERR_CAPACITY"),
    (dict(scale=-1.0), "SWA_ERR_BAD_SHAPE"),
    (dict(scale=float("inf")), "SWA_ERR_BAD_SHAPE"),
    (dict(eps=float("nan")), "SWA_ERR_BAD_SHAPE"),
    (dict(eps=-1.0), "SWA_ERR_BAD_SHAPE"),
    (dict(window=-1), "SWA_ERR_BAD_SHAPE"),
    (dict(len_bound=-1), "SWA_ERR_BAD_SHAPE"),
    (dict(flags=1), "SWA_ERR_BAD_SHAPE"),
    (dict(flags=8, dtype=0), "SWA_ERR_UNSUPPORTED_DTYPE"),
    (dict(rot_dim=24), "SWA_ERR_BAD_SHAPE"),         # not a multiple of 16
    (dict(rot_dim=80), "SWA_ERR_BAD_SHAPE"),         # beyond d
    (dict(rot_dim=-16), "SWA_ERR_BAD_SHAPE"),
    (dict(sections=[16, 15]), "SWA_ERR_BAD_SHAPE"),  # one pair too few
    (dict(sections=[40, -8]), "SWA_ERR_BAD_SHAPE"),
])
def test_bad_params_are_rejected_by_every_call(B, kw, code):
    p, want = params(B, **kw), getattr(B, code)
    assert plan(B, p) == want and append(B, p) == want and decode(B, p) == want
    assert B.lib().swa_paged_workspace_init(ctypes.byref(p), ok, None) == want
    st = ctypes.c_int32(0)
    assert B.lib().swa_paged_check_status(ctypes.byref(p), ok, None, ctypes.byref(st)) == want
    assert B.swa_paged_workspace_bytes(p) == 0


def test_axes_outside_the_range_are_refused(B):
    for axes in (0, 5):
        p = params(B)
        p.axes = axes
        assert decode(B, p) == B.SWA_ERR_BAD_SHAPE
    for parts in ([], [8] * 5):
        with pytest.raises(B.SwaError):
            params(B, sections=parts)


def test_null_pointers_are_refused(B):
    p, q8 = params(B), params(B, flags=B.SWA_KV_INT8)
    for call in (plan, append, decode):
        assert call(B, None) == B.SWA_ERR_NULL
    for n in ("new_cnt", "cache_len", "new_len", "block_table", "free_ring", "free_state", "free_state_out", "row_start", "slot", "pos", "workspace"):
        assert plan(B, p, **{n: None}) == B.SWA_ERR_NULL, n
    for n in ("pos", "slot", "inv_freq", "q_out", "k_pages", "v_pages", "workspace"):
        assert append(B, p, **{n: None}) == B.SWA_ERR_NULL, n
    for n in ("k_pages", "v_pages", "block_table", "cache_len", "out", "workspace"):
        assert decode(B, p, **{n: None}) == B.SWA_ERR_NULL, n
    for n in ("k_scale", "v_scale"):
        assert append(B, q8, **{n: None}) == B.SWA_ERR_NULL and decode(B, q8, **{n: None}) == B.SWA_ERR_NULL, n
    assert append(B, p, rows=[B.SwaRows(None, 256)] + [B.SwaRows(ok, 128)] * 2) == B.SWA_ERR_NULL
    assert decode(B, p, q=B.SwaRows(None, 256)) == B.SWA_ERR_NULL


def test_sizes_and_places_are_refused(B):
    p = params(B)
    for n in (0, -1, (1 << 24) + 1):
        assert plan(B, p, max_rows=n) == B.SWA_ERR_BAD_SHAPE
        assert append(B, p, n=n) == B.SWA_ERR_BAD_SHAPE
        assert decode(B, p, n=n) == B.SWA_ERR_BAD_SHAPE
    assert decode(B, p, n=1) == B.SWA_ERR_BAD_SHAPE                      # two sequences, one row
    assert plan(B, p, new_len=ok + 0x1000) == B.SWA_ERR_BAD_SHAPE        # the lengths need a second array
    assert plan(B, p, free_state_out=ok + 0x5000) == B.SWA_ERR_BAD_SHAPE
    R = B.SwaRows
    for i in range(3):
        for row, code in ((R(ok, 64 * (4, 2, 2)[i] - 8), B.SWA_ERR_BAD_SHAPE), (R(ok, 260), B.SWA_ERR_ALIGNMENT), (R(ok + 8, 256), B.SWA_ERR_ALIGNMENT),
                          (R(ok, -256), B.SWA_ERR_BAD_SHAPE), (R(ok, 1 << 41), B.SWA_ERR_BAD_SHAPE)):
            rows = [R(ok, 256), R(ok, 128), R(ok, 128)]
            rows[i] = row
            assert append(B, p, rows=rows) == code, (i, row.stride)
            if i == 0:
                assert decode(B, p, q=row) == code
    for n in ("q_out", "k_pages", "v_pages", "q_weight", "k_weight", "workspace"):
        assert append(B, p, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT, n
    for n in ("k_pages", "v_pages", "out", "workspace"):
        assert decode(B, p, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT, n
    assert plan(B, p, new_cnt=ok + 0x2000) == B.SWA_ERR_BAD_SHAPE        # (the new lengths' place)
    q8 = params(B, flags=B.SWA_KV_INT8)
    for n in ("k_scale", "v_scale"):
        assert append(B, q8, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT and decode(B, q8, **{n: ok + 8}) == B.SWA_ERR_ALIGNMENT, n
        assert append(B, p, **{n: ok + 8, "slot": None}) == B.SWA_ERR_NULL               # (not looked at without codes)
    rows = [R(ok, 512), R(ok, 128), R(ok, 128)]
    assert append(B, p, rows=rows, q_out=ok) == B.SWA_ERR_BAD_SHAPE      # in place, but with gaps between the rows


@pytest.mark.parametrize("general", [False, True])
def test_tensors_elsewhere_are_refused(B, monkeypatch, general):
    """Tensors of the CPU, rows that are not dense, and what is no tensor."""
    if general:
        monkeypatch.setattr(B, "_native", B._General())
    p, t = params(B), torch.zeros(64, dtype=torch.int32)
    rows = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current GPU"):
        B.swa_paged_plan(p, t, t, t, t, t, t, t, 4, t, t, t, t, 0)
    with pytest.raises(ValueError, match="current GPU"):
        B.swa_paged_append(p, rows, rows, rows, 4, t, t, t, None, None, t, t, t, None, None, t, 0)
    with pytest.raises(ValueError, match="current GPU"):
        B.swa_paged_decode(p, rows, 4, None, t, t, None, None, t, t, t, None, t, 0)
    for bad in (rows[..., ::2], rows.transpose(0, 1).expand(4, 4, 64).transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError, match="dense"):
            B.swa_paged_decode(p, bad, 4, None, t, t, None, None, t, t, t, None, t, 0)
    with pytest.raises((ValueError, AttributeError, TypeError)):
        B.swa_paged_decode(p, 5, 4, None, t, t, None, None, t, t, t, None, t, 0)
    with pytest.raises(ValueError):
        B.swa_paged_decode(p, rows[0], 4, None, t, t, None, None, t, t, t, None, t, 0)


def test_the_reference_plan_hands_out_and_takes_back():
    """The lists that the GPU's plan is compared with, by hand: pages of 4, sequence 1 finishes, 2 grows over a page's end, 3 finds no page."""
    import paged_reference as R
    new_len, table, ring, state, start, slot, pos, bits = R.plan(
        [0, -1, 3, 5, 1], [2, 5, 3, 4, 1], [[7, -1, -1], [3, 5, -1], [1, -1, -1], [2, -1, -1], [6, -1, -1]], [9, 9, 0, 4, 9, 9, 9, 9], [2, 2], 4, 16)
    assert new_len == [2, 0, 6, 4, 2] and table[2] == [1, 0, -1] and table[3] == [2, -1, -1]
    assert ring == [9, 9, 0, 4, 3, 5, 9, 9] and state == [3, 3] and start == [0, 0, 0, 3, 8, 9]
    assert slot == [7, 0, 1] + [-1] * 5 + [25] + [-1] * 7 and pos == [3, 4, 5] + [0] * 5 + [1] + [0] * 7 and bits == {"capacity"}
