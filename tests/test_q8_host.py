"""The 8-bit KV cache without a GPU: the oracle's number format against torch's float8 type and worked values, and what
the calls refuse before they launch anything."""
import numpy as np
import pytest
import torch

from oracle import cache_q8 as oq
from paper_2605_23296_b200 import binding as B

ALL = np.arange(256, dtype=np.uint8)


def _values(bits):
    return torch.from_numpy(bits.copy()).view(torch.float8_e4m3fn).double().numpy()


def test_every_code_keeps_its_bits():
    v = _values(ALL)
    keep = ~np.isnan(v)
    assert keep.sum() == 254
    assert np.array_equal(oq.e4m3_round(v[keep]), v[keep])
    assert np.array_equal(oq.e4m3_bits(v[keep]), ALL[keep])
    assert oq.e4m3_bits(np.array([np.nan]))[0] == 0x7F


def test_rounding_is_nearest_even_and_saturates():
    v = np.unique(np.abs(_values(ALL[:127])))
    mid = (v[:-1] + v[1:]) / 2
    want = torch.from_numpy(np.concatenate([mid, mid * (1 + 2 ** -20), mid * (1 - 2 ** -20)])).float()
    got = oq.e4m3_round(want.double().numpy())
    assert np.array_equal(got, want.to(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(oq.e4m3_round([500.0, -np.inf, np.inf]), [448.0, -448.0, 448.0])


@pytest.mark.parametrize("amax,scale", [(448.0, 1.0), (448.5, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.7501, 2.0 ** -7),
                                        (0.0, 2.0 ** -126), (3.3e38, 2.0 ** 120)])
def test_page_scale_worked_values(amax, scale):
    assert oq.page_scale(np.array([[amax, -amax / 2]])) == scale
    assert oq.page_scale(np.array([[amax, np.inf, np.nan]])) == scale


def test_append_in_pieces_holds_what_the_bounds_say():
    # growing magnitudes, one token at a time: every re-rounding is to the same significand unless it goes subnormal
    rng = np.random.default_rng(3)
    x = rng.standard_normal((16, 1, 64)) * 2.0 ** np.arange(16)[:, None, None] / 64
    c = oq.CacheQ8(2, 1, 64, [0], 16, np.array([1, 0]))
    for i in range(16):
        c.append(0, x[i:i + 1], x[i:i + 1])
    k = c.rows(0, 0, 16)[0].transpose(1, 0, 2)
    s = c.scales[1, 0, 0]
    # half a step of e4m3 (2^-4 relative, 2^-10 scales absolute), and at most once more where a value went subnormal
    assert (np.abs(k - x) <= 2.0 ** -4 * np.abs(x) + 2 * 2.0 ** -10 * s).all()


def _cfg(hq=8, hkv=2, d=64, page=16, scale=0.125, sms=0):
    return B.cpa_config(hq, hkv, d, page, scale, 0, 0, sms)


@pytest.mark.parametrize("cfg,want", [
    (_cfg(hq=7), B.CPA_EINVAL), (_cfg(hkv=0), B.CPA_EINVAL), (_cfg(scale=0.0), B.CPA_EINVAL),
    (_cfg(scale=float("nan")), B.CPA_EINVAL), (_cfg(sms=-1), B.CPA_EINVAL), (_cfg(d=96), B.CPA_EUNSUPPORTED),
    (_cfg(page=32), B.CPA_EUNSUPPORTED), (_cfg(hq=18), B.CPA_EUNSUPPORTED), (_cfg(sms=5000), B.CPA_EUNSUPPORTED)])
def test_bad_configurations_are_refused(cfg, want):
    dims = B.cpa_table_dims(4, 0, 8, 8, 8)
    assert B.cpa_tables_bytes(cfg, dims) == want
    assert B.cpa_decode_q8_workspace_bytes(cfg) == want
    assert B.cpa_tables_build(cfg, dims, 256, 256, 8, 256) == want


@pytest.mark.parametrize("dims,want", [
    ((0, 0, 8, 8, 8), B.CPA_EINVAL), ((4, -1, 8, 8, 8), B.CPA_EINVAL), ((4, 0, 0, 8, 8), B.CPA_EINVAL),
    ((4, 0, 8, -1, 8), B.CPA_EINVAL), ((4, 0, 8, 8, -1), B.CPA_EINVAL), ((1 << 21, 0, 8, 8, 8), B.CPA_EUNSUPPORTED),
    ((4, 0, 8, (1 << 30) + 1, 8), B.CPA_EUNSUPPORTED), ((4, 0, 1 << 28, 8, 8), B.CPA_EUNSUPPORTED), ((4, 0, 1 << 26, 8, 8), B.CPA_EUNSUPPORTED)])
def test_bad_sizes_are_refused(dims, want):
    dims = B.cpa_table_dims(*dims)
    assert B.cpa_tables_bytes(_cfg(), dims) == want
    assert B.cpa_tables_offset(_cfg(), dims, B.ARR_CU_SEQLENS) == want


def test_tables_arrays_lie_apart_inside_the_buffer():
    dims = B.cpa_table_dims(5, 3, 40, 23, 31)
    at = {w: B.cpa_tables_offset(_cfg(), dims, w)
          for w in (B.ARR_CU_SEQLENS, B.ARR_PAGE_INDPTR, B.ARR_PAGE_INDICES, B.ARR_SLOT_MAPPING)}
    size = {B.ARR_CU_SEQLENS: 6, B.ARR_PAGE_INDPTR: 6, B.ARR_PAGE_INDICES: 23, B.ARR_SLOT_MAPPING: 31}
    end = 0
    for w in sorted(at, key=at.get):
        assert at[w] % 16 == 0 and at[w] >= end
        end = at[w] + 4 * size[w]
    assert end + 4 * 5 * 2 <= B.cpa_tables_bytes(_cfg(), dims)      # the merge counters follow
    assert B.cpa_tables_offset(_cfg(), dims, B.ARR_SEQ_LENS) == B.CPA_EINVAL


def test_bad_pointers_are_refused():
    cfg, dims, ok = _cfg(), B.cpa_table_dims(4, 0, 8, 8, 8), 1 << 20      # (addresses are only looked at)
    other = ok + (1 << 16)
    build = lambda **k: B.cpa_tables_build(cfg, dims, **dict(dict(d_block_lens=ok, d_free_pages=ok, num_free=8, d_tables=ok), **k))
    for bad in (dict(d_block_lens=None), dict(d_free_pages=None), dict(d_tables=None), dict(d_tables=ok + 4),
                dict(d_block_lens=ok + 2), dict(d_free_pages=ok + 1), dict(num_free=-1)):
        assert build(**bad) == B.CPA_EINVAL, bad
    base = dict(d_tables=ok, k_new=ok, v_new=ok, d_cu_new=ok, num_rows=4, d_lens=ok, d_lens_out=other, kv_pool=ok, kv_scales=ok)
    for bad in (dict(d_tables=None), dict(k_new=None), dict(v_new=None), dict(kv_pool=None), dict(kv_scales=None),
                dict(num_rows=-1), dict(k_new=ok + 8), dict(v_new=ok + 2), dict(kv_pool=ok + 8), dict(kv_scales=ok + 4),
                dict(d_lens_out=ok), dict(d_lens=ok + 1), dict(d_cu_new=ok + 2), dict(d_cu_new=None, num_rows=3)):
        assert B.cpa_kv_append_q8(cfg, dims, **dict(base, **bad)) == B.CPA_EINVAL, bad
    base = dict(d_tables=ok, q=ok, d_lens=ok, d_active=None, kv_pool=ok, kv_scales=ok, o=ok, d_workspace=ok)
    for bad in ([{n: None} for n in ("d_tables", "q", "d_lens", "kv_pool", "kv_scales", "o", "d_workspace")] +
                [dict(q=ok + 2), dict(o=ok + 8), dict(d_lens=ok + 2), dict(d_active=ok + 1), dict(kv_pool=ok + 1),
                 dict(kv_scales=ok + 4), dict(d_workspace=ok + 4)]):
        assert B.cpa_decode_q8(cfg, dims, **dict(base, **bad)) == B.CPA_EINVAL, bad
        assert B.cpa_decode_append_q8(cfg, dims, **dict(base, k_new=ok, v_new=ok, d_lens_out=other, **bad)) == B.CPA_EINVAL, bad
    for bad in (dict(k_new=None), dict(v_new=None), dict(k_new=ok + 2), dict(v_new=ok + 8), dict(d_lens_out=None),
                dict(d_lens_out=ok)):
        assert B.cpa_decode_append_q8(cfg, dims, **dict(base, **dict(dict(k_new=ok, v_new=ok, d_lens_out=other), **bad))) == B.CPA_EINVAL, bad
    base = dict(d_tables=ok, d_first=None, d_cu=ok, num_rows=4, kv_pool=ok, kv_scales=ok, k_out=ok, v_out=ok)
    for bad in (dict(d_tables=None), dict(d_cu=None), dict(kv_pool=None), dict(kv_scales=None), dict(k_out=None),
                dict(v_out=None), dict(num_rows=-1), dict(d_first=ok + 1), dict(k_out=ok + 8), dict(v_out=ok + 2)):
        assert B.cpa_kv_read_q8(cfg, dims, **dict(base, **bad)) == B.CPA_EINVAL, bad
    assert B.cpa_tables_status(None) == B.CPA_EINVAL


def test_programmatic_kernels_read_global_memory_coherently():
    # a kernel that begins before its predecessor has ended may not load what that one writes through the non-coherent
    # path, by name or by the compiler's choice
    import os
    import re
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    for name in os.listdir(csrc):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(csrc, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        if '"cache_q8.cuh"' in text or name == "cache_q8.cuh":      # (their indexes and lengths are written on the device)
            assert "__ldg(" not in text and "global.nc" not in text, name
            assert not re.search(r"const\s+\w+\s*\*\s*__restrict__", text), name
