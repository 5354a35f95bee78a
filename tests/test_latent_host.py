"""Rotary positions and latent attention without a GPU: the frequencies against their definition, the oracle's two forms
against one another, and what the calls refuse before they launch anything."""
import os
import re
from fractions import Fraction

import numpy as np
import pytest

from oracle import latent as ol
from paper_2605_23296_b200 import binding as B


def _rope(R=64, layout=0, scaling=0, trained=4096, base=10000.0, factor=40.0, fast=32.0, slow=1.0, amplitude=1.0):
    return B.cpa_rope_config(R, layout, scaling, trained, base, factor, fast, slow, amplitude)


KINDS = {"none": 0, "all": 1, "base": 2, "parts": 3, "waves": 4}


@pytest.mark.parametrize("R", [2, 20, 64, 128, 256])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
def test_turns_are_the_frequencies(R, kind, base):
    if kind == "base" and R == 2:
        pytest.skip("no slower pair")
    turns = B.cpa_rope_turns(_rope(R, scaling=KINDS[kind], base=base))
    want = ol.frequencies(R, base, kind, 40.0, 32.0, 1.0, 4096) / (2 * np.pi)
    assert turns.shape == (R // 2,) and turns.dtype == np.uint64
    # float64 frequencies: a power and up to four more roundings, and one of pi
    off = np.abs(np.array([float(Fraction(int(t), 2 ** 64) - Fraction(float(w) % 1.0)) for t, w in zip(turns, want)]))
    assert (np.minimum(off, 1 - off) <= 64 * 2.0 ** -53 * np.maximum(want, 2.0 ** -11)).all()


def test_turns_keep_more_bits_than_a_double():
    # base 2^32, R = 64: f_i = 2^-i, so the fractions are 2^-i / (2 pi) to all their bits
    t = [int(x) for x in B.cpa_rope_turns(_rope(64, base=float(2 ** 32)))]
    # (2 pi, the quotient and the power are each rounded to 64 bits: 3 * 2^-64 of 0.16, and half a unit of the fraction)
    assert abs(t[0] - Fraction(2 ** 64) / Fraction("6.283185307179586476925286766559005768394338798750")) <= 1
    assert all(abs(2 * b - a) <= 3 for a, b in zip(t[:-1], t[1:]))


@pytest.mark.parametrize("bad", [dict(R=0), dict(R=7), dict(R=258), dict(R=-2), dict(layout=2), dict(layout=-1), dict(scaling=5),
                                 dict(base=0.0), dict(base=float("nan")), dict(base=1e31), dict(amplitude=0.0),
                                 dict(amplitude=float("nan")), dict(scaling=1, factor=0.0), dict(scaling=1, factor=float("inf")),
                                 dict(scaling=2, R=2), dict(scaling=3, trained=0), dict(scaling=3, slow=0.0),
                                 dict(scaling=3, fast=1.0), dict(scaling=3, fast=float("nan")), dict(scaling=4, slow=64.0),
                                 dict(scaling=3, base=1.0)])
def test_bad_rotary_configurations_are_refused(bad):
    cfg = _rope(**bad)
    assert B.cpa_rope_turns(cfg, check=False)[0] == B.CPA_EINVAL
    rows = B.cpa_rope_rows(256, 256, 64, 64, 64, 64, 1, 64, 0)
    assert B.cpa_rope(cfg, 256, 256, 1, rows) == B.CPA_EINVAL


def test_rope_refusals():
    ok = 1 << 20
    base = dict(x=ok, out=ok + (1 << 16), x_row_stride=512, x_head_stride=128, out_row_stride=512, out_head_stride=128, heads=4,
                head_dim=128, offset=64)
    call = lambda rows=3, turns=ok, pos=ok, **k: B.cpa_rope(_rope(), turns, pos, rows, B.cpa_rope_rows(**dict(base, **k)))
    for bad in (dict(x=0), dict(out=0), dict(x=ok + 1), dict(out=ok + 3), dict(heads=-1), dict(head_dim=63), dict(offset=-1),
                dict(offset=65), dict(out_head_stride=127), dict(out_row_stride=100), dict(out_row_stride=511),
                dict(out_head_stride=-128), dict(out_row_stride=0), dict(rows=-1), dict(turns=None), dict(turns=ok + 4),
                dict(pos=None), dict(pos=ok + 2), dict(out=ok, out_row_stride=1024)):
        assert call(**bad) == B.CPA_EINVAL, bad
    assert call(heads=1 << 17) == B.CPA_EUNSUPPORTED
    assert B.cpa_rope(_rope(), ok, ok, 1, B.cpa_rope_rows(ok, ok, 1 << 26, 1 << 12, 1 << 26, 1 << 12, 8192, 4096, 0)) == B.CPA_EUNSUPPORTED
    assert B._lib.cpa_rope(_rope(), ok, ok, 1, None, None, 0, None) == B.CPA_EINVAL
    assert call(rows=0) == 0 and call(heads=0) == 0          # nothing to do, nothing launched


def _cfg(H=16, L=512, R=64, nope=128, v=128, page=16, scale=0.07, eps=1e-6, sms=0):
    return B.cpa_latent_config(H, L, R, nope, v, page, scale, eps, sms)


@pytest.mark.parametrize("cfg,want", [
    (_cfg(H=0), B.CPA_EINVAL), (_cfg(L=0), B.CPA_EINVAL), (_cfg(scale=0.0), B.CPA_EINVAL), (_cfg(scale=float("nan")), B.CPA_EINVAL),
    (_cfg(scale=float("inf")), B.CPA_EINVAL), (_cfg(eps=-1.0), B.CPA_EINVAL), (_cfg(eps=float("nan")), B.CPA_EINVAL),
    (_cfg(sms=-1), B.CPA_EINVAL), (_cfg(H=129), B.CPA_EUNSUPPORTED), (_cfg(L=192), B.CPA_EUNSUPPORTED), (_cfg(L=640), B.CPA_EUNSUPPORTED),
    (_cfg(R=32), B.CPA_EUNSUPPORTED), (_cfg(nope=64), B.CPA_EUNSUPPORTED), (_cfg(v=64), B.CPA_EUNSUPPORTED),
    (_cfg(page=32), B.CPA_EUNSUPPORTED), (_cfg(sms=4096), B.CPA_EUNSUPPORTED)])
def test_bad_latent_configurations_are_refused(cfg, want):
    ok, dims = 1 << 20, B.cpa_table_dims(4, 0, 8, 8, 8)
    assert B.cpa_latent_decode_workspace_bytes(cfg) == want
    for call in (B.cpa_latent_tables_config, B.cpa_latent_plan_config):
        with pytest.raises(B.CpaError) as e:
            call(cfg)
        assert e.value.status == want
    io = B.cpa_latent_io(ok, 8192, 512, ok, 1024, 64, ok + (1 << 17), 8192, 512)
    assert B.cpa_latent_append(cfg, dims, ok, None, None, ok, 576, None, None, 4, None, ok, ok + 4, ok) == want
    assert B.cpa_latent_decode(cfg, dims, ok, io, ok, None, ok, ok) == want
    assert B.cpa_latent_step(cfg, dims, ok, None, None, io, ok, 576, None, None, ok, ok + 4, None, ok, ok) == want
    assert B.cpa_latent_prefill(cfg, 0, ok, ok, ok, 64, ok) == want


def test_latent_pointers_and_strides_are_refused():
    cfg, dims, ok = _cfg(), B.cpa_table_dims(4, 0, 8, 8, 8), 1 << 20
    other = ok + (1 << 16)
    base = dict(d_tables=ok, rope=_rope(), d_turns=ok, x=ok, x_row_stride=576, norm_weight=ok, d_cu_new=ok, num_rows=4, d_first=ok,
                d_lens=ok, d_lens_out=other, pool=ok, packed=ok)
    for bad in (dict(d_tables=None), dict(d_tables=ok + 8), dict(x=None), dict(x=ok + 1), dict(x_row_stride=575), dict(norm_weight=ok + 2),
                dict(d_cu_new=ok + 2), dict(num_rows=-1), dict(d_first=ok + 1), dict(d_lens=ok + 2), dict(d_lens_out=ok), dict(pool=None),
                dict(pool=ok + 8), dict(packed=ok + 2), dict(d_turns=None), dict(rope=None), dict(rope=_rope(32)), dict(rope=_rope(scaling=9)),
                dict(d_turns=ok + 4), dict(d_cu_new=None, num_rows=3), dict(d_lens_out=ok + 2)):
        assert B.cpa_latent_append(cfg, dims, **dict(base, **bad)) == B.CPA_EINVAL, bad
    io = dict(q_latent=ok, q_latent_block_stride=8192, q_latent_head_stride=512, q_rope=ok, q_rope_block_stride=1024, q_rope_head_stride=64,
              o=other, o_block_stride=8192, o_head_stride=512)
    dec = dict(d_tables=ok, io=B.cpa_latent_io(**io), d_lens=ok, d_active=None, pool=ok, d_workspace=ok)
    step = dict(dec, rope=_rope(), d_turns=ok, x=ok, x_row_stride=576, norm_weight=None, d_first=None, d_lens_out=other)
    bad_io = [dict(q_latent=0), dict(q_rope=0), dict(o=0), dict(q_latent=ok + 8), dict(q_rope=ok + 2), dict(o=other + 8), dict(o=ok),
              dict(q_latent_head_stride=516), dict(q_rope_block_stride=1), dict(o_head_stride=504), dict(o_block_stride=4096),
              dict(o_head_stride=-512), dict(o_block_stride=0), dict(q_latent_head_stride=0), dict(q_rope_block_stride=-1024),
              dict(q_rope_head_stride=0), dict(q_latent_block_stride=1 << 39)]
    for bad in [dict(io=B.cpa_latent_io(**dict(io, **b))) for b in bad_io] + [
            dict(d_tables=None), dict(d_lens=None), dict(pool=None), dict(d_workspace=None), dict(d_lens=ok + 2), dict(d_active=ok + 2),
            dict(pool=ok + 8), dict(d_workspace=ok + 8), dict(d_tables=ok + 4)]:
        assert B.cpa_latent_decode(cfg, dims, **dict(dec, **bad)) == B.CPA_EINVAL, bad
        assert B.cpa_latent_step(cfg, dims, **dict(step, **bad)) == B.CPA_EINVAL, bad
    for bad in (dict(x=None), dict(x=ok + 1), dict(x_row_stride=8), dict(d_lens_out=None), dict(d_lens_out=ok), dict(rope=None),
                dict(d_turns=None), dict(rope=_rope(128)), dict(norm_weight=ok + 8), dict(d_first=ok + 2)):
        assert B.cpa_latent_step(cfg, dims, **dict(step, **bad)) == B.CPA_EINVAL, bad
    bad_dims = B.cpa_table_dims(4, 0, 1 << 27, 8, 8)
    assert B.cpa_latent_append(cfg, bad_dims, **base) == B.CPA_EUNSUPPORTED
    assert B.cpa_latent_decode(cfg, bad_dims, **dec) == B.CPA_EUNSUPPORTED


def test_prefill_refusals():
    cfg, ok = _cfg(H=4), 1 << 20
    pc = B.cpa_latent_plan_config(cfg)
    assert (pc.num_q_heads, pc.num_kv_heads, pc.head_dim, pc.page_size) == (4, 4, 128, 16)
    plan = B.cpa_plan_create(pc, [100, 3], 0, list(range(8)))
    base = dict(plan=plan, q=ok, kv=ok + 4096, k_rope=ok + 8192, k_rope_row_stride=576, o=ok + 16384)
    assert B.cpa_latent_prefill(cfg, **base) == B.CPA_ESTATE               # not uploaded
    for bad in (dict(plan=0), dict(q=None), dict(kv=None), dict(k_rope=None), dict(o=None), dict(q=ok + 2), dict(kv=ok + 8), dict(k_rope=ok + 4),
                dict(o=ok + 8), dict(k_rope_row_stride=56), dict(k_rope_row_stride=100), dict(o=ok), dict(o=ok + 4096), dict(o=ok + 8192)):
        assert B.cpa_latent_prefill(cfg, **dict(base, **bad)) == B.CPA_EINVAL, bad
    for other in (_cfg(H=5), _cfg(H=4, scale=0.08)):
        assert B.cpa_latent_prefill(other, **base) == B.CPA_EINVAL
    pre = B.cpa_plan_create_prefix(pc, [100, 3], [0, 128], list(range(8, 16)), 0, list(range(8)))
    assert B.cpa_latent_prefill(cfg, **dict(base, plan=pre)) == B.CPA_EUNSUPPORTED
    B.cpa_plan_destroy(plan)
    B.cpa_plan_destroy(pre)


def test_tables_of_a_latent_cache_have_one_kv_head():
    for H in (1, 128):
        tc = B.cpa_latent_tables_config(_cfg(H=H, sms=7))
        assert (tc.num_q_heads, tc.num_kv_heads, tc.page_size, tc.num_sms) == (1, 1, 16, 7)
        assert B.cpa_tables_bytes(tc, B.cpa_table_dims(4, 0, 8, 8, 8)) > 0


def test_the_two_forms_are_one_attention():
    rng = np.random.default_rng(5)
    H, L, n, scale = 3, 128, 37, 0.1
    U, W = rng.standard_normal((H, 128, L)) / 8, rng.standard_normal((H, 128, L)) / 8
    rows, q = rng.standard_normal((n, L + 64)), rng.standard_normal((n, H, 192))
    kv = np.concatenate([np.einsum("hel,tl->the", U, rows[:, :L]), np.einsum("hel,tl->the", W, rows[:, :L])], 2)
    o = ol.prefill(q, kv, rows[:, L:], [0, n], scale)[0]
    for i in (0, 1, n - 1):
        qa = np.concatenate([np.einsum("hel,he->hl", U, q[i, :, :128]), q[i, :, 128:]], 1)
        got = np.einsum("hel,hl->he", W, ol.decode(qa, rows[:i + 1], L, scale)[0])
        assert np.allclose(got, o[i], atol=1e-12)


def test_oracle_turns_pairs_and_back():
    rng = np.random.default_rng(6)
    x, pos = rng.standard_normal((5, 3, 64)), rng.integers(-10 ** 6, 10 ** 6, (5, 1))
    f = ol.frequencies(64, 10000.0)
    for inter in (False, True):
        y = ol.turn(x, pos, f, inter, 1.25)
        assert np.allclose(ol.turn(y, pos, f, inter, 0.8, inverse=True), x, atol=1e-9)
        z = x[..., 0::2] + 1j * x[..., 1::2] if inter else x[..., :32] + 1j * x[..., 32:]
        w = z * 1.25 * np.exp(1j * pos[..., None] * f)
        got = y[..., 0::2] + 1j * y[..., 1::2] if inter else y[..., :32] + 1j * y[..., 32:]
        assert np.allclose(got, w)


@pytest.mark.parametrize("lens,H,want", [([1000], 16, 128), ([800, 900, 1000, 1050, 760], 3, 128), ([1024] * 32, 16, 256), ([8192, 4000, 1024], 64, 256),
                                         ([5], 1, 256), ([300] * 8, 16, 256), ([300, 500], 4, 128)])
def test_plans_of_a_latent_prefill_choose_their_items(lens, H, want):
    # few items: as many as there are SMs; long blocks: two sub-tiles that share K and V
    cfg = B.cpa_latent_config(H, 512, 64, 128, 128, 16, 0.07, 1e-6, 148)
    pc = B.cpa_latent_plan_config(cfg)
    assert pc.q_tile_rows == B.Q_TILE_LATENT
    pages = list(range(sum(-(-n // 16) for n in lens)))
    for rows, given in ((want, B.Q_TILE_LATENT), (128, 128), (256, 256)):
        pc.q_tile_rows = given
        plan = B.cpa_plan_create(pc, lens, 0, pages)
        assert B.cpa_plan_param(plan, B.PARAM_Q_TILE_ROWS) == rows
        B.cpa_plan_destroy(plan)


@pytest.mark.parametrize("first", [[], [5], [1, 2, 3], 7, [[1, 2]], [0, 2 ** 31 - 34], [-2 ** 31 - 1, 0], [2 ** 33, 0]])
def test_sessions_refuse_first_positions_that_are_not_one_per_block(first):
    # before anything touches a device: the kernels would read positions behind the array's end
    session = pytest.importorskip("paper_2605_23296_b200.session")
    with pytest.raises(ValueError, match="first"):
        session.LatentSession([10, 30], 4, 8, list(range(8)), 8, latent_dim=128, first=first)


def test_plans_of_a_latent_prefill_need_no_page_ids():
    # what the header promises: page 0 throughout, whatever the cache's own ids are, and the same schedule
    pc = B.cpa_latent_plan_config(_cfg(H=128, sms=148))
    lens = [300, 1, 700]
    pages = sum(-(-n // 16) for n in lens)
    with pytest.raises(B.CpaError):
        B.cpa_plan_create(pc, lens, 0, [1 << 25] * pages)
    plan = B.cpa_plan_create(pc, lens, 0, [0] * pages)
    assert B.cpa_plan_param(plan, B.PARAM_PAGES_USED) == pages
    B.cpa_plan_destroy(plan)
    tc = B.cpa_latent_tables_config(_cfg(H=128))
    assert B.cpa_tables_bytes(tc, B.cpa_table_dims(4, 0, (1 << 26) - 1, 8, 0)) > 0
    assert B.cpa_tables_bytes(tc, B.cpa_table_dims(4, 0, 1 << 26, 8, 0)) == B.CPA_EUNSUPPORTED


@pytest.mark.parametrize("name", ["latent_decode.cu", "latent_decode_pair.cu"])
def test_products_are_committed_by_the_lane_that_issues_them(name):
    # a commit follows the products of its own thread alone: the one behind which tensor memory is freed after a wait gave up has to come from
    # the elected lane too
    text = open(os.path.join(os.path.dirname(B.__file__), "csrc", name)).read().splitlines()
    drains = [i for i, line in enumerate(text) if re.search(r"commit_\w+\(bar\(&bars\.drain_", line)]
    assert len(drains) == 2
    for i in drains:
        assert "elect_one()" in text[i - 1], text[i - 1]


@pytest.mark.parametrize("scale", [1e-45, 1e-40, 2.0 ** -101, 2.0 ** 101, 2.9e38])
def test_scales_that_the_kernels_cannot_hold_are_refused(scale):
    # times log2(e) they would be flushed to zero (all tokens alike), or infinite (NaN throughout)
    assert B.cpa_latent_decode_workspace_bytes(_cfg(scale=scale)) == B.CPA_EINVAL
    for fine in (2.0 ** -100, 2.0 ** 100):
        assert B.cpa_latent_decode_workspace_bytes(_cfg(scale=fine)) > 0


def test_other_plans_do_not_take_the_latent_items():
    for Hq, Hkv, D in ((8, 2, 128), (8, 4, 128), (4, 4, 64), (8, 1, 64)):
        cfg = B.cpa_config(Hq, Hkv, D, 16, 0.1, B.Q_TILE_LATENT, 0, 148)
        with pytest.raises(B.CpaError) as e:
            B.cpa_plan_create(cfg, [100, 3], 0, list(range(8)))
        assert e.value.status == B.CPA_EUNSUPPORTED
        cfg.q_tile_rows = 0
        B.cpa_plan_destroy(B.cpa_plan_create(cfg, [100, 3], 0, list(range(8))))


def test_rows_are_packed_in_place_only_where_they_lie_packed():
    # a wider row would be overwritten by the row of another token before it is read
    cfg, dims, ok = _cfg(), B.cpa_table_dims(4, 0, 8, 8, 8), 1 << 20
    for stride in (577, 584, 1152):
        assert B.cpa_latent_append(cfg, dims, ok, None, None, ok, stride, None, None, 4, None, ok, ok + (1 << 16), ok, ok) == B.CPA_EINVAL


@pytest.mark.parametrize("amplitude", [1e-300, 1e-45, 1e-38, 9e-31])
def test_amplitudes_that_fp32_sines_cannot_hold_are_refused(amplitude):
    # they would come out as zeros
    assert B.cpa_rope_turns(_rope(amplitude=amplitude), check=False)[0] == B.CPA_EINVAL
    assert B.cpa_rope_turns(_rope(amplitude=1e-30), check=False)[0] == B.CPA_OK
