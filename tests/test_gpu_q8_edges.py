"""The 8-bit KV cache on the device at the edges of its numbers: values below fp32's normal range, scales of zero and
below it, scores beyond it; against the restatement in 64 bits (oracle/cache_q8.py)."""
import numpy as np
import pytest

from oracle import cache_q8 as oq
from test_gpu_q8 import B, Cache, _bf16, _i32, _values  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _steps(c, rng, what, kv=1.0):
    """A decode and two fused steps, each against the oracle."""
    n, hq = len(c.lens0), c.heads * c.group
    o, qf = c.decode(rng.standard_normal((n, hq, c.d)))
    c.check_rows(o, qf, what=f"{what} decode")
    for t in range(2):
        o, qf = c.step(rng.standard_normal((n, hq, c.d)), *(_values(rng, n, c.heads, c.d) * kv for _ in range(2)))
        c.check_rows(o, qf, what=f"{what} step {t}")
    c.check_pool(what)
    assert c.status() == c.B.CPA_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("num_sms", [0, 1])
def test_rows_below_the_normal_range_keep_their_values(B, d, num_sms):
    # V of 2^-131 .. 2^-127: bf16 holds them (down to 2^-133), and so has the output; one block is joined across CTAs
    lens = [3000, 20, 1]
    c = Cache(B, lens, 2, 2, d, seed=d, num_sms=num_sms)
    rng = np.random.default_rng(31)
    k, v = (_values(rng, sum(lens), 2, d) for _ in range(2))
    c.append(k, v * 2.0 ** -129, lens)
    q = rng.standard_normal((3, 8, d))
    o, qf = c.decode(q)
    c.check_rows(o, qf)
    assert (o[1:] != 0).any()
    o, qf = c.step(q, _values(rng, 3, 2, d), _values(rng, 3, 2, d) * 2.0 ** -129)
    c.check_rows(o, qf, what="step")
    c.check_pool()


def _set_scales(c, kind, pages, value):
    """Gives pages (positions in each block's list) of K (0) or V (1) a scale, on the device and in the oracle."""
    for b, n in enumerate(c.lens0):
        for j in range(-(-n // 16)):
            if pages(j, -(-n // 16)):
                pg = c.want.page_of(b, 16 * j)
                c.scales[pg, :, kind] = value
                c.want.scales[pg, :, kind] = value


WHERE = {"all": lambda j, n: True, "one warp": lambda j, n: j % 4 == 1, "another warp": lambda j, n: j % 4 == 2,
         "first round": lambda j, n: j < 16, "last round": lambda j, n: j >= n - 16, "even": lambda j, n: j % 2 == 0,
         "all but one": lambda j, n: j != 2}


@pytest.mark.parametrize("where", list(WHERE))
@pytest.mark.parametrize("value", [0.0, 2.0 ** -149, 2.0 ** -130, 1.25 * 2.0 ** -127])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_zero_and_below_the_normal_range(B, d, value, where):
    # what another writer gives a page of zeros; both directions of the walk (even and odd first lengths)
    for first, num_sms in ((700, 0), (701, 0), (700, 1), (701, 1)):
        c = Cache(B, [first, 33, 16, 640], 2, 2, d, 4, seed=d, num_sms=num_sms)
        rng = np.random.default_rng(first + d)
        n = sum(c.lens0)
        c.append(_values(rng, n, 2, d), _values(rng, n, 2, d), c.lens0)
        _set_scales(c, 1, WHERE[where], value)
        _steps(c, rng, f"{first} {num_sms}")


@pytest.mark.parametrize("value", [0.0, 2.0 ** -130])
def test_read_back_of_such_pages(B, value):
    c = Cache(B, [100], 0, 2, 64)
    rng = np.random.default_rng(3)
    c.append(_values(rng, 100, 2, 64), _values(rng, 100, 2, 64), [100])
    for kind in (0, 1):
        _set_scales(c, kind, WHERE["even"], value)
    out = torch.empty(2, 100, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, None, _i32([0, 100]), 100, c.pool, c.scales, out[0], out[1]) == 0
    want = torch.from_numpy(c.want.rows(0, 0, 100).transpose(0, 2, 1, 3)).bfloat16()     # (small ones are rounded once)
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_exp,k_exp,scale_exp", [(-118, 118, None), (118, -118, None), (118, None, -130), (100, None, -112),
                                                   (-100, 100, None)])
def test_scores_whose_factors_leave_the_normal_range(B, d, q_exp, k_exp, scale_exp):
    # scores of ordinary size out of a tiny query and huge keys, or the other way round
    c = Cache(B, [300, 17], 0, 2, d, 4, seed=d)
    rng = np.random.default_rng(41)
    k = _values(rng, 317, 2, d, 0.2).clip(-7, 7) * 2.0 ** (k_exp or 0)
    c.append(k, _values(rng, 317, 2, d), [300, 17])
    if scale_exp is not None:
        _set_scales(c, 0, WHERE["all"], 2.0 ** scale_exp)
    o, qf = c.decode(rng.standard_normal((2, 8, d)) * 2.0 ** q_exp)
    c.check_rows(o, qf)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_minus_infinity_beside_a_zero(B, d):
    # keys so large that their scores pass fp32's range downwards take no weight, and do not spoil the keys of zeros in
    # their own pages: the answer is the mean of the zero keys' values
    n = 330
    c = Cache(B, [n, n + 1], 0, 1, d, 1, seed=d)
    rng = np.random.default_rng(42)
    q = rng.choice([-1.0, 1.0], (2, 1, d)) * 2.0 ** 60
    zero = (rng.random(2 * n + 1) < 0.1) | (np.arange(2 * n + 1) % 8 == 3)       # some in every page
    k = np.concatenate([np.repeat(-q[0][None], n, 0), np.repeat(-q[1][None], n + 1, 0)]) * 2.0 ** 40
    k[zero] = 0.0
    v = rng.standard_normal((2 * n + 1, 1, d))
    c.append(k, v, [n, n + 1])
    o, _ = c.decode(q)
    for b, (lo, hi) in enumerate(((0, n), (n, 2 * n + 1))):
        rows = c.want.rows(b, 0, hi - lo)[1, 0][zero[lo:hi]]
        want, spread = rows.mean(0), np.abs(rows).mean(0)
        off = np.abs(o[b, 0].double().cpu().numpy() - want)
        assert (off <= oq.decode_tolerance(want, spread, 0.0, d)).all(), off.max()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 1, 5, 18, 41])
def test_whole_pages_of_minus_infinity(B, d, page):
    # every score but those of one page passes fp32's range downwards: warps, rounds and whole ranges meet nothing else
    n = 700
    for more in (0, 1):
        c = Cache(B, [n + more, 64], 0, 1, d, 1, seed=d)
        rng = np.random.default_rng(43)
        q = rng.choice([-1.0, 1.0], (2, 1, d)) * 2.0 ** 37
        k = np.repeat(-q[0][None], n + more + 64, 0) * 2.0 ** 63
        k[16 * page:16 * page + 16] = 0.0
        k[n + more:] = 0.0
        v = rng.standard_normal((n + more + 64, 1, d))
        c.append(k, v, [n + more, 64])
        o, _ = c.decode(q)
        for b, rows in enumerate((c.want.rows(0, 16 * page, min(16 * page + 16, n + more))[1, 0], c.want.rows(1, 0, 64)[1, 0])):
            want, spread = rows.mean(0), np.abs(rows).mean(0)
            off = np.abs(o[b, 0].double().cpu().numpy() - want)
            assert (off <= oq.decode_tolerance(want, spread, 0.0, d)).all(), (more, b, off.max())


def test_a_row_of_nothing_but_minus_infinity_is_nan(B):
    c = Cache(B, [100], 0, 1, 64, 1)
    q = np.full((1, 1, 64), 2.0 ** 37)
    c.append(np.full((100, 1, 64), -2.0 ** 100), np.ones((100, 1, 64)), [100])
    o, _ = c.decode(q)
    assert torch.isnan(o).all()


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("old", [2.0 ** -130, 2.0 ** -149, 1.5 * 2.0 ** -128, 0.0])
def test_append_to_pages_whose_scale_is_below_the_normal_range(B, d, old, fused):
    # another writer's page: its codes are rounded again to the new scale, not lost
    c = Cache(B, [21, 40], 8, 2, d, 2)
    rng = np.random.default_rng(51)
    c.append(_values(rng, 61, 2, d), _values(rng, 61, 2, d), [21, 40])
    for kind in (0, 1):
        _set_scales(c, kind, WHERE["all"], old)
    for t in range(3):
        k, v = (_values(rng, 2, 2, d) * 2.0 ** (6 * t - 122) for _ in range(2))
        if fused:
            o, qf = c.step(rng.standard_normal((2, 4, d)), k, v)
            c.check_rows(o, qf, what=f"step {t}")
        else:
            c.append(k, v)
        c.check_pool(f"token {t}")


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_tiny_rows_under_a_scale_that_is_no_power_of_two(B, d, fused):
    # rows below fp32's normal range, divided by a kept scale of 1.5 * 2^-126.  (A bf16 value over 1.5 is a midpoint of two
    # codes exactly or by 2^-9 of itself at least, so the 32-bit quotient rounds to the code that the 64-bit one gives.)
    c = Cache(B, [21, 40], 8, 2, d, 2)
    rng = np.random.default_rng(52)
    c.append(_values(rng, 61, 2, d) * 2.0 ** -120, _values(rng, 61, 2, d) * 2.0 ** -120, [21, 40])
    for kind in (0, 1):
        _set_scales(c, kind, WHERE["all"], 1.5 * 2.0 ** -126)
    for t in range(3):
        k, v = (_values(rng, 2, 2, d) * 2.0 ** (t - 129) for _ in range(2))
        if fused:
            c.step(rng.standard_normal((2, 4, d)), k, v)
        else:
            c.append(k, v)
        c.check_pool(f"token {t}")


def test_tables_rebuilt_between_calls_without_a_wait(B):
    # two events take turns on one table buffer, one workspace and one pool: build, append by the tables' own cu_seqlens,
    # decode, step and read-back follow one another with nothing between them, so that every call begins while the one
    # before it still writes what it is going to read
    heads, group, d, blocks = 2, 4, 128, 5
    rng = np.random.default_rng(71)
    events = [[700, 3, 0, 64, 17], [16, 41, 900, 1, 33]]
    need = max(sum(-(-(n + 1) // 16) for n in lens) for lens in events)
    rows = max(sum(lens) for lens in events)
    pages = 2 * need
    ids = rng.permutation(pages).astype(np.int32)
    cfg = B.cpa_config(heads * group, heads, d, 16, d ** -0.5, 0, 0, 0)
    dims = B.cpa_table_dims(blocks, 1, pages, need, 0)
    tables = torch.empty(B.cpa_tables_bytes(cfg, dims), dtype=torch.uint8, device="cuda")
    ws = torch.empty(B.cpa_decode_q8_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    at = B.cpa_tables_offset(cfg, dims, B.ARR_CU_SEQLENS)
    cu = tables[at:at + 4 * (blocks + 1)].view(torch.int32)
    pool = torch.full((pages, heads, 2, 16, d), 0x7F, dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, heads, 2), float("nan"), device="cuda")
    turns = 24
    ins, outs = [], []
    for i, lens in enumerate(events):
        k, v, q = (_bf16(x) for x in (_values(rng, rows, heads, d), _values(rng, rows, heads, d), rng.standard_normal((2, blocks, heads * group, d))))
        k1, v1 = (_bf16(_values(rng, blocks, heads, d)) for _ in range(2))
        ins.append((_i32(lens), _i32(ids[i * need:(i + 1) * need]), k, v, q, k1, v1))
    for _ in range(turns):
        outs.append([torch.full((2, blocks, heads * group, d), 9.0, dtype=torch.bfloat16, device="cuda"),
                     torch.full((2, rows, heads, d), 9.0, dtype=torch.bfloat16, device="cuda"),
                     torch.full((2, blocks), -7, dtype=torch.int32, device="cuda")])
    torch.cuda.synchronize()
    for t in range(turns):
        lens, free, (k, _), (v, _), (q, _), (k1, _), (v1, _) = ins[t % 2]
        o, kv, n = outs[t]
        rc = [B.cpa_tables_build(cfg, dims, lens, free, need, tables),
              B.cpa_kv_append_q8(cfg, dims, tables, k, v, cu, rows, None, n[0], pool, scales),
              B.cpa_decode_q8(cfg, dims, tables, q[0], n[0], None, pool, scales, o[0], ws),
              B.cpa_decode_append_q8(cfg, dims, tables, q[1], k1, v1, n[0], n[1], None, pool, scales, o[1], ws),
              B.cpa_kv_read_q8(cfg, dims, tables, None, cu, rows, pool, scales, kv[0], kv[1])]
        assert rc == [0] * 5
    assert B.cpa_tables_status(tables) == B.CPA_OK
    for i, lens in enumerate(events):
        want = oq.CacheQ8(pages, heads, d, lens, 1, ids[i * need:(i + 1) * need])
        (_, kf), (_, vf), (_, qf), (_, k1f), (_, v1f) = ins[i][2:]
        o, kv, n = outs[i]
        where = np.concatenate([[0], np.cumsum(lens)])
        scale = float(np.float32(d ** -0.5))
        for b, m in enumerate(lens):
            want.append(b, kf[where[b]:where[b] + m], vf[where[b]:where[b] + m])
            first = want.rows(b, 0, m)
            exact = want.decode(b, qf[0, b], scale)
            assert (np.abs(o[0, b].double().cpu().numpy() - exact[0]) <= oq.decode_tolerance(*exact, d)).all(), (i, b)
            want.append(b, k1f[b:b + 1], v1f[b:b + 1])
            exact = want.decode(b, qf[1, b], scale)
            assert (np.abs(o[1, b].double().cpu().numpy() - exact[0]) <= oq.decode_tolerance(*exact, d)).all(), (i, b)
            # (the read comes behind the step, whose token may have made the last page's scale grow: whole pages only)
            whole = m // 16 * 16
            assert np.array_equal(kv[:, where[b]:where[b] + whole].double().cpu().numpy(), first[:, :, :whole].transpose(0, 2, 1, 3))
        assert n.tolist() == [lens, [m + 1 for m in lens]] and (kv[:, where[-1]:] == 9).all()
        for t in range(i, turns, 2):
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs[t], outs[i])), t


RANGES = {"far back": [0, 320, 16, 160], "to the start": [0, 1000, 0, 16], "into the one before": [0, 100, 50, 150],
          "twice": [0, 500, 500, 20, 300, 10, 10, 700], "first not at 0": [64, 100, 37, 37, 90], "past the end": [0, 200, 5000, 100, 260],
          "negative": [0, 100, -50, 300, 400], "in order": [0, 100, 100, 117, 400]}
for _seed, _blocks in ((1, 40), (2, 40), (3, 33), (4, 1100)):
    RANGES[f"{_blocks} at random, {_seed}"] = [int(x) for x in np.random.default_rng(_seed).integers(0, 500, _blocks + 1)]
_r = [16 * i for i in range(1101)]
_r[600], _r[17], _r[1000] = 40, 17600, 0
RANGES["few of many"] = _r


@pytest.mark.parametrize("name", list(RANGES))
def test_a_bad_range_costs_no_other_block_its_rows(B, name):
    cu = RANGES[name]
    rows = max(1000, max(x for x in cu if x < 5000)) if "past" in name else max(max(cu), 1)
    blocks, d, heads = len(cu) - 1, 64, 1
    n = [b - a for a, b in zip(cu, cu[1:])]
    good = [b for b in range(blocks) if n[b] >= 0 and cu[b] >= 0 and cu[b + 1] <= rows]
    c = Cache(B, [5 + (n[b] if b in set(good) else 0) for b in range(blocks)], 0, heads, d, 1)
    rng = np.random.default_rng(61)
    c.append(_values(rng, 5 * blocks, heads, d), _values(rng, 5 * blocks, heads, d), [5] * blocks)
    (kd, kf), (vd, vf) = (_bf16(_values(rng, rows, heads, d)) for _ in range(2))
    out = torch.full_like(c.lens, -7)
    assert B.cpa_kv_append_q8(c.cfg, c.dims, c.tables, kd, vd, _i32(cu), rows, c.lens, out, c.pool, c.scales) == 0
    assert c.status() == (B.CPA_OK if len(good) == blocks else B.CPA_EINVAL)
    for b in good:
        c.want.append(b, kf[cu[b]:cu[b + 1]], vf[cu[b]:cu[b + 1]])
    c.lens = out
    c.check_pool()                       # every good block has its rows and its length, every other one what it had
    # the same ranges read back; a row that two blocks' ranges share may hold either's
    first = [5 if b in set(good) else 0 for b in range(blocks)]
    k_out, v_out = (torch.full((rows + 2, heads, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, _i32(first), _i32(cu), rows, c.pool, c.scales, k_out, v_out) == 0
    owners = np.zeros(rows + 2, dtype=int)
    for b in good:
        owners[cu[b]:cu[b + 1]] += 1
    got = [t.double().cpu().numpy() for t in (k_out, v_out)]
    for b in good:
        want = c.want.rows(b, 5, 5 + n[b])
        alone = np.flatnonzero(owners[cu[b]:cu[b + 1]] == 1)
        for i in range(2):
            assert np.array_equal(got[i][cu[b] + alone], want[i].transpose(1, 0, 2)[alone]), b
    for i in range(2):
        assert (got[i][owners == 0] == 9).all() and (got[i][owners > 0] != 9).any(axis=(1, 2)).all()


def _check_with_floors(c, o, qf, what):
    for b in range(len(c.lens0)):
        want = c.want.decode(b, qf[b], c.scale)
        tol = oq.decode_tolerance(*want, c.d, *c.want.floors(b, qf[b], c.scale))
        off = np.abs(o[b].double().cpu().numpy() - want[0])
        assert (off <= tol).all(), f"{what}: off {off.max():.3g}, {(off / tol).max():.2f} of the bound"
    return want[0]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [4, 12, 16, 20, 24, 32, 60])
def test_small_scales_beside_large_ones_in_other_dimensions(B, d, gap):
    # page 0 of each round holds 2^gap in dimension 0 alone, the others 1 in dimension 1 alone, at equal scores: dimension 1
    # is what the small scales add.  Up to 2^20 no weight is subnormal (the scales lie 2^gap apart), and nothing is lost
    c = Cache(B, [320], 0, 1, d, 2)
    rng = np.random.default_rng(81)
    v = np.zeros((320, 1, d))
    large = np.arange(320) // 16 % 4 == 0
    v[large, 0, 0], v[~large, 0, 1] = 2.0 ** gap, 1.0
    c.append(np.zeros((320, 1, d)), v, [320])
    o, qf = c.decode(rng.standard_normal((1, 2, d)))
    want = _check_with_floors(c, o, qf, gap)
    if gap <= 20:
        assert (np.abs(o[0, :, 1].double().cpu().numpy() / want[:, 1] - 1) <= 2.0 ** -8 + 2.0 ** -10).all()
    # all 320 tokens small but the page of one warp: the others do not share its maximum
    c = Cache(B, [320], 0, 1, d, 2, num_sms=1)
    v = rng.standard_normal((320, 1, d))
    v[:16] = 0.0
    v[:16, 0, 0] = 2.0 ** gap
    c.append(rng.standard_normal((320, 1, d)), v, [320])
    o, qf = c.decode(rng.standard_normal((1, 2, d)))
    _check_with_floors(c, o, qf, gap)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [4, 12, 18, 22, 28, 34, 60])
def test_small_weights_beside_a_large_one_in_other_dimensions(B, d, gap):
    # one key outweighs every other by 2^gap and has values in dimension 0 alone
    for at in (0, 17, 200, 319):
        c = Cache(B, [320], 0, 1, d, 1, scale=float(np.log(2)))
        rng = np.random.default_rng(82)
        k, v = np.zeros((320, 1, d)), rng.standard_normal((320, 1, d))
        k[at, 0, 0] = gap
        v[:, 0, 0], v[at] = 0.0, 0.0
        v[at, 0, 0] = 1.0
        c.append(k, v, [320])
        q = np.zeros((1, 1, d))
        q[0, 0, 0] = 1.0
        o, qf = c.decode(q)
        _check_with_floors(c, o, qf, (gap, at))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [10, 18, 22, 24, 26, 30, 34])
def test_small_query_elements_beside_a_large_one(B, d, gap):
    # the row's largest element meets keys of zeros: the scores come from elements 2^gap below it
    c = Cache(B, [150, 33], 0, 1, d, 2, scale=1.0)
    rng = np.random.default_rng(83)
    k = rng.standard_normal((183, 1, d)) * 2.0 ** (gap - 4)
    k[:, 0, 0] = 0.0
    c.append(k, rng.standard_normal((183, 1, d)), [150, 33])
    q = rng.standard_normal((2, 2, d)) * 2.0 ** -gap
    q[:, :, 0] = 1.5
    o, qf = c.decode(q)
    _check_with_floors(c, o, qf, gap)


def test_a_capture_with_copies_and_a_second_stream(B):
    # copies in front of the calls, a fork to another stream and a join: programmatic launches behind nodes of every kind
    rng = np.random.default_rng(91)
    lens = [200, 33]
    caches = []
    for i in range(2):
        c = Cache(B, lens, 8, 2, 64, seed=i)
        c.append(*(_values(rng, sum(lens), 2, 64) for _ in range(2)), lens)
        caches.append(c)
    src = [torch.zeros(2, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2)]
    buf = [torch.zeros_like(t) for t in src]
    new = [torch.zeros_like(c.lens) for c in caches]
    o = [torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in caches]
    total = torch.zeros(2, 8, 64, device="cuda")
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def step(i, on):
        c = caches[i]
        assert B.cpa_decode_append_q8(c.cfg, c.dims, c.tables, *buf, c.lens, new[i], None, c.pool, c.scales, o[i][0], c.ws, on.cuda_stream) == 0

    def decode(i, on):
        c = caches[i]
        assert B.cpa_decode_q8(c.cfg, c.dims, c.tables, buf[0], new[i], None, c.pool, c.scales, o[i][1], c.ws, on.cuda_stream) == 0

    def both():
        for a, b in zip(buf, src):
            a.copy_(b)
        step(0, main)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            step(1, side)
            caches[1].lens.copy_(new[1])
        decode(0, main)
        caches[0].lens.copy_(new[0])
        main.wait_stream(side)
        decode(1, main)
        total.copy_(o[0][1].float() + o[1][1].float())

    torch.cuda.synchronize()
    keep = [(c.pool.clone(), c.scales.clone(), c.lens.clone()) for c in caches]
    with torch.cuda.stream(main):
        both()
    torch.cuda.synchronize()
    for c, (pool, scales, n) in zip(caches, keep):
        c.pool.copy_(pool), c.scales.copy_(scales), c.lens.copy_(n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        both()
    for r in range(4):
        vals = [_bf16(x) for x in (rng.standard_normal((2, 8, 64)), _values(rng, 2, 2, 64), _values(rng, 2, 2, 64))]
        for t, (x, _) in zip(src, vals):
            t.copy_(x)
        graph.replay()
        for i, c in enumerate(caches):
            for b in range(2):
                c.want.append(b, vals[1][1][b:b + 1], vals[2][1][b:b + 1])
            c.check_rows(o[i][0], vals[0][1], what=f"replay {r} step {i}")
            assert torch.equal(o[i][0], o[i][1])
            c.check_pool(f"replay {r} cache {i}")
        assert torch.equal(total, o[0][1].float() + o[1][1].float())
    assert all(c.status() == B.CPA_OK for c in caches)
