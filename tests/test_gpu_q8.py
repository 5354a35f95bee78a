"""The 8-bit KV cache on the device against its restatement in 64 bits (oracle/cache_q8.py): the tables and the stored
codes and scales bit for bit, attention within the bounds that decode_tolerance derives."""
import numpy as np
import pytest

from oracle import cache_q8 as oq

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def B():
    from paper_2605_23296_b200 import binding
    return binding


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _bf16(x):
    """float64 values rounded to bf16: the device tensor, and the same values in float64."""
    t = torch.tensor(np.ascontiguousarray(x), dtype=torch.float64).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


class Cache:
    """A device cache beside the oracle's, filled by the calls under test.  Unfilled slots hold NaN."""

    def __init__(self, B, lens, max_new, heads, d, group=4, extra_pages=3, seed=0, num_sms=0, scale=None, page_ids=None):
        rng = np.random.default_rng(seed)
        self.B, self.lens0, self.heads, self.d, self.group = B, list(lens), heads, d, group
        need = sum(-(-(n + max_new) // oq.P) for n in lens)
        self.num_pages = need + extra_pages
        ids = rng.permutation(self.num_pages).astype(np.int32)
        if page_ids is not None:
            ids, self.num_pages = page_ids(need, rng)
        self.scale = float(np.float32(scale or d ** -0.5))
        self.cfg = B.cpa_config(heads * group, heads, d, 16, self.scale, 0, 0, num_sms)
        self.dims = B.cpa_table_dims(len(lens), max_new, self.num_pages, len(ids), max(1, sum(lens)))
        self.tables = torch.full((B.cpa_tables_bytes(self.cfg, self.dims),), 0xAB, dtype=torch.uint8, device="cuda")
        self.ids = _i32(ids)
        rc = B.cpa_tables_build(self.cfg, self.dims, _i32(lens), self.ids, len(ids), self.tables)
        assert rc == 0
        self.pool = torch.full((self.num_pages, heads, 2, 16, d), 0x7F, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((self.num_pages, heads, 2), float("nan"), device="cuda")
        self.ws = torch.full((B.cpa_decode_q8_workspace_bytes(self.cfg),), 0xFF, dtype=torch.uint8, device="cuda")
        self.lens = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
        self.want = oq.CacheQ8(self.num_pages if page_ids is None else 1, heads, d, lens, max_new, ids)

    def array(self, which, n):
        at = self.B.cpa_tables_offset(self.cfg, self.dims, which) // 4
        return self.tables.view(torch.int32)[at:at + n].cpu().numpy()

    def status(self):
        return self.B.cpa_tables_status(self.tables)

    def append(self, k, v, counts=None, want=True):
        """k, v float64 [rows, heads, d]; counts: rows per block (None: one each)."""
        (kd, kf), (vd, vf) = _bf16(k), _bf16(v)
        out = torch.full_like(self.lens, -7)
        cu = None if counts is None else _i32(np.concatenate([[0], np.cumsum(counts)]))
        rc = self.B.cpa_kv_append_q8(self.cfg, self.dims, self.tables, kd, vd, cu, len(k), self.lens, out, self.pool,
                                     self.scales)
        assert rc == 0
        if want:
            at = 0
            for b, n in enumerate(counts if counts is not None else [1] * len(self.lens0)):
                self.want.append(b, kf[at:at + n], vf[at:at + n])
                at += n
        self.lens = out
        return kd, vd

    def decode(self, q, active=None, fill=None):
        qd, qf = _bf16(q)
        o = torch.full_like(qd, 9.0 if fill is None else fill)
        rc = self.B.cpa_decode_q8(self.cfg, self.dims, self.tables, qd, self.lens, active, self.pool, self.scales, o, self.ws)
        assert rc == 0
        return o, qf

    def step(self, q, k, v, active=None):
        (qd, qf), (kd, kf), (vd, vf) = _bf16(q), _bf16(k), _bf16(v)
        o, out = torch.full_like(qd, 9.0), torch.full_like(self.lens, -7)
        rc = self.B.cpa_decode_append_q8(self.cfg, self.dims, self.tables, qd, kd, vd, self.lens, out, active, self.pool,
                                         self.scales, o, self.ws)
        assert rc == 0
        for b in range(len(self.lens0)):
            if active is None or int(active[b]):
                self.want.append(b, kf[b:b + 1], vf[b:b + 1])
        self.lens = out
        return o, qf

    def check_pool(self, what=""):
        assert self.lens.cpu().tolist() == self.want.lens.tolist(), what
        want = np.where(np.isnan(self.want.codes), 0x7F, oq.e4m3_bits(self.want.codes))
        got = self.pool.cpu().numpy()
        wrong = got != want
        assert not wrong.any(), f"{what}: {wrong.sum()} codes differ, first at {np.argwhere(wrong)[0]}"
        s = self.scales.cpu().numpy().astype(np.float64)
        assert np.array_equal(s, self.want.scales, equal_nan=True), what

    def check_rows(self, o, qf, blocks=None, what=""):
        got = o.double().cpu().numpy()
        for b in range(len(self.lens0)) if blocks is None else blocks:
            want, spread, shaken = self.want.decode(b, qf[b], self.scale)
            tol = oq.decode_tolerance(want, spread, shaken, self.d)
            off = np.abs(got[b] - want)
            assert (off <= tol).all(), f"{what} block {b} of {self.want.lens[b]}: off {off.max():.3g}, {(off / tol).max():.2f} of the bound"


def _values(rng, n, heads, d, spread=0.5):
    x = rng.standard_normal((n, heads, d)) * np.exp(spread * rng.standard_normal((n, heads, 1)))
    x[rng.random((n, heads)) < 1 / 64] *= 8
    return x


# ------------------------------------------------------------------------------------------------ tables

LENS = [[1], [16], [0], [7, 0, 0, 16, 17, 4097, 1, 0], [512 + 37 * i % 511 for i in range(192)], [0] * 70 + [5],
        [(i * 7919) % 40 for i in range(5000)], [100000, 3, 31111]]


@pytest.mark.parametrize("max_new", [0, 1, 33])
@pytest.mark.parametrize("lens", LENS, ids=lambda v: f"{len(v)}x{max(v)}")
def test_tables_match_the_definition(B, lens, max_new):
    rng = np.random.default_rng(len(lens))
    need = sum(-(-(n + max_new) // 16) for n in lens)
    num_pages = need + 5
    free = rng.permutation(num_pages).astype(np.int32)
    cfg, dims = B.cpa_config(8, 2, 64, 16, 1.0, 0, 0, 0), B.cpa_table_dims(len(lens), max_new, num_pages, num_pages, sum(lens) + 9)
    t = torch.full((B.cpa_tables_bytes(cfg, dims),), 0xAB, dtype=torch.uint8, device="cuda")
    for _ in range(2):                        # built twice over the same buffer
        assert B.cpa_tables_build(cfg, dims, _i32(lens), _i32(free), num_pages, t) == 0
    assert B.cpa_tables_status(t) == B.CPA_OK
    cu, indptr, pages, slots = oq.tables(lens, max_new, free)
    ints = t.view(torch.int32).cpu().numpy()
    for which, want, size in ((B.ARR_CU_SEQLENS, cu, len(cu)), (B.ARR_PAGE_INDPTR, indptr, len(cu)),
                              (B.ARR_PAGE_INDICES, pages, num_pages), (B.ARR_SLOT_MAPPING, slots, sum(lens) + 9)):
        at = B.cpa_tables_offset(cfg, dims, which) // 4
        got = ints[at:at + size]
        assert np.array_equal(got[:len(want)], want), which
        assert (got[len(want):].view(np.uint32) == 0xABABABAB).all(), which      # behind the last: as it was


def test_tables_match_the_host_plan(B):
    lens, max_new = [1, 16, 700, 33, 4095, 2], 19
    free = np.random.default_rng(1).permutation(400).astype(np.int32)
    cfg = B.cpa_config(8, 2, 64, 16, 1.0, 0, 0, 0)
    plan = B.cpa_plan_create(cfg, lens, max_new, free)
    dims = B.cpa_table_dims(len(lens), max_new, 400, 400, sum(lens))
    t = torch.empty(B.cpa_tables_bytes(cfg, dims), dtype=torch.uint8, device="cuda")
    assert B.cpa_tables_build(cfg, dims, _i32(lens), _i32(free), 400, t) == 0
    ints = t.view(torch.int32).cpu().numpy()
    for which in (B.ARR_CU_SEQLENS, B.ARR_PAGE_INDPTR, B.ARR_PAGE_INDICES, B.ARR_SLOT_MAPPING):
        want = B.cpa_plan_export(plan, which)
        at = B.cpa_tables_offset(cfg, dims, which) // 4
        assert np.array_equal(ints[at:at + len(want)], want), which
    B.cpa_plan_destroy(plan)


@pytest.mark.parametrize("lens,num_free,page_cap,token_cap,bad_id,want", [
    ([5, -1, 9], 10, 10, 64, None, "CPA_EINVAL"), ([5, 17, 9], 3, 10, 64, None, "CPA_ENOSPC"),
    ([5, 17, 9], 10, 3, 64, None, "CPA_ENOSPC"), ([5, 17, 9], 10, 10, 30, None, "CPA_ENOSPC"),
    ([2 ** 30, 2 ** 30, 2 ** 30], 10, 10, 0, None, "CPA_ENOSPC"), ([5, 17, 9], 4, 4, 31, None, "CPA_OK"),
    ([5, 17, 9], 10, 10, 31, -1, "CPA_EINVAL"), ([5, 17, 9], 10, 10, 31, 10, "CPA_EINVAL")])
def test_tables_of_bad_lengths_are_empty_and_say_so(B, lens, num_free, page_cap, token_cap, bad_id, want):
    cfg, dims = B.cpa_config(8, 2, 64, 16, 1.0, 0, 0, 0), B.cpa_table_dims(3, 0, 10, page_cap, token_cap)
    t = torch.full((B.cpa_tables_bytes(cfg, dims),), 0xAB, dtype=torch.uint8, device="cuda")
    ids = np.arange(10, dtype=np.int32)[::-1].copy()
    if bad_id is not None:
        ids[2] = bad_id
    assert B.cpa_tables_build(cfg, dims, _i32(lens), _i32(ids), num_free, t) == 0
    assert B.cpa_tables_status(t) == getattr(B, want)
    ints = t.view(torch.int32).cpu().numpy()
    cu, ip, pg, sl = (ints[B.cpa_tables_offset(cfg, dims, w) // 4:][:n] for w, n in (
        (B.ARR_CU_SEQLENS, 4), (B.ARR_PAGE_INDPTR, 4), (B.ARR_PAGE_INDICES, page_cap), (B.ARR_SLOT_MAPPING, token_cap)))
    if want != "CPA_OK" and bad_id is None:
        assert not cu.any() and not ip.any()
        # the calls on such tables touch nothing; blocks of length zero still get their rows of zeros
        pool = torch.full((10, 2, 2, 16, 64), 0x55, dtype=torch.uint8, device="cuda")
        scales, q = torch.ones(10, 2, 2, device="cuda"), torch.ones(3, 8, 64, dtype=torch.bfloat16, device="cuda")
        kv, o = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.full_like(q, 9.0)
        ws = torch.empty(B.cpa_decode_q8_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        out = _i32([-7, -7, -7])
        assert B.cpa_kv_append_q8(cfg, dims, t, kv, kv, None, 3, None, out, pool, scales) == 0
        assert out.tolist() == [0, 0, 0] and (pool == 0x55).all() and (scales == 1).all()
        assert B.cpa_decode_q8(cfg, dims, t, q, out, None, pool, scales, o, ws) == 0
        assert (o == 0).all()
        assert B.cpa_decode_append_q8(cfg, dims, t, q, kv, kv, out, _i32([0, 0, 0]), None, pool, scales, o.fill_(9), ws) == 0
        assert (o == 9).all() and (pool == 0x55).all()
    elif bad_id is not None:
        assert pg[2] == 0 and pg[0] == 9 and pg[1] == 8 and sl[5 + 16] == 0 and sl[5] == 8 * 16
    else:
        assert cu.tolist() == [0, 5, 22, 31] and sl[30] == 6 * 16 + 8


# ------------------------------------------------------------------------------------------------ append and read

@pytest.mark.parametrize("heads,d", [(1, 64), (2, 128), (8, 64), (3, 128)])
def test_append_prompts_chunks_and_tokens(B, heads, d):
    lens = [1, 15, 16, 17, 0, 95, 300]
    c = Cache(B, lens, 64, heads, d, seed=heads + d)
    rng = np.random.default_rng(heads * d)
    for counts in (lens, [3, 0, 16, 15, 1, 33, 0], None, [0, 1, 0, 0, 31, 0, 2], None, None):
        n = len(lens) if counts is None else sum(counts)
        # later rows are larger: pages that hold tokens have to grow their scale
        x = [_values(rng, n, heads, d) * rng.choice([1.0, 4.0, 64.0], (n, 1, 1)) for _ in range(2)]
        c.append(*x, counts)
        c.check_pool(str(counts))
    assert c.status() == B.CPA_OK
    # everything read back, and a range from odd positions
    for first in (None, [min(5 * b, int(n)) for b, n in enumerate(c.want.lens)]):
        f = first or [0] * len(lens)
        n = [int(t) - a for t, a in zip(c.want.lens, f)]
        cu = np.concatenate([[0], np.cumsum(n)])
        out = torch.full((2, int(cu[-1]) + 4, heads, d), 9.0, dtype=torch.bfloat16, device="cuda")
        assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, None if first is None else _i32(f), _i32(cu), out.shape[1], c.pool,
                                c.scales, out[0], out[1]) == 0
        want = np.concatenate([c.want.rows(b, a, a + m) for b, (a, m) in enumerate(zip(f, n))], 2).transpose(0, 2, 1, 3)
        assert np.array_equal(out[:, :-4].double().cpu().numpy(), want)      # code * 2^e is a bf16 value
        assert (out[:, -4:] == 9).all()


def test_append_special_values(B):
    c = Cache(B, [40], 0, 2, 64)
    rng = np.random.default_rng(5)
    k, v = _values(rng, 40, 2, 64), _values(rng, 40, 2, 64)
    k[3, 0, 7], k[4, 1, 0], v[5, 0, 1], v[20, 1, 2], v[21, 1, 3] = np.inf, -np.inf, np.nan, np.nan, np.inf
    k[16:32] = 0.0                       # a page of zeros
    v[32:, 0] *= 2.0 ** -120             # tiny, subnormal in bf16 in part
    v[32:, 1] *= 2.0 ** 120
    k[33, 0] = 448.0 / 8                 # the border of a scale
    c.append(k, v, [40])
    got = c.pool.cpu().numpy()
    want = oq.e4m3_bits(c.want.codes)
    nan = np.isnan(c.want.codes)
    assert np.array_equal(got[~nan], want[~nan])
    assert ((got[nan] & 0x7F) == 0x7F).all()
    assert np.array_equal(c.scales.cpu().numpy().astype(np.float64), c.want.scales, equal_nan=True)


def test_append_growth_from_the_smallest_to_the_largest_scale(B):
    c = Cache(B, [16], 0, 1, 64)
    rng = np.random.default_rng(6)
    for i in range(16):
        size = 2.0 ** (-130 + 17 * i)
        c.append(*(rng.standard_normal((1, 1, 64)) * size * (0.25 if i == 15 else 1) for _ in range(2)), [1])
        c.check_pool(f"token {i}")


def test_append_leaves_out_blocks_without_room_or_with_bad_ranges(B):
    c = Cache(B, [16, 16, 16, 16], 0, 2, 64)
    rng = np.random.default_rng(7)
    c.append(*(_values(rng, 40, 2, 64) for _ in range(2)), [10, 10, 10, 10])
    before, scales = c.pool.clone(), c.scales.clone()
    k, v = (_values(rng, 20, 2, 64) for _ in range(2))
    c.append(k, v, [6, 7, 0, 6], want=False)           # block 1 has room for 6
    assert c.lens.tolist() == [16, 10, 10, 16] and c.status() == B.CPA_ENOSPC
    p = [int(c.want.page_of(b, 0)) for b in range(4)]
    for b in (1, 2):
        assert torch.equal(c.pool[p[b]], before[p[b]]) and torch.equal(c.scales[p[b]], scales[p[b]])
    assert (c.pool[p[0], :, :, 10:] != 0x7F).any() and (c.pool[p[3], :, :, 10:] != 0x7F).any()
    # ranges that leave the packed rows, or run backwards; a negative length
    for lens, cu in (([10, 10, 10, 10], [0, 2, 1, 1, 2]), ([10, 10, 10, 10], [0, 0, 0, 0, 21]), ([10, -1, 10, 10], [0, 0, 1, 1, 1])):
        c2 = Cache(B, [16, 16, 16, 16], 0, 2, 64)
        before = c2.pool.clone()
        out, kd = _i32([-7] * 4), torch.ones(20, 2, 64, dtype=torch.bfloat16, device="cuda")
        assert B.cpa_kv_append_q8(c2.cfg, c2.dims, c2.tables, kd, kd, _i32(cu), 20, _i32(lens), out, c2.pool, c2.scales) == 0
        assert c2.status() == B.CPA_EINVAL
        changed = [b for b in range(4) if not torch.equal(c2.pool[int(c2.want.page_of(b, 0))], before[int(c2.want.page_of(b, 0))])]
        n = [b - a for a, b in zip(cu, cu[1:])]
        good = [i for i in range(4) if n[i] > 0 and lens[i] >= 0 and cu[i + 1] <= 20]
        assert set(changed) <= set(good) and out.tolist() == [a + (m if i in good or m == 0 else 0) for i, (a, m) in enumerate(zip(lens, n))]


def test_append_again_stores_the_same(B):
    c = Cache(B, [33, 5], 40, 2, 128)
    rng = np.random.default_rng(8)
    c.append(*(_values(rng, 38, 2, 128) for _ in range(2)), [33, 5])
    kd, vd = (_bf16(_values(rng, 30, 2, 128) * 16)[0] for _ in range(2))
    cu, out = _i32([0, 20, 30]), torch.empty_like(c.lens)
    for i in range(3):
        assert B.cpa_kv_append_q8(c.cfg, c.dims, c.tables, kd, vd, cu, 30, c.lens, out, c.pool, c.scales) == 0
        now = c.pool.clone(), c.scales.clone()
        if i:
            assert torch.equal(now[0], was[0]) and torch.equal(now[1].view(torch.int32), was[1].view(torch.int32))
        was = now


# ------------------------------------------------------------------------------------------------ decode

@pytest.mark.parametrize("lens", [[1], [16, 17], [0, 1, 2, 15, 16, 17, 31, 33, 0], [700, 3, 64, 129], [2500],
                                  [5] * 70, [40 + 13 * i for i in range(24)]], ids=lambda v: f"{len(v)}x{max(v)}")
@pytest.mark.parametrize("heads,group,d", [(1, 4, 64), (2, 8, 64), (8, 4, 128), (1, 1, 128), (3, 5, 128)])
def test_decode_matches_the_oracle(B, lens, heads, group, d):
    c = Cache(B, lens, 3, heads, d, group, seed=d)
    rng = np.random.default_rng(sum(lens) + heads)
    n = sum(lens)
    if n:
        c.append(_values(rng, n, heads, d), _values(rng, n, heads, d), lens)
    q = rng.standard_normal((len(lens), heads * group, d))
    o, qf = c.decode(q)
    c.check_rows(o, qf)
    again, _ = c.decode(q)                      # the workspace and the counters are left ready
    assert torch.equal(o, again)
    assert (o.cpu()[[i for i, m in enumerate(lens) if m == 0]] == 0).all()
    for t in range(3):
        o, qf = c.step(rng.standard_normal(q.shape), *(_values(rng, len(lens), heads, d) * 2.0 ** t for _ in range(2)))
        c.check_rows(o, qf, what=f"step {t}")
        c.check_pool(f"step {t}")
    assert c.status() == B.CPA_OK


@pytest.mark.parametrize("num_sms", [0, 1, 7])
def test_decode_splits_over_few_and_many_sms(B, num_sms):
    lens = [3000, 1, 0, 260, 517]
    c = Cache(B, lens, 2, 2, 128, num_sms=num_sms)
    rng = np.random.default_rng(9)
    c.append(_values(rng, sum(lens), 2, 128), _values(rng, sum(lens), 2, 128), lens)
    for t in range(2):
        o, qf = c.step(rng.standard_normal((5, 8, 128)), _values(rng, 5, 2, 128), _values(rng, 5, 2, 128))
        c.check_rows(o, qf)
    c.check_pool()


def test_decode_scales_far_apart(B):
    # pages whose scales lie 2^100 apart, in K (scores that decide the softmax) and in V (weights that must not vanish)
    c = Cache(B, [320], 0, 1, 64, 2)
    rng = np.random.default_rng(10)
    k, v = rng.standard_normal((320, 1, 64)), rng.standard_normal((320, 1, 64))
    page = np.arange(320) // 16
    k *= (2.0 ** -(page % 5 * 20.0))[:, None, None]
    v *= (2.0 ** ((page * 7 % 20 - 10) * 5.0))[:, None, None]
    c.append(k, v, [320])
    q = rng.standard_normal((1, 2, 64))
    o, qf = c.decode(q)
    c.check_rows(o, qf)
    # the key that takes all the weight has the smallest values of all
    k2 = np.zeros((320, 1, 64))
    k2[100] = 30 * q[0, 0] / np.abs(q[0, 0]).max()
    v2 = rng.standard_normal((320, 1, 64)) * 2.0 ** 40
    v2[96:112] *= 2.0 ** -80
    c = Cache(B, [320], 0, 1, 64, 1, scale=4.0)
    c.append(k2, v2, [320])
    o, qf = c.decode(q[:, :1])
    c.check_rows(o, qf)


def test_decode_takes_any_positive_scale(B):
    c = Cache(B, [50, 20], 4, 2, 128, 4)
    rng = np.random.default_rng(11)
    c.append(_values(rng, 70, 2, 128), _values(rng, 70, 2, 128), [50, 20])
    f = torch.rand_like(c.scales) + 0.5
    c.scales *= f
    c.want.scales = c.scales.cpu().numpy().astype(np.float64)
    o, qf = c.decode(rng.standard_normal((2, 8, 128)))
    c.check_rows(o, qf)
    out = torch.empty(70, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(70, 2, 128, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, None, _i32([0, 50, 70]), 70, c.pool, c.scales, *out) == 0
    want = np.concatenate([c.want.rows(0, 0, 50), c.want.rows(1, 0, 20)], 2).transpose(0, 2, 1, 3)
    for i in range(2):
        assert (np.abs(out[i].double().cpu().numpy() - want[i]) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want[i])).all()


def test_decode_extreme_queries(B):
    c = Cache(B, [37, 37, 37], 0, 1, 64, 4, scale=2.0 ** -40)
    rng = np.random.default_rng(12)
    c.append(_values(rng, 111, 1, 64), _values(rng, 111, 1, 64), [37] * 3)
    q = rng.standard_normal((3, 4, 64))
    q[0] *= 2.0 ** 38                    # far above f16's range
    q[1] *= 2.0 ** -60                   # far below it: uniform weights
    q[2, 0], q[2, 1, :32] = 0.0, 0.0
    q[2, 2, 0] = 2.0 ** 40
    q[2, 3] *= 2.0 ** (rng.integers(-20, 20, 64) + 15.0)
    o, qf = c.decode(q)
    c.check_rows(o, qf)


def test_nan_and_infinities_reach_the_rows_they_belong_to(B):
    c = Cache(B, [20, 20, 20], 0, 1, 64, 2)
    rng = np.random.default_rng(13)
    k, v = _values(rng, 60, 1, 64), _values(rng, 60, 1, 64)
    k[5, 0, 3], v[25, 0, 9] = np.nan, np.nan
    c.append(k, v, [20] * 3)
    q = rng.standard_normal((3, 2, 64))
    q[2, 1, 0] = np.nan
    o, qf = c.decode(q)
    nan = torch.isnan(o).cpu()
    assert nan[0].all() and nan[1, :, 9].all() and nan[1].sum() == 2 and nan[2, 1].all() and not nan[2, 0].any()
    want, spread, shaken = c.want.decode(2, np.nan_to_num(qf[2]), c.scale)
    tol = oq.decode_tolerance(want, spread, shaken, 64)
    assert (np.abs(o[2, 0].double().cpu().numpy() - want[0]) <= tol[0]).all()


def test_blocks_that_sit_out(B):
    lens = [30, 16, 0, 45, 32]
    c = Cache(B, lens, 0, 2, 64)
    rng = np.random.default_rng(14)
    c.append(*(_values(rng, sum(lens), 2, 64) for _ in range(2)), lens)
    active = _i32([1, 0, 1, 5, 0])
    q = rng.standard_normal((5, 8, 64))
    o, qf = c.decode(q, active)
    assert (o[[1, 4]] == 9).all() and (o[2] == 0).all()
    c.check_rows(o, qf, [0, 3])
    # a step: blocks 1 and 4 have no room left, block 2 has no page at all
    before = c.pool.clone()
    o, out = torch.full_like(o, 9.0), torch.full_like(c.lens, -7)
    (qd, qf), (kd, kf), (vd, vf) = _bf16(q), _bf16(_values(rng, 5, 2, 64)), _bf16(_values(rng, 5, 2, 64))
    assert B.cpa_decode_append_q8(c.cfg, c.dims, c.tables, qd, kd, vd, c.lens, out, None, c.pool, c.scales, o, c.ws) == 0
    assert out.tolist() == [31, 16, 0, 46, 32] and c.status() == B.CPA_ENOSPC
    assert (o[[1, 2, 4]] == 9).all()
    for b in (0, 3):
        c.want.append(b, kf[b:b + 1], vf[b:b + 1])
    c.check_rows(o, qf, [0, 3])
    for b in (1, 4):
        for i in range(lens[b] // 16):
            assert torch.equal(c.pool[c.want.page_of(b, 16 * i)], before[c.want.page_of(b, 16 * i)])
    # lengths that no table has: negative, and beyond the pages
    c.lens = _i32([31, -3, 0, 46, 33])
    o, qf = c.decode(q, fill=7.0)
    assert (o[[1, 4]] == 7).all()
    c.check_rows(o, qf, [0, 3])


def test_a_run_captured_and_replayed(B):
    # prompts, then pairs of steps that swap the two length arrays, replayed from a graph on a stream of its own
    lens = [100, 47, 260]
    c = Cache(B, lens, 8, 2, 128)
    rng = np.random.default_rng(15)
    c.append(*(_values(rng, sum(lens), 2, 128) for _ in range(2)), lens)
    bufs = [torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")] + [torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    a, b, o = c.lens, torch.zeros_like(c.lens), torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    pool0, scales0, a0 = c.pool.clone(), c.scales.clone(), a.clone()

    def two():
        on = torch.cuda.current_stream().cuda_stream
        for i, (x, y) in enumerate(((a, b), (b, a))):
            assert B.cpa_decode_append_q8(c.cfg, c.dims, c.tables, *bufs, x, y, None, c.pool, c.scales, o[i], c.ws, on) == 0

    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        two()                                   # warm: what is set up per device is set up
    side.synchronize()
    c.pool.copy_(pool0), c.scales.copy_(scales0), a.copy_(a0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        two()
    for r in range(3):
        vals = [_bf16(x) for x in (rng.standard_normal((3, 8, 128)), _values(rng, 3, 2, 128), _values(rng, 3, 2, 128))]
        for buf, (t, _) in zip(bufs, vals):
            buf.copy_(t)
        graph.replay()
        for i in range(2):                      # both steps of a replay take the same rows
            for blk in range(3):
                c.want.append(blk, vals[1][1][blk:blk + 1], vals[2][1][blk:blk + 1])
            if i == 1:
                c.check_rows(o[i], vals[0][1], what=f"replay {r}")
        c.lens = a
        c.check_pool(f"replay {r}")
    assert c.status() == B.CPA_OK


def test_steps_on_two_streams_with_their_own_tables(B):
    caches, rng = [], np.random.default_rng(16)
    for i in range(2):
        lens = [900 + 100 * i, 64]
        c = Cache(B, lens, 8, 2, 64, seed=i)
        c.append(*(_values(rng, sum(lens), 2, 64) for _ in range(2)), lens)
        caches.append(c)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]
    args = [[_bf16(x) for x in (rng.standard_normal((2, 8, 64)), _values(rng, 2, 2, 64), _values(rng, 2, 2, 64))] for _ in range(16)]
    torch.cuda.synchronize()
    outs = []
    for t in range(8):
        for i, c in enumerate(caches):
            with torch.cuda.stream(streams[i]):
                o, out = torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(c.lens)
                (qd, qf), (kd, kf), (vd, vf) = args[2 * t + i]
                assert B.cpa_decode_append_q8(c.cfg, c.dims, c.tables, qd, kd, vd, c.lens, out, None, c.pool, c.scales, o, c.ws,
                                              streams[i].cuda_stream) == 0
                c.lens = out
                outs.append(o)
    torch.cuda.synchronize()
    for t in range(8):
        for i, c in enumerate(caches):
            (_, qf), (_, kf), (_, vf) = args[2 * t + i]
            for b in range(2):
                c.want.append(b, kf[b:b + 1], vf[b:b + 1])
            c.check_rows(outs[2 * t + i], qf, what=f"step {t} of {i}")


def test_page_ids_on_both_sides_of_2_to_the_32_bytes(B):
    # a page of 8 heads of 128 is 32 KB: ids around 131072 lie on both sides of 2^32 bytes
    def ids(need, rng):
        far = np.array([131072 + (i // 2 if i % 2 else -1 - i // 2) for i in range(need)], dtype=np.int32)
        return far, 131072 + need
    c = Cache(B, [70, 33], 3, 8, 128, page_ids=ids)
    low = c.pool[:64].clone()
    rng = np.random.default_rng(17)
    small = oq.CacheQ8(20, 8, 128, [70, 33], 3, np.arange(20))
    c.want = small
    n = 103
    c.append(_values(rng, n, 8, 128), _values(rng, n, 8, 128), [70, 33])
    o, qf = c.decode(rng.standard_normal((2, 32, 128)))
    c.check_rows(o, qf)
    for _ in range(2):
        o, qf = c.step(rng.standard_normal((2, 32, 128)), _values(rng, 2, 8, 128), _values(rng, 2, 8, 128))
        c.check_rows(o, qf)
    out = torch.empty(2, n + 4, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, None, _i32([0, 72, 107]), n + 4, c.pool, c.scales, out[0], out[1]) == 0
    want = np.concatenate([small.rows(0, 0, 72), small.rows(1, 0, 35)], 2).transpose(0, 2, 1, 3)
    assert np.array_equal(out.double().cpu().numpy(), want)
    assert torch.equal(c.pool[:64], low)


def test_a_long_history_in_one_block(B):
    # 131072 tokens of one block, every answer checked in 64 bits on the device
    n, heads, group, d = 131072, 2, 4, 128
    c = Cache(B, [n], 1, heads, d, group)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(n, heads, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    k[77777] *= 6
    out = torch.empty_like(c.lens)
    assert B.cpa_kv_append_q8(c.cfg, c.dims, c.tables, k, v, _i32([0, n]), n, None, out, c.pool, c.scales) == 0
    c.lens = out
    q = torch.randn(1, heads * group, d, generator=gen, device="cuda").bfloat16()
    o = torch.empty_like(q)
    assert B.cpa_decode_q8(c.cfg, c.dims, c.tables, q, c.lens, None, c.pool, c.scales, o, c.ws) == 0
    pages = torch.from_numpy(c.want.pages[:n // 16].astype(np.int64)).cuda()
    x = (c.pool.view(torch.float8_e4m3fn)[pages].double() * c.scales[pages].double()[..., None, None])
    kk, vv = (x[:, :, i].transpose(0, 1).reshape(heads, n, d) for i in (0, 1))
    qq = q.double().view(heads, group, d)
    w = torch.softmax(c.scale * qq @ kk.transpose(1, 2), 2)
    want, spread = (w @ vv).reshape(-1, d), (w @ vv.abs()).reshape(-1, d)
    shaken = (c.scale * qq.abs() @ kk.abs().transpose(1, 2)).amax(2).reshape(-1, 1)
    tol = oq.decode_tolerance(*(t.cpu().numpy() for t in (want, spread, shaken)), d)
    assert (np.abs(o[0].double().cpu().numpy() - want.cpu().numpy()) <= tol).all()


@pytest.mark.parametrize("num_sms", [1, 3, 0, 300])
@pytest.mark.parametrize("blocks,hi", [(500, 40), (193, 3), (385, 130)])
def test_many_blocks(B, blocks, hi, num_sms):
    # more blocks than threads, a third of them empty, some sitting out; both directions of the walk
    rng = np.random.default_rng(blocks + num_sms)
    lens = [int(n) if rng.random() < 0.67 else 0 for n in rng.integers(1, hi + 1, blocks)]
    c = Cache(B, lens, 2, 2, 64, 3, num_sms=num_sms, seed=hi)
    c.append(_values(rng, sum(lens), 2, 64), _values(rng, sum(lens), 2, 64), lens)
    on = rng.random(blocks) < 0.8
    on[0] = True
    active = _i32(on)
    for t in range(2):
        o, qf = c.decode(rng.standard_normal((blocks, 6, 64)), active)
        c.check_rows(o, qf, np.flatnonzero(on), f"decode {t}")
        assert (o[~torch.from_numpy(on).cuda()] == 9).all()
        o, qf = c.step(rng.standard_normal((blocks, 6, 64)), _values(rng, blocks, 2, 64), _values(rng, blocks, 2, 64), active)
        c.check_rows(o, qf, np.flatnonzero(on), f"step {t}")
    c.check_pool()
    assert c.status() == B.CPA_OK


def test_cuts_at_every_place(B):
    # one to twelve SMs and blocks of one to eighty pages: range ends fall inside blocks, on their edges, and into the
    # cells that stand for a block's own cost
    rng = np.random.default_rng(21)
    for num_sms in range(1, 13):
        lens = [int(x) for x in rng.integers(1, 1280, rng.integers(1, 6))]
        c = Cache(B, lens, 2, 1, 128, 2, num_sms=num_sms, seed=num_sms)
        c.append(_values(rng, sum(lens), 1, 128), _values(rng, sum(lens), 1, 128), lens)
        for t in range(2):
            o, qf = c.step(rng.standard_normal((len(lens), 2, 128)), _values(rng, len(lens), 1, 128), _values(rng, len(lens), 1, 128))
            c.check_rows(o, qf, what=f"{num_sms} SMs")
        c.check_pool()


def test_calls_of_all_kinds_back_to_back(B):
    # every call starts while the one before it ends: append, read, decode and step of one cache without a wait between
    lens = [200, 31, 64]
    c = Cache(B, lens, 40, 2, 64)
    rng = np.random.default_rng(22)
    c.append(*(_values(rng, sum(lens), 2, 64) for _ in range(2)), lens)
    outs = []
    for t in range(6):
        q, k, v = rng.standard_normal((3, 8, 64)), _values(rng, 3, 2, 64), _values(rng, 3, 2, 64)
        c.append(k, v)
        o, qf = c.decode(q)
        outs.append((o, [c.want.decode(b, qf[b], c.scale) for b in range(3)]))
        k2, v2 = torch.empty(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 2, 64, dtype=torch.bfloat16, device="cuda")
        assert B.cpa_kv_read_q8(c.cfg, c.dims, c.tables, c.lens - 1, _i32([0, 1, 2, 3]), 3, c.pool, c.scales, k2, v2) == 0
        rows = np.concatenate([c.want.rows(b, int(c.want.lens[b]) - 1, int(c.want.lens[b])) for b in range(3)], 2).transpose(0, 2, 1, 3)
        o, qf = c.step(q[::-1], v, k)
        outs.append((o, [c.want.decode(b, qf[b], c.scale) for b in range(3)]))
        assert np.array_equal(k2.double().cpu().numpy(), rows[0]) and np.array_equal(v2.double().cpu().numpy(), rows[1])
    c.check_pool()
    for o, want in outs:
        for b in range(3):
            assert (np.abs(o[b].double().cpu().numpy() - want[b][0]) <= oq.decode_tolerance(*want[b], 64)).all()


@pytest.mark.parametrize("fused", [False, True])
def test_append_into_pages_of_any_scale(B, fused):
    # pages that another writer has filled: a scale that is no power of two is kept while it suffices, and a larger one
    # is again a power of two
    c = Cache(B, [21, 40], 8, 2, 128, 2)
    rng = np.random.default_rng(23)
    c.append(_values(rng, 61, 2, 128), _values(rng, 61, 2, 128), [21, 40])
    c.scales *= torch.rand_like(c.scales) * 0.9 + 0.6
    for t in range(6):
        old = c.pool.view(torch.float8_e4m3fn).double() * c.scales.double()[..., None, None]
        was, lens = c.scales.double().cpu().numpy(), c.lens.tolist()
        k, v = (_values(rng, 2, 2, 128) * 1.7 ** t for _ in range(2))
        if fused:
            c.step(rng.standard_normal((2, 4, 128)), k, v)
        else:
            c.append(k, v)
        now = (c.pool.view(torch.float8_e4m3fn).double() * c.scales.double()[..., None, None]).cpu().numpy()
        s, old_h = c.scales.double().cpu().numpy(), old.cpu().numpy()
        rows = np.stack([_bf16(k)[1], _bf16(v)[1]], 2)                     # [2, heads, 2, d]
        for b in range(2):
            pg, slot = c.want.page_of(b, lens[b]), lens[b] % 16
            top = np.abs(rows[b]).max(-1)
            need = oq.page_scale(rows[b][:, :, None])
            want_s = need if slot == 0 else np.where(need > was[pg], need, was[pg])
            assert np.array_equal(s[pg], want_s) and (top <= 448 * s[pg]).all()
            # half a step of e4m3, and the 32-bit quotient's own rounding
            off = np.abs(now[pg, :, :, slot] - rows[b])
            assert (off <= (2.0 ** -4 * np.abs(rows[b]) + 2.0 ** -10 * s[pg][..., None]) * (1 + 2.0 ** -20)).all()
            before = old_h[pg, :, :, :slot]
            grown = (s[pg] > was[pg])[..., None, None]
            off = np.abs(now[pg, :, :, :slot] - before)
            bound = np.where(grown, 2.0 ** -4 * np.abs(before) + 2.0 ** -10 * s[pg][..., None, None], 0.0) * (1 + 2.0 ** -20)
            assert (off <= bound).all()
