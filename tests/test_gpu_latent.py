"""Rotary positions and latent attention on the device against their definition in 64 bits (oracle/latent.py), within the bounds
that the oracle derives: sizes, masks, strides and inputs at which a kernel can go wrong, and a whole event through the calls."""
import numpy as np
import pytest

from oracle import latent as ol

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


def _np(t):
    return t.detach().double().cpu().numpy()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _check(got, want, tol, what=""):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]:.6g} for {want[bad][0]:.6g}"


SCALING = {"none": 0, "all": 1, "base": 2, "parts": 3, "waves": 4}


class Rope:
    def __init__(self, B, R=64, interleaved=True, scaling="parts", base=10000.0, factor=40.0, amplitude=1.0):
        self.cfg = B.cpa_rope_config(R, int(interleaved), SCALING[scaling], 4096, base, factor, 32.0, 1.0, amplitude)
        self.turns = torch.from_numpy(B.cpa_rope_turns(self.cfg).view(np.int64)).cuda()
        self.f = ol.frequencies(R, base, scaling, factor, 32.0, 1.0, 4096)
        self.interleaved, self.amplitude = interleaved, amplitude


# ------------------------------------------------------------------------------------------------ rotary positions

@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,kv,hd,R,offset", [
    (1, 1, 0, 64, 64, 0), (3, 32, 8, 128, 128, 0), (1200, 4, 1, 128, 32, 96), (700, 3, 3, 192, 64, 128), (7, 5, 2, 80, 20, 60),
    (5, 2, 1, 72, 8, 16), (4, 1, 1, 256, 256, 0), (9, 7, 1, 65, 2, 31), (2000, 1, 0, 48, 48, 0), (33, 128, 0, 192, 64, 128),
    (9501, 1, 1, 32, 32, 0), (20011, 1, 0, 24, 16, 8), (18945, 1, 0, 10, 6, 1)])
def test_rope_rows(B, rows, heads, kv, hd, R, offset, interleaved):
    rng = np.random.default_rng(rows + heads)
    rope = Rope(B, R, interleaved, "none" if rows % 2 else "parts", amplitude=1.0 if heads % 2 else 1.375)
    pos = rng.integers(-2 ** 31, 2 ** 31, rows)
    pos[:min(rows, 3)] = [0, 131071, -1][:min(rows, 3)]
    d_pos = _i32(pos)
    for in_place in (False, True):
        outs, want = [], []
        for n in (heads, kv):
            x, xf = _bf16(rng.standard_normal((rows, n, hd)))
            outs.append((x, x if in_place else torch.full_like(x, 9.0)))
            want.append(xf)
        args = [B.rope_rows(x, o, offset=offset) for x, o in outs]
        rc = B.cpa_rope(rope.cfg, rope.turns, d_pos, rows, args[0], args[1] if kv else None, False, _stream())
        assert rc == 0
        for (x, o), xf in zip(outs, want):
            part = xf[..., offset:offset + R]
            y = ol.turn(part, pos[:, None], rope.f, interleaved, rope.amplitude)
            # far positions: the oracle's angle is off by half a step of |position| f in 64 bits, the device's by 2^-64 turns each
            far = np.abs(pos)[:, None, None] * 2.0 ** -52 * 2 * (np.abs(part).max() if part.size else 0) * 2 * rope.amplitude
            _check(o[..., offset:offset + R], y, ol.turn_tolerance(part, y, interleaved, rope.amplitude) + far, "turned")
            keep = np.r_[0:offset, offset + R:hd]
            assert np.array_equal(_np(o)[..., keep], xf[..., keep])


def test_rope_strided_rows_and_back(B):
    # the positional part of projected queries (strided, in place), then back: x again to one rounding each way
    rope = Rope(B, 64, True, "parts")
    x = torch.randn(50, 6, 192, device="cuda").bfloat16()
    was, pos = x.clone(), torch.randint(0, 10 ** 6, (50,), device="cuda", dtype=torch.int32)
    part = x[..., 128:]
    assert B.cpa_rope(rope.cfg, rope.turns, pos, 50, B.rope_rows(part, None, 64), None, False, _stream()) == 0
    assert torch.equal(x[..., :128], was[..., :128]) and not torch.equal(part, was[..., 128:])
    # into heads-first memory and at an odd element, which moves by element
    out = torch.full((6, 50, 64), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    odd = torch.zeros(50 * 6 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(50, 6, 64)
    for o in (out, odd):
        assert B.cpa_rope(rope.cfg, rope.turns, pos, 50, B.rope_rows(part, o, 64), None, True, _stream()) == 0
        m = _np(was[..., 128:])
        # half a step of each of the pair's elements on the way there, half a step on the way back
        size = np.hypot(m[..., 0::2], m[..., 1::2]).repeat(2, -1)
        _check(o, m, 2.0 ** -7 * size + 2.0 ** -8 * size, "back")
    assert torch.equal(out, odd)


def test_rope_keeps_what_is_tiny_and_what_is_not_finite(B):
    rope = Rope(B, 64, False, "none")
    x = torch.zeros(4, 1, 64, device="cuda").bfloat16()
    x[0, 0, :] = 2.0 ** -130                                   # below fp32's normal range
    x[1, 0, 5] = float("inf")
    x[2, 0, 5] = float("nan")
    x[3, 0, :] = 3e38
    pos = _i32([0, 3, 3, 0])
    o = torch.empty_like(x)
    assert B.cpa_rope(rope.cfg, rope.turns, pos, 4, B.rope_rows(x, o, 64), None, False, _stream()) == 0
    y = _np(o)
    assert (y[0, 0] == 2.0 ** -130).all() and (y[3] == _np(x)[3]).all()
    assert not np.isfinite(y[1, 0, [5, 37]]).any() and np.isfinite(np.delete(y[1, 0], [5, 37])).all()
    assert np.isnan(y[2, 0, [5, 37]]).all() and np.isfinite(np.delete(y[2, 0], [5, 37])).all()


# ------------------------------------------------------------------------------------------------ the cache

class Cache:
    """A device cache beside the oracle's rows.  Unfilled slots hold NaN."""

    def __init__(self, B, room, L=512, H=16, seed=0, eps=1e-6, scale=192 ** -0.5, num_sms=0, extra=3, page_ids=None, rope=None):
        rng = np.random.default_rng(seed)
        self.B, self.L, self.H, self.eps, self.scale, self.rope = B, L, H, float(np.float32(eps)), float(np.float32(scale)), rope
        need = sum(-(-n // 16) for n in room)
        self.num_pages, ids = need + extra, rng.permutation(need + extra).astype(np.int32)
        if page_ids is not None:
            ids, self.num_pages = page_ids
        self.ids, self.n = ids, len(room)
        self.cfg = B.cpa_latent_config(H, L, 64, 128, 128, 16, scale, eps, num_sms)
        tc = B.cpa_latent_tables_config(self.cfg)
        self.dims = B.cpa_table_dims(self.n, 0, self.num_pages, len(ids), 0)
        self.tables = torch.full((B.cpa_tables_bytes(tc, self.dims),), 0xAB, dtype=torch.uint8, device="cuda")
        self.d_ids = _i32(ids)
        assert B.cpa_tables_build(tc, self.dims, _i32(room), self.d_ids, len(ids), self.tables, _stream()) == 0
        self.indptr = np.concatenate([[0], np.cumsum([-(-n // 16) for n in room])])
        self.pool = torch.full((self.num_pages, 16, L + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.ws = torch.full((B.cpa_latent_decode_workspace_bytes(self.cfg),), 0xFF, dtype=torch.uint8, device="cuda")
        self.lens = torch.zeros(self.n, dtype=torch.int32, device="cuda")
        self.rows = [np.zeros((0, L + 64)) for _ in room]      # what the pool holds, by the pool

    def status(self):
        return self.B.cpa_tables_status(self.tables, _stream())

    def slots(self, b, lo, hi):
        i = np.arange(lo, hi)
        return self.ids[self.indptr[b] + i // 16] * 16 + i % 16

    def fill(self, lens, rng, spread=1.0):
        """Cached rows written by hand, so that the attention's tests do not rest on the append."""
        flat = self.pool.view(-1, self.L + 64)
        for b, n in enumerate(lens):
            x, xf = _bf16(spread * rng.standard_normal((n, self.L + 64)))
            if n:
                flat[torch.as_tensor(self.slots(b, 0, n), dtype=torch.long, device="cuda")] = x
            self.rows[b] = xf
        self.lens = _i32(lens)

    def append(self, x, counts, weight=None, first=None, packed=True, stride=None, active=None):
        """x float64 rows; counts None: one per block.  Returns (packed rows, unrounded rows wanted, tolerance)."""
        stride = stride or self.L + 64
        wide = torch.full((max(1, len(x)), stride), 5.0, dtype=torch.bfloat16, device="cuda")
        xd, xf = _bf16(x)
        wide[:len(x), :self.L + 64] = xd
        out = torch.full_like(self.lens, -7)
        cu = None if counts is None else np.concatenate([[0], np.cumsum(counts)])
        pk = torch.full((len(x), self.L + 64), 3.0, dtype=torch.bfloat16, device="cuda") if packed else None
        wd, wf = (None, None) if weight is None else _bf16(weight)
        r = self.rope
        rc = self.B.cpa_latent_append(self.cfg, self.dims, self.tables, r and r.cfg, r and r.turns, wide, stride, wd,
                                      None if cu is None else _i32(cu), len(x), None if first is None else _i32(first), self.lens,
                                      out, self.pool, pk, _stream())
        assert rc == 0
        was = self.lens.cpu().numpy()
        self.lens = out
        at = np.arange(self.n + 1) if cu is None else cu
        pos = np.concatenate([np.arange(was[b], was[b] + at[b + 1] - at[b]) + (0 if first is None else first[b]) for b in range(self.n)])
        want = ol.new_rows(xf, self.L, wf, self.eps, pos, r and r.f, r is None or r.interleaved, r.amplitude if r else 1.0)
        tol = ol.rows_tolerance(xf, want, self.L, r is None or r.interleaved, r.amplitude if r else 1.0)
        flat = self.pool.view(-1, self.L + 64)
        for b in range(self.n):
            got = _np(flat[torch.as_tensor(self.slots(b, was[b], was[b] + at[b + 1] - at[b]), dtype=torch.long, device="cuda")])
            _check(got, want[at[b]:at[b + 1]], tol[at[b]:at[b + 1]], f"block {b}")
            self.rows[b] = np.concatenate([self.rows[b], got])
        if packed:
            for b in range(self.n):
                assert np.array_equal(_np(pk[at[b]:at[b + 1]]), self.rows[b][was[b]:], equal_nan=True)
        return pk

    def check_rest(self):
        """Nothing but the blocks' rows was written."""
        left = np.ones(self.num_pages * 16, dtype=bool)
        for b in range(self.n):
            left[self.slots(b, 0, len(self.rows[b]))] = False
        assert torch.isnan(self.pool.view(-1, self.L + 64)[torch.as_tensor(np.flatnonzero(left), device="cuda")]).all()
        assert self.lens.cpu().tolist() == [len(r) for r in self.rows]

    def queries(self, rng, spread=1.0):
        (qc, cf), (qr, rf) = _bf16(spread * rng.standard_normal((self.n, self.H, self.L))), _bf16(spread * rng.standard_normal((self.n, self.H, 64)))
        return qc, qr, cf, rf

    def decode(self, qc, qr, active=None, out=None, lens=None, ws=None):
        o = torch.full((self.n, self.H, self.L), 9.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        rc = self.B.cpa_latent_decode(self.cfg, self.dims, self.tables, self.B.latent_io(qc, qr, o), self.lens if lens is None else lens,
                                      active, self.pool, self.ws if ws is None else ws, _stream())
        assert rc == 0
        return o

    def check(self, o, cf, rf, blocks=None, what="", score=None):
        got = _np(o)
        for b in range(self.n) if blocks is None else blocks:
            want, spread, shaken = ol.decode(np.concatenate([cf[b], rf[b]], 1), self.rows[b], self.L, self.scale)
            tol = ol.attention_tolerance(want, spread, shaken, self.L + 64, 0.0 if score is None else score[b])
            _check(got[b], want, tol, f"{what} block {b} of {len(self.rows[b])}")


@pytest.mark.parametrize("L", [128, 256, 384, 512])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_prompts_chunks_and_single_rows(B, L, interleaved):
    rng = np.random.default_rng(L)
    room = [0, 1, 16, 17, 100, 333, 5]
    c = Cache(B, room, L, rope=Rope(B, 64, interleaved, "parts", amplitude=1.25))
    first, w = rng.integers(0, 10 ** 5, len(room)), 1 + 0.2 * rng.standard_normal(L)
    size = np.exp(rng.standard_normal((400, 1)))
    for counts in ([0, 0, 15, 3, 0, 211, 0], [0, 1, 1, 13, 64, 100, 4]):
        n = sum(counts)
        c.append(size[:n] * rng.standard_normal((n, L + 64)), counts, w, first, stride=L + 64 + 8 * (n % 2), packed=True)
        c.check_rest()
    assert c.status() == 0
    c = Cache(B, [3, 17, 40], L, rope=Rope(B, 64, interleaved, "none"))
    for i in range(3):
        c.append(rng.standard_normal((3, L + 64)), None, w, stride=L + 64 + (i == 1), packed=i != 2)      # an odd stride: by element
    c.check_rest()
    assert c.status() == 0


def test_append_without_norm_or_turn(B):
    rng = np.random.default_rng(2)
    c = Cache(B, [40, 7], 256)
    c.append(rng.standard_normal((33, 320)), [30, 3])
    assert c.status() == 0
    c = Cache(B, [40, 7], 256, rope=Rope(B, 64, True, "waves"))
    c.append(rng.standard_normal((33, 320)), [30, 3], None, [7, 99])


@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_append_norms_rows_of_any_magnitude(B, eps):
    rng = np.random.default_rng(3)
    c = Cache(B, [16], 512, eps=eps)
    size = 2.0 ** np.array([-120, -70, -64, -40, -20, 0, 10, 30, 60, 64, 90, 120])[:, None]
    x = rng.standard_normal((12, 576)) * size
    x[:, 512:] = 1.0
    c.append(x, [12], np.ones(512))
    assert c.status() == 0


def test_append_leaves_out_what_does_not_fit_or_is_bad(B):
    rng = np.random.default_rng(4)
    c = Cache(B, [16, 16, 32, 16], 128)
    x, _ = _bf16(rng.standard_normal((40, 192)))
    out = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    call = lambda cu, lens, rows=40: B.cpa_latent_append(c.cfg, c.dims, c.tables, None, None, x, 192, None, _i32(cu), rows, None, _i32(lens),
                                                         out, c.pool, None, _stream())
    assert call([0, 5, 25, 30, 34], [0, 0, 0, 0]) == 0                     # 20 rows into 16
    assert out.tolist() == [5, 0, 5, 4] and c.status() == B.CPA_ENOSPC
    flat = c.pool.view(-1, 192)
    at = lambda b, lo, hi: flat[torch.as_tensor(c.slots(b, lo, hi), dtype=torch.long, device="cuda")]
    assert torch.equal(at(0, 0, 5), x[:5]) and torch.equal(at(2, 0, 5), x[25:30]) and torch.equal(at(3, 0, 4), x[30:34])
    assert torch.isnan(at(1, 0, 16)).all()
    # ranges that run backwards, or leave the rows: theirs alone are left out
    for cu, lens, want in (([0, 10, 5, 12, 20], [0, 0, 0, 0], [10, 0, 7, 8]), ([0, 4, 8, 48, 52], [0, 0, 0, 0], [4, 4, 0, 0]),
                           ([0, 4, 8, 12, 16], [0, -1, 40, 12], [4, -1, 40, 16])):
        c.pool.fill_(float("nan"))
        assert call(cu, lens) == 0
        assert out.tolist() == want, (cu, lens)
        for b in range(4):
            n = want[b] - lens[b]
            if n > 0:
                assert torch.equal(at(b, lens[b], want[b]), x[cu[b]:cu[b + 1]]), (cu, b)
    # nothing to append: lengths go on
    assert B.cpa_latent_append(c.cfg, c.dims, c.tables, None, None, None, 192, None, _i32([0] * 5), 0, None, _i32([1, 2, 3, 4]), out, c.pool,
                               None, _stream()) == 0
    assert out.tolist() == [1, 2, 3, 4]


def test_append_packed_in_place(B):
    rng = np.random.default_rng(9)
    rope = Rope(B)
    made = []
    for in_place in (False, True):
        c = Cache(B, [40, 0, 25], 256, seed=2, rope=rope)
        x, _ = _bf16(np.random.default_rng(3).standard_normal((60, 320)))
        packed, w, out = x if in_place else torch.empty_like(x), torch.ones(256, dtype=torch.bfloat16, device="cuda"), torch.empty_like(c.lens)
        assert B.cpa_latent_append(c.cfg, c.dims, c.tables, rope.cfg, rope.turns, x, 320, w, _i32([0, 35, 35, 60]), 60, None, None, out, c.pool,
                                   packed, _stream()) == 0
        assert out.tolist() == [35, 0, 25] and c.status() == 0
        made.append((packed.clone(), c.pool.clone()))
    assert torch.equal(made[0][0], made[1][0]) and torch.equal(made[0][1].view(torch.int16), made[1][1].view(torch.int16))


def test_append_many_blocks_and_rows_behind_the_last(B):
    rng = np.random.default_rng(8)
    counts = rng.integers(0, 4, 1500)
    n = int(counts.sum())
    c = Cache(B, np.maximum(counts, 1), 128, rope=Rope(B))
    x, xf = _bf16(rng.standard_normal((n + 9, 192)))
    packed = torch.full_like(x, 3.0)
    out = torch.empty_like(c.lens)
    cu = np.concatenate([[0], np.cumsum(counts)])
    assert B.cpa_latent_append(c.cfg, c.dims, c.tables, c.rope.cfg, c.rope.turns, x, 192, None, _i32(cu), n + 9, None, None, out, c.pool,
                               packed, _stream()) == 0
    assert out.tolist() == counts.tolist() and c.status() == 0
    pos = np.concatenate([np.arange(k) for k in counts])
    want = ol.new_rows(xf[:n], 128, None, 0, pos, c.rope.f)
    _check(packed[:n], want, ol.rows_tolerance(xf[:n], want, 128))
    assert (packed[n:] == 3.0).all()                                        # rows behind the last sequence stay
    slots = np.concatenate([c.slots(b, 0, k) for b, k in enumerate(counts)])
    assert torch.equal(c.pool.view(-1, 192)[torch.as_tensor(slots, dtype=torch.long, device="cuda")], packed[:n])


@pytest.mark.parametrize("cu,rows", [([0, 10, 5, 12, 5, 5], 6000), ([0, 10, 5, 12, 5, 5], 40), ([0, 4000, 3999, 4737, 4700, 5001], 5001),
                                     ([0, 5000, 17, 18, 16, 4999], 5000), ([0, 4738, 4738, 4738, 4737, 4738], 4738),
                                     ([7, 3, 5000, 11, 11, 13], 5000), ([0, 0, 4800, 2400, 2401, 4800], 4800)])
def test_append_stores_every_good_range_beside_bad_ones(B, cu, rows):
    # ranges that run backwards, so that good ones overlap: each good block has all of its rows, whatever the search of a row leads to, with
    # one row of a warp in flight (40 rows) and with two
    rng = np.random.default_rng(rows)
    n = len(cu) - 1
    c = Cache(B, [5008] * n, 128, rope=Rope(B))
    x = torch.randn(rows, 192, device="cuda").bfloat16()
    first, out = _i32(rng.integers(0, 10 ** 5, n)), torch.full((n,), -7, dtype=torch.int32, device="cuda")
    assert B.cpa_latent_append(c.cfg, c.dims, c.tables, c.rope.cfg, c.rope.turns, x, 192, None, _i32(cu), rows, first, c.lens, out, c.pool, None,
                               _stream()) == 0
    assert c.status() == B.CPA_EINVAL
    lens = [max(0, cu[b + 1] - cu[b]) for b in range(n)]
    assert out.tolist() == lens
    for b in range(n):
        if not lens[b]:
            continue
        d = Cache(B, [5008], 128, rope=c.rope)
        part, one = x[cu[b]:cu[b + 1]].contiguous(), torch.empty(1, dtype=torch.int32, device="cuda")
        for lo in range(0, lens[b], 1000):                                   # by calls of few rows
            hi = min(lo + 1000, lens[b])
            assert B.cpa_latent_append(d.cfg, d.dims, d.tables, c.rope.cfg, c.rope.turns, part[lo:hi], 192, None, _i32([0, hi - lo]), hi - lo,
                                       first[b:b + 1].clone(), _i32([lo]), one, d.pool, None, _stream()) == 0
        got, want = (k.pool.view(-1, 192)[torch.as_tensor(k.slots(i, 0, lens[b]), dtype=torch.long, device="cuda")] for k, i in ((c, b), (d, 0)))
        assert torch.equal(got, want), (b, torch.nonzero((got != want).any(1)).flatten().tolist()[:4])


@pytest.mark.parametrize("rows", [4735, 4736, 4737, 4738, 6001])
@pytest.mark.parametrize("L,how", [(512, "apart"), (256, "odd stride"), (384, "in place"), (128, "as it is")])
def test_append_of_many_rows_is_that_of_few(B, rows, L, how):
    # one row of a warp in flight up to 4736 rows, two from there on: odd blocks (pairs lie across their borders), empty ones between
    # them, one without room and one whose length is bad; the same bits as by a call for every block
    rng = np.random.default_rng(rows + L)
    counts = [1, 0, 33, 0, 0, 1, 700, 17, 2, 0, 1501, 3, 1]
    counts.append(rows - 20 - sum(counts) - 96)
    counts += [95, 1, 0]
    cu = np.concatenate([[0], np.cumsum(counts)])                            # the last 20 rows are no block's
    n, full, bad = len(counts), 6, 10
    room = [k + 5 for k in counts]
    room[full] = 600
    rope = None if how == "as it is" else Rope(B, 64, L == 256, "parts")
    weight = None if how == "as it is" else torch.randn(L, device="cuda").bfloat16()
    before = rng.integers(0, 6, n)
    before[bad] = -1
    before = np.where(np.asarray(counts) > 0, before, 0)
    c, stride = Cache(B, room, L, rope=rope), L + 64 + (7 if how == "odd stride" else 0)
    x = torch.randn(rows, stride, device="cuda").bfloat16()
    was, first, out = x.clone(), _i32(rng.integers(0, 10 ** 5, n)), torch.full((n,), -7, dtype=torch.int32, device="cuda")
    packed = x if how == "in place" else torch.full((rows, L + 64), 3.0, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_append(c.cfg, c.dims, c.tables, rope and rope.cfg, rope and rope.turns, x, stride, weight, _i32(cu), rows, first, _i32(before),
                               out, c.pool, packed, _stream()) == 0
    assert c.status() in (B.CPA_ENOSPC, B.CPA_EINVAL)
    left_out = lambda b: b in (full, bad)
    assert out.tolist() == [int(before[b]) if left_out(b) else int(before[b]) + counts[b] for b in range(n)]
    stays = torch.ones(rows, dtype=torch.bool, device="cuda")
    d = Cache(B, room, L, rope=rope)
    for b in range(n):
        if counts[b] == 0 or left_out(b):
            continue
        lens, one = np.zeros(n, dtype=np.int64), torch.empty(n, dtype=torch.int32, device="cuda")
        lens[b] = before[b]
        own = torch.empty(counts[b], L + 64, dtype=torch.bfloat16, device="cuda")
        mine = np.concatenate([np.zeros(b + 1), np.full(n - b, counts[b])])
        part = was[cu[b]:cu[b + 1]].clone()
        assert counts[b] <= 4736 and B.cpa_latent_append(d.cfg, d.dims, d.tables, rope and rope.cfg, rope and rope.turns, part, stride, weight,
                                                         _i32(mine), counts[b], first, _i32(lens), one, d.pool, own, _stream()) == 0
        assert torch.equal(packed[cu[b]:cu[b + 1]], own), b
        stays[cu[b]:cu[b + 1]] = False
    assert torch.equal(c.pool.view(torch.int16), d.pool.view(torch.int16)) and d.status() == 0
    assert torch.equal(packed[stays], was[stays] if how == "in place" else torch.full_like(packed[stays], 3.0))


@pytest.mark.parametrize("n", [4735, 4737, 5001])
def test_append_one_row_for_each_of_many_blocks(B, n):
    rng = np.random.default_rng(n)
    c = Cache(B, [1 + b % 3 for b in range(n)], 128, rope=Rope(B))
    was = rng.integers(0, 3, n)                                              # some have no room left
    x, xf = _bf16(rng.standard_normal((n, 192)))
    first, out, packed = _i32(np.arange(n)), torch.empty_like(c.lens), torch.full((n, 192), 3.0, dtype=torch.bfloat16, device="cuda")
    was[::7] = 16
    assert B.cpa_latent_append(c.cfg, c.dims, c.tables, c.rope.cfg, c.rope.turns, x, 192, None, None, n, first, _i32(was), out, c.pool, packed,
                               _stream()) == 0
    fits = was < 16
    assert out.tolist() == (was + fits).tolist() and c.status() == B.CPA_ENOSPC
    want = ol.new_rows(xf, 128, None, 0, np.arange(n) + was, c.rope.f)
    got = _np(packed)
    _check(got[fits], want[fits], ol.rows_tolerance(xf, want, 128)[fits])
    assert (got[~fits] == 3.0).all()
    at = np.array([c.slots(b, was[b], was[b] + 1)[0] for b in np.flatnonzero(fits)])
    assert np.array_equal(_np(c.pool.view(-1, 192)[torch.as_tensor(at, dtype=torch.long, device="cuda")]), got[fits])
    assert int((~torch.isnan(c.pool.view(-1, 192)[:, 0])).sum()) == fits.sum()


# ------------------------------------------------------------------------------------------------ absorbed attention

EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 1000]


@pytest.mark.parametrize("L,H", [(512, 16), (512, 128), (512, 1), (512, 64), (256, 33), (128, 100), (384, 65), (512, 40), (128, 3)])
def test_decode_lengths_heads_and_latents(B, L, H):
    rng = np.random.default_rng(L + H)
    c = Cache(B, [n + 7 for n in EDGES], L, H)
    c.fill(EDGES, rng)
    qc, qr, cf, rf = c.queries(rng)
    o = c.decode(qc, qr)
    assert c.status() == 0
    c.check(o, cf, rf, what="decode")
    assert (o[0] == 0).all()                                                # no token: zeros


@pytest.mark.parametrize("lens,H", [([20000], 16), ([5000], 128), ([1], 128), ([3000, 1, 0, 9], 64), ([700] * 160, 8), ([64] * 300, 4),
                                    ([4096, 4096], 100)])
def test_decode_splits(B, lens, H):
    # one long block over the whole device, few and many blocks: every way in which ranges are cut and joined
    rng = np.random.default_rng(sum(lens))
    c = Cache(B, lens, 512 if H < 100 else 128, H)
    c.fill(lens, rng)
    qc, qr, cf, rf = c.queries(rng)
    o = c.decode(qc, qr)
    assert c.status() == 0
    some = range(len(lens)) if len(lens) < 20 else sorted(rng.choice(len(lens), 20, replace=False))
    c.check(o, cf, rf, some, "split")
    assert torch.equal(c.decode(qc, qr), o)                                 # the same call gives the same bits


@pytest.mark.parametrize("num_sms", [1, 2, 3, 7, 100])
@pytest.mark.parametrize("H", [16, 70])
def test_decode_on_fewer_sms(B, num_sms, H):
    lens = [300, 1, 0, 650, 17, 64]
    rng = np.random.default_rng(num_sms)
    c = Cache(B, lens, 256, H, num_sms=num_sms)
    c.fill(lens, rng)
    qc, qr, cf, rf = c.queries(rng)
    c.check(c.decode(qc, qr), cf, rf, what=f"{num_sms} SMs")
    assert c.status() == 0


def test_decode_takes_strided_queries_and_outputs(B):
    rng = np.random.default_rng(11)
    lens, H, L = [70, 3, 200], 24, 512
    c = Cache(B, lens, L, H)
    c.fill(lens, rng)
    qc, qr, cf, rf = c.queries(rng)
    hq = torch.empty(H, 3, L, dtype=torch.bfloat16, device="cuda").transpose(0, 1)       # as a product per head leaves them
    hq.copy_(qc)
    wide = torch.full((3, H, 192), float("nan"), dtype=torch.bfloat16, device="cuda")    # behind the part without position
    wide[..., 128:] = qr
    out = torch.full((H, 3, L + 8), 4.0, dtype=torch.bfloat16, device="cuda")
    o = c.decode(hq, wide[..., 128:], out=out[..., :L].transpose(0, 1))
    c.check(o, cf, rf, what="strided")
    assert (out[..., L:] == 4.0).all()


@pytest.mark.parametrize("lens,H", [([300], 24), ([300], 100), ([70, 3, 200], 1), ([1], 1)])
def test_strides_of_a_single_block_or_head_do_not_matter(B, lens, H):
    rng = np.random.default_rng(H)
    c = Cache(B, [n + 1 for n in lens], 256, H)
    c.fill(lens, rng)
    qc, qr, cf, rf = c.queries(rng)
    io = lambda o, f: B.cpa_latent_io(qc.data_ptr(), *f(qc.stride()), qr.data_ptr(), *f(qr.stride()), o.data_ptr(), *f(o.stride()))
    odd = lambda s: (13 if c.n == 1 else s[0], -5 if H == 1 else s[1])
    made = []
    for f in (lambda s: s[:2], odd):
        o, o2, out = torch.full_like(qc, 9.0), torch.full_like(qc, 9.0), torch.empty_like(c.lens)
        assert B.cpa_latent_decode(c.cfg, c.dims, c.tables, io(o, f), c.lens, None, c.pool, c.ws, _stream()) == 0
        x = torch.ones(c.n, 320, device="cuda").bfloat16()
        assert B.cpa_latent_step(c.cfg, c.dims, c.tables, None, None, io(o2, f), x, 320, None, None, c.lens, out, None, c.pool, c.ws, _stream()) == 0
        made.append((o, o2))
    c.check(made[0][0], cf, rf)
    assert c.status() == 0 and all(torch.equal(a, b) for a, b in zip(*made))


def test_decode_inactive_and_bad_blocks_sit_out(B):
    rng = np.random.default_rng(12)
    lens = [100, 64, 7, 30, 500]
    c = Cache(B, lens, 256, 20)
    c.fill(lens, rng)
    qc, qr, cf, rf = c.queries(rng)
    o = c.decode(qc, qr, active=_i32([1, 0, 5, 0, -1]))
    c.check(o, cf, rf, [0, 2, 4])
    assert (o[[1, 3]] == 9.0).all() and c.status() == 0
    o = c.decode(qc, qr, active=_i32([0] * 5))
    assert (o == 9.0).all()
    for bad, word in ((-1, B.CPA_EINVAL), (113, B.CPA_ENOSPC), (2 ** 31 - 1, B.CPA_ENOSPC), (-2 ** 31, B.CPA_EINVAL)):
        d = Cache(B, lens, 256, 20)
        d.pool, d.rows, d.ids, d.lens = c.pool, c.rows, c.ids, c.lens
        n = list(lens)
        n[0] = bad
        o = d.decode(qc, qr, lens=_i32(n))
        d.check(o, cf, rf, [1, 2, 3, 4], f"beside a length of {bad}")
        assert (o[0] == 9.0).all() and d.status() == word


@pytest.mark.parametrize("H,L", [(16, 512), (40, 256), (128, 512), (66, 128)])
def test_decode_masks_by_index_not_by_value(B, H, L):
    # what lies behind a block's length may be anything: NaN (as everywhere here), infinities, the largest values
    rng = np.random.default_rng(13)
    lens = [1, 17, 63, 65, 100, 190]
    for junk in (float("inf"), float("-inf"), 3e38):
        c = Cache(B, [256] * 6, L, H)
        c.pool.fill_(junk)
        c.fill(lens, rng)
        qc, qr, cf, rf = c.queries(rng)
        c.check(c.decode(qc, qr), cf, rf, what=str(junk))


@pytest.mark.parametrize("H,L", [(16, 512), (33, 256), (64, 128), (128, 512), (70, 128)])
@pytest.mark.parametrize("num_sms,lens", [(2, [1300, 40, 200]), (0, [5000]), (0, [1300, 40, 200, 1])])
@pytest.mark.parametrize("spread", [2.0 ** -131, 2.0 ** -126, 2.0 ** -123])
def test_decode_keeps_outputs_below_the_normal_range(B, H, L, num_sms, lens, spread):
    # latent parts that small come through, moves of the references (a token whose score lies 2^14 above the first one's, late) and joins too
    rng = np.random.default_rng(H + len(lens))
    c = Cache(B, lens, L, H, num_sms=num_sms)
    flat = c.pool.view(-1, L + 64)
    for b, n in enumerate(lens):
        x = np.zeros((n, L + 64))
        x[:, :L] = spread * (1 + rng.random((n, L)))
        x[n - min(n, 30), :] = 0.0
        x[n - min(n, 30), L] = 140.0
        x, c.rows[b] = _bf16(x)
        flat[torch.as_tensor(c.slots(b, 0, n), dtype=torch.long, device="cuda")] = x
    c.lens = _i32(lens)
    qc, qr = torch.zeros(c.n, H, L, device="cuda").bfloat16(), torch.zeros(c.n, H, 64, device="cuda").bfloat16()
    qr[:, :, 0] = 1.0
    c.check(c.decode(qc, qr), _np(qc), _np(qr), what="tiny values")
    assert c.status() == 0


@pytest.mark.parametrize("H", [16, 128])
def test_decode_scores_of_any_range(B, H):
    rng = np.random.default_rng(14)
    lens = [300, 1000, 129, 64]
    # growing scores move the running maximum at every tile; huge ones leave one token; tiny ones weigh all the same
    for grow, spread in ((1.0, 4.0), (1.0, 40.0), (1.02, 1.0), (1.0, 1e-4)):
        c = Cache(B, lens, 256, H)
        c.fill(lens, rng)
        flat = c.pool.view(-1, 320)
        for b, n in enumerate(lens):
            x, xf = _bf16(c.rows[b] * grow ** np.minimum(np.arange(n), 200)[:, None])
            flat[torch.as_tensor(c.slots(b, 0, n), dtype=torch.long, device="cuda")] = x
            c.rows[b] = xf
        qc, qr, cf, rf = c.queries(rng, spread)
        c.check(c.decode(qc, qr), cf, rf, what=f"{grow} {spread}")


@pytest.mark.parametrize("H", [4, 33, 100])
def test_decode_scores_that_are_minus_infinity_or_nan(B, H):
    rng = np.random.default_rng(15)
    lens = [200, 200, 70, 128]
    c = Cache(B, lens, 128, H)
    c.fill(lens, rng)
    flat = c.pool.view(-1, 192)
    qc, qr, cf, rf = c.queries(rng)
    qr[:, :, 0], rf[:, :, 0] = 1.0, 1.0
    low = torch.as_tensor(c.slots(0, 0, 130), dtype=torch.long, device="cuda")
    flat[low, 128] = float("-inf")                                          # block 0: the first two tiles have no weight
    one = torch.as_tensor(c.slots(1, 150, 151), dtype=torch.long, device="cuda")
    flat[one, 128] = float("nan")                                           # block 1: a NaN score
    flat[torch.as_tensor(c.slots(3, 0, 128), dtype=torch.long, device="cuda"), 128] = float("-inf")   # block 3: all of them
    o = c.decode(qc, qr)
    c.rows[0] = c.rows[0][130:]
    c.check(o, cf, rf, [0, 2], "minus infinity")
    assert torch.isnan(o[1]).all() and torch.isnan(o[3]).all()


@pytest.mark.parametrize("H", [16, 128])
def test_decode_far_pages(B, H):
    # page ids on both sides of the pool's 2^32-byte line
    page = 16 * 576 * 2
    edge = 2 ** 32 // page
    free = torch.cuda.mem_get_info()[0]
    if free < 6 * 2 ** 30:
        pytest.skip("too little memory")
    ids = np.array([edge + 40, 3, edge - 1, edge, edge + 1, 0, 2 * edge // 2 + 7], dtype=np.int32)
    rng = np.random.default_rng(16)
    c = Cache(B, [100], 512, H, page_ids=(ids, edge + 64), rope=Rope(B))
    c.fill([90], rng)
    qc, qr, cf, rf = c.queries(rng)
    c.check(c.decode(qc, qr), cf, rf, what="far pages")
    c.append(rng.standard_normal((1, 576)), None, np.ones(512))
    c.check(c.decode(qc, qr), cf, rf, what="far pages")
    assert c.status() == 0


@pytest.mark.parametrize("H", [8, 64, 96])
def test_decode_and_step_of_many_short_blocks(B, H):
    # several blocks to a thread of the cut, many segments to a CTA, empty and inactive ones between them
    rng = np.random.default_rng(H)
    lens = rng.integers(0, 90, 1300)
    lens[rng.random(1300) < 0.2] = 0
    c = Cache(B, lens + 1, 128, H, rope=Rope(B))
    c.fill(list(lens), rng)
    qc, qr, cf, rf = c.queries(rng)
    some = sorted(rng.choice(1300, 40, replace=False))
    o = c.decode(qc, qr)
    assert c.status() == 0
    c.check(o, cf, rf, some, "many")
    assert (o[torch.as_tensor(np.flatnonzero(lens == 0), device="cuda")] == 0).all()
    active = (rng.random(1300) < 0.7).astype(np.int32)
    _step(c, rng, np.ones(128), rng.integers(0, 1000, 1300), _i32(active), blocks=some)
    assert c.status() == 0


# ------------------------------------------------------------------------------------------------ steps

def _step(c, rng, weight, first, active=None, qspread=1.0, blocks=None):
    """One step of all blocks; checks rows, lengths and outputs."""
    B, r = c.B, c.rope
    x, xf = _bf16(rng.standard_normal((c.n, c.L + 64)))
    wd, wf = _bf16(weight)
    qc, qr, cf, rf = c.queries(rng, qspread)
    o, out = torch.full((c.n, c.H, c.L), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full_like(c.lens, -7)
    was = c.lens.cpu().numpy()
    rc = B.cpa_latent_step(c.cfg, c.dims, c.tables, r and r.cfg, r and r.turns, B.latent_io(qc, qr, o), x, c.L + 64, wd, _i32(first), c.lens, out,
                           active, c.pool, c.ws, _stream())
    assert rc == 0
    pos = np.asarray(first) + was
    want = ol.new_rows(xf, c.L, wf, c.eps, pos, r and r.f, r is None or r.interleaved)
    tol = ol.rows_tolerance(xf, want, c.L, r is None or r.interleaved)
    on = [b for b in range(c.n) if active is None or int(active[b])]
    flat = c.pool.view(-1, c.L + 64)
    for b in on:
        got = _np(flat[torch.as_tensor(c.slots(b, was[b], was[b] + 1), dtype=torch.long, device="cuda")])
        _check(got, want[b:b + 1], tol[b:b + 1], f"new row of block {b}")
        c.rows[b] = np.concatenate([c.rows[b], got])
    c.lens = out
    c.check_rest()
    if r:
        rf = ol.turn(rf, pos[:, None], r.f, r.interleaved)
    # the turned query is rounded to bf16: 2^-8 of each element, times the positional key, in the score
    score = [c.scale * 2.0 ** -8 * (np.abs(rf[b]) @ np.abs(c.rows[b][:, c.L:]).T).max(1)[:, None] if len(c.rows[b]) else 0.0 for b in range(c.n)]
    c.check(o, cf, rf, [b for b in on if blocks is None or b in blocks], "step", score if r else None)
    for b in range(c.n):
        if b not in on:
            assert (o[b] == 9.0).all()
    return o


@pytest.mark.parametrize("H,L,interleaved", [(16, 512, True), (128, 512, False), (5, 128, True), (64, 256, False)])
def test_steps(B, H, L, interleaved):
    rng = np.random.default_rng(H)
    lens = [0, 1, 14, 15, 16, 17, 62, 63, 64, 65, 300, 1000]
    c = Cache(B, [n + 4 for n in lens], L, H, rope=Rope(B, 64, interleaved, "parts"))
    c.fill(lens, rng)
    first, w = rng.integers(0, 10 ** 5, len(lens)), 1 + 0.1 * rng.standard_normal(L)
    for i in range(4):
        _step(c, rng, w, first, None if i % 2 else _i32([(b + i) % 3 for b in range(len(lens))]))
    assert c.status() == 0
    c = Cache(B, [n + 4 for n in lens], L, H)                               # without positions
    c.fill(lens, rng)
    _step(c, rng, w, first)


def test_step_without_room_sits_out(B):
    rng = np.random.default_rng(22)
    c = Cache(B, [16, 16, 32], 128, 8)
    c.fill([16, 3, 31], rng)
    qc, qr, cf, rf = c.queries(rng)
    x, xf = _bf16(rng.standard_normal((3, 192)))
    o, out = torch.full((3, 8, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.empty_like(c.lens)
    before = c.pool.clone()
    assert B.cpa_latent_step(c.cfg, c.dims, c.tables, None, None, B.latent_io(qc, qr, o), x, 192, None, None, c.lens, out, None, c.pool, c.ws,
                             _stream()) == 0
    assert out.tolist() == [16, 4, 32] and c.status() == B.CPA_ENOSPC
    for b, n in ((1, 3), (2, 31)):
        c.rows[b] = np.concatenate([c.rows[b], xf[b:b + 1]])
    c.check(o, cf, rf, [1, 2])
    assert (o[0] == 9.0).all()
    same = torch.as_tensor(c.slots(0, 0, 16), dtype=torch.long, device="cuda")
    assert torch.equal(c.pool.view(-1, 192)[same], before.view(-1, 192)[same])


def test_steps_captured_and_replayed(B):
    # two steps in one graph, replayed: lengths go on as in a loop; the same steps outside of it give the same cache and outputs
    rng = np.random.default_rng(23)
    lens, H, L = [60, 0, 130, 15], 16, 512
    w, first = torch.ones(L, dtype=torch.bfloat16, device="cuda"), _i32([5, 0, 10 ** 5, 77])
    rope = Rope(B)
    made = []
    for graph in (True, False):
        c = Cache(B, [n + 8 for n in lens], L, H, seed=1, rope=rope)
        c.fill(lens, np.random.default_rng(1))
        gen = np.random.default_rng(2)
        qs = [c.queries(gen)[:2] for _ in range(2)]
        xs = [_bf16(gen.standard_normal((4, L + 64)))[0] for _ in range(2)]
        a, b = c.lens, torch.empty_like(c.lens)
        outs = [torch.empty(4, H, L, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

        def two():
            for i, (src, dst) in enumerate(((a, b), (b, a))):
                assert B.cpa_latent_step(c.cfg, c.dims, c.tables, rope.cfg, rope.turns, B.latent_io(*qs[i], outs[i]), xs[i], L + 64, w, first, src,
                                         dst, None, c.pool, c.ws, _stream()) == 0
        if graph:
            g = torch.cuda.CUDAGraph()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
                two()
            torch.cuda.current_stream().wait_stream(side)
            for _ in range(3):
                g.replay()
        else:
            for _ in range(3):
                two()
        torch.cuda.synchronize()
        assert a.tolist() == [n + 6 for n in lens] and c.status() == 0
        made.append((c.pool.clone().view(torch.int16), [o.clone() for o in outs]))
    assert torch.equal(made[0][0], made[1][0])
    assert all(torch.equal(x, y) for x, y in zip(made[0][1], made[1][1]))


def test_two_caches_on_two_streams(B):
    rng = np.random.default_rng(24)
    caches = []
    for i in range(2):
        lens = [900, 30, 411] if i else [2000, 5]
        c = Cache(B, lens, 512, 64 if i else 16, seed=i)
        c.fill(lens, rng)
        caches.append((c, c.queries(rng)))
    want = [c.decode(*q[:2]) for c, q in caches]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(10):
        for i, (c, q) in enumerate(caches):
            with torch.cuda.stream(streams[i]):
                got[i].append(c.decode(*q[:2]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])
        caches[i][0].check(want[i], *caches[i][1][2:])


@pytest.mark.parametrize("H", [64, 128])
def test_graphs_of_two_caches_replayed_at_once(B, H):
    # a step and the decode behind it, captured for each of two caches with tables and workspaces of their own, replayed side by side
    rng = np.random.default_rng(H)
    w, first = torch.ones(512, dtype=torch.bfloat16, device="cuda"), _i32([3, 0, 99])
    rope, runs = Rope(B), []
    for i in range(2):
        lens = [1500, 0, 77] if i else [9, 2300, 640]
        c = Cache(B, [n + 1 for n in lens], 512, H, seed=i, rope=rope)
        c.fill(lens, rng)
        qc, qr = c.queries(rng)[:2]
        x = _bf16(rng.standard_normal((3, 576)))[0]
        out, o, o2 = torch.empty_like(c.lens), *(torch.empty(3, H, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2))

        def run(c=c, qc=qc, qr=qr, x=x, out=out, o=o, o2=o2):
            assert B.cpa_latent_step(c.cfg, c.dims, c.tables, rope.cfg, rope.turns, B.latent_io(qc, qr, o), x, 576, w, first, c.lens, out, None,
                                     c.pool, c.ws, _stream()) == 0
            assert B.cpa_latent_decode(c.cfg, c.dims, c.tables, B.latent_io(qc, qr, o2), out, None, c.pool, c.ws, _stream()) == 0
        run()                                             # (the step stores the same row again whenever it is repeated)
        torch.cuda.synchronize()
        want = [o.clone(), o2.clone(), out.clone()]
        g, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=stream):
            run()
        runs.append((g, stream, (o, o2, out), want, c, run))         # (run holds the graph's inputs)
    torch.cuda.synchronize()
    for _ in range(20):
        for g, stream, *_ in runs:
            with torch.cuda.stream(stream):
                g.replay()
    torch.cuda.synchronize()
    for _, _, got, want, c, _ in runs:
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and c.status() == 0


@pytest.mark.parametrize("H", [4, 72])
def test_few_blocks_with_tokens_among_many_without(B, H):
    rng = np.random.default_rng(H)
    n = 6000
    lens = np.zeros(n, dtype=np.int64)
    lens[[0, 2700, n - 1]] = [700, 1, 130]
    c = Cache(B, lens, 128, H)
    c.fill(list(lens), rng)
    q = [torch.randn(n, H, e, device="cuda").bfloat16() for e in (128, 64)]
    o = c.decode(*q)
    assert c.status() == 0
    at = np.flatnonzero(lens)
    on = torch.as_tensor(at, device="cuda")
    cf, rf = ({b: _np(t[b]) for b in at} for t in q)
    c.check(o, cf, rf, at, "few")
    o[on] = 0
    assert (o == 0).all()


# ------------------------------------------------------------------------------------------------ every token, once
#
# Values of zero and one show a token that is lost or taken twice at any length: element e of the output is the weight of the tokens
# marked e over that of all, and no more than 60 tokens share a mark.  Bounds: queries score the positional part's first element k, a whole
# number, with scale ln 2 to fp32, so that a weight is 2^k but for |k| 2^-23 at most (2^-18 for |k| <= 32, and the same again of every factor by
# which a reference moves); rounded to bf16 it is 2^k.  Sums of such weights, two reciprocals' and products' roundings: below 2^-20.
# The output: 2^-8.  In all |o| (2^-8 + 2^-14).  The lightest of sixty, a quarter of the heaviest, is 2^-7.1.  The last element, marked in all tokens, is one, exactly.

MARKED = 2.0 ** -8 + 2.0 ** -14


def _marks(n, m, k):
    """[n, m + 1]: where the scores k are equal, token j has mark j % m, else stretches of equal length in either half of the tokens (whose
    weights are of one size) have one mark; and one for all."""
    v, j, a, half = np.zeros((n, m + 1)), np.arange(n), n // 2, m // 2
    v[j, j % m if (k == k[:1]).all() else np.where(j < a, j * half // max(a, 1), half + (j - a) * (m - half) // max(n - a, 1))] = 1.0
    v[:, m] = 1.0
    return v


def _scores(n, kind):
    """Whole numbers: all alike; moving up by more than a reference allows; falling, so that the first tile's reference stays."""
    j = np.arange(n)
    if kind == "alike":
        return np.zeros(n)
    return (16.0 if kind == "rising" else -16.0) * (j >= n // 2) + (j % 3)


def _check_marked(got, k, m, what):
    w = 2.0 ** k
    want = (w[:, None] * _marks(len(k), m, k)).sum(0) / w.sum()
    _check(got, np.broadcast_to(want, got.shape), np.broadcast_to(MARKED * want, got.shape), what)
    assert (got[..., m] == 1.0).all(), what


@pytest.mark.parametrize("kind", ["alike", "rising", "falling"])
@pytest.mark.parametrize("H", [16, 40, 64, 128])
@pytest.mark.parametrize("num_sms,lens", [(0, EDGES), (0, [30000]), (0, [20011, 5, 3000, 1]), (3, [2011, 700, 64, 65]), (0, [997] * 40)])
def test_decode_and_step_take_every_token_once(B, H, num_sms, lens, kind):
    c = Cache(B, [n + 1 for n in lens], 512, H, num_sms=num_sms, scale=float(np.float32(np.log(2.0))))
    rng, flat = np.random.default_rng(H), c.pool.view(-1, 576)
    # (the tokens behind the first are what a step adds)
    rows = [np.concatenate([_marks(n + 1, 511, _scores(n + 1, kind)), _scores(n + 1, kind)[:, None], rng.standard_normal((n + 1, 63))], 1) for n in lens]
    for b, n in enumerate(lens):
        if n:
            flat[torch.as_tensor(c.slots(b, 0, n), dtype=torch.long, device="cuda")] = _bf16(rows[b][:n])[0]
    c.lens = _i32(lens)
    qc, qr = torch.zeros(c.n, H, 512, device="cuda").bfloat16(), torch.zeros(c.n, H, 64, device="cuda").bfloat16()
    qr[:, :, 0] = 1.0
    o = _np(c.decode(qc, qr))
    for b, n in enumerate(lens):
        if n:
            k = _scores(n + 1, kind)
            w, v = 2.0 ** k[:n], rows[b][:n, :512]
            want = np.broadcast_to((w[:, None] * v).sum(0) / w.sum(), o[b].shape)
            _check(o[b], want, MARKED * want, f"decode, block of {n}")
            assert (o[b][:, 511] == 1.0).all()
    x, _ = _bf16(np.stack([r[-1] for r in rows]))
    out, o = torch.empty_like(c.lens), torch.empty(c.n, H, 512, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_step(c.cfg, c.dims, c.tables, None, None, B.latent_io(qc, qr, o), x, 576, None, None, c.lens, out, None, c.pool, c.ws,
                             _stream()) == 0
    o = _np(o)
    for b, n in enumerate(lens):
        _check_marked(o[b], _scores(n + 1, kind), 511, f"step, block of {n + 1}")
    assert out.tolist() == [n + 1 for n in lens] and c.status() == 0


@pytest.mark.parametrize("kind", ["alike", "rising", "falling"])
@pytest.mark.parametrize("rows", [128, 256])
@pytest.mark.parametrize("lens,H,num_sms", [([1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 128, 129], 2, 3), ([255, 256, 257, 383, 384, 385], 3, 0),
                                            ([2500, 18, 1300], 1, 0)])
def test_prefill_takes_every_token_once(B, lens, H, num_sms, rows, kind):
    T, scale = sum(lens), float(np.float32(np.log(2.0)))
    qf, kvf, rf = np.zeros((T, H, 192)), np.zeros((T, H, 256)), np.zeros((T, 64))
    qf[:, :, 128] = 1.0
    cu = np.concatenate([[0], np.cumsum(lens)])
    for a, n in zip(cu, lens):
        k = _scores(n, kind)
        kvf[a:a + n, :, 128:], rf[a:a + n, 0] = _marks(n, 127, k)[:, None], k
    (q, _), (kv, _), (r, _) = _bf16(qf), _bf16(kvf), _bf16(rf)
    cfg = B.cpa_latent_config(H, 512, 64, 128, 128, 16, scale, 1e-6, num_sms)
    pc = B.cpa_latent_plan_config(cfg)
    pc.q_tile_rows = rows
    plan = B.cpa_plan_create(pc, lens, 0, [0] * sum(-(-n // 16) for n in lens))
    index = torch.empty(B.cpa_plan_param(plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
    assert B.cpa_plan_upload(plan, index, index.numel(), _stream()) == 0
    o = torch.full((T, H, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_prefill(cfg, plan, q, kv, r, 64, o, _stream()) == 0 and B.cpa_plan_status(plan, _stream()) == 0
    o = _np(o)
    for a, n in zip(cu, lens):
        w = 2.0 ** rf[a:a + n, :1] * kvf[a:a + n, 0, 128:]
        want = (np.cumsum(w, 0) / np.cumsum(2.0 ** rf[a:a + n, :1], 0))[:, None]
        _check(o[a:a + n], np.broadcast_to(want, (n, H, 128)), np.broadcast_to(MARKED * want, (n, H, 128)), f"block of {n}")
        assert (o[a:a + n, :, 127] == 1.0).all()
    B.cpa_plan_destroy(plan)


# ------------------------------------------------------------------------------------------------ expanded attention

def _prefill(B, lens, H, rng, spread=1.0, stride=576, num_sms=0, scale=192 ** -0.5, rows=None):
    T = sum(lens)
    cfg = B.cpa_latent_config(H, 512, 64, 128, 128, 16, scale, 1e-6, num_sms)
    pc = B.cpa_latent_plan_config(cfg)
    pc.q_tile_rows = rows or pc.q_tile_rows
    plan = B.cpa_plan_create(pc, lens, 0, list(range(sum(-(-n // 16) for n in lens))))
    index = torch.empty(B.cpa_plan_param(plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
    assert B.cpa_plan_upload(plan, index, index.numel(), _stream()) == 0
    (q, qf), (kv, kvf) = _bf16(spread * rng.standard_normal((T, H, 192))), _bf16(rng.standard_normal((T, H, 256)))
    (r, rf) = _bf16(rng.standard_normal((T, stride)))
    part = r[:, stride - 64:]
    o = torch.full((T + 2, H, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_prefill(cfg, plan, q, kv, part, stride, o, _stream()) == 0
    assert B.cpa_plan_status(plan, _stream()) == 0
    want, wide, shaken = ol.prefill(qf, kvf, rf[:, stride - 64:], np.concatenate([[0], np.cumsum(lens)]), float(np.float32(scale)))
    _check(o[:T], want, ol.attention_tolerance(want, wide, shaken, 192), f"prefill {lens[:6]}")
    assert (o[T:] == 9.0).all()                                             # rows behind the last block
    B.cpa_plan_destroy(plan)


@pytest.mark.parametrize("lens,H", [([1], 1), ([1, 2, 3], 4), ([127, 128, 129], 2), ([255, 256, 257, 1], 3), ([700], 1), ([64, 63, 65, 385], 16),
                                    ([1500, 40], 2), ([30] * 40, 5), ([513, 640, 300], 20)])
def test_prefill_lengths_and_heads(B, lens, H):
    for rows in (256, 128):
        _prefill(B, lens, H, np.random.default_rng(sum(lens) + H), rows=rows)


@pytest.mark.parametrize("lens,H", [([40, 131], 128), ([260, 1, 64], 65), ([385], 40)])
def test_prefill_of_many_heads(B, lens, H):
    _prefill(B, lens, H, np.random.default_rng(H))


@pytest.mark.parametrize("lens,H,num_sms", [([18] * 60, 5, 4), ([1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 66], 3, 2),
                                            ([129, 144, 145, 160, 161, 191, 192, 193, 257, 300, 320, 321], 2, 3),
                                            ([20, 300, 64, 1, 513, 130, 7, 40, 256, 2, 383], 4, 5), ([5, 200, 3, 450] * 8, 2, 1)])
def test_prefill_short_and_long_units_in_turn(B, lens, H, num_sms):
    # many units to a CTA: short blocks, short ends of long ones and whole tiles follow one another through the same buffers
    for spread, rows in ((1.0, 256), (20.0, 256), (1.0, 128)):
        _prefill(B, lens, H, np.random.default_rng(len(lens) + H), spread, 64, num_sms, rows=rows)


@pytest.mark.parametrize("spread,stride,num_sms", [(30.0, 64, 0), (1e-3, 72, 0), (1.0, 576, 3), (4.0, 192, 1)])
def test_prefill_scores_strides_and_sms(B, spread, stride, num_sms):
    _prefill(B, [300, 17, 600], 3, np.random.default_rng(stride), spread, stride, num_sms)


def test_prefill_keeps_what_is_not_finite_to_its_own(B):
    # NaN and infinities in the next block, and in keys of the row's future, change nothing; values that are not finite reach
    # the rows from their own on (and, of their own block, the earlier ones of their 128-token tile)
    rng = np.random.default_rng(30)
    lens, H = [70, 130, 200], 2
    T = sum(lens)
    cfg = B.cpa_latent_config(H, 512, 64, 128, 128, 16, 192 ** -0.5, 1e-6, 0)
    plan = B.cpa_plan_create(B.cpa_latent_plan_config(cfg), lens, 0, list(range(27)))
    index = torch.empty(B.cpa_plan_param(plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
    assert B.cpa_plan_upload(plan, index, index.numel(), _stream()) == 0
    (q, _), (kv, _), (r, _) = _bf16(rng.standard_normal((T, H, 192))), _bf16(rng.standard_normal((T, H, 256))), _bf16(rng.standard_normal((T, 64)))
    run = lambda: (lambda o: (B.cpa_latent_prefill(cfg, plan, q, kv, r, 64, o, _stream()), o)[1])(torch.empty(T, H, 128, dtype=torch.bfloat16, device="cuda"))
    plain = run()
    for bad in (float("nan"), float("inf")):
        was = kv[70:200].clone(), r[70:200].clone()
        kv[70:200], r[70:200] = bad, bad                       # all of block 1
        o = run()
        assert torch.equal(o[:70], plain[:70]) and torch.equal(o[200:], plain[200:])
        assert not torch.isfinite(o[70:200].float()).any()
        kv[70:200], r[70:200] = was
        key = kv[300, 0, :128].clone()
        kv[300, 0, :128] = bad                                 # a key of block 2: earlier rows and the other head do not see it
        o = run()
        assert torch.equal(o[:300], plain[:300]) and torch.equal(o[:, 1], plain[:, 1])
        assert torch.isnan(o[300:, 0]).all() or bad != bad
        kv[300, 0, :128] = key
        value = kv[390, 1, 130].clone()
        kv[390, 1, 130] = bad                                  # a value in block 2's second tile: its first tile does not see it
        o = run()
        assert torch.equal(o[:328], plain[:328]) and torch.equal(o[:, 0], plain[:, 0])
        assert not torch.isfinite(o[390:, 1, 2].float()).any()
        kv[390, 1, 130] = value
    assert torch.equal(run(), plain)
    B.cpa_plan_destroy(plan)


@pytest.mark.parametrize("rows", [128, 256])
@pytest.mark.parametrize("lens", [[1300], [129, 40, 257, 1000]])
@pytest.mark.parametrize("spread", [2.0 ** -130, 2.0 ** -126, 2.0 ** -123])
def test_prefill_keeps_outputs_below_the_normal_range(B, rows, lens, spread):
    # values that small come through, the references' moves too: a key whose score lies 2^9 above the others' in a later tile
    H, T, scale = 2, sum(lens), float(np.float32(192 ** -0.5))
    rng = np.random.default_rng(len(lens))
    qf, kvf, rf = np.zeros((T, H, 192)), np.zeros((T, H, 256)), np.zeros((T, 64))
    qf[:, :, 128] = 1.0
    kvf[..., 128:] = spread * (1 + rng.random((T, H, 128)))
    for a, n in zip(np.cumsum([0] + lens), lens):
        at = a + n - min(n, 30)
        rf[at, 0], kvf[at, :, 128:] = 91.0, 0.0
    (q, qf), (kv, kvf), (r, rf) = _bf16(qf), _bf16(kvf), _bf16(rf)
    cfg = B.cpa_latent_config(H, 512, 64, 128, 128, 16, scale, 1e-6, 0)
    pc = B.cpa_latent_plan_config(cfg)
    pc.q_tile_rows = rows
    plan = B.cpa_plan_create(pc, lens, 0, [0] * sum(-(-n // 16) for n in lens))
    index = torch.empty(B.cpa_plan_param(plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
    assert B.cpa_plan_upload(plan, index, index.numel(), _stream()) == 0
    o = torch.full((T, H, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_prefill(cfg, plan, q, kv, r, 64, o, _stream()) == 0 and B.cpa_plan_status(plan, _stream()) == 0
    want, wide, shaken = ol.prefill(qf, kvf, rf, np.concatenate([[0], np.cumsum(lens)]), scale)
    _check(o, want, ol.attention_tolerance(want, wide, shaken, 192), "tiny values")
    B.cpa_plan_destroy(plan)


# ------------------------------------------------------------------------------------------------ a whole event

@pytest.mark.parametrize("H,L", [(8, 256), (40, 512)])
def test_event_expanded_and_absorbed_agree(B, H, L):
    """Prompts through append and expanded prefill, then steps in the absorbed form, against one attention in 64 bits over the
    rows that the cache holds."""
    rng = np.random.default_rng(H)
    lens, T, scale = [130, 1, 77], 3, 192 ** -0.5
    rope = Rope(B)
    c = Cache(B, [n + T for n in lens], L, H, rope=rope, scale=scale)
    n, first = sum(lens), [0, 500, 9000]
    U, W = (rng.standard_normal((H, 128, L)) * L ** -0.5 for _ in range(2))
    w = 1 + 0.1 * rng.standard_normal(L)
    packed = c.append(rng.standard_normal((n, L + 64)), lens, w, first)
    rows = _np(packed)
    # expanded: the caller's products, rounded to bf16
    kv, kvf = _bf16(np.concatenate([np.einsum("hel,tl->the", U, rows[:, :L]), np.einsum("hel,tl->the", W, rows[:, :L])], 2))
    q, qf = _bf16(rng.standard_normal((n, H, 192)))
    pos = np.concatenate([np.arange(k) + f for k, f in zip(lens, first)])
    assert B.cpa_rope(rope.cfg, rope.turns, _i32(pos), n, B.rope_rows(q[..., 128:], None, 64), None, False, _stream()) == 0
    qf = _np(q)
    plan = B.cpa_plan_create(B.cpa_latent_plan_config(c.cfg), lens, 0, list(range(20)))
    index = torch.empty(B.cpa_plan_param(plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
    assert B.cpa_plan_upload(plan, index, index.numel(), _stream()) == 0
    o = torch.empty(n, H, 128, dtype=torch.bfloat16, device="cuda")
    assert B.cpa_latent_prefill(c.cfg, plan, q, kv, packed[:, L:], L + 64, o, _stream()) == 0
    cu = np.concatenate([[0], np.cumsum(lens)])
    want, wide, shaken = ol.prefill(qf, kvf, rows[:, L:], cu, c.scale)
    _check(o, want, ol.attention_tolerance(want, wide, shaken, 192), "expanded")
    # absorbed, for the last token of every block: the same output but for the roundings of keys, values and taken-over queries
    last = cu[1:] - 1
    qa, qaf = _bf16(np.einsum("hel,bhe->bhl", U, qf[last, :, :128]))
    oa = c.decode(qa, q[torch.as_tensor(last, device="cuda")][..., 128:].contiguous())
    c.check(oa, qaf, qf[last, :, 128:], what="absorbed")
    back = np.einsum("hel,bhl->bhe", W, _np(oa))
    for b in range(3):
        r = rows[cu[b]:cu[b + 1]]
        for h in range(H):
            k, v = np.concatenate([r[:, :L] @ U[h].T, r[:, L:]], 1), r[:, :L] @ W[h].T
            s = c.scale * (k @ qf[last[b], h])
            p = np.exp(s - s.max())
            p /= p.sum()
            exact = p @ v
            # roundings: operands of the scores by 2^-8 each in either form (2 x 2^-8 of the products' magnitudes), weights and
            # values by 2^-8, the output by 2^-8, and the absorbed output's 2^-8 through W
            e = 2 * 2.0 ** -8 * c.scale * max((np.abs(k) @ np.abs(qf[last[b], h])).max(), (np.abs(r[:, :L]) @ np.abs(qaf[b, h])).max())
            through = np.abs(W[h]) @ np.abs(_np(oa)[b, h])
            tol = 4 * 2.0 ** -8 * (p @ np.abs(v) + np.abs(exact)) + 2 * e * (p @ np.abs(v)) + 2.0 ** -7 * through
            assert (np.abs(_np(o)[last[b], h] - exact) <= tol).all() and (np.abs(back[b, h] - exact) <= tol).all(), (b, h)
    for _ in range(T):
        _step(c, rng, w, first)
    assert c.status() == 0 and B.cpa_plan_status(plan, _stream()) == 0
    B.cpa_plan_destroy(plan)
