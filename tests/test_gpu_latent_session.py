"""Latent attention and rotary positions through the sessions: a whole event, captured steps, another stream, refusals, and
rotary positions ahead of an event of grouped-query attention."""
import numpy as np
import pytest

from oracle import latent as ol

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16).cuda()


def _session(rng, lens, T, H, L, rope=True, **more):
    from paper_2605_23296_b200 import binding as B
    from paper_2605_23296_b200.session import LatentSession, Rotary
    pages = sum(-(-(n + T) // 16) for n in lens)
    ids = rng.permutation(pages + 2).astype(np.int32)
    r = Rotary(64, interleaved=True, scaling=B.ROPE_SCALED_PARTS, factor=40.0, trained_len=4096) if rope else None
    w = (1 + 0.1 * torch.from_numpy(rng.standard_normal(L))).to(torch.bfloat16).cuda()
    s = LatentSession(lens, T, H, ids, pages + 2, L, rope=r, norm_weight=w, poison_pools=True, **more)
    return s, ids


def _row(s, ids, lens, T, b, at):
    page = ids[sum(-(-(n + T) // 16) for n in lens[:b]) + at // 16]
    return _np(s.pool[int(page), at % 16])


@pytest.mark.parametrize("H,L,first", [(16, 512, None), (70, 256, [5, 0, 123456, 77])])
def test_event(H, L, first):
    rng = np.random.default_rng(H)
    lens, T = [130, 1, 40, 257], 4
    s, ids = _session(rng, lens, T, H, L, first=first)
    n, f = sum(lens), ol.frequencies(64, 10000.0, "parts", 40.0, 32.0, 1.0, 4096)
    start = first or [0] * 4
    wide = _bf16(rng, n, L + 64 + 8)                         # rows inside a wider projection
    x = wide[:, :L + 64]
    packed = s.append_prefill(x)
    pos = np.concatenate([np.arange(k) + p for k, p in zip(lens, start)])
    want = ol.new_rows(_np(x), L, _np(s.norm_weight), float(np.float32(1e-6)), pos, f)
    assert (np.abs(_np(packed) - want) <= ol.rows_tolerance(_np(x), want, L)).all()
    raw = _bf16(rng, n, H, 192)
    q = s.turn_queries(raw.clone())
    y = ol.turn(_np(raw)[..., 128:], pos[:, None], f, True)
    assert (np.abs(_np(q)[..., 128:] - y) <= ol.turn_tolerance(_np(raw)[..., 128:], y, True)).all()
    assert torch.equal(q[..., :128], raw[..., :128])
    kv = _bf16(rng, n, H, 256)
    o = s.prefill(q, kv, packed)
    rows = _np(packed)
    want, spread, shaken = ol.prefill(_np(q), _np(kv), rows[:, L:], np.cumsum([0] + lens), s.scale)
    assert (np.abs(_np(o) - want) <= ol.attention_tolerance(want, spread, shaken, 192)).all()
    cached = np.split(rows, np.cumsum(lens)[:-1])
    for t in range(T):
        qc, qr, x = _bf16(rng, 4, H, L), _bf16(rng, 4, H, 64), _bf16(rng, 4, L + 64)
        if t == 2:                                            # append and decode apart, the query turned by hand
            assert torch.equal(s.append(x, packed=True)[2], torch.from_numpy(_row(s, ids, lens, T, 2, lens[2] + t)).to(torch.bfloat16).cuda())
            at = torch.tensor([p + k + t for p, k in zip(start, lens)], dtype=torch.int32, device="cuda")
            turned = qr.clone()
            s.rope.turn(at, turned)
            got = s.decode(qc, turned)
        else:
            got = s.step(qc, qr, x)
        assert s.lens.tolist() == [k + t + 1 for k in lens]
        for b in range(4):
            cached[b] = np.concatenate([cached[b], _row(s, ids, lens, T, b, lens[b] + t)[None]])
            r = ol.turn(_np(qr[b]), np.full(H, start[b] + lens[b] + t), f, True)
            want, spread, shaken = ol.decode(np.concatenate([_np(qc[b]), r], 1), cached[b], L, s.scale)
            score = s.scale * 2.0 ** -8 * (np.abs(r) @ np.abs(cached[b][:, L:]).T).max(1)[:, None]      # the turned query's rounding
            assert (np.abs(_np(got[b]) - want) <= ol.attention_tolerance(want, spread, shaken, L + 64, score)).all(), (t, b)
    assert s.status() == 0
    from paper_2605_23296_b200 import binding as B
    s.step(_bf16(rng, 4, H, L), _bf16(rng, 4, H, 64), _bf16(rng, 4, L + 64))
    assert s.lens.tolist()[0] == lens[0] + T + 1                # room is left in its last page
    for _ in range(16):
        s.step(_bf16(rng, 4, H, L), _bf16(rng, 4, H, 64), _bf16(rng, 4, L + 64))
    assert s.status() == B.CPA_ENOSPC                           # every block has run out of pages and kept its length
    assert s.lens.tolist() == [-(-(k + T) // 16) * 16 for k in lens]
    s.close()


def test_chunks_and_steps_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(3)
    lens, T, H, L = [60, 33, 90], 12, 16, 256
    made = []
    for how in ("plain", "stream", "graph"):
        gen = np.random.default_rng(4)
        s, _ = _session(np.random.default_rng(5), lens, T, H, L)
        xs = [_bf16(gen, 100, L + 64), _bf16(gen, 83, L + 64)]
        steps = [(_bf16(gen, 3, H, L), _bf16(gen, 3, H, 64), _bf16(gen, 3, L + 64)) for _ in range(2)]
        outs = [torch.empty(3, H, L, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        side = torch.cuda.Stream() if how != "plain" else torch.cuda.current_stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.append(xs[0], [30, 0, 70])
            s.append(xs[1], [30, 33, 20])
            both = lambda: [s.step(*steps[i], out=outs[i]) for i in range(2)]
            if how == "graph":
                side.synchronize()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    both()
                for _ in range(4):
                    g.replay()
            else:
                for _ in range(4):
                    both()
        torch.cuda.synchronize()
        assert s.status() == 0 and s.lens.tolist() == [n + 8 for n in lens]
        made.append((s.pool.clone().view(torch.int16), [o.clone() for o in outs]))
        s.close()
    for pool, outs in made[1:]:
        assert torch.equal(pool, made[0][0]) and all(torch.equal(a, b) for a, b in zip(outs, made[0][1]))


def test_inactive_blocks():
    rng = np.random.default_rng(6)
    lens, H, L = [20, 30], 8, 128
    s, _ = _session(rng, lens, 4, H, L, rope=False)
    s.append_prefill(_bf16(rng, 50, L + 64))
    out = torch.full((2, H, L), 5.0, dtype=torch.bfloat16, device="cuda")
    s.step(_bf16(rng, 2, H, L), _bf16(rng, 2, H, 64), _bf16(rng, 2, L + 64), out=out,
           active=torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    assert (out[0] == 5.0).all() and not (out[1] == 5.0).any() and s.lens.tolist() == [20, 31] and s.status() == 0
    s.close()


def test_refusals():
    from paper_2605_23296_b200 import binding as B
    from paper_2605_23296_b200.session import LatentSession, Rotary
    rng = np.random.default_rng(7)
    s, _ = _session(rng, [20, 30], 4, 8, 128)
    ok = dict(q_latent=_bf16(rng, 2, 8, 128), q_rope=_bf16(rng, 2, 8, 64), x=_bf16(rng, 2, 192))
    for bad in (dict(q_latent=_bf16(rng, 2, 8, 64)), dict(q_rope=_bf16(rng, 2, 4, 64)), dict(x=_bf16(rng, 3, 192)), dict(x=_bf16(rng, 2, 128)),
                dict(x=_bf16(rng, 2, 192).float()), dict(q_latent=_bf16(rng, 2, 8, 128).float()), dict(q_latent=_bf16(rng, 2, 128, 8).transpose(1, 2)),
                dict(x=_bf16(rng, 2, 192).cpu()), dict(active=torch.ones(2, device="cuda")), dict(out=_bf16(rng, 2, 8, 64))):
        with pytest.raises(ValueError):
            s.step(**dict(ok, **bad))
    for counts in ([1], [1, -1], [[1, 2]]):
        with pytest.raises(ValueError):
            s.append(_bf16(rng, 2, 192), counts)
    packed = s.append_prefill(_bf16(rng, 50, 192))
    with pytest.raises(ValueError):
        s.prefill(_bf16(rng, 50, 8, 128), _bf16(rng, 50, 8, 256), packed)
    with pytest.raises(ValueError):
        s.prefill(_bf16(rng, 50, 8, 192), _bf16(rng, 50, 8, 256), packed[:, :128])
    with pytest.raises(B.CpaError):
        LatentSession([10], 0, 8, [0], 1, latent_dim=100)
    with pytest.raises(B.CpaError):
        LatentSession([10], 0, 200, [0], 1)
    with pytest.raises(B.CpaError):
        LatentSession([100], 0, 8, [0], 1)                  # too few pages
    r = Rotary(64)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for q, k, p in ((_bf16(rng, 2, 4, 64), None, pos), (_bf16(rng, 3, 4, 64), _bf16(rng, 2, 1, 64), pos), (_bf16(rng, 3, 4, 64), None, pos.long()),
                    (_bf16(rng, 3, 4, 64).float(), None, pos), (_bf16(rng, 3, 64), None, pos)):
        with pytest.raises(ValueError):
            r.turn(p, q, k)
    with pytest.raises(B.CpaError):
        r.turn(pos, _bf16(rng, 3, 4, 32))                   # a head shorter than its rotated part
    with pytest.raises(B.CpaError):
        Rotary(63)
    assert s.status() == 0
    s.close()


def test_rotary_ahead_of_a_grouped_query_event():
    """Queries and keys turned, prefilled and cached by the plain session: the same attention as over turned inputs in 64 bits."""
    from oracle import attention as oa
    from paper_2605_23296_b200 import workloads as wl
    from paper_2605_23296_b200.session import CompactionSession, Rotary, bits_to_tensor, tensor_to_bits
    from _util import assert_attention_close
    w = wl.custom([150, 40], 8, 2, 128, steps=1, seed=9).materialise()
    s = CompactionSession(w.block_lens, 1, 8, 2, 128, w.free_pages, w.num_pages, scale=w.scale, poison_pools=True)
    q, k, v = (bits_to_tensor(a, "cuda:0") for a in (w.q, w.k, w.v))
    r = Rotary(128, base=500000.0)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in (150, 40)]).cuda()
    was = _np(k)
    r.turn(pos, q, k)
    y = ol.turn(was, pos.cpu().numpy()[:, None], ol.frequencies(128, 500000.0), False)
    assert (np.abs(_np(k) - y) <= ol.turn_tolerance(was, y, False)).all()
    cu = np.array([0, 150, 190])
    o = s.prefill(q, k, v)
    assert_attention_close(tensor_to_bits(o), oa.prefill(tensor_to_bits(q), tensor_to_bits(k), w.v, cu, w.scale), "turned prompts")
    assert s.status() == 0
    s.close()


def test_weights_and_frequencies_elsewhere_are_refused():
    from paper_2605_23296_b200.session import LatentSession, Rotary
    w = torch.ones(128, dtype=torch.bfloat16)
    for bad in (dict(norm_weight=w), dict(norm_weight=w.cuda().float()), dict(norm_weight=w[:64].cuda()), dict(rope=Rotary(64, device="cpu")),
                dict(rope=Rotary(32))):
        with pytest.raises(ValueError):
            LatentSession([10], 0, 8, [0], 1, latent_dim=128, **bad)


@pytest.mark.parametrize("H,L,far", [(128, 128, 524290), (64, 128, 1048580)])
def test_far_pages_of_a_large_pool(H, L, far):
    # page ids that a cache of H key heads could not have: the same event as in the first pages
    from paper_2605_23296_b200 import binding as B
    from paper_2605_23296_b200.session import LatentSession
    if torch.cuda.mem_get_info()[0] < 4 * far * 16 * (L + 64):
        pytest.skip("too little memory")
    lens, T, made = [100, 37], 2, []
    for at in (0, far):
        rng = np.random.default_rng(H)
        ids = at + rng.permutation(12)
        s = LatentSession(lens, T, H, ids, at + 12, L)
        packed = s.append_prefill(_bf16(rng, 137, L + 64))
        outs = [packed, s.prefill(_bf16(rng, 137, H, 192), _bf16(rng, 137, H, 256), packed)]
        outs += [s.step(_bf16(rng, 2, H, L), _bf16(rng, 2, H, 64), _bf16(rng, 2, L + 64)) for _ in range(T)]
        assert s.status() == 0 and s.lens.tolist() == [102, 39]
        made.append(outs)
        s.close()
        del s
    assert all(torch.equal(a, b) for a, b in zip(*made))
    with pytest.raises(B.CpaError):
        LatentSession(lens, T, H, [-1] * 12, 12, L)


def test_a_device_without_a_number_is_the_current_one_of_then():
    from paper_2605_23296_b200.session import LatentSession, Rotary
    here = torch.device("cuda", torch.cuda.current_device())
    r = Rotary(64, device="cuda")
    s = LatentSession([20], 2, 4, [0, 1], 2, 128, rope=r, device="cuda")
    assert r.device == s.device == here
    s.append_prefill(_bf16(np.random.default_rng(0), 20, 192))
    assert s.status() == 0 and s.lens.tolist() == [20]
    s.close()
