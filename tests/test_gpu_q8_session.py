"""A compaction event whose cache is held in 8 bits, through CompactionSession: prefill, the prompts' append, fused and
separate decode steps, read-back; against the 64-bit oracles."""
import numpy as np
import pytest

from _util import assert_attention_close
from oracle import attention as oa
from oracle import cache_q8 as oq
from paper_2605_23296_b200 import workloads as wl

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _f64(bits):
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("lens,hq,hkv,d", [([96, 160, 224, 288], 4, 1, 64), ([700, 1, 129, 64], 16, 2, 128),
                                           ([17, 33], 8, 8, 128), ([40] * 9, 16, 2, 64)])
def test_event(lens, hq, hkv, d):
    from paper_2605_23296_b200.session import CompactionSession, bits_to_tensor, tensor_to_bits

    T = 12
    w = wl.custom(lens, hq, hkv, d, steps=T, seed=len(lens) + d).materialise()
    s = CompactionSession(w.block_lens, T, hq, hkv, d, w.free_pages, w.num_pages, scale=w.scale, poison_pools=True, kv_bits=8)
    dev = lambda a: bits_to_tensor(a, "cuda:0")
    k, v = dev(w.k), dev(w.v)
    o = s.prefill(dev(w.q), k, v)
    s.append_prefill(k, v)
    cu = np.concatenate([[0], np.cumsum(w.block_lens.astype(np.int64))])
    assert_attention_close(tensor_to_bits(o), oa.prefill(w.q, w.k, w.v, cu, w.scale), "prefill")
    want = oq.CacheQ8(w.num_pages, hkv, d, lens, T, w.free_pages)
    for b in range(len(lens)):
        want.append(b, _f64(w.k[cu[b]:cu[b + 1]]), _f64(w.v[cu[b]:cu[b + 1]]))
    from paper_2605_23296_b200 import binding as B
    at = B.cpa_tables_offset(s.cfg, s.dims, B.ARR_SLOT_MAPPING) // 4
    assert np.array_equal(s.tables.view(torch.int32)[at:at + s.total_tokens].cpu().numpy(), s.export(B.ARR_SLOT_MAPPING))
    for t in range(T):
        if t % 3 == 0:
            s.append(dev(w.k_dec[t]), dev(w.v_dec[t]))
            got = s.decode(dev(w.q_dec[t]))
        elif t % 3 == 1:
            got = s.decode_append(dev(w.q_dec[t]), dev(w.k_dec[t]), dev(w.v_dec[t]))
        else:
            got = s.decode_append_steps(dev(w.q_dec[t:t + 1]), dev(w.k_dec[t:t + 1]), dev(w.v_dec[t:t + 1]))[0]
        for b in range(len(lens)):
            want.append(b, _f64(w.k_dec[t, b])[None], _f64(w.v_dec[t, b])[None])
            exact, spread, shaken = want.decode(b, _f64(w.q_dec[t, b]), float(np.float32(w.scale)))
            off = np.abs(got[b].double().cpu().numpy() - exact)
            assert (off <= oq.decode_tolerance(exact, spread, shaken, d)).all(), (t, b)
    assert s.status() == 0 and s.export(B.ARR_SEQ_LENS).tolist() == [n + T for n in lens]
    # read-back leaves the cache as it is
    before = s.kv_pool.view(torch.uint8).clone()
    kk, vv = s.read_cache([0] * len(lens), [n + T for n in lens])
    rows = np.concatenate([want.rows(b, 0, n + T) for b, n in enumerate(lens)], 2).transpose(0, 2, 1, 3)
    assert np.array_equal(kk.double().cpu().numpy(), rows[0]) and np.array_equal(vv.double().cpu().numpy(), rows[1])
    assert torch.equal(before, s.kv_pool.view(torch.uint8))
    s.close()


def test_chunks_of_any_length_and_a_full_reservation():
    from paper_2605_23296_b200 import binding as B
    from paper_2605_23296_b200.session import CompactionSession

    s = CompactionSession([30, 4], 2, 8, 2, 64, np.arange(8), 8, kv_bits=8, poison_pools=True)     # 32 and 6 tokens: 2 + 1 pages
    rng = np.random.default_rng(1)
    rows = lambda n, h=2: torch.tensor(rng.standard_normal((n, h, 64)), dtype=torch.bfloat16, device="cuda")
    s.append(rows(11), rows(11), [11, 0])
    s.append(rows(23), rows(23), [19, 4])
    assert s.lens.tolist() == [30, 4] and s.status() == 0
    s.decode_append(rows(2, 8), rows(2), rows(2), active=torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
    assert s.lens.tolist() == [31, 4]
    s.append(rows(3), rows(3), [2, 1])                  # block 0 has room for one
    assert s.lens.tolist() == [31, 5] and s.status() == B.CPA_ENOSPC
    s.close()


def test_refusals():
    from paper_2605_23296_b200 import binding as B
    from paper_2605_23296_b200.session import CompactionSession

    for more in (dict(chunk_tokens=128), dict(dynamic_pages=True), dict(prefix_lens=[0, 0], shared_pages=[]),
                 dict(pools=(None, None)), dict(kv_bits=4)):
        with pytest.raises(ValueError):
            CompactionSession([30, 4], 2, 8, 2, 64, np.arange(8), 8, **dict(dict(kv_bits=8), **more))
    s = CompactionSession([30, 4], 2, 8, 2, 64, np.arange(8), 8, kv_bits=8)
    good_q, good_k = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    for q in (good_q.float(), good_q[:1], good_q.cpu(), torch.zeros(2, 64, 8, dtype=torch.bfloat16, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            s.decode(q)
    for k in (good_k.half(), good_k[:1], torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            s.append(k, good_k)
        with pytest.raises(ValueError):
            s.decode_append(good_q, good_k, k)
    with pytest.raises(ValueError):
        s.decode(good_q, active=torch.ones(2, device="cuda"))
    with pytest.raises(B.CpaError):
        s.append(good_k, good_k, [3, -1])
    with pytest.raises(ValueError):
        s.read_cache([0], [1])
    for call in (lambda: s.step_mixed(0, None, None, None, None), lambda: s.event_from_host(None, None, None, None),
                 lambda: s.decode_append_dynamic(good_q, good_k, good_k), lambda: s.step_mixed_range(0, 1, None, None, None, None)):
        with pytest.raises(B.CpaError):
            call()
    assert s.lens.tolist() == [0, 0] and s.status() == 0
    s.close()
    s = CompactionSession([30, 4], 2, 8, 2, 64, np.arange(8), 8)
    with pytest.raises(B.CpaError):
        s.read_cache([0, 0], [1, 1])
    with pytest.raises(B.CpaError):
        s.decode(good_q, active=torch.ones(2, dtype=torch.int32, device="cuda"))
    s.close()


def test_read_back_refuses_ranges_outside_the_blocks_pages():
    from paper_2605_23296_b200.session import CompactionSession

    s = CompactionSession([30, 4], 2, 8, 2, 64, np.arange(8), 8, kv_bits=8, poison_pools=True)     # pages for 32 and 16 tokens
    rows = torch.ones(34, 2, 64, dtype=torch.bfloat16, device="cuda")
    s.append(rows, rows, [30, 4])
    for first, counts in (([0, 0], [33, 1]), ([0, 0], [1, 17]), ([31, 0], [2, 0]), ([33, 0], [0, 0]), ([0, 17], [1, 0]),
                          ([0, -1], [1, 1]), ([0, 0], [1, -1]), ([2 ** 40, 0], [1, 1]), ([0, 0], [2 ** 40, 1]),
                          ([2 ** 62, 0], [2 ** 62, 0]), ([0], [1, 1]), ([0, 0], [1]), ([0.0, 0.0], [1, 1])):
        with pytest.raises(ValueError):
            s.read_cache(first, counts)
    for first, counts in (([0, 0], [30, 4]), ([29, 3], [1, 1]), ([30, 4], [0, 0]), (np.array([7, 0]), torch.tensor([3, 4]))):
        k, v = s.read_cache(first, counts)
        assert k.shape == v.shape == (int(sum(counts)), 2, 64) and (k == 1).all() and (v == 1).all()
    assert s.read_cache([32, 16], [0, 0])[0].shape[0] == 0 and s.status() == 0
    s.close()


def test_steps_of_different_counts_are_refused_before_any_is_taken():
    from paper_2605_23296_b200.session import CompactionSession

    s = CompactionSession([30, 4], 4, 8, 2, 64, np.arange(8), 8, kv_bits=8)
    q, k = (torch.zeros(3, 2, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2))
    for args in ((q, k[:2], k), (q, k, k[:1]), (q[:2], k, k), (q, k, k, torch.empty_like(q)[:2])):
        with pytest.raises(ValueError):
            s.decode_append_steps(*args)
    assert s.lens.tolist() == [0, 0]
    s.decode_append_steps(q, k, k)
    assert s.lens.tolist() == [3, 3] and s.status() == 0
    s.close()


def test_an_event_in_8_bits_beside_one_in_bf16_on_one_stream():
    # the two caches' steps alternate without a wait: both kinds of launch begin before the other kind has ended
    from paper_2605_23296_b200.session import CompactionSession, bits_to_tensor

    T, hq, hkv, d = 10, 16, 2, 128
    w = wl.custom([300, 17, 64, 900], hq, hkv, d, steps=T, seed=5).materialise()
    dev = lambda a: bits_to_tensor(a, "cuda:0")
    k, v, q_dec, k_dec, v_dec = (dev(a) for a in (w.k, w.v, w.q_dec, w.k_dec, w.v_dec))

    def run(kinds):
        s = [CompactionSession(w.block_lens, T, hq, hkv, d, w.free_pages, w.num_pages, scale=w.scale, kv_bits=bits) for bits in kinds]
        out = [torch.zeros(T, 4, hq, d, dtype=torch.bfloat16, device="cuda") for _ in s]
        for x in s:
            x.append_prefill(k, v)
        for t in range(T):
            for x, o in zip(s, out):
                if t % 2:
                    x.append(k_dec[t], v_dec[t])
            for x, o in zip(s, out):
                if t % 2:
                    x.decode(q_dec[t], o[t])
                else:
                    x.decode_append(q_dec[t], k_dec[t], v_dec[t], o[t])
        assert all(x.status() == 0 for x in s)
        for x in s:
            x.close()
        return out

    alone = [run([bits])[0] for bits in (8, 16)]
    for kinds in ((8, 16), (16, 8), (16, 8, 16, 8)):
        for bits, o in zip(kinds, run(kinds)):
            assert torch.equal(o, alone[0 if bits == 8 else 1]), (kinds, bits)
