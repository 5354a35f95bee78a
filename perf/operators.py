"""Measured cases of the KV cache held in 8 bits: tables built on the device, quantising append, decode and read-back.

The cache.  A page holds 16 tokens of a block; the pool is [num_pages, kv_heads, 2 (K, V), 16, head_dim] in
float8_e4m3fn, with one fp32 scale per (page, kv head, K or V), a power of two: a stored value is code * scale.  The
scale of a page is the smallest power of two (not below 2^-126) that keeps its tokens' largest magnitude within 448 codes; when a
later token needs a larger one, the page's earlier codes are rounded again to it.

The operators (`op` of a case):
  tables  request lengths and a list of free pages, both on the device -> cu_seqlens, page_indptr, the blocks' page
          lists and the slot of every prompt token
  append  new K/V rows of every block, in bf16, into the block's pages behind the tokens that it has
  decode  attention of one query token per block over the block's cached tokens
  step    one decode step: append of one token per block, then decode over the cache with that token in it
  read    a range of every block's cached rows back as packed bf16 rows

A case's lengths come from its own `lens` number, so that shapes do not depend on the seed; values, page order and
queries come from the seed.  With `own` false every operator is computed with elementary torch operations in 32 bits.
"""
import random

import torch

own = False

P = 16          # tokens per page
TOP = 448.0     # largest e4m3 magnitude


# ---------------------------------------------------------------------------------------------------- cases

def _case(name, op, blocks, lo, hi, q_heads=32, kv_heads=8, head_dim=128, new_lo=0, new_hi=0, reserve=0, lens=1):
    """`lo`..`hi`: cached tokens per block (tables: prompt lengths); `new_lo`..`new_hi`: new or read tokens per block;
    `reserve`: tokens reserved behind the cached ones; `lens`: the number that the lengths are drawn from."""
    c = {"op": op, "blocks": blocks, "lo": lo, "hi": hi, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "new_lo": new_lo, "new_hi": new_hi, "reserve": reserve, "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # many short documents with several questions each, admitted together
        _case("tables short documents", "tables", 192, 512, 1024, reserve=256, lens=11),
        # a whole queue of requests of any length, admitted at once
        _case("tables long queue", "tables", 2000, 1, 2048, reserve=64, lens=12),
        # the prompts of a ragged compaction event, cached after their prefill
        _case("append ragged prompts", "append", 32, 0, 0, new_lo=1024, new_hi=8192, lens=13),
        # one decode step's tokens of many short sequences, stored without attention: smallest call
        _case("append one token", "append", 192, 512, 1280, new_lo=1, new_hi=1, lens=14),
        # a chunk of every prompt behind what is cached, heads of 64, ragged and odd
        _case("append odd chunks", "append", 24, 1, 4095, q_heads=64, head_dim=64, new_lo=1, new_hi=1021, lens=15),
        # a small event of one kv head: latency of a single call
        _case("decode small", "decode", 4, 96, 288, q_heads=4, kv_heads=1, head_dim=64, lens=16),
        # a ragged compaction event
        _case("decode ragged", "decode", 32, 1024, 8192, lens=17),
        # sequential compaction: the whole history is one block
        _case("decode one history", "decode", 1, 131072, 131072, lens=18),
        # many short sequences, each with its step's token
        _case("step short documents", "step", 192, 512, 1024, new_lo=1, new_hi=1, lens=19),
        # 64 query heads over 8 kv heads of 64
        _case("step wide groups", "step", 16, 8000, 8192, q_heads=64, head_dim=64, new_lo=1, new_hi=1, lens=20),
        # a cached history handed on in bf16
        _case("read history", "read", 8, 4096, 4096, new_lo=4096, new_hi=4096, lens=21),
        # the summaries alone, from odd positions
        _case("read summaries", "read", 192, 512, 1280, new_lo=33, new_hi=255, lens=22),
    ]


def _log(rng, lo, hi):
    """A whole number spread over its logarithm."""
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["tables", "append", "decode", "decode", "step", "step", "read"])
    lens = rng.randrange(1 << 30)
    if op == "tables":
        blocks = _log(rng, 1, 2000)
        hi = _log(rng, 1, min(131072, 2000000 // blocks))
        return _case(None, op, blocks, rng.randrange(0, hi + 1), hi, reserve=rng.randrange(0, 513), lens=lens)
    d = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8])
    q = kv * rng.choice([1, 2, 3, 4, 5, 8])
    total = 131072 * 8 * 128 // (kv * d)         # cached tokens that cost no more than the largest listed case
    blocks = _log(rng, 1, 192)
    hi = _log(rng, 2, min(131072, total // blocks))
    few = blocks < 4                              # a few blocks all hold something; of many, some may be empty
    lo = rng.randrange(few, hi + 1)
    if op == "decode":
        return _case(None, op, blocks, lo, hi, q, kv, d, lens=lens)
    if op == "step":
        return _case(None, op, blocks, lo, hi, q, kv, d, 1, 1, lens=lens)
    new = _log(rng, 1, max(1, min(hi, 65536 * 8 * 128 // (kv * d) // blocks)))
    lo = max(lo, op == "read")
    return _case(None, op, blocks, lo, hi, q, kv, d, rng.randrange(few or new < 2, new + 1), new, lens=lens)


def _lengths(case):
    """(cached, new, first) per block: `first` is where a read starts."""
    r = random.Random(case["lens"])
    cached = [r.randint(case["lo"], case["hi"]) for _ in range(case["blocks"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["blocks"])]
    if case["op"] != "read":
        return cached, new, [0] * case["blocks"]
    new = [min(n, c) for n, c in zip(new, cached)]
    return cached, new, [c - n for n, c in zip(new, cached)]


def work(case):
    cached, new, _ = _lengths(case)
    q, kv, d, op = case["q_heads"], case["kv_heads"], case["head_dim"], case["op"]
    B, tok, n = len(cached), sum(cached), sum(new)
    pages = sum(-(-c // P) for c in cached)
    if op == "tables":
        used = sum(-(-(c + case["reserve"]) // P) for c in cached)
        return {"bytes": 4 * (B + 2 * (B + 1) + 2 * used + tok), "flops": 0}
    row = 2 * kv * d                                      # bytes of a token's K and V in the cache
    if op == "append":                                    # bf16 rows in; codes and the touched pages' scales out
        touched = sum(-(-(c % P + x) // P) if x else 0 for c, x in zip(cached, new))
        return {"bytes": 3 * row * n + 8 * kv * touched + 12 * B, "flops": 0}
    if op == "read":
        return {"bytes": 3 * row * n + 8 * B, "flops": 0}
    bytes_ = row * tok + 8 * kv * pages + 2 * 2 * B * q * d + 4 * (B + pages)    # with the lengths and page ids
    if op == "step":
        return {"bytes": bytes_ + 3 * row * B + 4 * B, "flops": 4 * (tok + B) * q * d}
    return {"bytes": bytes_, "flops": 4 * tok * q * d}


# ---------------------------------------------------------------------------------------------------- inputs

def _pow2_scale(amax):
    """fp32: the smallest power of two s, not below 2^-126, with amax <= 448 s (448 = 1.75 * 2^8)."""
    e = ((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 135
    return ((e.clamp_min(-126) + 127) << 23).view(torch.float32)


def _rows(gen, n, kv, d):
    """bf16 K or V rows: normal values, tokens of different magnitude, a few outliers of eight times the size."""
    size = torch.randn(n, 1, 1, generator=gen, device="cuda").mul_(0.5).exp_()
    size *= 1 + 7 * (torch.rand(n, 1, 1, generator=gen, device="cuda") < 1 / 512)
    return (torch.randn(n, kv, d, generator=gen, device="cuda") * size).bfloat16()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _sum0(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def _fill(gen, case, cached, ids, num_pages):
    """A pool and its scales with `cached` tokens in every block; what no token has filled holds NaN."""
    kv, d = case["kv_heads"], case["head_dim"]
    pool = torch.full((num_pages, kv, 2, P, d), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.full((num_pages, kv, 2), float("nan"), device="cuda")
    used = [-(-c // P) for c in cached]
    fill = [min(P, c - P * j) for c, u in zip(cached, used) for j in range(u)]   # tokens in each page that holds any
    if fill:
        pages = torch.cat([ids[a:a + u] for a, u in zip(_sum0(case["_pages"]), used)]).long()
        there = torch.arange(P, device="cuda") < _i32(fill)[:, None]             # [n, 16]
        for at in range(0, len(fill), 8192):
            pg, on = pages[at:at + 8192], there[at:at + 8192][:, None, :, None]
            for kind in (0, 1):
                x = _rows(gen, pg.numel() * P, kv, d).view(-1, P, kv, d).transpose(1, 2).float() * on
                s = _pow2_scale(x.abs().amax((2, 3)))
                scales[pg, :, kind] = s
                codes = (x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
                pool.view(torch.uint8)[pg, :, kind] = torch.where(on, codes, 0x7F)
    return pool, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cached, new, first = _lengths(case)
    op, B, kv, d = case["op"], case["blocks"], case["kv_heads"], case["head_dim"]
    reserve = case["reserve"] if op == "tables" else 0
    room = [c + (n if op in ("append", "step") else reserve) for c, n in zip(cached, new)]
    pages = [-(-r // P) for r in room]
    total = sum(pages)
    num_pages = total + 3                                                # a pool with a few pages to spare
    ids = torch.randperm(num_pages, generator=gen, device="cuda").int()  # the free list: any order
    st = {"case": case, "free": ids, "num_pages": num_pages, "total_pages": total, "tokens": sum(cached), "rows": sum(new),
          "room": _i32(room), "lens": _i32(cached), "lens_out": torch.zeros(B, dtype=torch.int32, device="cuda"),
          "reserve": reserve}
    if op != "tables":
        case = dict(case, _pages=pages)
        st["indptr"], st["ids"] = _i32(_sum0(pages)), ids[:total]
        st["pool"], st["scales"] = _fill(gen, case, cached, ids, num_pages)
        st["max_pages"] = max([1] + [-(-(c + (1 if op == "step" else 0)) // P) for c in cached])
    if op in ("append", "step"):
        st["k"], st["v"] = (_rows(gen, sum(new), kv, d) for _ in range(2))
    if op in ("append", "read"):
        st["cu_new"] = _i32(_sum0(new))
    if op == "read":
        st["first"] = _i32(first)
        st["k_out"], st["v_out"] = (torch.empty(sum(new), kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if op in ("decode", "step"):
        st["q"] = torch.randn(B, case["q_heads"], d, generator=gen, device="cuda").bfloat16()
        st["o"] = torch.empty_like(st["q"])
    if own:
        from paper_2605_23296_b200 import binding as lib

        st["cfg"] = lib.cpa_config(case["q_heads"], kv, d, P, d ** -0.5, 0, 0, 0)
        st["dims"] = lib.cpa_table_dims(B, reserve, num_pages, num_pages, st["tokens"] if op == "tables" else 0)
        st["tables"] = torch.empty(lib.cpa_tables_bytes(st["cfg"], st["dims"]), dtype=torch.uint8, device="cuda")
        if op == "tables":
            ints = st["tables"].view(torch.int32)
            sizes = ((lib.ARR_CU_SEQLENS, B + 1), (lib.ARR_PAGE_INDPTR, B + 1), (lib.ARR_PAGE_INDICES, total),
                     (lib.ARR_SLOT_MAPPING, st["tokens"]))
            at = [(lib.cpa_tables_offset(st["cfg"], st["dims"], which) // 4, n) for which, n in sizes]
            st["views"] = [ints[a:a + n] for a, n in at]
        else:
            lib.cpa_tables_build(st["cfg"], st["dims"], st["room"], ids, num_pages, st["tables"],
                                 torch.cuda.current_stream().cuda_stream)
        st["workspace"] = torch.empty(lib.cpa_decode_q8_workspace_bytes(st["cfg"]), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------- run

def run(st):
    op = st["case"]["op"]
    if own:
        return _own(st, op)
    return {"tables": _tables, "append": _append, "decode": _decode, "step": _step, "read": _read}[op](st)


def _own(st, op):
    from paper_2605_23296_b200 import binding as lib

    on = torch.cuda.current_stream().cuda_stream
    cfg, dims, t = st["cfg"], st["dims"], st["tables"]
    if op == "tables":
        rc = lib.cpa_tables_build(cfg, dims, st["lens"], st["free"], st["num_pages"], t, on)
        out = st["views"]
    elif op == "append":
        rc = lib.cpa_kv_append_q8(cfg, dims, t, st["k"], st["v"], st["cu_new"], st["rows"], st["lens"], st["lens_out"],
                                  st["pool"], st["scales"], on)
        out = st["pool"], st["scales"], st["lens_out"]
    elif op == "decode":
        rc = lib.cpa_decode_q8(cfg, dims, t, st["q"], st["lens"], None, st["pool"], st["scales"], st["o"],
                               st["workspace"], on)
        out = st["o"]
    elif op == "step":
        rc = lib.cpa_decode_append_q8(cfg, dims, t, st["q"], st["k"], st["v"], st["lens"], st["lens_out"], None,
                                      st["pool"], st["scales"], st["o"], st["workspace"], on)
        out = st["o"], st["pool"], st["scales"], st["lens_out"]
    else:
        rc = lib.cpa_kv_read_q8(cfg, dims, t, st["first"], st["cu_new"], st["rows"], st["pool"], st["scales"],
                                st["k_out"], st["v_out"], on)
        out = st["k_out"], st["v_out"]
    if rc:
        raise lib.CpaError(rc, op)
    return out


def _zero_first(v):
    return torch.cat([v.new_zeros(1), v.cumsum(0, dtype=torch.int32)])


def _tables(st):
    lens, free = st["lens"], st["free"]
    cu, indptr = _zero_first(lens), _zero_first((lens + (st["reserve"] + P - 1)) // P)
    token = torch.arange(st["tokens"], dtype=torch.int32, device="cuda")
    block = torch.searchsorted(cu[1:], token, right=True)
    at = token - cu[block]
    slots = free[indptr[block] + at // P] * P + at % P
    return [cu, indptr, free[:st["total_pages"]].clone(), slots]


def _places(st, first, cu, rows):
    """Of every packed row: its block, its position, its page's place in the page list."""
    row = torch.arange(rows, dtype=torch.int32, device="cuda")
    block = torch.searchsorted(cu[1:], row, right=True)
    at = first[block] + row - cu[block]
    return at, st["ids"][st["indptr"][block] + at // P].long()


def _codes(pool, pages):
    return pool.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float()


def _store(st, k, v, cu, rows):
    lens, pool, scales = st["lens"], st["pool"], st["scales"]
    at, page = _places(st, lens, cu, rows)
    x = torch.stack([k, v], 2).float()                                  # [rows, kv, 2, d]
    amax = torch.zeros_like(scales).index_reduce_(0, page, x.abs().amax(3), "amax")
    need = _pow2_scale(amax)
    # pages that held tokens of their block already keep their scale, or grow it and round their codes again
    has = (lens % P != 0) & (cu[1:] > cu[:-1])
    at_spare = st["total_pages"]                                        # a page of no block stands for "none"
    part = st["free"][torch.where(has, st["indptr"][:-1] + lens // P, at_spare)].long()
    held = torch.arange(P, device="cuda") < (lens % P * has)[:, None]   # [B, 16]
    old = scales[part]
    grown = torch.maximum(need[part], old)
    raw = pool.view(torch.uint8)
    again = (_codes(pool, part) * (old / grown)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    raw[part] = torch.where(held[:, None, None, :, None], again, raw[part])
    need[part] = grown
    scales[page] = need[page]
    codes = (x / need[page][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    raw[page, :, :, at % P] = codes
    torch.add(lens, cu[1:] - cu[:-1], out=st["lens_out"])


def _append(st):
    _store(st, st["k"], st["v"], st["cu_new"], st["rows"])
    return st["pool"], st["scales"], st["lens_out"]


def _attend(st, lens):
    q, B, kv, d = st["q"], st["case"]["blocks"], st["case"]["kv_heads"], st["case"]["head_dim"]
    n = st["max_pages"]
    place = st["indptr"][:-1, None] + torch.arange(n, device="cuda")
    place = torch.minimum(place, st["indptr"][1:, None] - 1).clamp_min(0)
    pages = st["ids"][place].long() if st["ids"].numel() else torch.zeros_like(place)        # [B, n]
    x = _codes(st["pool"], pages) * st["scales"][pages][..., None, None]                      # [B, n, kv, 2, 16, d]
    k, v = (x[:, :, :, i].transpose(1, 2).reshape(B, kv, n * P, d) for i in (0, 1))
    seen = (torch.arange(n * P, device="cuda") < lens[:, None])[:, None, None]                # [B, 1, 1, n * 16]
    s = torch.matmul(q.float().view(B, kv, -1, d), k.transpose(2, 3)) * d ** -0.5
    s = s.masked_fill(~seen, float("-inf"))
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), 0.0, m))
    o = torch.matmul(p, v.masked_fill(~seen.transpose(2, 3), 0.0))
    o = o / p.sum(3, keepdim=True).masked_fill(lens[:, None, None, None] == 0, 1.0)           # no token: zero
    return st["o"].copy_(o.reshape(q.shape))


def _decode(st):
    return _attend(st, st["lens"])


def _step(st):
    B = st["case"]["blocks"]
    _store(st, st["k"], st["v"], torch.arange(B + 1, dtype=torch.int32, device="cuda"), B)
    return _attend(st, st["lens_out"]), st["pool"], st["scales"], st["lens_out"]


def _read(st):
    at, page = _places(st, st["first"], st["cu_new"], st["rows"])
    codes = st["pool"].view(torch.uint8)[page, :, :, at % P].view(torch.float8_e4m3fn)
    x = codes.float() * st["scales"][page][..., None]                                         # [rows, kv, 2, d]
    return st["k_out"].copy_(x[:, :, 0]), st["v_out"].copy_(x[:, :, 1])


# ---------------------------------------------------------------------------------------------------- 64 bits

def _e4m3(x):
    """float64 values rounded to the nearest e4m3 value, ties to even: 4 significant bits, spacing 2^-9 at least."""
    _, e = torch.frexp(x)                                   # |x| = m 2^e, 1/2 <= m < 1
    step = torch.ldexp(torch.ones_like(x), e.clamp_min(-5) - 4)
    return torch.round(x / step) * step


def _scale64(amax):
    m, e = torch.frexp(amax.double() / TOP)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.ldexp(torch.ones_like(m), torch.where(amax == 0, -126, e).clamp_min(-126))


def _exact_store(st, cached, new):
    """The pool's codes and scales in float64 after the append, block by block and page by page of the definition."""
    codes, scales = st["pool"].double(), st["scales"].double()
    indptr, ids = st["indptr"].tolist(), st["ids"].tolist()
    parts = []       # (rows, page, slot of the first row): runs of rows that share a page
    row = 0
    for b, (c, n) in enumerate(zip(cached, new)):
        while n > 0:
            take = min(n, P - c % P)
            parts.append((row, take, ids[indptr[b] + c // P], c % P))
            row, c, n = row + take, c + take, n - take
    x = torch.stack([st["k"], st["v"]], 2).double()
    for size, slot in sorted({(p[1], p[3]) for p in parts}):
        some = [p for p in parts if (p[1], p[3]) == (size, slot)]
        first = torch.tensor([p[0] for p in some], device="cuda")
        page = torch.tensor([p[2] for p in some], device="cuda")
        y = x[first[:, None] + torch.arange(size, device="cuda")].permute(0, 2, 3, 1, 4)      # [n, kv, 2, size, d]
        s = _scale64(y.abs().amax((3, 4)))
        if slot:
            s = torch.maximum(s, scales[page])
            before = codes[page][:, :, :, :slot]
            codes[page, :, :, :slot] = _e4m3(before * (scales[page] / s)[..., None, None])
        codes[page, :, :, slot:slot + size] = _e4m3(y / s[..., None, None])
        scales[page] = s
    return codes, scales


def exact(case, seed):
    global own
    if case["op"] == "tables":
        return None                 # whole numbers alone
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op, d, kv = case["op"], case["head_dim"], case["kv_heads"]
    cached, new, first = _lengths(case)
    indptr, ids = st["indptr"].tolist(), st["ids"].long()
    if op == "append":
        codes, scales = _exact_store(st, cached, new)
        return codes, scales, None
    if op == "step":
        codes, scales = _exact_store(st, cached, new)
        cached = [c + 1 for c in cached]
    else:
        codes, scales = st["pool"].float(), st["scales"].double()

    def block(b, lo, hi):
        """K and V of positions lo..hi of block b: [2][kv, hi - lo, d]."""
        pg = ids[indptr[b] + lo // P: indptr[b] + -(-hi // P)]
        y = codes[pg].double() * scales[pg][..., None, None]
        y = y.permute(2, 1, 0, 3, 4).reshape(2, kv, -1, d)
        return y[:, :, lo % P: lo % P + hi - lo]

    if op == "read":
        out = [block(b, f, f + n).transpose(1, 2) if n else torch.zeros(2, 0, kv, d, dtype=torch.float64, device="cuda")
               for b, (f, n) in enumerate(zip(first, new))]
        return tuple(torch.cat(out, 1))
    o = torch.zeros(case["blocks"], case["q_heads"], d, dtype=torch.float64, device="cuda")
    for b, n in enumerate(cached):
        if n:
            k, v = block(b, 0, n)
            w = torch.softmax(st["q"][b].double().view(kv, -1, d) @ k.transpose(1, 2) / d ** 0.5, 2)
            o[b] = (w @ v).reshape(-1, d)
    return (o, codes, scales, None) if op == "step" else o
