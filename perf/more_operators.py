"""Measured cases of latent attention (keys and values from one shared vector a token) and of rotary positions.

The cache.  Of every token it holds one row [latent_dim + 64] in bf16, shared by all heads: the normalised latent vector c
and behind it the rotated positional key r.  A page holds 16 tokens of a block; the pool is [num_pages, 16, latent_dim + 64].

The operators (`op` of a case):
  rope     rotary positions of packed rows of query heads and of key heads
  append   new rows x = [latent | positional key] of every block, in bf16: c = x / rms(x) * weight, r rotated to the token's
           position, both into the block's pages behind the tokens that it has; the stored rows packed as well
  decode   absorbed form, one query token per block: score_j = scale (q_c . c_j + q_r . r_j), output = sum_j p_j c_j
  step     one decode step: append of one token per block, the query's positional part rotated, then decode with that token
  prefill  expanded form, causal over every block: keys [nope | r] and values per head, r shared by the heads

Rotary positions.  Pair i of a rotated part of R elements turns by position * f_i; f_i = base^(-2i/R), "parts": divided by
`factor` where the pair turns few times over the length that the model was trained on, blended in between.  "half": pair i
is (i, i + R/2); "interleaved": (2i, 2i + 1).

A case's lengths come from its own `lens` number, so that shapes do not depend on the seed; values, page order, queries and
positions come from the seed.  With `own` false every operator is computed with elementary torch operations in 32 bits, the
angles of far positions in 64.
"""
import math
import random

import torch

own = False

P = 16              # tokens per page
R = 64              # rotated part of a cached row
NOPE, VDIM = 128, 128
EPS = 1e-6
PARTS = dict(base=10000.0, factor=40.0, fast=32.0, slow=1.0, trained=4096)   # scaled for long contexts
PLAIN = dict(base=10000.0)


# ---------------------------------------------------------------------------------------------------- cases

def _case(name, op, blocks, lo, hi, heads=16, latent=512, new_lo=0, new_hi=0, lens=1, **more):
    """`lo`..`hi`: cached tokens per block (prefill, rope: tokens of a block); `new_lo`..`new_hi`: new tokens per block;
    `lens`: the number that the lengths are drawn from.  rope: `heads` query and `kv_heads` key heads of `head_dim`, whose
    last `rot` elements turn."""
    c = {"op": op, "blocks": blocks, "lo": lo, "hi": hi, "heads": heads, "latent": latent, "new_lo": new_lo,
         "new_hi": new_hi, "lens": lens}
    c.update(more)
    return dict(c, name=name) if name else c


def _rope(name, blocks, lo, hi, heads, kv_heads, head_dim, rot, layout, scaling, lens):
    return _case(name, "rope", blocks, lo, hi, heads, 0, lens=lens, kv_heads=kv_heads, head_dim=head_dim, rot=rot,
                 layout=layout, scaling=scaling)


def listed():
    return [
        # queries and keys of a ragged compaction event's prompts, ahead of their prefill
        _rope("rope ragged prompts", 32, 1024, 8192, 32, 8, 128, 128, "half", "none", 31),
        # the positional part of one decode step's queries, heads of 128 + 64: smallest call
        _rope("rope one token", 192, 1, 1, 16, 0, 192, 64, "interleaved", "parts", 32),
        # the latent rows of a ragged event's prompts
        _case("append ragged prompts", "append", 32, 0, 0, new_lo=1024, new_hi=8192, lens=33),
        # one decode step's rows of many short sequences, stored without attention
        _case("append one token", "append", 192, 512, 1280, new_lo=1, new_hi=1, lens=34),
        # a chunk of every prompt behind what is cached, a smaller latent vector, ragged and odd
        _case("append odd chunks", "append", 24, 1, 4095, latent=256, new_lo=1, new_hi=1021, lens=35),
        # a small event: latency of a single call
        _case("decode small", "decode", 4, 96, 288, 16, lens=36),
        # a ragged compaction event, 64 heads on this device
        _case("decode ragged", "decode", 32, 1024, 8192, 64, lens=37),
        # sequential compaction: the whole history is one block, all heads on one device
        _case("decode one history", "decode", 1, 131072, 131072, 128, lens=38),
        # many short sequences, each with its step's token, an eighth of the heads on this device
        _case("step short documents", "step", 192, 512, 1024, 16, new_lo=1, new_hi=1, lens=39),
        # long sequences with all heads on one device
        _case("step all heads", "step", 16, 8000, 8192, 128, new_lo=1, new_hi=1, lens=40),
        # a few short prompts of odd lengths
        _case("prefill odd prompts", "prefill", 9, 1, 700, 16, lens=41),
        # the prompts of a ragged event
        _case("prefill ragged prompts", "prefill", 32, 1024, 8192, 16, lens=42),
    ]


def _log(rng, lo, hi):
    """A whole number spread over its logarithm."""
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["rope", "append", "decode", "decode", "step", "step", "prefill"])
    lens = rng.randrange(1 << 30)
    blocks = _log(rng, 1, 192)
    if op == "rope":
        heads, kv_heads = rng.choice([(32, 8), (16, 0), (20, 4), (64, 8), (7, 1)])
        head_dim, rot = rng.choice([(64, 64), (128, 128), (128, 32), (192, 64), (80, 20)])
        hi = _log(rng, 1, max(1, 131072 * 40 * 128 // ((heads + kv_heads) * head_dim) // blocks))
        return _rope(None, blocks, rng.randrange(1, hi + 1), hi, heads, kv_heads, head_dim, rot,
                     rng.choice(["half", "interleaved"]), rng.choice(["none", "parts"]), lens)
    if op == "prefill":
        heads = rng.choice([1, 3, 8, 16, 20])
        hi = _log(rng, 1, max(1, min(8192, int((32 * 4608 ** 2 * 16 / (blocks * heads)) ** 0.5))))
        return _case(None, op, blocks, rng.randrange(1, hi + 1), hi, heads, lens=lens)
    latent = rng.choice([128, 256, 384, 512, 512])
    heads = rng.choice([1, 5, 8, 16, 16, 24, 32, 64, 128])
    few = blocks < 4                              # a few blocks all hold something; of many, some may be empty
    hi = _log(rng, 2, min(131072, 131072 // blocks))
    lo = rng.randrange(few, hi + 1)
    if op == "decode":
        return _case(None, op, blocks, lo, hi, heads, latent, lens=lens)
    if op == "step":
        return _case(None, op, blocks, lo, hi, heads, latent, 1, 1, lens)
    new = _log(rng, 1, max(1, min(hi, 131072 // blocks)))
    return _case(None, op, blocks, lo, hi, heads, latent, rng.randrange(few or new < 2, new + 1), new, lens)


def _lengths(case):
    """(cached, new) tokens per block."""
    r = random.Random(case["lens"])
    cached = [r.randint(case["lo"], case["hi"]) for _ in range(case["blocks"])]
    return cached, [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["blocks"])]


def work(case):
    cached, new = _lengths(case)
    op, B, tok, n, H = case["op"], len(cached), sum(cached), sum(new), case["heads"]
    if op == "rope":
        return {"bytes": tok * (4 * (H + case["kv_heads"]) * case["head_dim"] + 4), "flops": 0}
    if op == "prefill":     # queries, keys, values and the shared positional keys in, outputs out
        pairs = sum(c * (c + 1) // 2 for c in cached)
        return {"bytes": 2 * tok * (H * (NOPE + R + NOPE + VDIM + VDIM) + R), "flops": 2 * pairs * H * (NOPE + R + VDIM)}
    L = case["latent"]
    row, pages = 2 * (L + R), sum(-(-c // P) for c in cached)
    if op == "append":      # rows in; rows to their pages and packed
        return {"bytes": 3 * row * n + 2 * L + 12 * B, "flops": 0}
    bytes_ = row * tok + 2 * B * H * (2 * L + R) + 4 * (B + pages)
    if op == "step":
        return {"bytes": bytes_ + 2 * row * B + 4 * B, "flops": 2 * (tok + B) * H * (2 * L + R)}
    return {"bytes": bytes_, "flops": 2 * tok * H * (2 * L + R)}


# ---------------------------------------------------------------------------------------------------- inputs

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _rows(gen, n, L):
    """bf16 rows [n, L + 64] of a down projection: tokens of different magnitude, a few outliers."""
    size = (0.5 * _normal(gen, n, 1)).exp_()
    size *= 1 + 7 * (torch.rand(n, 1, generator=gen, device="cuda") < 1 / 512)
    return (_normal(gen, n, L + R) * size).bfloat16()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _sum0(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def _fill(gen, cached, pages, ids, num_pages, L):
    """A pool with `cached` tokens in every block; what no token has filled holds NaN."""
    pool = torch.full((num_pages, P, L + R), float("nan"), dtype=torch.bfloat16, device="cuda")
    used = [-(-c // P) for c in cached]
    fill = [min(P, c - P * j) for c, u in zip(cached, used) for j in range(u)]   # tokens in each page that holds any
    if fill:
        at = torch.cat([ids[a:a + u] for a, u in zip(_sum0(pages), used)]).long()
        there = torch.arange(P, device="cuda") < _i32(fill)[:, None]
        pool[at] = torch.where(there[..., None], _normal(gen, len(fill), P, L + R), float("nan")).bfloat16()
    return pool


def _rope_kind(case):
    """(rotated elements, layout, scaling) of the case's positions."""
    return (case["rot"], case["layout"], case["scaling"]) if case["op"] == "rope" else (R, "interleaved", "parts")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, B, H, L = case["op"], case["blocks"], case["heads"], case["latent"]
    cached, new = _lengths(case)
    tok, rows = sum(cached), sum(new)
    st = {"case": case, "lens_host": cached}
    if op == "rope":
        start = torch.randint(0, 131072, (B,), generator=gen, device="cuda", dtype=torch.int32)   # blocks of a history
        st["positions"] = torch.cat([s + torch.arange(c, device="cuda", dtype=torch.int32) for s, c in zip(start, cached)])
        st["q"] = _normal(gen, tok, H, case["head_dim"]).bfloat16()
        st["q_out"] = torch.empty_like(st["q"])
        if case["kv_heads"]:
            st["k"] = _normal(gen, tok, case["kv_heads"], case["head_dim"]).bfloat16()
            st["k_out"] = torch.empty_like(st["k"])
    elif op == "prefill":
        st["q"] = _normal(gen, tok, H, NOPE + R).bfloat16()
        st["kv"] = _normal(gen, tok, H, NOPE + VDIM).bfloat16()         # a head's key and value parts, as one product gives them
        st["rows"] = _normal(gen, tok, 512 + R).bfloat16()              # the packed rows of the append: r is their last part
        st["o"] = torch.empty(tok, H, VDIM, dtype=torch.bfloat16, device="cuda")
    else:
        room = [c + n for c, n in zip(cached, new)]
        pages = [-(-r // P) for r in room]
        total = sum(pages)
        num_pages = total + 3                                                # a pool with a few pages to spare
        ids = torch.randperm(num_pages, generator=gen, device="cuda").int()  # the free list: any order
        st.update(total=total, indptr=_i32(_sum0(pages)), ids=ids[:total], pool=_fill(gen, cached, pages, ids, num_pages, L),
                  lens=_i32(cached), lens_out=torch.zeros(B, dtype=torch.int32, device="cuda"), rows=rows,
                  max_pages=max([1] + [-(-(c + (op == "step")) // P) for c in cached]))
        if op != "decode":
            st["x"] = _rows(gen, rows, L)
            st["weight"] = (1 + 0.1 * _normal(gen, L)).bfloat16()
            st["first"] = torch.randint(0, 100000, (B,), generator=gen, device="cuda", dtype=torch.int32)
        if op == "append":
            st["cu"] = _i32(_sum0(new))
            st["packed"] = torch.empty(rows, L + R, dtype=torch.bfloat16, device="cuda")
        else:
            st["q_c"] = _normal(gen, H, B, L).bfloat16().transpose(0, 1)     # a batched product per head gives [H, B, L]
            st["q_r"] = _normal(gen, B, H, NOPE + R).bfloat16()[..., NOPE:]  # the last part of the projected query
            st["o"] = torch.empty(B, H, L, dtype=torch.bfloat16, device="cuda")
    if own:
        _own_prepare(st, op)
    return st


def _own_prepare(st, op):
    import numpy as np

    from paper_2605_23296_b200 import binding as lib

    case, on = st["case"], torch.cuda.current_stream().cuda_stream
    rot, layout, scaling = _rope_kind(case)
    kind = PARTS if scaling == "parts" else PLAIN
    st["rope"] = lib.cpa_rope_config(rot, lib.ROPE_HALF if layout == "half" else lib.ROPE_INTERLEAVED,
                                     lib.ROPE_SCALED_PARTS if scaling == "parts" else lib.ROPE_UNSCALED,
                                     kind.get("trained", 0), kind["base"], kind.get("factor", 1.0), kind.get("fast", 0.0),
                                     kind.get("slow", 0.0), 1.0)
    st["turns"] = torch.from_numpy(lib.cpa_rope_turns(st["rope"]).view(np.int64)).cuda()
    if op == "rope":
        return
    H, L = case["heads"], case["latent"]
    st["cfg"] = lib.cpa_latent_config(H, L or 512, R, NOPE, VDIM, P, (NOPE + R) ** -0.5, EPS, 0)
    tcfg = lib.cpa_latent_tables_config(st["cfg"])
    if op == "prefill":
        lens = st["lens_host"]
        pages = sum(-(-c // P) for c in lens)
        st["plan"] = plan = _Plan(lib, lib.cpa_latent_plan_config(st["cfg"]), lens, list(range(pages)))
        st["index"] = torch.empty(lib.cpa_plan_param(plan.handle, lib.PARAM_INDEX_BYTES), dtype=torch.uint8, device="cuda")
        lib.cpa_plan_upload(plan.handle, st["index"], st["index"].numel(), on)
        return
    num_pages = st["pool"].shape[0]
    st["dims"] = lib.cpa_table_dims(case["blocks"], 0, num_pages, num_pages, 0)
    st["tables"] = torch.empty(lib.cpa_tables_bytes(tcfg, st["dims"]), dtype=torch.uint8, device="cuda")
    room = (st["indptr"][1:] - st["indptr"][:-1]) * P
    rc = lib.cpa_tables_build(tcfg, st["dims"], room, st["ids"], st["total"], st["tables"], on)
    if rc:
        raise lib.CpaError(rc, "tables")
    st["workspace"] = torch.empty(lib.cpa_latent_decode_workspace_bytes(st["cfg"]), dtype=torch.uint8, device="cuda")


class _Plan:
    """A plan handle that goes with the state."""

    def __init__(self, lib, cfg, lens, pages):
        self.lib, self.handle = lib, lib.cpa_plan_create(cfg, lens, 0, pages)

    def __del__(self):
        self.lib.cpa_plan_destroy(self.handle)


# ---------------------------------------------------------------------------------------------------- run

def run(st):
    op = st["case"]["op"]
    if own:
        return _own(st, op)
    return {"rope": _rotate, "append": _append, "decode": _decode, "step": _step, "prefill": _prefill}[op](st)


def _own(st, op):
    from paper_2605_23296_b200 import binding as lib

    on = torch.cuda.current_stream().cuda_stream
    if op == "rope":
        rot = st["case"]["rot"]
        k = lib.rope_rows(st["k"], st["k_out"], rot) if "k" in st else None
        rc = lib.cpa_rope(st["rope"], st["turns"], st["positions"], st["q"].shape[0], lib.rope_rows(st["q"], st["q_out"], rot), k,
                          False, on)
        out = (st["q_out"], st["k_out"]) if k else st["q_out"]
    elif op == "append":
        rc = lib.cpa_latent_append(st["cfg"], st["dims"], st["tables"], st["rope"], st["turns"], st["x"], st["x"].stride(0),
                                   st["weight"], st["cu"], st["rows"], st["first"], st["lens"], st["lens_out"], st["pool"],
                                   st["packed"], on)
        out = st["pool"], st["packed"], st["lens_out"]
    elif op == "decode":
        rc = lib.cpa_latent_decode(st["cfg"], st["dims"], st["tables"], lib.latent_io(st["q_c"], st["q_r"], st["o"]),
                                   st["lens"], None, st["pool"], st["workspace"], on)
        out = st["o"]
    elif op == "step":
        rc = lib.cpa_latent_step(st["cfg"], st["dims"], st["tables"], st["rope"], st["turns"],
                                 lib.latent_io(st["q_c"], st["q_r"], st["o"]), st["x"], st["x"].stride(0), st["weight"],
                                 st["first"], st["lens"], st["lens_out"], None, st["pool"], st["workspace"], on)
        out = st["o"], st["pool"], st["lens_out"]
    else:
        r = st["rows"][:, -R:]
        rc = lib.cpa_latent_prefill(st["cfg"], st["plan"].handle, st["q"], st["kv"], r, r.stride(0), st["o"], on)
        out = st["o"]
    if rc:
        raise lib.CpaError(rc, op)
    return out


def _frequencies(rot, scaling):
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    f = PLAIN["base"] ** (-2 * i / rot)
    if scaling == "none":
        return f
    p = PARTS
    at = [rot * math.log(p["trained"] / (2 * math.pi * t)) / (2 * math.log(p["base"])) for t in (p["fast"], p["slow"])]
    lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
    ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
    return f / p["factor"] * ramp + f * (1 - ramp)


def _turn(x, positions, rot, layout, scaling):
    """x [..., rows, heads, rot] in 32 bits, turned to `positions` [rows]; angles in 64 bits."""
    a = positions.double()[:, None] * _frequencies(rot, scaling)
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    if layout == "half":
        u, v = x[..., :rot // 2], x[..., rot // 2:]
        return torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    u, v = x[..., 0::2], x[..., 1::2]
    return torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)


def _rotate(st):
    rot, layout, scaling = _rope_kind(st["case"])
    out = []
    for x, y in [(st["q"], st["q_out"])] + ([(st["k"], st["k_out"])] if "k" in st else []):
        rest = x.shape[2] - rot
        y[..., :rest] = x[..., :rest]
        y[..., rest:] = _turn(x[..., rest:].float(), st["positions"], rot, layout, scaling)
        out.append(y)
    return tuple(out) if len(out) > 1 else out[0]


def _new_rows(st, positions):
    """The rows as they are cached: normalised latent part, turned positional part; rounded once."""
    L, x = st["case"]["latent"], st["x"].float()
    c = x[:, :L]
    c = c * torch.rsqrt((c * c).mean(1, keepdim=True) + EPS) * st["weight"].float()
    return torch.cat([c, _turn(x[:, None, L:], positions, *_rope_kind(st["case"]))[:, 0]], 1).bfloat16()


def _store(st, cu):
    row = torch.arange(st["rows"], dtype=torch.int32, device="cuda")
    block = torch.searchsorted(cu[1:], row, right=True)
    at = st["lens"][block] + row - cu[block]
    y = _new_rows(st, st["first"][block] + at)
    st["pool"][st["ids"][st["indptr"][block] + at // P].long(), (at % P).long()] = y
    torch.add(st["lens"], cu[1:] - cu[:-1], out=st["lens_out"])
    return y


def _append(st):
    st["packed"].copy_(_store(st, st["cu"]))
    return st["pool"], st["packed"], st["lens_out"]


def _attend(st, lens, q_r):
    n, L = st["max_pages"], st["case"]["latent"]
    place = st["indptr"][:-1, None] + torch.arange(n, device="cuda")
    place = torch.minimum(place, st["indptr"][1:, None] - 1).clamp_min(0)
    pages = st["ids"][place].long() if st["ids"].numel() else torch.zeros_like(place)              # [B, n]
    seen = torch.arange(n * P, device="cuda") < lens[:, None]                                       # [B, n * 16]
    x = st["pool"][pages].flatten(1, 2).float().masked_fill(~seen[..., None], 0.0)                  # [B, n * 16, L + R]
    s = torch.matmul(torch.cat([st["q_c"].float(), q_r], 2), x.transpose(1, 2)) * (NOPE + R) ** -0.5
    s = s.masked_fill(~seen[:, None], float("-inf"))
    m = s.amax(2, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), 0.0, m))
    o = torch.matmul(p, x[..., :L]) / p.sum(2, keepdim=True).masked_fill(lens[:, None, None] == 0, 1.0)   # no token: zero
    return st["o"].copy_(o)


def _decode(st):
    return _attend(st, st["lens"], st["q_r"].float())


def _step(st):
    _store(st, torch.arange(st["case"]["blocks"] + 1, dtype=torch.int32, device="cuda"))
    q_r = _turn(st["q_r"].float(), st["first"] + st["lens"], *_rope_kind(st["case"]))
    return _attend(st, st["lens_out"], q_r), st["pool"], st["lens_out"]


def _prefill(st):
    q, kv, r, at = st["q"], st["kv"], st["rows"][:, -R:], 0
    for n in st["lens_host"]:                                                 # blocks do not see one another
        u = slice(at, at + n)
        k = torch.cat([kv[u, :, :NOPE], r[u, None].expand(n, q.shape[1], R)], 2).transpose(0, 1).float()   # [H, n, 192]
        s = torch.matmul(q[u].transpose(0, 1).float(), k.transpose(1, 2)) * (NOPE + R) ** -0.5
        i = torch.arange(n, device="cuda")
        s = s.masked_fill_(i > i[:, None], float("-inf"))
        p = s.sub_(s.amax(2, keepdim=True) if n else 0.0).exp_()
        o = torch.matmul(p, kv[u, :, NOPE:].transpose(0, 1).float()) / p.sum(2, keepdim=True)
        st["o"][u] = o.transpose(0, 1)
        at += n
    return st["o"]


# ---------------------------------------------------------------------------------------------------- 64 bits

def _turn64(x, positions, rot, layout, scaling):
    """As complex numbers: element pairs times e^(i angle)."""
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), positions.double()[:, None] * _frequencies(rot, scaling))
    pair = x.double().unflatten(-1, (2, rot // 2)).transpose(-1, -2) if layout == "half" else x.double().unflatten(-1, (rot // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
    return (y.transpose(-1, -2) if layout == "half" else y).flatten(-2)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op, H, L, B = case["op"], case["heads"], case["latent"], case["blocks"]
    cached, new = _lengths(case)
    kind = _rope_kind(case)
    if op == "rope":
        rest = case["head_dim"] - case["rot"]
        out = [torch.cat([x[..., :rest].double(), _turn64(x[..., rest:], st["positions"], *kind)], -1)
               for x in ([st["q"], st["k"]] if "k" in st else [st["q"]])]
        return tuple(out) if len(out) > 1 else out[0]
    if op == "prefill":
        o, at = torch.zeros(sum(cached), H, VDIM, dtype=torch.float64, device="cuda"), 0
        for n in cached:
            for h in range(H):
                q, kv, r = st["q"][at:at + n, h].double(), st["kv"][at:at + n, h].double(), st["rows"][at:at + n, -R:].double()
                s = (q[:, :NOPE] @ kv[:, :NOPE].T + q[:, NOPE:] @ r.T) / (NOPE + R) ** 0.5
                above = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
                o[at:at + n, h] = torch.softmax(s.masked_fill_(above, float("-inf")), 1) @ kv[:, NOPE:]
            at += n
        return o
    indptr, ids = st["indptr"].tolist(), st["ids"].long()
    pool, q_r = st["pool"].double(), st["q_r"].double() if op != "append" else None
    if op != "decode":
        x, first = st["x"].double(), st["first"].tolist()
        c = x[:, :L] / (x[:, :L].square().mean(1, keepdim=True) + EPS).sqrt() * st["weight"].double()
        where = [(b, cached[b] + i) for b in range(B) for i in range(new[b])]
        at = torch.tensor([first[b] + i for b, i in where], device="cuda")
        y = torch.cat([c, _turn64(x[:, None, L:], at, *kind)[:, 0]], 1)
        page = ids[torch.tensor([indptr[b] + i // P for b, i in where], device="cuda")]
        pool[page, torch.tensor([i % P for b, i in where], device="cuda")] = y
        if op == "append":
            return pool, y, None
        q_r = _turn64(st["q_r"], torch.tensor([f + n for f, n in zip(first, cached)], device="cuda"), *kind)
        cached = [n + 1 for n in cached]
    o = torch.zeros(B, H, L, dtype=torch.float64, device="cuda")
    for b, n in enumerate(cached):
        if n:
            y = pool[ids[indptr[b]:indptr[b] + -(-n // P)]].flatten(0, 1)[:n]
            w = torch.softmax((st["q_c"][b].double() @ y[:, :L].T + q_r[b] @ y[:, L:].T) / (NOPE + R) ** 0.5, 1)
            o[b] = w @ y[:, :L]
    return (o, pool, None) if op == "step" else o
