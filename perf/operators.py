"""Operators around the decode-attention step, case by case: their plain form in elementary torch operations, and the same
through this package's calls.

A case names an operator and the sizes of a batch:

  append     one token a request: q, k, v of a fused projection normed per head and rotated, k and v stored in the cache
  ingest     whole prefixes handed over as raw projections: k normed, rotated and stored, v stored
  rows       the queries of newly appended context tokens, normed and rotated
  gather     stored prefixes read back into contiguous tensors
  summaries  the largest and smallest key of every block and channel, in eight bits
  select     the blocks of its context that a request attends to, by the products of its queries with the summaries
  sparse     one decode step over those blocks and the private tokens: the selection, then the attention

Lengths follow from the case alone (its `lens` seed), values and block placement from the seed given to prepare().
"""
import math

import numpy as np
import torch

own = False

ESZ = {"f32": 4, "bf16": 2, "fp8_e4m3": 1}
EPS = 1e-6
BASE = 500000.0
H8B, H70B, H64, H28, H256 = (32, 8, 128), (64, 8, 128), (32, 8, 64), (28, 4, 128), (16, 4, 256)


def _case(op, kv, heads, prompts, models, prefix, suffix, block=16, lens=0, rot=None, pairing="halves", norm=True, start=0,
          blocks=0, first=1, last=2, **more):
    return dict(op=op, kv=kv, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], block=block, prompts=prompts, models=models,
                prefix_lo=prefix[0], prefix_hi=prefix[1], suffix_hi=suffix, lens=lens, rot=heads[2] if rot is None else rot,
                pairing=pairing, norm=norm, start=start, blocks=blocks, first=first, last=last, **more)


def listed():
    return [
        # the decode step of a lone session, four models, deep in a long context: nothing but latency
        _case("append", "bf16", H8B, 1, 4, (32, 32), 200, lens=1, start=120000, name="append_lone"),
        # a loaded decode GPU: 240 requests of a model with 64 query heads, e4m3 cache
        _case("append", "fp8_e4m3", H70B, 60, 4, (20, 60), 120, lens=2, start=9000, name="append_fp8"),
        # a prefill worker's raw projections of ragged contexts handed over, neighbouring elements paired, half of a head rotated
        _case("ingest", "bf16", H8B, 11, 1, (700, 9000), 0, lens=3, rot=64, pairing="neighbours", name="ingest_bf16"),
        # the same for a model with an e4m3 cache, many contexts
        _case("ingest", "fp8_e4m3", H70B, 40, 1, (2048, 12288), 0, lens=4, name="ingest_fp8"),
        # the queries of a batch of partial prefills
        _case("rows", "bf16", H70B, 24, 1, (100, 301), 0, lens=5, start=8192, name="rows_prefill"),
        # a short float32 context read back, as a comparison against a reference does
        _case("gather", "f32", (4, 2, 64), 1, 1, (1037, 1037), 0, lens=6, name="gather_f32"),
        # cached contexts of an e4m3 pool handed to a worker that computes in bf16
        _case("gather", "fp8_e4m3", H70B, 32, 1, (2048, 12288), 0, lens=7, name="gather_fp8"),
        # summaries of one context that has just been handed over
        _case("summaries", "bf16", H8B, 1, 1, (5003, 5003), 0, lens=8, name="summaries_lone"),
        # ... and of a batch of long ones
        _case("summaries", "fp8_e4m3", H70B, 24, 1, (8192, 32768), 0, lens=9, name="summaries_fp8"),
        # one very long context under four models: 8192 blocks to choose from
        _case("select", "bf16", H8B, 1, 4, (131001, 131001), 64, lens=10, blocks=128, name="select_long"),
        # a decode step of a lone session that attends to 1024 tokens of a context of 60000
        _case("sparse", "bf16", H8B, 1, 4, (60013, 60013), 256, lens=11, blocks=64, name="sparse_lone"),
        # 96 requests on 32 long contexts, e4m3 cache, 2048 tokens each and up to 500 private ones
        _case("sparse", "fp8_e4m3", H70B, 32, 3, (6000, 30000), 500, lens=12, blocks=128, name="sparse_fp8"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["append", "append", "ingest", "ingest", "rows", "gather", "summaries", "select", "sparse", "sparse"])
    kv = rng.choice(["bf16", "bf16", "fp8_e4m3", "f32"])
    heads = {"bf16": rng.choice([H8B, H8B, H64, H28, H256, (16, 16, 128)]), "fp8_e4m3": rng.choice([H70B, H8B, H28, H64]),
             "f32": rng.choice([H8B, (4, 2, 64), H256, (8, 1, 128)])}[kv]
    block = rng.choice([16, 16, 16, 32, 64])
    d = heads[2]
    common = dict(block=block, lens=rng.randrange(1 << 20), rot=rng.choice([d, d, d // 2, d // 4]), norm=rng.random() < 0.75,
                  pairing=rng.choice(["halves", "halves", "neighbours"]), start=log_int(1, 200000) - 1)
    token = 2 * heads[1] * d * (4 if kv == "f32" else 2)   # bytes of K and V of one token, unquantised
    if op == "append":
        return _case(op, kv, heads, log_int(1, 64), rng.randint(1, 8), (16, 64), log_int(4, 200), **common)
    prompts, longest = log_int(1, 64), log_int(40, 32000)
    lo = max(1, longest // rng.choice([1, 3, 12]))
    if op == "rows":
        longest = log_int(1, 512)
        return _case(op, kv, heads, prompts, 1, (max(1, longest // 4), longest), 0, **common)
    most = 1.0e9
    models = 1 if op in ("ingest", "gather", "summaries") else rng.randint(1, 6)
    chosen = 0
    if op in ("select", "sparse"):
        chosen = log_int(4, 2048 // block)
        longest = max(longest, 2 * chosen * block)
        lo = max(1, longest // rng.choice([1, 2, 8]))
        while prompts > 1 and prompts * models * heads[1] * chosen * block * d > 1.5e8:
            prompts = prompts * 3 // 4
    while prompts > 1 and prompts * longest * token > most:
        prompts = prompts * 3 // 4
    return _case(op, kv, heads, prompts, models, (min(lo, longest), longest), log_int(1, 512) if chosen else 0, blocks=chosen,
                 first=rng.randint(0, 2), last=rng.randint(1, 2), **common)


# ---- lengths and tables --------------------------------------------------------------------------------------------

class Lengths:
    """Segment lengths of a case and the blocks they take (roots aside, prompts first, then requests, from the head of the
    free list; an appended token takes one more block where the private segment is at a block boundary)."""

    def __init__(self, case):
        rng = np.random.default_rng([23, case["lens"]])
        n, blk = case["prompts"], case["block"]
        self.prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, n).astype(np.int32)
        self.req_prompt = np.repeat(np.arange(n, dtype=np.int32), case["models"])
        self.req_model = np.tile(np.arange(case["models"], dtype=np.int32), n)
        self.num_requests = n * case["models"]
        hi = case["suffix_hi"]
        self.suffix = rng.integers(0, hi + 1, self.num_requests).astype(np.int32)
        self.prefix_blocks = -(-self.prefix // blk)
        self.suffix_blocks = -(-self.suffix // blk)
        self.grown = (self.suffix % blk == 0).astype(np.int32) if case["op"] == "append" else np.zeros_like(self.suffix)
        self.num_blocks = int(self.prefix_blocks.sum() + self.suffix_blocks.sum() + self.grown.sum()) + 3


def _padded(order, counts, first):
    """[segments, most] block ids (0 past a segment's end) of segments that take `counts` blocks each from order[first:]."""
    most = max(1, int(counts.max()))
    at = first + np.cumsum(counts) - counts
    index = at[:, None] + np.arange(most)[None, :]
    live = np.arange(most)[None, :] < counts[:, None]
    return np.where(live, order[np.minimum(index, len(order) - 1)], 0).astype(np.int64), live


def _dtype(kv):
    return torch.float32 if kv == "f32" else torch.bfloat16


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _fill(case, gen, num_blocks, topics):
    """Pool contents: keys and values of unit spread, the keys of a block around one of a few topics."""
    h, d, blk, kv = case["kv_heads"], case["head_dim"], case["block"], case["kv"]
    pool = torch.empty((num_blocks, h, 2, blk, d), dtype=torch.uint8 if kv == "fp8_e4m3" else _dtype(kv), device="cuda")
    scales = None
    if kv == "fp8_e4m3":
        scales = (0.8 + 0.4 * torch.rand((num_blocks, h, 2), device="cuda", generator=gen)) / 100.0
    per = max(1, (1 << 27) // (h * 2 * blk * d))
    for b0 in range(0, num_blocks, per):
        n = min(per, num_blocks - b0)
        x = torch.randn((n, h, 2, blk, d), device="cuda", generator=gen)
        x[:, :, 0] += topics[torch.randint(topics.shape[0], (n,), device="cuda", generator=gen)][:, None, None, :]
        if scales is not None:
            x = (x / scales[b0:b0 + n, :, :, None, None]).clamp_(-448, 448)
            pool[b0:b0 + n] = x.to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            pool[b0:b0 + n] = x.to(pool.dtype)
    return pool, scales


def _inputs(case, seed):
    lens = Lengths(case)
    gen = torch.Generator(device="cuda").manual_seed(1000003 * (seed % (1 << 32)) + 11)
    hq, h, d, blk, op, t = case["q_heads"], case["kv_heads"], case["head_dim"], case["block"], case["op"], _dtype(case["kv"])
    order = np.random.default_rng([seed, 6]).permutation(lens.num_blocks).astype(np.int32)
    s = {"case": case, "lens": lens, "order": order}
    ids, live = _padded(order, lens.prefix_blocks, 0)
    s["prefix_ids"], s["prefix_live"] = _dev(ids), _dev(live)
    sids, slive = _padded(order, lens.suffix_blocks, int(lens.prefix_blocks.sum()))
    s["suffix_ids"] = _dev(sids)
    s["prefix_len"], s["suffix_len"] = _dev(lens.prefix.astype(np.int64)), _dev(lens.suffix.astype(np.int64))
    topics = 1.5 * torch.randn((32, d), device="cuda", generator=gen)

    def rows(*shape):
        x = torch.randn(shape, device="cuda", generator=gen)
        return (x * torch.exp2(3.0 * torch.rand((*shape[:-1], 1), device="cuda", generator=gen) - 2.0)).to(t)

    if op in ("append", "ingest", "rows"):
        s["radians"] = BASE ** (-np.arange(0, case["rot"], 2) / max(1, case["rot"]))
        for name in ("q_weight", "k_weight"):
            s[name] = (1.0 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(t) if case["norm"] else None
    if op == "append":
        s["pool"], s["scales"] = _fill(case, gen, lens.num_blocks, topics)
        qkv = rows(lens.num_requests, hq + 2 * h, d)           # one projection's output: q, k, v heads side by side
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
        s["positions"] = _dev((case["start"] + lens.prefix[lens.req_prompt] + lens.suffix).astype(np.int32))
        last = np.array([sids[r, lens.suffix[r] // blk] if not lens.grown[r] else 0 for r in range(lens.num_requests)], np.int64)
        fresh = int(lens.prefix_blocks.sum() + lens.suffix_blocks.sum())
        last[lens.grown == 1] = order[fresh:fresh + int(lens.grown.sum())]
        s["dest_block"], s["dest_slot"] = _dev(last), _dev((lens.suffix % blk).astype(np.int64))
    elif op == "rows":
        n = int(lens.prefix.sum())
        s["q"] = rows(n, hq + 2 * h, d)[:, :hq]
        s["positions"] = _dev(np.concatenate([case["start"] + np.arange(x) for x in lens.prefix]).astype(np.int32))
    elif op == "ingest":
        n = int(lens.prefix.sum())
        kv = rows(n, 2 * h, d)
        s["k"], s["v"] = kv[:, :h], kv[:, h:]
        s["positions"] = _dev(np.concatenate([case["start"] + np.arange(x) for x in lens.prefix]).astype(np.int32))
        s["pool"] = torch.zeros((lens.num_blocks, h, 2, blk, d), dtype=torch.uint8 if case["kv"] == "fp8_e4m3" else t, device="cuda")
        s["scales"] = torch.zeros((lens.num_blocks, h, 2), device="cuda") if case["kv"] == "fp8_e4m3" else None
    elif op != "select":
        s["pool"], s["scales"] = _fill(case, gen, lens.num_blocks, topics)
    if op == "gather":
        n = int(lens.prefix.sum())
        s["dst"] = torch.empty((2, n, h, d), dtype=t, device="cuda")
    if op in ("select", "sparse"):
        q = torch.randn((lens.num_requests, hq, d), device="cuda", generator=gen)
        s["q"] = (q + topics[torch.randint(32, (lens.num_requests, 1), device="cuda", generator=gen)]).to(t)
    if op == "select":                                        # summaries of blocks around a topic each
        mid = topics[torch.randint(32, (lens.num_blocks,), device="cuda", generator=gen)][:, None, None, :]
        width = 1.5 + 0.5 * torch.randn((lens.num_blocks, h, 2, d), device="cuda", generator=gen)
        s["summaries"], s["summary_scales"] = _eight_bits(mid + width * torch.tensor([[1.0], [-1.0]], device="cuda"))
    elif op == "sparse":
        full = torch.full((lens.num_blocks,), blk, device="cuda")
        full[s["prefix_ids"][s["prefix_live"]]] = _valid(s)[s["prefix_live"]]
        s["summaries"], s["summary_scales"] = _eight_bits(_bounds(s, torch.arange(lens.num_blocks, device="cuda"), full))
    elif op == "summaries":
        s["summaries"] = torch.zeros((lens.num_blocks, h, 2, d), dtype=torch.int8, device="cuda")
        s["summary_scales"] = torch.zeros((lens.num_blocks, h), device="cuda")
    return s


def _valid(s):
    """Tokens stored in each block of the prefixes, [prompts, most]."""
    blk = s["case"]["block"]
    first = torch.arange(s["prefix_ids"].shape[1], device="cuda") * blk
    return (s["prefix_len"][:, None] - first[None, :]).clamp(0, blk)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["batch"] = _batch(s)
    return s


# ---- the framework's calls ---------------------------------------------------------------------------------------------

def _batch(s):
    """What a program keeps between calls: the layout over a pool, its uploaded tables, the rotation's parameters."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd import runtime
    case, lens, op = s["case"], s["lens"], s["case"]["op"]
    geo = B.geometry(case["q_heads"], case["kv_heads"], case["head_dim"], case["block"], "f32" if case["kv"] == "f32" else "bf16", case["kv"])
    if op in ("append", "ingest", "rows"):
        s["rope"] = runtime.Rope(s["radians"], case["pairing"], s["q_weight"], s["k_weight"], EPS)
    if op == "rows":
        s["geo"], s["out"] = geo, torch.empty((s["q"].shape[0], case["q_heads"], case["head_dim"]), dtype=s["q"].dtype, device="cuda")
        return None
    pool = B.ps_pool_create(lens.num_blocks, s["order"])
    layout = B.ps_kv_layout(pool, geo, lens.prefix, lens.req_prompt, lens.req_model, lens.suffix)
    if op == "append":
        B.ps_layout_append(pool, layout, lens.num_requests)
    q = s["q"] if op in ("select", "sparse") else torch.zeros((lens.num_requests, case["q_heads"], case["head_dim"]), dtype=_dtype(case["kv"]), device="cuda")
    batch = runtime.DecodeBatch(layout, geo, lens.num_requests, q, s.get("pool", q), s.get("scales"))
    if op in ("select", "sparse"):
        return batch.select(case["blocks"], case["first"], case["last"])
    return batch


def _run_own(s):
    op, batch = s["case"]["op"], s["batch"]
    if op == "append":
        batch.kv_append_rope(s["rope"], s["q"], s["k"], s["v"], s["positions"])
        return {"q": batch.q, **_cache(s)}
    if op == "ingest":
        batch.kv_ingest_rope(0, s["rope"], s["k"], s["v"], s["positions"])
        return _cache(s)
    if op == "rows":
        from paper_2602_12029_amd import runtime
        return runtime.rope_rows(s["geo"], s["rope"], s["q"], s["positions"], s["out"])
    if op == "gather":
        batch.kv_gather(0, s["dst"][0], s["dst"][1])
        return s["dst"]
    if op == "summaries":
        batch.block_summaries(0, s["summaries"], s["summary_scales"])
        return _summary_values(s["summaries"], s["summary_scales"])
    batch.select_blocks(s["summaries"], s["summary_scales"])
    if op == "select":
        return batch.lists()
    batch.decode_attention()
    return {"lists": batch.lists(), "out": batch.out, "lse": batch.lse}


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "ingest": _ingest, "rows": _rows, "gather": _gather, "summaries": _summaries, "select": _select,
            "sparse": _sparse}[s["case"]["op"]](s)


def _cache(s):
    """The pool: of an e4m3 one its codes as numbers, and the scale of every tile beside them."""
    if s["scales"] is None:
        return {"kv": s["pool"]}
    return {"kv": s["pool"].view(torch.float8_e4m3fn), "scales": s["scales"]}


def _norm_rotate(s, x, weight):
    """Rows [tokens, heads, d] in float32, normed and rotated."""
    case = s["case"]
    y = x.to(torch.float32)
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.to(torch.float32)
    rot = case["rot"]
    angle = s["positions"].to(torch.float64)[:, None] * torch.from_numpy(s["radians"]).cuda()[None, :]
    cos, sin = torch.cos(angle).to(torch.float32)[:, None, :], torch.sin(angle).to(torch.float32)[:, None, :]
    out = y.clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if case["pairing"] == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    out[..., a] = y[..., a] * cos - y[..., b] * sin
    out[..., b] = y[..., a] * sin + y[..., b] * cos
    return out


def _codes(x, scale):
    return (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _append(s):
    case, pool = s["case"], s["pool"]
    q = _norm_rotate(s, s["q"], s["q_weight"]).to(s["q"].dtype)
    new = torch.stack([_norm_rotate(s, s["k"], s["k_weight"]), s["v"].to(torch.float32)], 2)      # [R, heads, K|V, d]
    at, slot = s["dest_block"], s["dest_slot"]
    row = torch.arange(at.shape[0], device="cuda")
    if s["scales"] is None:
        tiles = pool[at]
        tiles[row, :, :, slot] = new.to(pool.dtype)
        pool[at] = tiles
        return {"q": q, **_cache(s)}
    old, top = s["scales"][at], new.abs().amax(-1)
    fresh = (slot == 0)[:, None, None]
    grown = torch.where(fresh, torch.where(top > 0, top / 448, 1.0), torch.maximum(old, top / 448))
    tiles = pool[at]
    held = tiles.view(torch.float8_e4m3fn).to(torch.float32) * old[..., None, None]
    again = torch.where((grown != old)[..., None, None], _codes(held, grown[..., None, None]), tiles)
    before = (torch.arange(case["block"], device="cuda")[None, :] < slot[:, None])[:, None, None, :, None]
    tiles = torch.where(before, again, tiles)
    tiles[row, :, :, slot] = _codes(new, grown[..., None])
    pool[at] = tiles
    s["scales"][at] = grown
    return {"q": q, **_cache(s)}


def _ingest(s):
    case, pool, live = s["case"], s["pool"], s["prefix_live"]
    new = torch.stack([_norm_rotate(s, s["k"], s["k_weight"]), s["v"].to(torch.float32)], 2)      # [T, heads, K|V, d]
    at, valid = s["prefix_ids"][live], _valid(s)[live]                                            # blocks in token order
    first = torch.cumsum(valid, 0) - valid
    slot = torch.arange(case["block"], device="cuda")
    held = slot[None, :] < valid[:, None]
    token = torch.where(held, first[:, None] + slot[None, :], 0)
    tiles = new[token].permute(0, 2, 3, 1, 4) * held[:, None, None, :, None]                      # [blocks, heads, K|V, slots, d]
    if s["scales"] is None:
        codes = tiles.to(pool.dtype)
    else:
        top = tiles.abs().amax((-1, -2))
        scale = torch.where(top > 0, top / 448, 1.0)
        codes = _codes(tiles, scale[..., None, None])
        s["scales"][at] = scale
    pool[at] = torch.where(held[:, None, None, :, None], codes, pool[at])
    return _cache(s)


def _rows(s):
    return _norm_rotate(s, s["q"], s["q_weight"]).to(s["q"].dtype)


def _floats(s, ids):
    """Blocks of the pool in float32, [..., heads, K|V, slots, d]."""
    x = s["pool"][ids]
    if s["scales"] is None:
        return x.to(torch.float32)
    return x.view(torch.float8_e4m3fn).to(torch.float32) * s["scales"][ids][..., None, None]


def _gather(s):
    live = s["prefix_live"]
    held = torch.arange(s["case"]["block"], device="cuda")[None, :] < _valid(s)[live][:, None]
    x = _floats(s, s["prefix_ids"][live]).to(s["dst"].dtype)
    return x.permute(2, 0, 3, 1, 4)[:, held]                                                      # [K|V, T, heads, d]


def _bounds(s, ids, valid):
    """Largest and smallest key of each block, head and channel over its stored tokens, [blocks, heads, 2, d]."""
    x = s["pool"][ids, :, 0]
    k = x.view(torch.float8_e4m3fn).to(torch.float32) * s["scales"][ids, :, 0][..., None, None] if s["scales"] is not None else x.to(torch.float32)
    hidden = (torch.arange(s["case"]["block"], device="cuda")[None, :] >= valid[:, None])[:, None, :, None]
    return torch.stack([k.masked_fill(hidden, -math.inf).amax(2), k.masked_fill(hidden, math.inf).amin(2)], 2)


def _eight_bits(x):
    """[..., 2, d] as codes of -127 to 127 and one scale for both rows; the quotient is a float32 one."""
    top = x.abs().amax((-1, -2))
    scale = top / 127
    scale = torch.where(scale >= 2.0 ** -126, scale, 1.0)
    return torch.round(x / scale[..., None, None]).clamp(-127, 127).to(torch.int8), scale


def _summary_values(codes, scales):
    return codes.to(torch.float32) * scales[..., None, None]


def _summaries(s):
    live = s["prefix_live"]
    ids = s["prefix_ids"][live]
    s["summaries"][ids], s["summary_scales"][ids] = _eight_bits(_bounds(s, ids, _valid(s)[live]))
    return _summary_values(s["summaries"], s["summary_scales"])


def _chosen(s):
    """Positions of the blocks that a request attends to in its context, ascending, [R, heads, most], and how many they are [R]."""
    case, ids, live = s["case"], s["prefix_ids"], s["prefix_live"]
    p, h, d, m = case["prompts"], case["kv_heads"], case["head_dim"], case["models"]
    g, most = case["q_heads"] // h, case["blocks"]
    q = s["q"].to(torch.float32)
    top = q.abs().amax(-1) / 127
    q_scale = torch.where(top >= 2.0 ** -126, top, 1.0)
    code = torch.round(q / q_scale[..., None]).clamp(-127, 127)
    halves = torch.cat([code.clamp(min=0), code.clamp(max=0)], -1).reshape(p, m, h, g, 2 * d).permute(0, 2, 1, 3, 4)
    keys = s["summaries"][ids].to(torch.float32).reshape(p, -1, h, 2 * d).permute(0, 2, 3, 1).contiguous()
    dots = torch.matmul(halves.reshape(p, h, m * g, 2 * d).contiguous(), keys)                   # whole numbers under 2^24: exact
    score = dots * s["summary_scales"][ids].permute(0, 2, 1)[:, :, None, :]
    score = score.reshape(p, h, m, g, -1) * q_scale.reshape(p, m, h, g).permute(0, 2, 1, 3)[..., None]
    score = score.amax(3).permute(0, 2, 1, 3).reshape(p * m, h, -1)                              # [R, heads, blocks]
    n = live.sum(1).repeat_interleave(m)[:, None, None]
    j = torch.arange(ids.shape[1], device="cuda")
    score = score.masked_fill((j < case["first"]) | (j >= n - case["last"]), math.inf).masked_fill(j >= n, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :most]
    count = torch.minimum(n, torch.tensor(most, device="cuda"))
    best = torch.where(torch.arange(best.shape[-1], device="cuda") < count, best, ids.shape[1])
    return torch.sort(best, -1).values, count[:, 0, 0]


def _lists(s, chosen, count):
    """Block ids of the selections of all requests, one behind another, [heads, sum of the counts]."""
    ids = s["prefix_ids"].repeat_interleave(s["case"]["models"], 0)
    listed = torch.gather(ids[:, None, :].expand(-1, chosen.shape[1], -1), 2, chosen.clamp(max=ids.shape[1] - 1))
    kept = torch.arange(chosen.shape[2], device="cuda")[None, :] < count[:, None]
    return listed.permute(1, 0, 2)[:, kept].to(torch.int32), listed


def _select(s):
    return _lists(s, *_chosen(s))[0]


def _sparse(s):
    case = s["case"]
    h, d, blk, m = case["kv_heads"], case["head_dim"], case["block"], case["models"]
    chosen, count = _chosen(s)
    lists, listed = _lists(s, chosen, count)
    q = s["q"].to(torch.float32).reshape(-1, h, case["q_heads"] // h, d)
    head = torch.arange(h, device="cuda")
    slot = torch.arange(blk, device="cuda")

    def tokens(ids, seen):                       # ids, seen [R, heads, blocks]: K, V [R, heads, tokens, d], which of them count
        x = s["pool"][ids, head[None, :, None]]
        x = x.view(torch.float8_e4m3fn).to(torch.float32) * s["scales"][ids, head[None, :, None]][..., None, None] if s["scales"] is not None else x.to(torch.float32)
        x = x.permute(3, 0, 1, 2, 4, 5).reshape(2, ids.shape[0], h, -1, d)
        return x[0], x[1], (slot < seen[..., None]).reshape(ids.shape[0], h, -1)

    length = s["prefix_len"].repeat_interleave(m)[:, None, None]
    pk, pv, pm = tokens(listed, (length - chosen * blk).clamp(0, blk))
    ids = s["suffix_ids"][:, None, :].expand(-1, h, -1)
    first = torch.arange(ids.shape[2], device="cuda") * blk
    sk, sv, sm = tokens(ids, (s["suffix_len"][:, None, None] - first).clamp(0, blk).expand(-1, h, -1))
    k, v, seen = torch.cat([pk, sk], 2), torch.cat([pv, sv], 2), torch.cat([pm, sm], 2)[:, :, None, :]
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, v.masked_fill(~seen.transpose(2, 3), 0)) / total
    lse = (top + torch.log(total))[..., 0]
    return {"lists": lists, "out": out.reshape(-1, case["q_heads"], d).to(s["q"].dtype), "lse": lse.reshape(-1, case["q_heads"])}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    lens = Lengths(case)
    hq, h, d, op, esz = case["q_heads"], case["kv_heads"], case["head_dim"], case["op"], ESZ[case["kv"]]
    src = 4 if case["kv"] == "f32" else 2
    tokens, blocks, r = int(lens.prefix.sum(dtype=np.int64)), int(lens.prefix_blocks.sum(dtype=np.int64)), lens.num_requests
    tile_scales = 8 * h if case["kv"] == "fp8_e4m3" else 0
    summary = h * (2 * d + 4)
    if op == "append":
        return {"bytes": r * ((hq + 2 * h) * d * src + hq * d * src + 2 * h * d * esz + tile_scales + 4), "flops": 10 * r * (hq + h) * d}
    if op == "rows":
        return {"bytes": tokens * (2 * hq * d * src + 4), "flops": 10 * tokens * hq * d}
    if op in ("ingest", "gather"):
        return {"bytes": tokens * (2 * h * d * (src + esz) + 4) + blocks * tile_scales, "flops": 10 * tokens * h * d if op == "ingest" else 0}
    if op == "summaries":
        return {"bytes": tokens * h * d * esz + blocks * (summary + tile_scales // 2), "flops": 2 * tokens * h * d}
    kept = np.minimum(lens.prefix_blocks, case["blocks"]).astype(np.int64)
    choosing = lens.prefix_blocks > case["blocks"]
    total = int(lens.prefix_blocks[choosing].sum(dtype=np.int64)) * summary + r * hq * d * src + int(kept.sum()) * case["models"] * h * 4
    flops = 4 * d * hq * case["models"] * int(lens.prefix_blocks[choosing].sum(dtype=np.int64))
    if op == "sparse":
        # the models of a context choose apart: the blocks that at least one of them took, if they chose at random
        n = lens.prefix_blocks.astype(np.float64)
        read = int((n * (1.0 - (1.0 - kept / n) ** case["models"])).sum())
        own_tokens = int(lens.suffix.sum(dtype=np.int64))
        total += (read * case["block"] + own_tokens) * 2 * h * d * esz + read * tile_scales + r * hq * (d * src + 4)
        flops += 4 * d * hq * (int(kept.sum()) * case["models"] * case["block"] + own_tokens)
    return {"bytes": total, "flops": flops}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------------

def _turned(s, x, weight):
    """float64 rows, normed and turned pair by pair as complex numbers."""
    case = s["case"]
    y = x.to(torch.float64)
    if weight is not None:
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) * weight.to(torch.float64)
    rot = case["rot"]
    if rot == 0:
        return y
    z = y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["pairing"] == "halves" else y[..., :rot].unflatten(-1, (rot // 2, 2))
    z = torch.view_as_complex(z.contiguous())
    phase = s["positions"].to(torch.float64)[:, None, None] * torch.from_numpy(s["radians"]).cuda()
    z = torch.view_as_real(z * torch.polar(torch.ones_like(phase), phase))
    z = z.transpose(-1, -2) if case["pairing"] == "halves" else z
    return torch.cat([z.reshape(*z.shape[:-2], rot), y[..., rot:]], -1)


def _nearest_e4m3(x):
    return x.clamp(-448, 448).to(torch.float32).to(torch.float8_e4m3fn).to(torch.float64)


def exact(case, seed):
    op = case["op"]
    if op == "select":
        return None                              # block ids
    s = _inputs(case, seed)
    lens, blk, h, d = s["lens"], case["block"], case["kv_heads"], case["head_dim"]
    if op == "rows":
        return _turned(s, s["q"], s["q_weight"])
    if op in ("append", "ingest"):
        k, v = _turned(s, s["k"], s["k_weight"]), s["v"].to(torch.float64)
        e4m3 = s["scales"] is not None
        pool = s["pool"].view(torch.float8_e4m3fn).to(torch.float64) if e4m3 else s["pool"].to(torch.float64)
        scales = s["scales"].to(torch.float64) if e4m3 else None
        if op == "append":
            for r, (b, slot) in enumerate(zip(s["dest_block"].tolist(), s["dest_slot"].tolist())):
                for i, x in enumerate((k[r], v[r])):
                    if e4m3:
                        need = x.abs().amax(-1) / 448
                        new = torch.where(need > 0, need, 1.0) if slot == 0 else torch.maximum(scales[b, :, i], need)
                        moved = (new > scales[b, :, i])[:, None, None] if slot else False
                        if slot:
                            stored = pool[b, :, i, :slot]
                            pool[b, :, i, :slot] = torch.where(moved, _nearest_e4m3(stored * (scales[b, :, i] / new)[:, None, None]), stored)
                        scales[b, :, i] = new
                        x = _nearest_e4m3(x / new[:, None])
                    pool[b, :, i, slot] = x
        else:
            t0 = 0
            for p, n in enumerate(lens.prefix.tolist()):
                nb = -(-n // blk)
                ids = s["prefix_ids"][p, :nb]
                for i, x in enumerate((k[t0:t0 + n], v[t0:t0 + n])):
                    x = torch.cat([x, torch.zeros((nb * blk - n, h, d), dtype=torch.float64, device="cuda")]).reshape(nb, blk, h, d).transpose(1, 2)
                    if e4m3:
                        need = x.abs().amax((2, 3)) / 448
                        need = torch.where(need > 0, need, 1.0)
                        scales[ids, :, i] = need
                        x = _nearest_e4m3(x / need[:, :, None, None])
                    pool[ids, :, i] = x          # (what lies past the end was zero and stays so)
                t0 += n
        got = {"kv": pool, "scales": scales} if e4m3 else {"kv": pool}
        return {"q": _turned(s, s["q"], s["q_weight"]), **got} if op == "append" else got

    def stored(ids, head=slice(None)):
        x = s["pool"][ids][:, head]
        return x.to(torch.float64) if s["scales"] is None else \
            x.view(torch.float8_e4m3fn).to(torch.float64) * s["scales"][ids][:, head].to(torch.float64)[..., None, None]

    if op == "gather":
        parts = []
        for p, n in enumerate(lens.prefix.tolist()):
            x = stored(s["prefix_ids"][p, :-(-n // blk)])
            parts.append(x.permute(2, 0, 3, 1, 4).reshape(2, -1, h, d)[:, :n])
        return torch.cat(parts, 1)
    if op == "summaries":
        out = torch.zeros((lens.num_blocks, h, 2, d), dtype=torch.float64, device="cuda")
        for p, n in enumerate(lens.prefix.tolist()):
            nb = -(-n // blk)
            ids = s["prefix_ids"][p, :nb]
            k = stored(ids)[:, :, 0]
            if n % blk:
                k[-1, :, n % blk:] = k[-1, :, :1]                        # a token of the block again
            ends = torch.stack([k.amax(2), k.amin(2)], 2).to(torch.float32)   # (e4m3: a key is the float32 product)
            unit = ends.abs().amax((2, 3), keepdim=True) / 127                # a float32 scale, a float32 quotient: so defined
            out[ids] = torch.round(ends / unit).to(torch.float64) * unit.to(torch.float64)
        return out
    # sparse: the selection as it is defined, on whole numbers; the attention in 64 bits
    g, out, lse = case["q_heads"] // h, [], []
    for r in range(lens.num_requests):
        p = int(lens.req_prompt[r])
        n = int(lens.prefix[p])
        nb = -(-n // blk)
        ids = s["prefix_ids"][p, :nb]
        q = s["q"][r].to(torch.float32).reshape(h, g, d)
        unit = q.abs().amax(-1, keepdim=True) / 127
        code = torch.round(q / unit).to(torch.float64)
        hi, lo = s["summaries"][ids].to(torch.float64).permute(2, 1, 3, 0).contiguous()
        dots = (torch.bmm(code.clamp(min=0), hi) + torch.bmm(code.clamp(max=0), lo)).to(torch.float32)
        rank = ((dots * s["summary_scales"][ids].t()[:, None, :]) * unit).amax(1)
        rank[:, :case["first"]] = math.inf
        rank[:, max(0, nb - case["last"]):] = math.inf
        keep = torch.sort(torch.sort(-rank, dim=1, stable=True).indices[:, :case["blocks"]], 1).values
        ns = int(lens.suffix[r])
        own_k, own_v = stored(s["suffix_ids"][r, :-(-ns // blk)]).permute(2, 1, 0, 3, 4).flatten(2, 3)[:, :, :ns]
        os_, ls = [], []
        for i in range(h):
            x = stored(ids[keep[i]], i).reshape(-1, 2, blk, d).transpose(0, 1).reshape(2, -1, d)
            t = (keep[i][:, None] * blk + torch.arange(blk, device="cuda")).reshape(-1) < n
            kk, vv = torch.cat([x[0][t], own_k[i]]), torch.cat([x[1][t], own_v[i]])
            sc = s["q"][r].to(torch.float64).reshape(h, g, d)[i] @ kk.t().contiguous() / math.sqrt(d)
            ls.append(torch.logsumexp(sc, 1))
            os_.append(torch.softmax(sc, 1) @ vv)
        out.append(torch.cat(os_))
        lse.append(torch.cat(ls))
    return {"lists": None, "out": torch.stack(out), "lse": torch.stack(lse)}
