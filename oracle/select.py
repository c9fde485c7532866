"""Block summaries and block selection (oracle side, test infrastructure).

The paper's decode step attends to the whole cache; attending to a bounded number of blocks of a long shared context, chosen by
the query, is this build's own.  Everything up to the choice is defined in float32 steps on whole numbers, so that an
implementation can match bit for bit:

  * summary of a (block, KV head): per channel the largest and the smallest of the block's stored keys (e4m3: the float32 product
    of code and scale); keys that are not numbers passed over, a channel with none other is 0, infinities the largest finite
    float32.  a = the largest magnitude, scale = a * float32(1/127) (1 where that is under 2^-126), code = rint(x / scale) held to
    127 in magnitude.
  * query codes likewise per row (what is not a number counts as 0).
  * score(r, h, j) = max over the heads g of KV head h of (float32(sum_c max(q_gc, 0) hi_jc + min(q_gc, 0) lo_jc) * s_j) * s_g.
  * Of a request's context (root blocks, then the visible blocks of its prefix) `blocks` are taken: the first keep_first, the last
    keep_last, a root's partly filled last block, and the highest scores, lower positions first where they are equal (no number: the lowest); all of a context
    of no more than that.
"""
from __future__ import annotations

import numpy as np

from . import attention, fp8

_F = np.float32
_MOST = np.finfo(np.float32).max
_RCP = _F(1.0) / _F(127.0)


def _scale(top):
    with np.errstate(over="ignore", under="ignore"):
        s = (top * _RCP).astype(np.float32)
    return np.where(s >= _F(2.0 ** -126), s, _F(1.0))


def _codes(x, scale):
    return np.clip(np.rint((x / scale).astype(np.float32)), -127, 127).astype(np.int8)


def keys_f32(kv, scales, kv_dtype, blk, n):
    """Keys of the first n slots of a block, float32 [heads, n, d]."""
    k = kv[blk, :, 0, :n]
    if kv_dtype == "f32":
        return k.astype(np.float32)
    if kv_dtype == "bf16":
        return (k.astype(np.uint32) << np.uint32(16)).view(np.float32)
    return (fp8.decode(k).astype(np.float32) * scales[blk, :, 0].astype(np.float32)[:, None, None]).astype(np.float32)


def summarise(kv, scales, kv_dtype, blk, n):
    """(codes int8 [heads, 2, d], scales float32 [heads]) of a block with n stored tokens."""
    k = keys_f32(kv, scales, kv_dtype, blk, n)
    hi = np.fmax.reduce(k, axis=1)
    lo = np.fmin.reduce(k, axis=1)
    ends = np.stack([hi, lo], 1)
    ends = np.clip(np.where(np.isnan(ends), _F(0), ends), -_MOST, _MOST).astype(np.float32)
    s = _scale(np.abs(ends).max((1, 2)))
    return _codes(ends, s[:, None, None]), s


def scores(q: np.ndarray, codes: np.ndarray, block_scales: np.ndarray, num_kv_heads: int) -> np.ndarray:
    """q float32 [Hq, d]; codes int8 [n, heads, 2, d], block_scales [n, heads] -> float32 [heads, n]."""
    q = np.clip(np.where(np.isnan(q), _F(0), q), -_MOST, _MOST).astype(np.float32)
    s = _scale(np.abs(q).max(-1))
    c = _codes(q, s[:, None]).astype(np.int64).reshape(num_kv_heads, -1, q.shape[-1])
    s = s.reshape(num_kv_heads, -1)
    hi, lo = codes[:, :, 0].astype(np.int64), codes[:, :, 1].astype(np.int64)
    dots = np.einsum("hgc,nhc->hgn", np.maximum(c, 0), hi) + np.einsum("hgc,nhc->hgn", np.minimum(c, 0), lo)
    with np.errstate(over="ignore"):
        v = (dots.astype(np.float32) * block_scales.T[:, None, :].astype(np.float32)).astype(np.float32)
        return (v * s[:, :, None]).astype(np.float32).max(1)


def context(lay, r, block, visible=None):
    """(block ids, valid tokens) of request r's context, root first, and the position of a partly filled last root block (-1: none)."""
    p = int(lay.req_prompt[r])
    t = -1 if getattr(lay, "prompt_root", None) is None else int(lay.prompt_root[p])
    seen = int(lay.prefix_len[p]) if visible is None else int(visible[r])
    ids, valid, partial = [], [], -1
    if t >= 0:
        n = int(lay.root_len[t])
        blk = lay.root_blk[lay.root_blk_indptr[t]:lay.root_blk_indptr[t + 1]]
        ids += [int(b) for b in blk]
        valid += [min(block, n - i * block) for i in range(len(blk))]
        partial = len(blk) - 1 if n % block else -1
    nb = -(-seen // block)
    ids += [int(b) for b in lay.prefix_blk[lay.prefix_blk_indptr[p]:lay.prefix_blk_indptr[p] + nb]]
    valid += [min(block, seen - i * block) for i in range(nb)]
    return ids, valid, partial


def choose(score: np.ndarray, n: int, partial: int, blocks: int, keep_first: int, keep_last: int) -> list:
    """Positions taken of one (request, KV head), ascending, without the partly filled root block."""
    others = [j for j in range(n) if j != partial]
    most = blocks - (partial >= 0)
    if len(others) <= most:
        return others
    always = [j for j in others if j < keep_first or j >= n - keep_last]
    score = np.where(np.isnan(score), -np.inf, score)
    rest = sorted((j for j in others if keep_first <= j < n - keep_last), key=lambda j: (-float(score[j]), j))
    return sorted(always + rest[:most - len(always)])


def select(q_f32, lay, block, codes, block_scales, num_kv_heads, blocks, keep_first, keep_last, visible=None):
    """Per request, per KV head: (positions, block ids) of the choice."""
    out = []
    for r in range(len(lay.req_prompt)):
        ids, _, partial = context(lay, r, block, visible)
        sc = scores(q_f32[r], codes[ids], block_scales[ids], num_kv_heads) if ids else np.zeros((num_kv_heads, 0))
        rows = []
        for h in range(num_kv_heads):
            pos = choose(sc[h], len(ids), partial, blocks, keep_first, keep_last)
            rows.append((pos, [ids[j] for j in pos]))
        out.append(rows)
    return out


def attend(q_bits, q_dtype, kv, scales, kv_dtype, lay, chosen, block, visible=None):
    """fp64 attention of every request over its chosen blocks, a partly filled root block, and its private tokens."""
    q = attention.widen(q_bits, q_dtype)
    out, lse = np.zeros(q.shape), np.zeros(q.shape[:2])
    heads = kv.shape[1]
    g = q.shape[1] // heads
    for r in range(q.shape[0]):
        ids, valid, partial = context(lay, r, block, visible)
        sb = lay.suffix_blk[lay.suffix_blk_indptr[r]:lay.suffix_blk_indptr[r + 1]]
        own = attention.gather_segment(kv, scales, kv_dtype, sb, int(lay.suffix_len[r]))
        for h in range(heads):
            pos = sorted(chosen[r][h][0] + ([partial] if partial >= 0 else []))
            parts = [attention.gather_segment(kv, scales, kv_dtype, [ids[j]], valid[j]) for j in pos] + [own]
            k = np.concatenate([p[0] for p in parts])[:, h:h + 1]
            v = np.concatenate([p[1] for p in parts])[:, h:h + 1]
            out[r, h * g:(h + 1) * g], lse[r, h * g:(h + 1) * g] = attention.attention_state(q[r, h * g:(h + 1) * g], k, v)
    return out, lse
