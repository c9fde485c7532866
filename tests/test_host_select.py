"""Selections and rotation rates on the host, no GPU: the derived tables and plan, following a growing base, what is refused."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

import workloads as wl
from helpers import oracle_setup
from oracle import layout as ol
from oracle import rope as orope
from oracle import select as osel
from paper_2602_12029_amd import binding as B

HOST_ONLY = bool(__import__("os").environ.get(B.HOST_ONLY_LIB_ENV))


def _geometry(g):
    return B.geometry(g.num_q_heads, g.num_kv_heads, g.head_dim, g.block_size, g.q_dtype, g.kv_dtype)


def _random_workload(rng, seed, roots):
    geo = [wl.Geometry(8, 2, 128, 16, "bf16", "bf16"), wl.Geometry(8, 2, 128, 32, "bf16", "fp8_e4m3"),
           wl.Geometry(4, 2, 64, 48, "f32", "f32"), wl.Geometry(28, 4, 128, 16, "bf16", "bf16")][int(rng.integers(4))]
    prompts = int(rng.integers(1, 5))
    member = [list(range(int(rng.integers(1, 4)))) for _ in range(prompts)]
    prefix = rng.integers(0, 700, prompts).tolist()
    suffix = rng.integers(0, 90, sum(map(len, member))).tolist()
    if roots:
        where = rng.integers(-1, 2, prompts).tolist()
        where = [0, 1][:prompts] + where[2:]
        lens = rng.integers(0, 300, max(where) + 1).tolist()
        return wl.make_tree_workload(f"sel{seed}", geo, 4, lens, where, prefix, member, suffix, 1.5, seed)
    return wl.make_workload(f"sel{seed}", geo, 4, prefix, member, suffix, 1.5, seed)


def _layouts(w):
    pool = B.ps_pool_create(w.num_blocks, w.free_order)
    geo = _geometry(w.geometry)
    if w.num_roots:
        lay = B.ps_kv_layout_tree(pool, geo, w.root_len, w.prompt_root, w.prefix_len, w.req_prompt, w.req_model, w.suffix_len)
    else:
        lay = B.ps_kv_layout(pool, geo, w.prefix_len, w.req_prompt, w.req_model, w.suffix_len)
    return pool, lay, oracle_setup(w)[:2]


def _check(w, sel, olay, blocks, first, last, visible=None):
    """Lists, lengths and plan of a selection against the oracle's context."""
    g, R, bs = w.geometry, w.num_requests, w.geometry.block_size
    t = B.ps_layout_tables(sel, R, R)
    lens = B.ps_layout_lengths(sel, R, R)
    indptr, stride = B.ps_select_lists(sel, R)
    roots = B.ps_layout_root_tables(sel)
    assert np.array_equal(indptr, t["prefix_blk_indptr"])
    assert np.array_equal(t["suffix_blk"], olay.suffix_blk) and np.array_equal(lens["suffix_len"], olay.suffix_len)
    assert stride == len(t["prefix_blk"]) + len(t["suffix_blk"]) + len(roots["root_blk"])
    n_root = 0
    for r in range(R):
        ids, valid, partial = osel.context(olay, r, bs, visible)
        mine = t["prefix_blk"][indptr[r]:indptr[r + 1]].tolist()
        others = [b for j, b in enumerate(ids) if j != partial]
        assert len(mine) == min(len(others), blocks - (partial >= 0)) and len(set(mine)) == len(mine)
        at = [others.index(b) for b in mine]
        assert at == sorted(at)
        tokens = [v for j, v in enumerate(valid) if j != partial]
        assert lens["prefix_len"][r] == sum(tokens[j] for j in at)              # (the tail, if any, is the last of the list)
        if partial >= 0:
            assert roots["root_blk"][n_root] == ids[partial]
            assert roots["root_group_req"][n_root] == r
            n_root += 1
    assert len(roots["root_blk"]) == n_root
    # the plan: every token of every request and KV head once, all block indexes inside its head's part of the block array
    plan = B.ps_layout_plan(sel, R)
    req = B.ps_layout_request_list(sel)
    seen = np.zeros((R, g.num_kv_heads), np.int64)
    for blk, t0, t1, off, n, h, split, kind in plan["items"].tolist():
        assert h * stride <= blk and blk + -(-t1 // bs) <= (h + 1) * stride and t0 < t1
        for r in req[off:off + n]:
            seen[r, h] += t1 - t0
    for r in range(R):
        _, valid, partial = osel.context(olay, r, bs, visible)
        want = int(lens["prefix_len"][r] + lens["suffix_len"][r]) + (valid[partial] if partial >= 0 else 0)
        assert (seen[r] == want).all()
    for which in (0, 1, 2):
        s = B.ps_layout_schedule(sel, which)
        if s:
            per = plan["items"][plan["items"][:, 7] & 1 == which] if which < 2 else plan["items"]
            assert sorted(map(tuple, s["items"].tolist())) == sorted(map(tuple, per.tolist()))
    choosing = [r for r in range(R) for ids, _, partial in [osel.context(olay, r, bs, visible)] if len(ids) - (partial >= 0) > blocks - (partial >= 0)]
    words = sum(g.num_kv_heads * -(-len(osel.context(olay, r, bs, visible)[0]) // 4) * 4 for r in choosing)
    assert B.ps_select_workspace_bytes(sel) == max(16, 4 * words)


@pytest.mark.parametrize("roots", [False, True])
def test_selection_tables_and_plan(roots):
    rng = np.random.default_rng(7 + roots)
    for seed in range(25):
        w = _random_workload(rng, seed, roots)
        pool, lay, (opool, olay) = _layouts(w)
        before = B.ps_pool_refcounts(pool, w.num_blocks)
        for blocks, first, last in ((4, 1, 2), (3, 0, 1), (9, 2, 2), (1000, 1, 1)):
            sel = B.ps_layout_select(lay, blocks, first, last)
            _check(w, sel, olay, blocks, first, last)
            B.ps_layout_replan(sel, B.plan_options(prefix_chunk_tokens=64, suffix_chunk_tokens=64))
            _check(w, sel, olay, blocks, first, last)
            assert B.ps_layout_state(sel) == (0, False)
            B.ps_layout_release(pool, sel)
        if w.num_requests and not roots:
            visible = np.array([rng.integers(0, w.prefix_len[p] + 1) for p in w.req_prompt], np.int32)
            sel = B.ps_layout_select(lay, 5)
            B.ps_layout_set_visible(lay, w.num_requests, visible)
            B.ps_layout_select_follow(lay, sel)
            _check(w, sel, olay, 5, 1, 2, visible)
            B.ps_layout_release(pool, sel)
        assert np.array_equal(before, B.ps_pool_refcounts(pool, w.num_blocks))
        B.ps_layout_release(pool, lay)
        B.ps_pool_destroy(pool)


def test_a_selection_follows_its_growing_base():
    rng = np.random.default_rng(11)
    for seed in range(8):
        w = _random_workload(rng, 100 + seed, seed % 2 == 1)
        w.num_blocks += 12 * w.num_requests
        w.free_order = np.random.default_rng(seed).permutation(w.num_blocks).astype(np.int32)
        pool, lay, (opool, olay) = _layouts(w)
        sel = B.ps_layout_select(lay, 4)
        for step in range(40):
            active = None if step % 3 == 0 else (rng.random(w.num_requests) < 0.6).astype(np.int32)
            B.ps_layout_append(pool, lay, w.num_requests, active)
            ol.append_step(opool, olay, active)
            if step % 7 != 5:                                # (a follow may come after several appends)
                B.ps_layout_select_follow(lay, sel)
                _check(w, sel, olay, 4, 1, 2)
        B.ps_layout_release(pool, sel)
        B.ps_layout_release(pool, lay)
        B.ps_pool_destroy(pool)


def test_an_empty_batch():
    pool = B.ps_pool_create(4)
    lay = B.ps_kv_layout(pool, B.geometry(4, 2, 64, 16, "f32", "f32"), [], [], [], [])
    sel = B.ps_layout_select(lay, 3)
    assert B.ps_select_lists(sel, 0)[1] == 0 and B.ps_select_workspace_bytes(sel) == 16 and B.ps_workspace_bytes(sel) == 16
    for h in (sel, lay):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def _refused(status, fn, *args):
    with pytest.raises(B.PsError) as e:
        fn(*args)
    assert e.value.status == status


def test_refusals():
    geo = B.geometry(4, 2, 64, 16, "f32", "f32")
    pool = B.ps_pool_create(64)
    lay = B.ps_kv_layout(pool, geo, [200], [0], [0], [3])
    for options in ((0, 0, 1), (4, -1, 1), (4, 1, 0), (3, 2, 2), (-1, 0, 1), (2 ** 31 - 1, 2 ** 31 - 1, 1)):
        _refused(B.PS_ERR_INVALID_ARG, B.ps_layout_select, lay, *options)
    tree = B.ps_kv_layout_tree(pool, geo, [20], [0], [50], [0], [0], [3])
    _refused(B.PS_ERR_INVALID_ARG, B.ps_layout_select, tree, 3, 1, 2)
    B.ps_layout_release(pool, B.ps_layout_select(tree, 4, 1, 2))
    sel = B.ps_layout_select(lay, 4)
    for fn, args in ((B.ps_layout_select, (sel, 4)), (B.ps_layout_append, (pool, sel, 1)), (B.ps_layout_set_visible, (sel, 1)),
                     (B.ps_layout_park, (pool, sel)), (B.ps_layout_resume, (pool, sel)), (B.ps_stage_layout, (sel,)),
                     (B.ps_layout_select_follow, (sel, sel)), (B.ps_layout_select_follow, (lay, lay)), (B.ps_layout_select_follow, (tree, sel)),
                     (B.ps_select_lists, (lay, 1)), (B.ps_ingest_tokens, (lay, 3)), (B.ps_ingest_tokens, (lay, -1))):
        _refused(B.PS_ERR_INVALID_ARG, fn, *args)
    assert B.ps_select_workspace_bytes(lay) == -1
    B.ps_layout_park(pool, lay)
    _refused(B.PS_ERR_INVALID_ARG, B.ps_layout_select, lay, 4)
    _refused(B.PS_ERR_INVALID_ARG, B.ps_layout_select_follow, lay, sel)
    wide = B.ps_kv_layout(pool, B.geometry(65, 1, 64, 16, "f32", "f32"), [200], [0], [0], [3])
    odd = B.ps_kv_layout(pool, B.geometry(4, 2, 96, 16, "f32", "f32"), [200], [0], [0], [3])
    for other in (wide, odd):
        _refused(B.PS_ERR_UNSUPPORTED, B.ps_layout_select, other, 4)
    for h in (sel, lay, tree, wide, odd):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_a_context_of_too_many_blocks():
    geo = B.geometry(1, 1, 64, 16, "bf16", "bf16")
    n = 65537
    pool = B.ps_pool_create(n + 1)
    lay = B.ps_kv_layout(pool, geo, [n * 16], [0], [0], [0])
    _refused(B.PS_ERR_UNSUPPORTED, B.ps_layout_select, lay, 4)
    B.ps_layout_set_visible(lay, 1, [(n - 1) * 16])
    sel = B.ps_layout_select(lay, 4)
    assert B.ps_select_workspace_bytes(sel) == 4 * (n - 1)
    for h in (sel, lay):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_a_follow_that_fails():
    """Nothing is launched from a selection whose follow failed, and the next follow plans it afresh."""
    geo = B.geometry(4, 1, 64, 16, "bf16", "bf16")
    n = 65540
    pool = B.ps_pool_create(n + 64)
    lay = B.ps_kv_layout(pool, geo, [n * 16, 100], [0, 1], [0, 0], [30, 0])
    B.ps_layout_set_visible(lay, 2, [900, 100])
    sel = B.ps_layout_select(lay, 4)
    for appends in (1, 2, 40):
        B.ps_layout_set_visible(lay, 2)
        for _ in range(appends):
            B.ps_layout_append(pool, lay, 2)
        _refused(B.PS_ERR_UNSUPPORTED, B.ps_layout_select_follow, lay, sel)
        _refused(B.PS_ERR_INVALID_ARG, B.ps_layout_replan, sel, B.plan_options())
        if not HOST_ONLY:                                 # (addresses that nothing may follow)
            _refused(B.PS_ERR_INVALID_ARG, B.ps_decode_attention, sel, 4096, 4096, 4096, 0, 4096, 4096, 0)
            _refused(B.PS_ERR_INVALID_ARG, B.ps_merge_states, sel, 4096, 4096, 4096, 0)
            _refused(B.PS_ERR_INVALID_ARG, B.ps_select_blocks, lay, 4096, sel, 4096, 4096, 4096, 4096, 4096)
        B.ps_layout_set_visible(lay, 2, [900, 100])
        B.ps_layout_append(pool, lay, 2)
        B.ps_layout_select_follow(lay, sel)
        fresh = B.ps_layout_select(lay, 4)
        for a, b in ((B.ps_layout_tables(sel, 2, 2), B.ps_layout_tables(fresh, 2, 2)), (B.ps_layout_plan(sel, 2), B.ps_layout_plan(fresh, 2))):
            assert a.keys() == b.keys() and all(np.array_equal(a[key], b[key]) for key in a)
        assert np.array_equal(B.ps_select_lists(sel, 2)[0], B.ps_select_lists(fresh, 2)[0])
        B.ps_layout_release(pool, fresh)
    for h in (sel, lay):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_ingest_tokens():
    pool = B.ps_pool_create(64)
    geo = B.geometry(4, 2, 64, 16, "f32", "f32")
    lay = B.ps_kv_layout_tree(pool, geo, [20, 0], [0, 1], [50, 7], [0, 0, 1], [0, 1, 0], [3, 0, 9])
    assert [B.ps_ingest_tokens(lay, which) for which in (0, 1, 2)] == [57, 12, 20]
    first = B.ps_kv_layout(pool, geo, [50], [0], [0], [3])
    ids = B.ps_layout_tables(first, 1, 1)["prefix_blk"][:2]
    more = B.ps_kv_layout_adopt(pool, geo, [70], [ids], [0], [0], [0])
    assert B.ps_ingest_tokens(more, 0) == 38
    for h in (more, first, lay):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_rates():
    rad = np.concatenate([[0.0, 1.0, np.pi, 2 * np.pi, 7.0, 1e-12, 5e-324, 1e6], 500000.0 ** (-np.arange(64) / 64)])
    got = B.ps_rope_turns(rad)
    for r, turns in zip(rad, got):
        exact = Fraction(float(r)) / orope._TWO_PI
        exact = (exact - exact.numerator // exact.denominator) * 2 ** 64
        # long double: 2^-64 of the turns, whole ones included, and half a step of the result
        off = abs(int(turns) - exact)
        assert min(off, 2 ** 64 - off) <= 1 + float(r) / 6
    for bad in (-1.0, float("nan"), float("inf")):
        _refused(B.PS_ERR_INVALID_ARG, B.ps_rope_turns, [0.5, bad])
    assert B.ps_rope_turns([]).size == 0


@pytest.mark.skipif(HOST_ONLY, reason="the device entry points are not in this library")
def test_device_calls_refuse_before_they_launch():
    """Addresses here are numbers that nothing may follow: every one of these calls has to return by its arguments alone."""
    P = 4096                                              # an aligned address
    geo = B.geometry(4, 2, 64, 16, "bf16", "fp8_e4m3")
    pool = B.ps_pool_create(64)
    lay = B.ps_kv_layout(pool, geo, [200], [0], [0], [3])
    sel = B.ps_layout_select(lay, 4)
    bad, shape, unsupported = B.PS_ERR_INVALID_ARG, B.PS_ERR_SHAPE, B.PS_ERR_UNSUPPORTED

    def rope(turns=P, qw=P, kw=P, eps=1e-6, rot=64, pairing=0):
        return B.ps_rope(turns, qw, kw, eps, rot, pairing)

    def rows(q=P, k=P, v=P, a=256, b=64, c=128, d=64, pos=P):
        return B.ps_token_rows(q, k, v, a, b, c, d, pos)

    ropes = [(bad, rope(turns=0)), (bad, rope(eps=-1.0)), (bad, rope(eps=float("nan"))), (bad, rope(eps=float("inf"))), (bad, rope(rot=66)),
             (bad, rope(rot=-2)), (bad, rope(rot=7)), (bad, rope(pairing=2)), (unsupported, rope(rot=24)), (shape, rope(qw=P + 8)),
             (shape, rope(kw=P + 2)), (shape, rope(turns=P + 4))]
    for status, r in ropes:
        _refused(status, B.ps_rope_rows, geo, r, 5, P, 256, 64, P, P)
        _refused(status, B.ps_kv_append_rope, lay, P, r, rows(), P, P, P)
        _refused(status, B.ps_kv_ingest_rope, lay, P, 0, r, P, P, 128, 64, P, P, P)
    for status, args in ((bad, (geo, rope(), -1, P, 256, 64, P, P)), (bad, (geo, rope(), 5, 0, 256, 64, P, P)), (bad, (geo, rope(), 5, P, 256, 64, 0, P)),
                         (bad, (geo, rope(), 5, P, 256, 64, P, 0)), (shape, (geo, rope(), 5, P + 8, 256, 64, P, P)), (shape, (geo, rope(), 5, P, 252, 64, P, P)),
                         (shape, (geo, rope(), 5, P, 256, 56, P, P)), (shape, (geo, rope(), 5, P, 256, 64, P, P + 2))):
        _refused(status, B.ps_rope_rows, *args)
    B.ps_rope_rows(geo, rope(), 0, 0, 0, 0, 0, 0)         # no rows: nothing to do
    for status, args in ((bad, (lay, 0, rope(), rows(), P, P, P)), (bad, (lay, P, rope(), rows(k=0), P, P, P)), (bad, (lay, P, rope(), rows(v=0), P, P, P)),
                         (bad, (lay, P, rope(), rows(pos=0), P, P, P)), (bad, (lay, P, rope(), rows(), 0, P, P)), (bad, (lay, P, rope(), rows(q=0), P, P, P)),
                         (bad, (lay, P, rope(), rows(), P, 0, P)), (bad, (lay, P, rope(), rows(), P, P, 0)), (bad, (sel, P, rope(), rows(), P, P, P)),
                         (shape, (lay, P, rope(), rows(k=P + 8), P, P, P)), (shape, (lay, P, rope(), rows(v=P + 8), P, P, P)),
                         (shape, (lay, P, rope(), rows(q=P + 8), P, P, P)), (shape, (lay, P, rope(), rows(a=255), P, P, P)),
                         (shape, (lay, P, rope(), rows(d=60), P, P, P)), (shape, (lay, P, rope(), rows(), P + 8, P, P)), (shape, (lay, P, rope(), rows(), P, P + 8, P))):
        _refused(status, B.ps_kv_append_rope, *args)
    for status, args in ((bad, (lay, 0, 0, rope(), P, P, 128, 64, P, P, P)), (bad, (lay, P, 3, rope(), P, P, 128, 64, P, P, P)),
                         (bad, (lay, P, 0, rope(), 0, P, 128, 64, P, P, P)), (bad, (lay, P, 0, rope(), P, P, 128, 64, 0, P, P)),
                         (bad, (lay, P, 0, rope(), P, P, 128, 64, P, P, 0)), (bad, (sel, P, 0, rope(), P, P, 128, 64, P, P, P)),
                         (shape, (lay, P, 0, rope(), P, P, 124, 64, P, P, P)), (shape, (lay, P, 0, rope(), P, P + 8, 128, 64, P, P, P))):
        _refused(status, B.ps_kv_ingest_rope, *args)
    for status, args in ((bad, (lay, 0, 0, P, P, 1, P, P, 128, 64)), (bad, (lay, P, -1, P, P, 1, P, P, 128, 64)), (bad, (lay, P, 0, 0, P, 1, P, P, 128, 64)),
                         (bad, (lay, P, 0, P, 0, 1, P, P, 128, 64)), (bad, (lay, P, 0, P, P, 1, 0, P, 128, 64)), (bad, (sel, P, 0, P, P, 1, P, P, 128, 64)),
                         (unsupported, (lay, P, 0, P, P, 2, P, P, 128, 64)), (shape, (lay, P, 0, P, P, 1, P, P, 100, 64)), (shape, (lay, P, 0, P, P, 1, P, P + 2, 128, 64))):
        _refused(status, B.ps_kv_gather, *args)
    for status, args in ((bad, (lay, 0, 0, P, P, P, P)), (bad, (lay, P, 5, P, P, P, P)), (bad, (lay, P, 0, 0, P, P, P)), (bad, (lay, P, 0, P, 0, P, P)),
                         (bad, (lay, P, 0, P, P, 0, P)), (bad, (lay, P, 0, P, P, P, 0)), (bad, (sel, P, 0, P, P, P, P)), (shape, (lay, P, 0, P, P, P + 8, P))):
        _refused(status, B.ps_block_summaries, *args)
    good = (lay, P, sel, P, P, P, P, P)
    for i, arg in enumerate(good):
        if i not in (0, 2):
            _refused(bad, B.ps_select_blocks, *good[:i], 0, *good[i + 1:])
    for status, args in ((bad, (sel, P, sel, P, P, P, P, P)), (bad, (lay, P, lay, P, P, P, P, P)), (shape, (lay, P, sel, P, P + 2, P, P, P)),
                         (shape, (lay, P, sel, P, P, P + 8, P, P)), (shape, (lay, P, sel, P, P, P, P, P + 4))):
        _refused(status, B.ps_select_blocks, *args)
    for fn, args in ((B.ps_kv_ingest, (sel, P, 0, P, P, 128, 64, P, P)), (B.ps_kv_append, (sel, P, P, P, P, P)), (B.ps_kv_stage_out, (sel, P, P, P, P)),
                     (B.ps_kv_stage_in, (sel, P, P, P, P)), (B.ps_layout_upload_append, (sel, P, P, P, P, P))):
        _refused(bad, fn, *args)
    B.ps_layout_append(pool, lay, 1)                      # the base has moved on: the selection has to follow first
    _refused(bad, B.ps_select_blocks, *good)
    odd = B.ps_kv_layout(pool, B.geometry(4, 2, 96, 16, "bf16", "bf16"), [40], [0], [0], [3])
    _refused(unsupported, B.ps_kv_append_rope, odd, P, rope(rot=32), rows(), P, P, 0)
    _refused(unsupported, B.ps_block_summaries, odd, P, 0, P, 0, P, P)
    for h in (odd, sel, lay):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_wrappers_check_tensors():
    import torch
    from paper_2602_12029_amd import runtime
    geo = B.geometry(4, 2, 64, 16, "bf16", "bf16")
    rope = runtime.Rope(np.ones(32), device="cpu")
    src, pos = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    for s, p, out in ((src.float(), pos, None), (src[:, :3], pos, None), (src.transpose(0, 2), pos, None), (src, pos.long(), None),
                      (src, pos[:4], None), (src, pos, torch.zeros(5, 4, 64)), (src, pos, torch.zeros(4, 5, 64, dtype=torch.bfloat16).transpose(0, 1))):
        with pytest.raises(ValueError):
            runtime.rope_rows(geo, rope, s, p, out)
    with pytest.raises(ValueError):
        runtime.Rope(np.ones(32), q_weight=torch.ones(128)[::2], device="cpu")
    b = runtime.DecodeBatch.__new__(runtime.DecodeBatch)
    b.geometry, b.num_requests, b.q, b.device = geo, 5, src, torch.device("cpu")
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for q, kk, v, p in ((src, k, k.float(), pos), (src, k[:4], k[:4], pos), (src.float(), k, k, pos), (src, k, torch.zeros(5, 3, 64, dtype=torch.bfloat16)[:, :2], pos),
                        (src, k, k, pos[::2])):
        with pytest.raises(ValueError):
            b._token_rows(q, kk, v, p)
    good = b._token_rows(src, k, k, pos)
    assert (good.q_stride_row, good.q_stride_head, good.kv_stride_row, good.kv_stride_head) == (256, 64, 128, 64)
    meta = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="meta")                   # tensors of another device
    for q, kk, v, p in ((src, meta, k, pos), (src, k, meta, pos), (torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="meta"), k, k, pos),
                        (src, k, k, torch.zeros(5, dtype=torch.int32, device="meta"))):
        with pytest.raises(ValueError):
            b._token_rows(q, kk, v, p)
    with pytest.raises(ValueError):                                                     # not on a GPU at all
        b.kv_append_rope(rope, src, k, k, pos)
    with pytest.raises(ValueError):
        runtime.rope_rows(geo, rope, src, pos)
    weights = runtime.Rope(np.ones(32), q_weight=torch.ones(64), k_weight=torch.ones(32, dtype=torch.bfloat16), device="cpu")
    for q_dtype, k_dtype in ((torch.bfloat16, None), (None, torch.bfloat16)):
        with pytest.raises(ValueError):
            weights.check(torch.device("cpu"), 64, q_dtype, k_dtype)
    weights.check(torch.device("cpu"), 64, torch.float32, None)
    with pytest.raises(ValueError):
        runtime.Rope(np.ones(32), q_weight=torch.ones(64, device="meta"), device="cpu")
    for codes, scales in ((torch.zeros(3, 2, 2, 64), torch.zeros(3, 2)), (torch.zeros(3, 2, 2, 64, dtype=torch.int8), torch.zeros(4, 2)),
                          (torch.zeros(3, 2, 64, 2, dtype=torch.int8).transpose(2, 3), torch.zeros(3, 2))):
        with pytest.raises(ValueError):
            b._check_summaries(codes, scales)
