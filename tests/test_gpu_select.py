"""Block summaries, block selection and the step over the selected blocks on the GPU, against the oracle.

Summaries and lists are defined bit for bit and compared so; the attention over them keeps the bars of the attention tests.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from helpers import errors
from oracle import attention as oa
from oracle import layout as ol
from oracle import select as osel

pytestmark = pytest.mark.gpu

TOL = {"f32": (1e-5, 1e-5), "bf16": (1e-2, 5e-3), "fp8_e4m3": (1e-2, 5e-3)}   # as in gpu_helpers: max-abs, relative RMS
GEO = {
    "bf16": (8, 2, 128, 16, "bf16", "bf16"), "fp8": (32, 4, 128, 16, "bf16", "fp8_e4m3"), "fp8_b64": (28, 4, 128, 64, "bf16", "fp8_e4m3"),
    "f32_d64": (4, 2, 64, 16, "f32", "f32"), "bf16_d256": (16, 4, 256, 32, "bf16", "bf16"), "mha": (3, 3, 128, 16, "bf16", "bf16"),
    "wide_group": (40, 2, 128, 16, "bf16", "bf16"), "b48": (12, 1, 128, 48, "f32", "f32"), "mixed_types": (4, 2, 128, 16, "f32", "fp8_e4m3"),
    "pair": (4, 2, 64, 32, "bf16", "bf16"), "group64": (64, 1, 64, 16, "bf16", "bf16"),
}


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from gpu_helpers import GpuCase
    return GpuCase


def _workload(name, seed=1, tree=False):
    geo = wl.Geometry(*GEO[name])
    member = [[0], [1, 2], [0, 1, 2, 3], [2]]
    pre, suf = [5, 700, 333, 1041], [0, 5, 17, 77, 130, 1, 16, 33]
    if tree:
        return wl.make_tree_workload(name, geo, 4, [215, 64], [0, 1, 0, -1], pre, member, suf, 1.4, seed)
    return wl.make_workload(name, geo, 4, pre, member, suf, 1.4, seed)


def _summary_tensors(w):
    g = w.geometry
    return (torch.full((w.num_blocks, g.num_kv_heads, 2, g.head_dim), 77, dtype=torch.int8, device="cuda"),
            torch.full((w.num_blocks, g.num_kv_heads), -3.0, device="cuda"))


def _segments(w, lay):
    yield from ((lay.prefix_blk[lay.prefix_blk_indptr[p]:lay.prefix_blk_indptr[p + 1]], int(w.prefix_len[p])) for p in range(w.num_prompts))
    yield from ((lay.root_blk[lay.root_blk_indptr[t]:lay.root_blk_indptr[t + 1]], int(w.root_len[t])) for t in range(w.num_roots))


def _oracle_summaries(case):
    w, g = case.w, case.w.geometry
    codes = np.full((w.num_blocks, g.num_kv_heads, 2, g.head_dim), 77, np.int8)
    scales = np.full((w.num_blocks, g.num_kv_heads), -3.0, np.float32)
    for ids, n in _segments(w, case.olay):
        for i, b in enumerate(ids):
            codes[b], scales[b] = osel.summarise(case.data.kv, case.data.scales, g.kv_dtype, b, min(g.block_size, n - i * g.block_size))
    return codes, scales


def _summarise(case):
    codes, scales = _summary_tensors(case.w)
    case.batch.block_summaries(0, codes, scales)
    if case.w.num_roots:
        case.batch.block_summaries(2, codes, scales)
    torch.cuda.synchronize()
    want, want_scales = _oracle_summaries(case)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy().view(np.int32), want_scales.view(np.int32))
    return codes, scales, want, want_scales


def _q32(case):
    return oa.widen(case.q_bits, case.w.geometry.q_dtype).astype(np.float32)


def _check_lists(sel, chosen, label):
    torch.cuda.synchronize()
    lists, indptr = sel.lists().cpu().numpy(), sel.list_indptr()
    for r, rows in enumerate(chosen):
        for h, (_, ids) in enumerate(rows):
            assert lists[h, indptr[r]:indptr[r + 1]].tolist() == ids, (label, r, h)


def _check_step(case, sel, chosen, label, visible=None):
    w, g = case.w, case.w.geometry
    sel.workspace.view(torch.float32).fill_(float("nan"))
    sel.out.fill_(float("nan"))
    sel.decode_attention()
    torch.cuda.synchronize()
    ref, ref_lse = osel.attend(case.q_bits, g.q_dtype, case.data.kv, case.data.scales, g.kv_dtype, case.olay, chosen, g.block_size, visible)
    got, lse = sel.out.cpu().to(torch.float64).numpy(), sel.lse.cpu().numpy()
    max_abs, rel, _ = errors(got, ref)
    print(f"[{label}] max_abs={max_abs:.3e} rel_rms={rel:.3e}", flush=True)
    tol_abs, tol_rel = TOL[g.kv_dtype]
    # (rows that see a handful of tokens reach |O| of 2 to 4: there the bar is relative, as half a step of bf16 alone is 2^-8 of the value)
    assert (np.abs(got - ref) <= tol_abs * np.maximum(1.0, np.abs(ref))).all() and rel <= tol_rel
    finite = np.isfinite(ref_lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse))
    assert np.abs(lse[finite] - ref_lse[finite]).max(initial=0.0) <= (1e-4 if g.kv_dtype == "f32" else 2e-3)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("name", list(GEO))
def test_selected_step(gpu, name, tree):
    w = _workload(name, tree=tree)
    case = gpu(w)
    g = w.geometry
    codes, scales, hcodes, hscales = _summarise(case)
    for blocks, first, last in ((6, 1, 2), (4, 0, 1), (3, 1, 1), (1000, 1, 1)):
        sel = case.batch.select(blocks, first, last)
        sel.decode_attention()                           # before the first choice the lists name blocks of the context
        torch.cuda.synchronize()
        assert torch.isfinite(sel.out.float()).all()
        sel.scratch.fill_(0xff)
        sel.select_blocks(codes, scales)
        chosen = osel.select(_q32(case), case.olay, g.block_size, hcodes, hscales, g.num_kv_heads, blocks, first, last)
        _check_lists(sel, chosen, f"{name} {blocks}")
        _check_step(case, sel, chosen, f"{name} tree={tree} blocks={blocks}")
        from paper_2602_12029_amd import binding as B
        torch.cuda.synchronize()
        B.ps_layout_release(case.pool, sel.layout)
    case.close()


@pytest.mark.parametrize("pool_layout", ["token_major", "planes"])
def test_summaries_of_other_pool_layouts(gpu, pool_layout):
    for name in ("bf16", "fp8_b64", "b48"):
        case = gpu(_workload(name), pool_layout=pool_layout)
        _summarise(case)
        case.close()


def test_summaries_of_odd_keys(gpu):
    """Zeros, denormals, infinities, NaN (all of a channel, some of it), the largest numbers, -0."""
    for name in ("bf16", "f32_d64", "fp8"):
        w = _workload(name)
        case = gpu(w)
        g = w.geometry
        b = case.olay.prefix_blk
        kv = case.data.kv
        if g.kv_dtype == "fp8_e4m3":
            kv[b[3], 0, 0, :, 5] = 0x7f                  # NaN
            kv[b[4], 0, 0, 2:9, 6] = 0xff
            kv[b[5], 1, 0] = 0
            kv[b[6], 1, 0] = 0x80
            kv[b[7], 0, 0] = np.resize([0x01, 0x81, 0x7e, 0xfe], kv[b[7], 0, 0].shape)
        else:
            odd = np.array([np.nan, np.inf, -np.inf, 3.3e38, -3.3e38, 1e-40, -1e-44, 0.0, -0.0, 1.0], np.float32)
            odd = odd if g.kv_dtype == "f32" else (odd.view(np.uint32) >> 16).astype(np.uint16)
            kv[b[3], 0, 0, :, 5] = odd[0]
            kv[b[4], 0, 0, 2:9, 6] = odd[0]
            kv[b[5], 1, 0] = odd[7]
            kv[b[6], 1, 0] = np.resize(odd[5:9], kv[b[6], 1, 0].shape)      # scale under the smallest normal number
            kv[b[7], 0, 0] = np.resize(odd, kv[b[7], 0, 0].shape)
            kv[b[8], 0, 0, 1] = odd[1]
        case.batch.kv.copy_(torch.from_numpy(kv.view({4: np.float32, 2: np.int16, 1: np.uint8}[kv.itemsize])).view(case.batch.kv.dtype))
        _summarise(case)
        case.close()


def test_equal_scores_and_odd_queries(gpu):
    """Queries of zeros (all scores equal), NaN, infinities and the largest numbers; summaries that are all the same."""
    w = _workload("bf16")
    case = gpu(w)
    g = w.geometry
    codes, scales, hcodes, hscales = _summarise(case)
    q = _q32(case).copy()
    q[0], q[1, :, 3], q[2, 1], q[3], q[4, 0, 0], q[5] = 0, np.nan, np.inf, 3e38, -np.inf, -q[5]
    case.q_bits = wl.bf16_bits_from_f32(np.nan_to_num(q, nan=0.0, posinf=0.0, neginf=0.0))
    odd = torch.from_numpy(q).to(torch.bfloat16)
    q = odd.to(torch.float32).numpy()
    case.batch.q.copy_(odd)
    sel = case.batch.select(5, 1, 1)
    sel.select_blocks(codes, scales)
    _check_lists(sel, osel.select(q, case.olay, 16, hcodes, hscales, 2, 5, 1, 1), "odd queries")
    for value, scale in ((0, 1.0), (100, 0.5), (-100, 2.0 ** 120), (127, 3e38)):
        codes.fill_(value)
        scales.fill_(scale)
        sel.select_blocks(codes, scales)
        same = np.full_like(hcodes, value)
        _check_lists(sel, osel.select(q, case.olay, 16, same, np.full_like(hscales, scale), 2, 5, 1, 1), f"summaries of {value}")
    case.close()


def test_scales_that_are_no_numbers(gpu):
    """Blocks that nobody has summarised: their scales may be anything, and the choice ends all the same, such blocks last."""
    w = _workload("fp8")
    case = gpu(w)
    codes, scales, hcodes, hscales = _summarise(case)
    rng = np.random.default_rng(2)
    hcodes, hscales = rng.integers(1, 128, hcodes.shape).astype(np.int8), hscales.copy()   # (no product of 0 with an infinite scale)
    codes.copy_(torch.from_numpy(hcodes))
    sel = case.batch.select(9, 1, 2)
    for share in (0.3, 0.97, 1.0):
        odd = rng.random(hscales.shape) < share
        values = np.where(odd, rng.choice(np.array([np.nan, -np.nan, np.inf, -np.inf], np.float32), hscales.shape), hscales).astype(np.float32)
        scales.copy_(torch.from_numpy(values))
        sel.select_blocks(codes, scales)
        with np.errstate(invalid="ignore"):
            _check_lists(sel, osel.select(_q32(case), case.olay, 16, hcodes, values, 4, 9, 1, 2), f"odd scales {share}")
    case.close()


@pytest.mark.parametrize("blocks_of", [900, 1500, 2049, 3001, 5000, 8192, 8193, 16384, 16385, 20011])
def test_long_contexts(gpu, blocks_of):
    """Every size of the choice kernel, scores with many equal ones and wide ranges; the lists alone."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import DecodeBatch
    rng = np.random.default_rng(blocks_of)
    geo = B.geometry(6, 2, 64, 16, "bf16", "bf16")
    lens, req, model = [blocks_of * 16 - 5, 300], [0, 0, 1], [0, 1, 0]
    total = blocks_of + 19
    order = rng.permutation(total).astype(np.int32)
    pool = B.ps_pool_create(total, order)
    lay = B.ps_kv_layout(pool, geo, lens, req, model, [0, 0, 0])
    q = torch.from_numpy(rng.standard_normal((3, 6, 64)).astype(np.float32)).to(torch.bfloat16)
    batch = DecodeBatch(lay, geo, 3, q.cuda(), q.cuda())
    codes = rng.integers(-127, 128, (total, 2, 2, 64)).astype(np.int8)
    scales = np.exp2(rng.uniform(-20, 20, (total, 2))).astype(np.float32)
    codes[order[:blocks_of // 2]] = codes[order[0]]                 # half of them the same
    scales[order[:blocks_of // 3]] = scales[order[0]]
    tables = [order[:blocks_of], order[blocks_of:]]
    dc, ds = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    for blocks in (3, 64, blocks_of // 2 + 7, blocks_of - 1):
        sel = batch.select(blocks, 1, 2)
        sel.scratch.fill_(0xff)
        sel.select_blocks(dc, ds)
        torch.cuda.synchronize()
        lists, ip = sel.lists().cpu().numpy(), sel.list_indptr()
        for r in range(3):
            ids = tables[req[r]]
            sc = osel.scores(q[r].to(torch.float32).numpy(), codes[ids], scales[ids], 2)
            for h in range(2):
                want = ids[osel.choose(sc[h], len(ids), -1, blocks, 1, 2)]
                assert np.array_equal(lists[h, ip[r]:ip[r + 1]], want), (blocks, r, h)
        B.ps_layout_release(pool, sel.layout)
    B.ps_layout_release(pool, lay)
    B.ps_pool_destroy(pool)


def test_visible_contexts(gpu):
    """Rows of a partial prefill, each with its own view of the context (none of it, too), and many of them."""
    geo = wl.Geometry(8, 2, 128, 16, "bf16", "bf16")
    w, visible = wl.chunk_prefill_workload("chunk", geo, [400, 7], [45, 30], 1.3, 5)
    visible[3], visible[4], visible[-1] = 0, 1, 37
    case = gpu(w)
    case.set_visible(visible)
    codes, scales, hcodes, hscales = _summarise(case)
    sel = case.batch.select(7, 1, 2)
    sel.select_blocks(codes, scales)
    chosen = osel.select(_q32(case), case.olay, 16, hcodes, hscales, 2, 7, 1, 2, visible)
    _check_lists(sel, chosen, "visible")
    _check_step(case, sel, chosen, "visible", visible)
    case.set_visible(None)
    with pytest.raises(Exception):                                  # the base has changed: follow first
        sel.select_blocks(codes, scales)
    sel.follow()
    sel.select_blocks(codes, scales)
    _check_lists(sel, osel.select(_q32(case), case.olay, 16, hcodes, hscales, 2, 7, 1, 2), "all visible")
    case.close()


def test_serving_loop(gpu):
    """A cache handed over as raw projections, summaries, then steps: append with rotation, follow, select, attend, read back."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope
    for name in ("bf16", "fp8", "f32_d64"):
        w = _workload(name)
        g = w.geometry
        w.num_blocks += 3 * w.num_requests
        w.free_order = np.random.default_rng(1).permutation(w.num_blocks).astype(np.int32)
        case = gpu(w)
        dtype = torch.float32 if g.kv_dtype == "f32" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(3)

        def rows(n, heads):
            return torch.randn((n, heads, g.head_dim), device="cuda", generator=gen).to(dtype)

        rope = Rope(10000.0 ** (-np.arange(0, g.head_dim, 2) / g.head_dim), "halves", rows(1, 1)[0, 0].contiguous(), rows(1, 1)[0, 0].contiguous())
        for which, lens, base in ((0, w.prefix_len, np.zeros(w.num_prompts, int)), (1, w.suffix_len, w.prefix_len[w.req_prompt])):
            pos = np.concatenate([b + np.arange(n) for b, n in zip(base, lens)]).astype(np.int32)
            case.batch.kv_ingest_rope(which, rope, rows(len(pos), g.num_kv_heads), rows(len(pos), g.num_kv_heads), torch.from_numpy(pos).cuda())
        codes, scales = _summary_tensors(w)
        case.batch.block_summaries(0, codes, scales)
        sel = case.batch.select(6, 1, 2)
        positions = torch.from_numpy((w.prefix_len[w.req_prompt] + w.suffix_len).astype(np.int32)).cuda()
        for step in range(20):
            active = None if step % 5 == 0 else (np.arange(w.num_requests) % 3 != step % 3).astype(np.int32)
            B.ps_layout_append(case.pool, case.layout, w.num_requests, active)
            ol.append_step(case.opool, case.olay, active)
            case.batch._sync_plan(wait=False)
            case.batch.kv_append_rope(rope, rows(w.num_requests, g.num_q_heads), rows(w.num_requests, g.num_kv_heads), rows(w.num_requests, g.num_kv_heads), positions)
            positions += 1 if active is None else torch.from_numpy(active).cuda()
            sel.follow()
            sel.select_blocks(codes, scales)
            sel.decode_attention()
            if step % 6:
                continue
            torch.cuda.synchronize()
            kv = case.batch.kv.cpu()                                # what the device holds: attended to as it is
            case.data.kv[...] = kv.numpy() if kv.dtype != torch.bfloat16 else kv.view(torch.int16).numpy().view(np.uint16)
            if case.data.scales is not None:
                case.data.scales[...] = case.batch.scales.cpu().numpy()
            q = case.batch.q.cpu()
            case.q_bits = q.numpy() if q.dtype != torch.bfloat16 else q.view(torch.int16).numpy().view(np.uint16)
            hcodes, hscales = _oracle_summaries(case)
            chosen = osel.select(_q32(case), case.olay, g.block_size, hcodes, hscales, g.num_kv_heads, 6, 1, 2)
            _check_lists(sel, chosen, f"{name} step {step}")
            _check_step(case, sel, chosen, f"{name} step {step}")
        n = B.ps_ingest_tokens(case.layout, 1)
        back = torch.empty((2, n, g.num_kv_heads, g.head_dim), dtype=torch.float32, device="cuda")
        case.batch.kv_gather(1, back[0], back[1])
        torch.cuda.synchronize()
        at = 0
        for r in range(w.num_requests):
            m = int(case.olay.suffix_len[r])
            k, v = oa.gather_segment(case.batch.kv.cpu().numpy() if g.kv_dtype != "bf16" else case.batch.kv.cpu().view(torch.int16).numpy().view(np.uint16),
                                     None if case.batch.scales is None else case.batch.scales.cpu().numpy(), g.kv_dtype,
                                     case.olay.suffix_blk[case.olay.suffix_blk_indptr[r]:case.olay.suffix_blk_indptr[r + 1]], m)
            assert np.array_equal(back[0, at:at + m].cpu().numpy(), k.astype(np.float32)) and np.array_equal(back[1, at:at + m].cpu().numpy(), v.astype(np.float32))
            at += m
        B.ps_layout_release(case.pool, sel.layout)
        case.close()


def test_captured_selection_replays(gpu):
    """Selection and attention recorded once, replayed with other queries, eager work of the program in between."""
    w = _workload("fp8")
    case = gpu(w)
    codes, scales, _, _ = _summarise(case)
    sel, eager = case.batch.select(6, 1, 2), case.batch.select(6, 1, 2)
    sel.select_blocks(codes, scales)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sel.select_blocks(codes, scales)
        sel.decode_attention()
    for step in range(4):
        case.batch.q.copy_(torch.randn(case.batch.q.shape, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        eager.select_blocks(codes, scales)
        eager.decode_attention()
        torch.cuda.synchronize()
        assert torch.equal(sel.lists(), eager.lists()) and torch.equal(sel.out.view(torch.int16), eager.out.view(torch.int16))
    case.close()


def test_another_stream(gpu):
    """Everything on a stream that is not the one the tables were uploaded on, behind a follow that does not wait on the host."""
    from paper_2602_12029_amd import binding as B
    w = _workload("bf16")
    w.num_blocks += w.num_requests
    w.free_order = np.random.default_rng(1).permutation(w.num_blocks).astype(np.int32)
    case = gpu(w)
    codes, scales, hcodes, hscales = _summarise(case)
    sel = case.batch.select(6, 1, 2)
    token = torch.zeros((w.num_requests, 2, 128), dtype=torch.bfloat16, device="cuda")
    case.batch.append_step(case.pool, token, token)
    ol.append_step(case.opool, case.olay)
    sel.follow()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sel.select_blocks(codes, scales)
        sel.decode_attention()
    torch.cuda.synchronize()
    case.data.kv[...] = case.batch.kv.cpu().view(torch.int16).numpy().view(np.uint16)
    chosen = osel.select(_q32(case), case.olay, 16, hcodes, hscales, 2, 6, 1, 2)
    _check_lists(sel, chosen, "another stream")
    _check_step(case, sel, chosen, "another stream")
    assert B.ps_layout_state(sel.layout) == (0, False)
    case.close()


def test_adopted_blocks_have_their_summaries_already(gpu):
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import DecodeBatch
    geo = B.geometry(4, 2, 128, 16, "bf16", "bf16")
    pool = B.ps_pool_create(32)
    first = B.ps_kv_layout(pool, geo, [50], [0], [0], [0])
    ids = B.ps_layout_tables(first, 1, 1)["prefix_blk"][:3]
    more = B.ps_kv_layout_adopt(pool, geo, [90], [ids], [0], [0], [0])
    q, kv = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.randn(32, 2, 2, 16, 128, device="cuda").bfloat16()
    codes, scales = torch.full((32, 2, 2, 128), 5, dtype=torch.int8, device="cuda"), torch.full((32, 2), 9.0, device="cuda")
    DecodeBatch(more, geo, 1, q, kv).block_summaries(0, codes, scales)
    torch.cuda.synchronize()
    written = (scales != 9.0).all(1).cpu().numpy()
    assert set(np.nonzero(written)[0]) == set(B.ps_layout_tables(more, 1, 1)["prefix_blk"][3:].tolist())
    assert (codes[torch.from_numpy(~written).cuda()] == 5).all()
    for h in (more, first):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)
