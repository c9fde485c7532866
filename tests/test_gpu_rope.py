"""Norm and rotation of head rows on the GPU, alone and on the way into the cache, against the fp64 oracle and the plain cache writes.

Bars, per element and derived: the result is rounded once to its format (half a step: 2^-8 of the value for bf16, 2^-24 for float32)
after float32 arithmetic on the row.  That arithmetic: the norm's factor (a sum of d squares by a tree, a division, v_rsq: under
8 float32 roundings), two products, the cosine and sine (argument and series: under 4 roundings absolute) and the pair's two products
and sum: 32 roundings of 2^-24 of the pair's magnitude hold all of it; F32 = 2^-19.  e4m3: half a step is 2^-4 of the value, or
2^-10 of the scale below the normal range; the same float32 slack.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa
from oracle import fp8
from oracle import layout as ol
from oracle import rope as orope

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -19
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from gpu_helpers import GpuCase
    return GpuCase


def _tensor(x, dtype):
    from paper_2602_12029_amd.runtime import to_device
    return to_device(x if dtype == "f32" else wl.bf16_bits_from_f32(x), dtype)


def _values(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _rows(rng, tokens, heads, d, dtype, layout="dense"):
    """Rows [T, heads, d] on the device, of different magnitudes; "padded": with gaps between heads and tokens."""
    x = rng.standard_normal((tokens, heads, d)).astype(np.float32) * np.exp2(rng.uniform(-3, 3, (tokens, heads, 1))).astype(np.float32)
    t = _tensor(x, dtype)
    if layout == "padded":
        wide = torch.full((tokens, heads + 2, d + 16), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 1:1 + heads, 16:] = t
        return wide[:, 1:1 + heads, 16:]
    return t


def _rope(rng, rot, pairing, norm, d, dtype):
    from paper_2602_12029_amd.runtime import Rope
    rad = 500000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    qw, kw = [(_tensor((1 + 0.3 * rng.standard_normal(d)).astype(np.float32), dtype) if norm else None) for _ in range(2)]
    return Rope(rad, pairing, qw, kw, 1e-5), rad, qw, kw


def _oracle(x, pos, rad, pairing, weight):
    return orope.norm_rotate(_values(x), pos, rad, pairing, None if weight is None else _values(weight), 1e-5)


def _magnitude(x, weight):
    """Per element, what the float32 slack is relative to: the largest magnitude of its row before the rotation."""
    y = np.abs(orope.norm_rotate(_values(x), np.zeros(x.shape[0]), [], "halves", None if weight is None else _values(weight), 1e-5))
    return y.max(-1, keepdims=True)


def _check(got, ref, mag, dtype, label):
    off = np.abs(got - ref)
    bar = HALF_STEP[dtype] * np.abs(ref) + F32 * mag
    print(f"[{label}] worst {np.max(off / np.maximum(bar, 1e-300), initial=0.0):.3f} of the bar", flush=True)
    assert (off <= bar).all()


CASES = [  # dtype, heads, d, rot, pairing, norm, tokens, layout
    ("bf16", 32, 128, 128, "halves", True, 5, "dense"), ("bf16", 32, 128, 64, "neighbours", True, 130, "padded"),
    ("bf16", 7, 128, 128, "halves", False, 1, "padded"), ("bf16", 1, 64, 64, "halves", True, 33, "dense"),
    ("bf16", 28, 64, 16, "neighbours", False, 3, "dense"), ("bf16", 5, 256, 256, "halves", True, 9, "padded"),
    ("f32", 4, 64, 64, "neighbours", True, 17, "padded"), ("f32", 9, 128, 128, "halves", True, 65, "dense"),
    ("f32", 3, 256, 32, "halves", False, 2, "padded"), ("f32", 16, 128, 0, "halves", True, 7, "dense"),
    ("f32", 2, 256, 254, "neighbours", True, 4, "dense"), ("bf16", 64, 128, 32, "halves", True, 700, "dense"),
]


@pytest.mark.parametrize("dtype,heads,d,rot,pairing,norm,tokens,layout", CASES)
def test_rows(gpu, dtype, heads, d, rot, pairing, norm, tokens, layout):
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import rope_rows
    rng = np.random.default_rng(rot + d + tokens)
    rope, rad, qw, _ = _rope(rng, rot, pairing, norm, d, dtype)
    x = _rows(rng, tokens, heads, d, dtype, layout)
    pos = np.concatenate([[0, 2 ** 31 - 1, -1, 131072, 77][:tokens], rng.integers(0, 1 << 20, max(0, tokens - 5))]).astype(np.int32)
    geo = B.geometry(heads, 1, d, 16, dtype, "f32" if dtype == "f32" else "bf16")
    room = torch.full((tokens + 2, heads, d), float("nan"), dtype=x.dtype, device="cuda")
    got = rope_rows(geo, rope, x, torch.from_numpy(pos).cuda(), room[1:1 + tokens])
    torch.cuda.synchronize()
    _check(_values(got), _oracle(x, pos, rad, pairing, qw), _magnitude(x, qw), dtype, f"rows {dtype} {heads}x{d} rot {rot}")
    assert torch.isnan(room[0]).all() and torch.isnan(room[-1]).all()             # rows in front and behind are left alone
    if layout == "dense":                                                          # in place
        assert torch.equal(rope_rows(geo, rope, x, torch.from_numpy(pos).cuda(), x), got)


def test_no_rows(gpu):
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope, rope_rows
    geo = B.geometry(4, 2, 64, 16, "bf16", "bf16")
    got = rope_rows(geo, Rope(np.ones(32)), torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert got.shape == (0, 4, 64)


def test_rows_that_are_not_numbers_stay_their_own(gpu):
    """A row with NaN or infinities spoils itself alone."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import rope_rows
    rng = np.random.default_rng(3)
    rope, rad, qw, _ = _rope(rng, 128, "halves", True, 128, "bf16")
    x = _rows(rng, 6, 8, 128, "bf16")
    x[2, 3, 17], x[4, 0, 5] = float("nan"), float("inf")
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    got = rope_rows(B.geometry(8, 1, 128, 16, "bf16", "bf16"), rope, x, pos)
    ok = torch.ones(6, 8, dtype=torch.bool, device="cuda")
    ok[2, 3] = ok[4, 0] = False
    assert torch.isfinite(got[ok].float()).all() and torch.isnan(got[2, 3].float()).all() and torch.isnan(got[4, 0].float()).any()


def _workloads():
    bf, f8, f32 = (wl.Geometry(8, 2, 128, 16, "bf16", "bf16"), wl.Geometry(8, 2, 128, 16, "bf16", "fp8_e4m3"), wl.Geometry(4, 2, 64, 48, "f32", "f32"))
    member, pre, suf = [[0], [1, 2], [0, 1, 2], [2]], [1, 333, 1000, 16], [0, 5, 17, 77, 300, 1, 16]
    return [
        wl.make_workload("bf16", bf, 3, pre, member, suf, 1.6, seed=2), wl.make_workload("fp8", f8, 3, pre, member, suf, 1.6, seed=3),
        wl.make_workload("fp8_b64", wl.Geometry(28, 4, 128, 64, "bf16", "fp8_e4m3"), 3, pre, member, suf, 2.0, seed=4),
        wl.make_workload("fp8_b128", wl.Geometry(8, 1, 128, 128, "bf16", "fp8_e4m3"), 3, pre, member, suf, 2.0, seed=14),
        wl.make_workload("f32_b48", f32, 3, pre, member, suf, 2.0, seed=5), wl.make_workload("fp8_d64", wl.Geometry(8, 3 + 1, 64, 32, "bf16", "fp8_e4m3"), 3, pre, member, suf, 2.0, seed=6),
        wl.make_workload("bf16_d256", wl.Geometry(10, 5, 256, 16, "bf16", "bf16"), 3, pre, member, suf, 2.0, seed=7),
        wl.make_workload("fp8_d256", wl.Geometry(4, 2, 256, 32, "f32", "fp8_e4m3"), 3, pre, member, suf, 2.0, seed=8),
        wl.make_workload("f32_d128", wl.Geometry(4, 1, 128, 16, "bf16", "f32"), 3, pre, member, suf, 2.0, seed=9),
    ]


NAMES = [w.name for w in _workloads()]


def _poison(case):
    case.batch.kv.view(torch.uint8).fill_(0xff)
    if case.batch.scales is not None:
        case.batch.scales.fill_(float("nan"))


def _pool(case):
    """The device's pool in the dense axis order: stored values (e4m3: codes), scales."""
    bits = case.batch.kv.cpu()
    v = fp8.decode(bits.numpy()) if bits.dtype == torch.uint8 else bits.to(torch.float64).numpy()
    return v.transpose(np.argsort(case.pool_axes)), None if case.batch.scales is None else case.batch.scales.cpu().numpy()


def _bits(t):
    return t.view({2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()])


def _check_tile(values, scale, ref, mag, kv_dtype, label):
    """Stored rows [n, d] of one tile against exact ones; e4m3: values are codes, scale the tile's."""
    if kv_dtype != "fp8_e4m3":
        return _check_quiet(values, ref, HALF_STEP[kv_dtype] * np.abs(ref) + F32 * mag, label)
    top = np.abs(ref).max()
    want = top / 448 if top > 0 else 1.0
    assert abs(scale - want) <= want * F32 * 4 + F32 * mag.max() / 448, label
    step = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * scale)
    _check_quiet(values * scale, ref, step * (1 + F32) + F32 * mag, label)


def _check_quiet(got, ref, bar, label):
    assert np.isfinite(got).all() and (np.abs(got - ref) <= bar).all(), (label, np.max(np.abs(got - ref) / bar))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("pool_layout,layout,pairing", [("dense", "dense", "halves"), ("token_major", "padded", "neighbours"), ("planes", "padded", "halves")])
def test_ingest(gpu, name, pool_layout, layout, pairing):
    w = next(x for x in _workloads() if x.name == name)
    g = w.geometry
    rng = np.random.default_rng(w.seed)
    case = gpu(w, pool_layout=pool_layout)
    _poison(case)
    src = "f32" if g.kv_dtype == "f32" else "bf16"
    rot = g.head_dim if layout == "dense" else g.head_dim // 2
    rope, rad, _, kw = _rope(rng, rot, pairing, layout == "dense", g.head_dim, src)
    for which in (0, 1):
        lens = w.prefix_len if which == 0 else w.suffix_len
        n = int(lens.sum())
        kv = _rows(rng, n, 2 * g.num_kv_heads, g.head_dim, src, layout)
        k, v = kv[:, :g.num_kv_heads], kv[:, g.num_kv_heads:]
        pos = rng.integers(0, 300000, n).astype(np.int32)
        case.batch.kv_ingest_rope(which, rope, k, v, torch.from_numpy(pos).cuda())
        torch.cuda.synchronize()
        stored, scales = _pool(case)
        rows = (_oracle(k, pos, rad, pairing, kw), _values(v))
        mags = (_magnitude(k, kw), _magnitude(v, None))
        indptr, blk = (case.olay.prefix_blk_indptr, case.olay.prefix_blk) if which == 0 else (case.olay.suffix_blk_indptr, case.olay.suffix_blk)
        t0 = 0
        for s, length in enumerate(lens):
            for i, b in enumerate(blk[indptr[s]:indptr[s + 1]]):
                m = min(g.block_size, int(length) - i * g.block_size)
                at = slice(t0 + i * g.block_size, t0 + i * g.block_size + m)
                for h in range(g.num_kv_heads):
                    for kind in (0, 1):
                        _check_tile(stored[b, h, kind, :m], None if scales is None else scales[b, h, kind], rows[kind][at, h], mags[kind][at, h],
                                    g.kv_dtype, (name, which, int(b), h, kind))
                bits = _bits(case.batch.kv).cpu().numpy().transpose(np.argsort(case.pool_axes))
                assert (bits[b, :, :, m:] == bits.dtype.type(-1 if bits.dtype != np.uint8 else 255)).all()      # slots past the end: as they were
            t0 += int(length)
    case.close()


@pytest.mark.parametrize("name", NAMES)
def test_without_norm_and_rotation_the_plain_cache_writes(gpu, name):
    """rot_dim 0 and no weights, or position 0 without weights: the bits of kv_ingest and kv_append."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope
    w = next(x for x in _workloads() if x.name == name)
    g = w.geometry
    src = "f32" if g.kv_dtype == "f32" else "bf16"
    w.num_blocks += 8 * w.num_requests
    w.free_order = np.random.default_rng(1).permutation(w.num_blocks).astype(np.int32)
    plain, fused = gpu(w), gpu(w)
    for rope in (Rope([], "halves"), Rope(np.ones(16) / 3, "halves"), Rope(np.ones(3), "neighbours")):
        rng = np.random.default_rng(5)
        for case in (plain, fused):
            _poison(case)
        for which in (0, 1):
            n = B.ps_ingest_tokens(plain.layout, which)           # (the steps below grow the private segments)
            k, v = _rows(rng, n, g.num_kv_heads, g.head_dim, src), _rows(rng, n, g.num_kv_heads, g.head_dim, src)
            k[0], v[n // 2] = 0, 0
            plain.batch.kv_ingest(which, k, v)
            fused.batch.kv_ingest_rope(which, rope, k, v, torch.zeros(n, dtype=torch.int32, device="cuda"))
        for step in range(5):
            active = None if step == 0 else (rng.random(w.num_requests) < 0.6).astype(np.int32)
            k, v = (_rows(rng, w.num_requests, g.num_kv_heads, g.head_dim, src) for _ in range(2))
            plain.batch.append_step(plain.pool, k, v, active)
            B.ps_layout_append(fused.pool, fused.layout, w.num_requests, active)
            fused.batch._sync_plan()
            fused.batch.kv_append_rope(rope, None, k, v, torch.zeros(w.num_requests, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        used = np.concatenate([plain.olay.prefix_blk, B.ps_layout_tables(plain.layout, w.num_prompts, w.num_requests)["suffix_blk"]])
        assert torch.equal(_bits(plain.batch.kv), _bits(fused.batch.kv))
        if plain.batch.scales is not None:
            assert torch.equal(plain.batch.scales[used].view(torch.int32), fused.batch.scales[used].view(torch.int32))
    plain.close()
    fused.close()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("layout,pairing", [("dense", "halves"), ("padded", "neighbours")])
def test_append(gpu, name, layout, pairing):
    """Steps of appends with changing magnitudes and some requests inactive: queries and new tokens against the oracle; an e4m3
    tile's earlier tokens, re-encoded from their stored values, against those (half a step each time its scale grew)."""
    w = next(x for x in _workloads() if x.name == name)
    g = w.geometry
    src, steps = ("f32" if g.kv_dtype == "f32" else "bf16"), 20
    w.num_blocks += (steps // g.block_size + 1) * w.num_requests
    w.free_order = np.random.default_rng(1).permutation(w.num_blocks).astype(np.int32)
    rng = np.random.default_rng(w.seed + 50)
    case = gpu(w)
    qrope, rad, qw, _ = _rope(rng, g.head_dim, pairing, True, g.head_dim, g.q_dtype)
    kw = _tensor((1 + 0.3 * rng.standard_normal(g.head_dim)).astype(np.float32), src)
    from paper_2602_12029_amd.runtime import Rope
    rope = Rope(rad, pairing, qw, kw, 1e-5)
    from paper_2602_12029_amd import binding as B
    for step in range(steps):
        active = None if step % 4 == 0 else (rng.random(w.num_requests) < 0.7).astype(np.int32)
        dest = B.ps_layout_append(case.pool, case.layout, w.num_requests, active)
        assert np.array_equal(dest, ol.append_step(case.opool, case.olay, active))
        case.batch._sync_plan()
        q = _rows(rng, w.num_requests, g.num_q_heads, g.head_dim, g.q_dtype, layout)
        kv = _rows(rng, w.num_requests, 2 * g.num_kv_heads, g.head_dim, src, layout)
        k, v = kv[:, :g.num_kv_heads], kv[:, g.num_kv_heads:]
        pos = rng.integers(0, 200000, w.num_requests).astype(np.int32)
        before, old = _pool(case)
        case.batch.kv_append_rope(rope, q, k, v, torch.from_numpy(pos).cuda())
        torch.cuda.synchronize()
        _check(_values(case.batch.q), _oracle(q, pos, rad, pairing, qw), _magnitude(q, qw), g.q_dtype, f"{name} step {step} q")
        after, scales = _pool(case)
        rows = (_oracle(k, pos, rad, pairing, kw), _values(v))
        mags = (_magnitude(k, kw), _magnitude(v, None))
        touched = np.zeros(before.shape[0], bool)
        for r in np.nonzero(dest >= 0)[0]:
            b, slot = divmod(int(dest[r]), g.block_size)
            touched[b] = True
            for h in range(g.num_kv_heads):
                for kind in (0, 1):
                    ref, mag = rows[kind][r, h], mags[kind][r, h]
                    if g.kv_dtype != "fp8_e4m3":
                        _check_tile(after[b, h, kind, slot], None, ref, mag, g.kv_dtype, (name, step, r, h, kind))
                        continue
                    s, need = float(scales[b, h, kind]), np.abs(ref).max() / 448
                    want = max(need, float(old[b, h, kind])) if slot else need
                    assert abs(s - want) <= F32 * (want + mag.max() / 448)
                    step_of = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * s)
                    _check_quiet(after[b, h, kind, slot] * s, ref, step_of * (1 + F32) + F32 * mag, (name, step, r, h, kind))
                    held = before[b, h, kind, :slot] * float(old[b, h, kind]) if slot else np.zeros((0, g.head_dim))
                    _check_quiet(after[b, h, kind, :slot] * s, held, np.maximum(2.0 ** -4 * np.abs(held), 2.0 ** -10 * s) * (1 + F32), (name, step, r, "stored"))
        bits = np.isnan(before[~touched])
        assert np.array_equal(np.where(bits, 0, before[~touched]), np.where(bits, 0, after[~touched]))
    case.close()


def test_adopted_blocks_are_left_alone(gpu):
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import DecodeBatch, Rope
    geo = B.geometry(4, 2, 128, 16, "bf16", "fp8_e4m3")
    pool = B.ps_pool_create(32)
    first = B.ps_kv_layout(pool, geo, [50], [0], [0], [0])
    ids = B.ps_layout_tables(first, 1, 1)["prefix_blk"][:3]
    more = B.ps_kv_layout_adopt(pool, geo, [90], [ids], [0], [0], [0])
    q = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")
    kv = torch.full((32, 2, 2, 16, 128), 0xff, dtype=torch.uint8, device="cuda")
    scales = torch.full((32, 2, 2), float("nan"), device="cuda")
    batch = DecodeBatch(more, geo, 1, q, kv, scales)
    rng = np.random.default_rng(0)
    n = 90 - 48
    k, v = _rows(rng, n, 2, 128, "bf16"), _rows(rng, n, 2, 128, "bf16")
    pos = torch.arange(48, 90, dtype=torch.int32, device="cuda")
    batch.kv_ingest_rope(0, Rope(np.ones(64) / 7), k, v, pos)
    torch.cuda.synchronize()
    assert (kv[torch.from_numpy(ids).long().cuda()] == 0xff).all() and torch.isnan(scales[torch.from_numpy(ids).long().cuda()]).all()
    dst = torch.full((2, n + 1, 2, 128), 7.0, device="cuda")
    batch.kv_gather(0, dst[0, :n], dst[1, :n])
    ref = orope.norm_rotate(_values(k), np.arange(48, 90), np.ones(64) / 7, "halves")
    for got, want in ((dst[0, :n], ref), (dst[1, :n], _values(v))):
        for i in range(0, n, 16):
            for h in range(2):
                r = want[i:i + 16, h]
                s = np.abs(r).max() / 448
                assert (np.abs(_values(got)[i:i + 16, h] - r) <= np.maximum(2.0 ** -4 * np.abs(r), 2.0 ** -10 * s) * (1 + F32) + F32 * np.abs(r).max()).all()
    assert (dst[:, n:] == 7).all()
    torch.cuda.synchronize()
    for h in (more, first):
        B.ps_layout_release(pool, h)
    B.ps_pool_destroy(pool)


def test_a_captured_step_replays(gpu):
    """Rotation and cache write recorded into a graph: replays with other tokens and positions, the program's own work in between."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope
    w = wl.make_workload("captured", wl.Geometry(8, 2, 128, 16, "bf16", "fp8_e4m3"), 2, [40, 7], [[0, 1], [0]], [3, 16, 0], 3.0, seed=3)
    eager, replayed = gpu(w), gpu(w)
    rng = np.random.default_rng(2)
    rope = Rope(np.ones(64) / 9)
    q, kv = _rows(rng, 3, 8, 128, "bf16"), _rows(rng, 3, 4, 128, "bf16")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for case in (eager, replayed):
        B.ps_layout_append(case.pool, case.layout, 3)
        case.batch._sync_plan()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        replayed.batch.kv_append_rope(rope, q, kv[:, :2], kv[:, 2:], pos)
    for step in range(4):
        q.copy_(_rows(rng, 3, 8, 128, "bf16"))
        kv.copy_(_rows(rng, 3, 4, 128, "bf16"))
        pos.fill_(1000 * step + 5)
        torch.cuda.synchronize()
        graph.replay()
        eager.batch.kv_append_rope(rope, q, kv[:, :2], kv[:, 2:], pos)
        torch.cuda.synchronize()
        assert torch.equal(eager.batch.q.view(torch.int16), replayed.batch.q.view(torch.int16))
        assert torch.equal(eager.batch.kv, replayed.batch.kv)
        assert torch.equal(eager.batch.scales.view(torch.int32), replayed.batch.scales.view(torch.int32))
    eager.close()
    replayed.close()


@pytest.mark.parametrize("magnitude", [2.0 ** -130, 2.0 ** -120, 2.0 ** -95, 2.0 ** -82, 1.0, 2.0 ** 90, 2.0 ** 126])
def test_tiles_of_extreme_magnitude(gpu, magnitude):
    """e4m3 tiles whose scale is subnormal, tiny or huge, zeros of both signs among them: the bits of the oracle's quantiser, by the plain
    ingest and by the fused one."""
    from oracle import kv_update as ku
    from paper_2602_12029_amd.runtime import Rope
    w = wl.make_workload("extreme", wl.Geometry(4, 2, 128, 16, "bf16", "fp8_e4m3"), 1, [70], [[0]], [0], seed=3)
    case = gpu(w)
    rng = np.random.default_rng(4)
    src = []
    for _ in range(2):
        x = rng.uniform(-1, 1, (70, 2, 128)) * np.exp2(-rng.integers(0, 16, (70, 2, 128)).astype(float))
        x[rng.random(x.shape) < 0.05] = 0.0
        x[rng.random(x.shape) < 0.05] = -0.0
        src.append(wl.bf16_bits_from_f32((x * magnitude).astype(np.float32)))
    from paper_2602_12029_amd.runtime import to_device
    k, v = (to_device(s, "bf16") for s in src)
    _poison(case)
    case.data.kv[...] = 0xff
    case.data.scales[...] = np.nan
    ku.ingest_segment(case.data.kv, case.data.scales, "fp8_e4m3", case.olay.prefix_blk, *src)
    for fused in (False, True):
        _poison(case)
        if fused:
            case.batch.kv_ingest_rope(0, Rope([]), k, v, torch.zeros(70, dtype=torch.int32, device="cuda"))
        else:
            case.batch.kv_ingest(0, k, v)
        torch.cuda.synchronize()
        ids = case.olay.prefix_blk
        assert np.array_equal(case.batch.scales.cpu().numpy()[ids].view(np.int32), case.data.scales[ids].view(np.int32)), fused
        assert np.array_equal(case.batch.kv.cpu().numpy(), case.data.kv), fused
    case.close()


@pytest.mark.parametrize("d,block", [(64, 256), (128, 128), (256, 64)])
def test_the_largest_e4m3_tiles(gpu, d, block):
    """As many tokens' angles at once as the ingest ever holds, all of their pairs turned."""
    w = wl.make_workload("large", wl.Geometry(4, 2, d, block, "bf16", "fp8_e4m3"), 1, [2 * block + 9], [[0]], [0], 1.0, seed=3)
    case = gpu(w)
    rng = np.random.default_rng(8)
    n = 2 * block + 9
    rope, rad, _, kw = _rope(rng, d, "halves", True, d, "bf16")
    pos = np.arange(n, dtype=np.int32) + 100000
    k, v = (torch.from_numpy(rng.standard_normal((n, 2, d)).astype(np.float32)).to(torch.bfloat16).cuda() for _ in range(2))
    _poison(case)
    case.batch.kv_ingest_rope(0, rope, k, v, torch.from_numpy(pos).cuda())
    torch.cuda.synchronize()
    values, scales = _pool(case)
    ref, mag = _oracle(k, pos, rad, "halves", kw), _magnitude(k, kw)
    for i, b in enumerate(case.olay.prefix_blk):
        m = min(block, n - i * block)
        for h in range(2):
            _check_tile(values[b, h, 0, :m], scales[b, h, 0], ref[i * block:i * block + m, h], mag[i * block:i * block + m, h], "fp8_e4m3", f"{b} {h}")
    case.close()


@pytest.mark.parametrize("heads", [8, 3, 1])
@pytest.mark.parametrize("blocks", [5, 300, 500, 800, 1300])
def test_however_many_blocks(gpu, heads, blocks):
    """A block's tiles in one workgroup or shared out over several: bf16 keys as the rows alone come out, e4m3 tiles as by the plain ingest."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope, rope_rows
    n = 16 * blocks - 7
    gen = torch.Generator(device="cuda").manual_seed(blocks + heads)
    k, v = (torch.randn((n, heads, 128), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    for dtype in ("bf16", "fp8_e4m3"):
        w = wl.make_workload("many", wl.Geometry(heads, heads, 128, 16, "bf16", dtype), 1, [n], [[0]], [0], 1.0, seed=1)
        case = gpu(w)
        _poison(case)
        if dtype == "bf16":
            rope = Rope(500000.0 ** (-np.arange(64) / 64), q_weight=v[0, 0].contiguous(), k_weight=v[0, 0].contiguous())
            case.batch.kv_ingest_rope(0, rope, k, v, pos)
            back = torch.empty((2, n, heads, 128), dtype=torch.bfloat16, device="cuda")
            case.batch.kv_gather(0, back[0], back[1])
            rows = rope_rows(B.geometry(heads, heads, 128, 16, "bf16", "bf16"), rope, k, pos)
            torch.cuda.synchronize()
            assert torch.equal(_bits(back[0]), _bits(rows)) and torch.equal(_bits(back[1]), _bits(v))
        else:
            case.batch.kv_ingest_rope(0, Rope([]), k, v, pos)
            torch.cuda.synchronize()
            got, scales = case.batch.kv.clone(), case.batch.scales.clone()
            _poison(case)
            case.batch.kv_ingest(0, k, v)
            torch.cuda.synchronize()
            assert torch.equal(got, case.batch.kv) and torch.equal(_bits(scales), _bits(case.batch.scales))
        case.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 256)])
def test_rows_whose_squares_are_subnormal(gpu, dtype, d):
    """Without an eps, magnitudes of 2^-65 to 2^-64: squares of 2^-130 and more, on a grid of 2^-149, are off by 2^-20 of themselves, as is
    their mean, its root by half of each: 2^-20, which the few roundings of the rest leave room for in F32."""
    from paper_2602_12029_amd import binding as B
    from paper_2602_12029_amd.runtime import Rope, rope_rows
    rng = np.random.default_rng(d)
    x = _tensor((rng.choice([-1.0, 1.0], (9, 4, d)) * rng.uniform(1, 2, (9, 4, d)) * 2.0 ** -65).astype(np.float32), dtype)
    weight = _tensor((1 + 0.3 * rng.standard_normal(d)).astype(np.float32), dtype)
    got = rope_rows(B.geometry(4, 1, d, 16, dtype, "f32" if dtype == "f32" else "bf16"), Rope([], "halves", weight, None, 0.0), x,
                    torch.zeros(9, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    ref = orope.norm_rotate(_values(x), np.zeros(9), [], "halves", _values(weight), 0.0)
    _check(_values(got), ref, np.abs(ref).max(-1, keepdims=True), dtype, f"subnormal squares {dtype} {d}")
