"""Reading stored segments back into contiguous tensors: bit for bit what the pool stands for, float32 product and one rounding."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa
from oracle import fp8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from gpu_helpers import GpuCase
    return GpuCase


def _workloads():
    member, pre, suf = [[0], [1, 2], [0, 1, 2], [2]], [1, 333, 1000, 16], [0, 5, 17, 77, 300, 1, 16]
    geos = [("bf16", (8, 2, 128, 16, "bf16", "bf16")), ("fp8", (8, 2, 128, 16, "bf16", "fp8_e4m3")), ("fp8_b64", (6, 3, 128, 64, "bf16", "fp8_e4m3")),
            ("f32", (4, 2, 64, 48, "f32", "f32")), ("fp8_d256", (4, 1, 256, 32, "bf16", "fp8_e4m3")), ("bf16_d96", (4, 2, 96, 16, "bf16", "bf16")),
            ("fp8_d80", (4, 2, 80, 16, "bf16", "fp8_e4m3"))]
    return {n: wl.make_workload(n, wl.Geometry(*g), 3, pre, member, suf, 1.6, seed=3) for n, g in geos}


def _expected(case, which, dst):
    """Stored values as the destination's bits: numpy float32 product, rounded once."""
    w, g, lay = case.w, case.w.geometry, case.olay
    lens, indptr, blk = (w.prefix_len, lay.prefix_blk_indptr, lay.prefix_blk) if which == 0 else \
        (w.suffix_len, lay.suffix_blk_indptr, lay.suffix_blk) if which == 1 else (w.root_len, lay.root_blk_indptr, lay.root_blk)
    out = [[], []]
    for s, n in enumerate(lens):
        for i, b in enumerate(blk[indptr[s]:indptr[s + 1]]):
            m = min(g.block_size, int(n) - i * g.block_size)
            for kind in (0, 1):
                x = oa.widen(case.data.kv[b, :, kind, :m], g.kv_dtype).astype(np.float32)
                if g.kv_dtype == "fp8_e4m3":
                    x = x * case.data.scales[b, :, kind][:, None, None].astype(np.float32)
                out[kind].append(x.transpose(1, 0, 2))
    x = np.stack([np.concatenate(o) if o else np.zeros((0, g.num_kv_heads, g.head_dim), np.float32) for o in out])
    return torch.from_numpy(x if dst == "f32" else wl.bf16_bits_from_f32(x).view(np.int16).copy()), x.shape[1]


@pytest.mark.parametrize("name", list(_workloads()))
@pytest.mark.parametrize("pool_layout,dst,padded", [("dense", "bf16", False), ("token_major", "f32", True), ("planes", "bf16", True), ("dense", "f32", False)])
def test_gather(gpu, name, pool_layout, dst, padded):
    w = _workloads()[name]
    g = w.geometry
    case = gpu(w, pool_layout=pool_layout)
    dtype = torch.float32 if dst == "f32" else torch.bfloat16
    for which in (0, 1):
        want, n = _expected(case, which, dst)
        room = torch.full((2, n + 2, g.num_kv_heads + padded, g.head_dim + 16 * padded), 7.0, dtype=dtype, device="cuda")
        out = room[:, 1:n + 1, :g.num_kv_heads, :g.head_dim]
        case.batch.kv_gather(which, out[0], out[1])
        torch.cuda.synchronize()
        bits = torch.int32 if dst == "f32" else torch.int16
        assert torch.equal(out.cpu().contiguous().view(bits), want.view(bits)), (name, which)
        rest = room.clone()
        rest[:, 1:n + 1, :g.num_kv_heads, :g.head_dim] = 7.0
        assert (rest == 7).all()                                 # nothing outside the rows
    case.close()


def test_gather_roots(gpu):
    w = wl.make_tree_workload("roots", wl.Geometry(4, 2, 64, 16, "f32", "f32"), 2, [40, 16], [0, 1, 0], [24, 50, 7], [[0, 1], [0], [1]], [3, 0, 9, 20], 1.0, 3)
    case = gpu(w)
    want, n = _expected(case, 2, "f32")
    out = torch.empty(2, n, 2, 64, device="cuda")
    case.batch.kv_gather(2, out[0], out[1])
    assert n == 56 and torch.equal(out.cpu(), want)
    case.close()


def test_every_code(gpu):
    """All 254 finite codes against a scale that is no power of two."""
    w = wl.make_workload("codes", wl.Geometry(1, 1, 128, 16, "bf16", "fp8_e4m3"), 1, [16], [[0]], [0], seed=9)
    case = gpu(w)
    codes = np.resize(np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8), 16 * 128).reshape(16, 128)
    b = int(case.olay.prefix_blk[0])
    case.data.kv[b, 0, 0], case.data.kv[b, 0, 1] = codes, codes[::-1]
    case.data.scales[b, 0] = [0.37, 1.0 / 3.0]
    case.batch.kv.copy_(torch.from_numpy(case.data.kv))
    case.batch.scales.copy_(torch.from_numpy(case.data.scales))
    for dst, dtype in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        want, n = _expected(case, 0, dst)
        out = torch.empty(2, n, 1, 128, dtype=dtype, device="cuda")
        case.batch.kv_gather(0, out[0], out[1])
        bits = torch.int32 if dst == "f32" else torch.int16
        assert torch.equal(out.cpu().view(bits), want.view(bits))
    case.close()


@pytest.mark.parametrize("kv_dtype", ["bf16", "f32"])
def test_what_was_ingested_comes_back(gpu, kv_dtype):
    w = wl.make_workload("round", wl.Geometry(8, 2, 128, 16, kv_dtype, kv_dtype), 2, [100, 17], [[0], [1]], [3, 0], 1.0, seed=3)
    case = gpu(w)
    src = [torch.randn(117, 2, 128, device="cuda").to(case.batch.kv.dtype) for _ in range(2)]
    case.batch.kv_ingest(0, *src)
    dst = [torch.empty_like(s) for s in src]
    case.batch.kv_gather(0, *dst)
    assert all(torch.equal(a, b) for a, b in zip(src, dst))
    case.close()


def test_wrong_tensors_are_refused(gpu):
    w = wl.make_workload("refused", wl.Geometry(8, 2, 128, 16, "bf16", "bf16"), 2, [100, 17], [[0], [1]], [3, 0], 1.0, seed=3)
    case = gpu(w)
    good = torch.empty(117, 2, 128, device="cuda")
    for k, v in ((good[:116], good[:116]), (good, good[:, :1]), (good.half(), good.half()), (good, good.bfloat16()), (good.transpose(0, 2), good),
                 (good, torch.empty(117, 4, 128, device="cuda")[:, :2])):
        with pytest.raises(ValueError):
            case.batch.kv_gather(0, k, v)
    case.close()
