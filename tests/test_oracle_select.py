"""The oracle of block summaries and selection: brute force in Python integers, the bound that a summary is, odd keys, ties."""
from types import SimpleNamespace

import numpy as np

import workloads as wl
from helpers import oracle_setup
from oracle import attention, select


def _f32_pool(rng, blocks=6, heads=2, slots=4, d=8):
    return rng.standard_normal((blocks, heads, 2, slots, d)).astype(np.float32)


def test_scores_by_hand():
    rng = np.random.default_rng(2)
    kv = _f32_pool(rng)
    made = [select.summarise(kv, None, "f32", b, 4) for b in range(6)]
    codes, scales = np.stack([m[0] for m in made]), np.stack([m[1] for m in made])
    q = rng.standard_normal((6, 8)).astype(np.float32)
    got = select.scores(q, codes, scales, 2)
    for h in range(2):
        for j in range(6):
            best = None
            for g in range(3):
                row = q[3 * h + g]
                s = np.float32(np.abs(row).max() * (np.float32(1) / np.float32(127)))
                total = 0
                for c in range(8):
                    qc = int(np.rint(np.float32(row[c] / s)))
                    total += qc * int(codes[j, h, 0 if qc > 0 else 1, c])
                v = np.float32(np.float32(np.float32(total) * scales[j, h]) * s)
                best = v if best is None else max(best, v)
            assert got[h, j] == best


def test_a_score_bounds_the_products_of_its_block():
    """Up to the eight bits: every code is off by at most half a step of its scale, the query's and the summary's."""
    rng = np.random.default_rng(3)
    kv, q = _f32_pool(rng), rng.standard_normal((2, 8)).astype(np.float32)
    made = [select.summarise(kv, None, "f32", b, 3) for b in range(6)]
    codes, scales = np.stack([m[0] for m in made]), np.stack([m[1] for m in made])
    got = select.scores(q, codes, scales, 2)
    for h in range(2):
        sq = np.abs(q[h]).max() / 127
        for j in range(6):
            slack = 8 * (np.abs(q[h]).max() * scales[j, h] / 2 + 127 * scales[j, h] * sq / 2 + scales[j, h] * sq)
            assert (kv[j, h, 0, :3] @ q[h]).max() <= got[h, j] + slack


def test_keys_that_are_no_numbers():
    kv = np.zeros((1, 1, 2, 4, 4), np.float32)
    kv[0, 0, 0] = [[np.nan, 1.0, np.inf, 5.0], [np.nan, np.nan, -2.0, 5.0], [np.nan, -3.0, 0.0, 5.0], [7.0, 7.0, 7.0, 7.0]]
    codes, scale = select.summarise(kv, None, "f32", 0, 3)                     # the fourth slot is not stored
    top = np.finfo(np.float32).max
    assert scale[0] == np.float32(top * (np.float32(1) / np.float32(127)))
    assert codes[0, :, 0].tolist() == [0, 0] and codes[0, 0, 2] == 127 and codes[0, 1, 2] == 0
    codes, scale = select.summarise(np.zeros((1, 1, 2, 4, 4), np.float32), None, "f32", 0, 4)
    assert scale[0] == 1.0 and not codes.any()


def test_choice():
    score = np.array([0, 5, 5, 1, 5, -1, 2, 0], np.float32)
    assert select.choose(score, 8, -1, 4, 1, 1) == [0, 1, 2, 7]               # equal scores: the lower positions
    assert select.choose(score, 8, -1, 8, 1, 1) == list(range(8))
    assert select.choose(score, 8, 2, 4, 0, 1) == [1, 4, 7]                   # the partly filled root block counts, and is not listed
    assert select.choose(score, 3, 2, 9, 0, 1) == [0, 1]


def test_everything_selected_is_the_whole_step():
    w = wl.make_tree_workload("sel", wl.Geometry(4, 2, 64, 16, "f32", "f32"), 2, [40], [0, -1, 0], [24, 50, 7], [[0, 1], [0], [1]],
                              [3, 0, 9, 20], 1.0, 3)
    _, lay, data = oracle_setup(w)
    q = attention.widen(w.q_bits(), "f32").astype(np.float32)
    codes = np.zeros((w.num_blocks, 2, 2, 64), np.int8)
    chosen = select.select(q, lay, 16, codes, np.ones((w.num_blocks, 2), np.float32), 2, 100, 1, 1)
    out, lse = select.attend(w.q_bits(), "f32", data.kv, None, "f32", lay, chosen, 16)
    ref, ref_lse = attention.decode_attention(w.q_bits(), "f32", data.kv, None, "f32", lay)
    assert np.allclose(out, ref, rtol=1e-12, atol=1e-12) and np.allclose(lse, ref_lse, rtol=1e-12)
    few = select.select(q, lay, 16, codes, np.ones((w.num_blocks, 2), np.float32), 2, 3, 1, 1)
    assert few[0][0][0] == [0, 4] and few[2][1][0] == [0, 1, 3]               # equal scores everywhere


def test_visible_contexts():
    lay = SimpleNamespace(req_prompt=[0, 0], prefix_len=[50], prefix_blk_indptr=[0, 4], prefix_blk=np.array([9, 8, 7, 6]))
    assert select.context(lay, 0, 16, [0, 33]) == ([], [], -1)
    assert select.context(lay, 1, 16, [0, 33]) == ([9, 8, 7], [16, 16, 1], -1)
