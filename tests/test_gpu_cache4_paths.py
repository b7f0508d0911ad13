"""GPU parity of the attention over the 4-bit cache in every form that its sizes
choose: one and two row tiles, keys unsplit, in few and in many splits, logits kept
in LDS, kept in the workspace, taken again and not wanted. Bounds as in
test_gpu_cache4. tests/test_cache4_paths.py checks on the host that the cases here
reach every form.
"""
import numpy as np
import pytest
import torch

import paper_2506_07416_amd as lv
from oracle import cache4 as c4
from parity_util import log
from test_gpu_cache4 import DT, check_attn, cumulate, dev, random_cache

pytestmark = pytest.mark.gpu

PATHS = [
    # lens, queries, Hq, H, D, cap, dtype, weight_rows, extra max_len
    # many heads, two row tiles in one block: few splits at D = 128, many at 64
    ([1700, 3, 900, 1699], [9, 9, 1, 8], 32, 16, 128, 1728, "bf16", 4, 0),
    ([1700, 1000, 0, 17], [9, 2, 9, 9], 32, 16, 64, 1728, "bf16", 4, 11),
    ([1700, 1550, 40, 1601], [9, 9, 3, 0], 32, 16, 128, 1728, "f32", 9, 0),
    ([1690, 1200, 1, 300], [9, 5, 1, 9], 32, 16, 64, 1696, "f32", 9, 6),
    # heads enough to leave the keys unsplit, several blocks of rows
    ([450, 449, 70], [70, 33, 64], 32, 32, 128, 480, "bf16", 5, 20),
    ([450, 200, 69], [70, 1, 70], 32, 32, 128, 480, "f32", 8, 0),
    ([420, 419, 1, 300, 33, 97], [70, 65, 33, 64, 40, 70], 32, 32, 64, 448, "bf16", 70, 0),
    ([420, 100, 420, 7, 64, 385], [70, 64, 17, 16, 31, 70], 32, 32, 64, 448, "f32", 20, 3),
    ([450, 449, 70], [70, 33, 64], 32, 32, 128, 480, "bf16", 33, 0),
    ([450, 449, 70], [64, 33, 70], 32, 32, 128, 480, "f32", 70, 0),
    ([420, 419, 1, 300, 33, 97], [70, 65, 33, 64, 40, 70], 32, 32, 64, 448, "bf16", 8, 0),
    ([420, 100, 420, 7, 64, 385], [70, 64, 17, 16, 31, 70], 32, 32, 64, 448, "f32", 2, 3),
    # a prompt of few heads that follows: many blocks, split keys
    ([1500], [300], 8, 2, 128, 1504, "bf16", 2, 0),
    ([1490], [300], 8, 2, 128, 1504, "f32", 2, 7),
    ([1500], [300], 8, 2, 64, 1504, "f32", 300, 0),
    ([2700], [300], 4, 1, 64, 2720, "f32", 2, 0),
    ([2700], [299], 4, 1, 64, 2720, "bf16", 1, 20),
    ([3100], [300], 4, 1, 128, 3104, "bf16", 300, 0),
    ([3100, 20], [130, 200], 4, 1, 128, 3104, "f32", 1, 0),
    # few splits of two row tiles at D = 64
    ([900, 899, 30, 512, 1, 0, 640, 700], [9, 8, 9, 1, 3, 9, 5, 2], 32, 16, 64, 928, "bf16", 4, 0),
    ([900, 257, 30, 512, 1, 0, 640, 899], [9, 8, 9, 1, 3, 9, 5, 2], 32, 16, 64, 928, "f32", 9, 5),
    # up to 512 keys with 17..32 rows: one workgroup a head, weights added by it or not
    ([512, 300], [7, 8], 8, 2, 64, 512, "f32", 2, 0),
    ([511, 31], [8, 5], 8, 2, 64, 512, "bf16", 2, 1),
    ([130, 512, 0], [8, 1, 8], 8, 2, 128, 544, "f32", 2, 0),
    ([130, 500, 0], [8, 6, 8], 8, 2, 128, 544, "bf16", 1, 0),
    ([512, 300], [7, 8], 8, 2, 64, 512, "f32", 8, 0),
    ([512, 129], [8, 8], 8, 2, 128, 512, "bf16", 7, 0),
    # one row tile: one workgroup a head, and what the cases of test_gpu_cache4 leave out
    ([512, 511], [2, 3], 8, 2, 64, 512, "bf16", 2, 0),
    ([512, 77], [2, 3], 8, 2, 128, 512, "f32", 2, 0),
    ([1000], [20], 8, 8, 64, 1024, "bf16", 8, 0),
    ([1000], [20], 8, 8, 64, 1024, "bf16", 20, 0),
    ([1000], [20], 8, 8, 128, 1024, "f32", 20, 0),
    ([600, 601], [20, 1], 8, 2, 128, 608, "f32", 2, 0),
    # few splits and none with one row tile: many short heads
    ([250] * 20, [1] * 20, 32, 32, 128, 256, "bf16", 0, 0),
    ([250] * 18, [9] * 18, 32, 32, 64, 256, "bf16", 9, 0),
    ([250] * 18, [9] * 18, 32, 32, 64, 256, "f32", 9, 0),
    ([250, 249] * 9, [9, 2] * 9, 32, 32, 128, 256, "f32", 9, 0),
    ([650, 20] * 5, [2, 1] * 5, 32, 16, 128, 672, "f32", 1, 0),
    ([650, 20] * 5, [2, 1] * 5, 32, 16, 64, 672, "bf16", 1, 0),
    ([650, 20] * 5, [2, 1] * 5, 32, 16, 64, 672, "f32", 2, 0),
    ([2500, 2499], [2, 2], 8, 2, 64, 2528, "bf16", 2, 0),
    ([2500, 10], [1, 2], 8, 2, 64, 2528, "f32", 2, 0),
    ([2500, 10], [1, 2], 8, 2, 128, 2528, "f32", 2, 0),
]


@pytest.mark.parametrize("case", range(len(PATHS)))
def test_attention_forms_match_oracle(case):
    lens, nq, Hq, H, D, cap, dtype, wr, extra = PATHS[case]
    what = f"form {case}: lens {lens[:4]} queries {nq[:4]} batch {len(lens)} heads {Hq}/{H} D {D} {dtype} weight rows {wr}"
    log(what)
    rng = np.random.default_rng(700 + case)
    B, cu = len(lens), cumulate(nq)
    cache = random_cache(rng, B, H, D, cap)
    qt = torch.as_tensor(rng.standard_normal((cu[-1] + 1, Hq, D)) * 2).to(DT[dtype])
    weight = rng.random((B, H, cap)).astype(np.float32)
    wt = torch.as_tensor(weight).cuda()
    wo = wt.clone()
    o = torch.full(qt.shape, 3.0, dtype=DT[dtype], device="cuda")
    top = min(cap, max(lens) + extra)
    args = (torch.as_tensor(cache).cuda(), qt.cuda(), dev(cu), dev(lens), max(nq), top)
    ws = torch.full((lv.cache4_attn_workspace_bytes(DT[dtype], B, Hq, H, D, max(nq), top, wr),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    lv.cache4_attn(*args, weight=wt, weight_out=wo, weight_rows=wr, out=o, workspace=ws)
    got, w = o.double().cpu().numpy(), wo.double().cpu().numpy()
    assert (got[cu[-1]:] == 3).all()
    q = qt.double().numpy()[:cu[-1]]
    check_attn(cache, q, cu, lens, Hq, D, dtype, wr, weight.astype(np.float64), got[:cu[-1]], w, f"form {case}")
    # the same bits over another workspace's contents, in place, and without weights
    ws.fill_(0x7F)
    o2 = lv.cache4_attn(*args, weight=wt, weight_rows=wr, workspace=ws)
    assert torch.equal(o2[:cu[-1]], o[:cu[-1]]) and torch.equal(wt, wo)
    o3 = lv.cache4_attn(*args)
    check_attn(cache, q, cu, lens, Hq, D, dtype, 0, None, o3.double().cpu().numpy()[:cu[-1]], None,
               f"form {case}, no weights")


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_nan_and_stale_rows_with_two_row_tiles_and_split_keys(dtype, D):
    """NaN blocks reach the queries that see them and no other, whichever tile and split they are in."""
    rng = np.random.default_rng(950)
    B, Hq, H, cap, n, m = 1, 8, 2, 1696, 1650, 300
    log(f"NaN blocks, two row tiles, {dtype} D {D}")
    cache = random_cache(rng, B, H, D, cap)
    kc, ks, vc, vs = c4.split_cache(cache, D)
    clean = c4.join_cache(kc, ks, vc, vs)
    for a in (kc, vc):
        a[:, :, n:] = 15
    for s in (ks, vs):
        s[:, :, n:] = 255
    bad = np.zeros((m, Hq, D), bool)
    first = n - m + 1                  # rows that query 0 sees
    for at in (first + 5, n - 1, first + 140):     # values, seen from the query 'at - first + 1' on
        vs[0, 0, at, 1] = 255
        bad[at - first + 1:, 0:4, 32:64] = True
    at = first + 39                    # queries 40..43 fill a row tile: the others' bits do not change
    ks[0, 1, at, 0] = 255
    bad[at - first + 1:, 4:8] = True
    qt = torch.as_tensor(rng.standard_normal((m, Hq, D))).to(DT[dtype])
    outs, ws = [], []
    for c in (clean, c4.join_cache(kc, ks, vc, vs)):
        w = torch.zeros((B, H, cap), device="cuda")
        o = lv.cache4_attn(torch.as_tensor(c).cuda(), qt.cuda(), dev([0, m]), dev([n]), m, cap, weight_out=w, weight_rows=40)
        outs.append(o.double().cpu().numpy())
        ws.append(w.cpu().numpy())
    assert np.array_equal(np.isnan(outs[1]), bad)
    assert np.array_equal(outs[0][~bad], outs[1][~bad])
    # the first 40 queries see no NaN key: query 40 is the first that does
    assert np.array_equal(ws[0], ws[1]) and np.isfinite(ws[1]).all() and (ws[1][:, :, n:] == 0).all()
    w = torch.zeros((B, H, cap), device="cuda")
    lv.cache4_attn(torch.as_tensor(c4.join_cache(kc, ks, vc, vs)).cuda(), qt.cuda(), dev([0, m]), dev([n]), m, cap,
                   weight_out=w, weight_rows=41)
    assert torch.isfinite(w[0, 0]).all()
    # the query's probabilities are NaN for the rows that it sees, and for no other
    assert torch.isnan(w[0, 1, :at + 1]).all() and not w[0, 1, at + 1:].any()
