"""GPU parity of the attention over the 4-bit cache in every form that its sizes
choose: one and two row tiles, keys unsplit, in few and in many splits, logits kept
in LDS, kept in the workspace, taken again and not wanted, keys of caches beyond
128 MiB; numbers at the ends of the format; and the cache behind the framework's own
selection. Bounds as in test_gpu_cache4.
tests/test_cache4_paths.py checks on the host that the cases here reach every form.
"""
import math

import numpy as np
import pytest
import torch

import paper_2506_07416_amd as lv
import synth
from oracle import cache4 as c4
from parity_util import log, to_device
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


# batch, Hq, H, D, cap, queries of a sample at most: caches just over 128 MiB, one block of rows
LONG = [(16, 32, 8, 128, 7744, 3), (16, 32, 8, 128, 7744, 5), (32, 32, 8, 64, 7744, 3), (32, 32, 8, 64, 7744, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_attention_of_caches_beyond_the_last_level_cache(case, dtype):
    """Random codes and scales everywhere; three samples' first and last heads against the oracle."""
    B, Hq, H, D, cap, mq = LONG[case]
    assert B * H * cap * (D + D // 16) > 128 << 20
    rng = np.random.default_rng(800 + case)
    gen = torch.Generator(device="cuda").manual_seed(800 + case)
    half = cap * D
    cache = torch.randint(0, 256, (B, H, half + cap * D // 16), generator=gen, device="cuda", dtype=torch.uint8)
    cache[:, :, half:] = cache[:, :, half:] % 5 + 122
    lens = rng.integers(cap // 2, cap + 1, B)
    lens[0], lens[B // 2] = cap, 37
    nq = rng.integers(1, mq + 1, B)
    nq[B - 1], nq[0] = mq, mq - 1
    cu = cumulate(nq)
    qt = torch.as_tensor(rng.standard_normal((cu[-1], Hq, D)) * 2).to(DT[dtype])
    qd = qt.cuda()
    G = Hq // H
    for wr in (0, 1, 3):
        log(f"long caches: batch {B} heads {Hq}/{H} D {D} {dtype}, up to {mq} queries, weight rows {wr}")
        w0 = torch.rand((B, H, cap), generator=gen, device="cuda")
        wo = w0.clone()
        o = lv.cache4_attn(cache, qd, dev(cu), dev(lens), mq, cap, weight=w0, weight_out=wo, weight_rows=wr)
        for b in (0, B // 2, B - 1):
            heads = [0, H - 1]
            rows = slice(cu[b], cu[b + 1])
            qh = [g * G + i for g in heads for i in range(G)]
            pick = lambda t: t[b:b + 1, heads].double().cpu().numpy()  # noqa: E731
            check_attn(cache[b:b + 1, heads].cpu().numpy(), qt[rows][:, qh].double().numpy(), np.array([0, nq[b]]),
                       [int(lens[b])], 2 * G, D, dtype, wr, pick(w0), o[rows][:, qh].double().cpu().numpy(), pick(wo),
                       f"sample {b}")


def test_attention_of_random_rows_beyond_32_bit_offsets():
    """16777216 rows of two heads of random codes, in 64 bits on the GPU by parts.

    The kernels add: in a wave, 16 steps of 32 keys in the matrix products (at most 512
    roundings) or 8 exponentials a lane (128); 4 waves; 8192 splits by 8 slots of 1024,
    then the slots. So an output is within 1600 roundings of fp32, 2^-24 of the sum of
    p |V| each, and the sum of a softmax within 300; the logits as in check_attn."""
    cap, D, H = lv._abi.MAX_CACHE4, 128, 2
    log("16777216 random rows of two heads")
    gen = torch.Generator(device="cuda").manual_seed(900)
    cache = torch.empty((1, H, cap * (D + D // 16)), dtype=torch.uint8, device="cuda")
    for g in range(H):  # by heads and parts: whole numbers of 8 bytes at a time
        cache[0, g, :cap * D].random_(0, 256, generator=gen)
        cache[0, g, cap * D:].random_(122, 127, generator=gen)
    q = torch.randn((1, H, D), generator=gen, device="cuda")
    w = torch.full((1, H, cap), 9.0, device="cuda")
    n = cap - 5
    o = lv.cache4_attn(cache, q, dev([0, 1]), dev([n]), 1, cap, weight_out=w, weight_rows=1)
    assert (w[:, :, n:] == 9).all()
    code = torch.tensor(list(c4.E2M1) + [-x for x in c4.E2M1], dtype=torch.float64, device="cuda")
    part = 1 << 19
    for g in range(H):
        kc, vc = (cache[0, g, i * cap * D // 2:(i + 1) * cap * D // 2].view(cap, D // 2) for i in (0, 1))
        ks, vs = (cache[0, g, cap * D + i * cap * 4:cap * D + (i + 1) * cap * 4].view(4, cap) for i in (0, 1))

        def rows(codes, scales, j):
            c = codes[j:j + part].long()
            x = torch.stack((code[c & 15], code[c >> 4]), -1).view(-1, 4, 32)
            s = torch.exp2(scales[:, j:j + part].double().T - 127)
            return (x * s[:, :, None]).view(-1, D)

        x = torch.empty((cap,), dtype=torch.float64, device="cuda")
        size = 0.0
        qg = q[0, g].double()
        for j in range(0, cap, part):
            k = rows(kc, ks, j)
            x[j:j + part] = (k * qg).sum(-1) / math.sqrt(D)
            size = max(size, float((k * qg).abs().sum(-1).max()) / math.sqrt(D))
        x = x[:n]
        p = torch.exp(x - x.max())
        p /= p.sum()
        want, A = (torch.zeros((D,), dtype=torch.float64, device="cuda") for _ in range(2))
        for j in range(0, n, part):
            v = rows(vc, vs, j)[:n - j]
            pj = p[j:j + part, None]
            want += (pj * v).sum(0)
            A += (pj * v.abs()).sum(0)
        rel = math.expm1(2 * size * (D + 4) * 2.0 ** -24) + 2.0 ** -22
        err = (o[0, g].double() - want).abs()
        assert (err <= (rel + 1900 * 2.0 ** -24) * A + 2.0 ** -23 * want.abs()).all(), float((err / A).max())
        werr = ((w[0, g, :n].double() - p).abs() / p).max()
        assert float(werr) <= rel + 310 * 2.0 ** -24, float(werr)
        log(f"  head {g}: outputs {float((err / A).max()):.2e} of sum p|V|, weights {float(werr):.2e}")


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


# ----------------------------------------------------------------------------- numbers at the format's ends

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_the_smallest_numbers(dtype):
    """Blocks below 2^-126 keep the scale 2^-125, whose first step is 2^-126: what lies
    above 2^-127 rounds up to it, a subnormal input or not."""
    log(f"append of the smallest numbers, {dtype}")
    D, cap = 64, 32
    x = np.zeros((3, 1, D))
    x[0, 0, :8] = np.array([1.0, 1.5, 1.01, 1.99, -1.5, -1.0, 0.99, 2.0]) * 2.0 ** -127
    x[0, 0, 32:36] = np.array([3.0, 1.5, -2.5, 0.5]) * 2.0 ** -127     # beside a normal number
    x[1, 0, :4] = np.array([12.0, 1.5, 7.0, -1.75]) * 2.0 ** -127
    x[1, 0, 32:35] = [1.0, 1e-38, -1e-38]                           # far below the block's scale
    x[2, 0, :] = 2.0 ** -127 * (1 + np.arange(D) / D)
    kt = torch.as_tensor(x).float().to(DT[dtype])
    cache = lv.cache4_empty(1, 1, D, cap)
    lv.cache4_append(cache, kt.cuda(), kt.flip(0).cuda(), dev([0, 3]), dev([0]), 3)
    got = c4.split_cache(cache.cpu().numpy(), D)
    for t, codes, scales in ((kt, got[0], got[1]), (kt.flip(0), got[2], got[3])):
        wc, ws = c4.encode(t.double().numpy()[:, 0])
        assert np.array_equal(scales[0, 0, :3], ws) and np.array_equal(codes[0, 0, :3], wc)


def test_read_of_every_scale():
    """All 256 scale bytes with every code whose value fp32 has (bf16 then has it too),
    the subnormal ones among them; byte 255 is NaN."""
    log("every scale byte")
    D, cap = 64, 256
    codes = np.zeros((1, 1, cap, D), np.uint8)
    codes[0, 0] = np.arange(D) % 16
    codes[0, 0, 253] = [0, 1, 2, 3, 4, 5, 8, 9, 10, 11, 12, 13, 0, 1, 2, 3] * 4      # up to 3 * 2^126
    codes[0, 0, 254] = [0, 1, 2, 3, 8, 9, 10, 11] * 8                                # up to 1.5 * 2^127
    scales = np.broadcast_to(np.arange(256, dtype=np.uint8)[None, None, :, None], (1, 1, cap, 2))
    cache = torch.as_tensor(c4.join_cache(codes, scales, codes[:, :, :, ::-1], scales)).cuda()
    want = c4.decode(codes, scales)[0, 0]
    for dt in (torch.bfloat16, torch.float32):
        k, v = lv.cache4_read(cache, D, dev([0, cap]), dev([0]), cap, dtype=dt)
        np.testing.assert_array_equal(k[:, 0].double().cpu().numpy(), want)
        np.testing.assert_array_equal(v[:, 0].double().cpu().numpy(), want[:, ::-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m,top", [(512, 1, 107), (1500, 40, 105)])
def test_attention_at_the_end_of_the_values_range(dtype, n, m, top):
    """n rows of up to 6 * 2^top, n * max|V| just below 2^119: the largest that the header
    allows. All keys but a wave's first have logits 7.9 (log2) above those: the reference
    stays behind the maximum, where the unnormalised outputs are largest."""
    log(f"values of up to 6 * 2^{top}, {n} rows, {m} queries, {dtype}")
    assert 2.0 ** 118 < n * 6 * 2.0 ** top < 2.0 ** 119
    rng = np.random.default_rng(970)
    Hq, H, D, cap = 4, 1, 128, (n + 31) // 32 * 32
    kc, ks, vc, vs = c4.split_cache(random_cache(rng, 1, H, D, cap), D)
    kc[:], ks[:], vs[:] = 0, 127, top + 127
    vc[..., :64] = 7                                   # half of the elements 6 * 2^top in every row: sums that grow
    kc[0, 0, 128:, 0] = 2                              # 1.0, behind the four waves' first steps
    cache = c4.join_cache(kc, ks, vc, vs)
    qt = torch.zeros((m, Hq, D))
    qt[..., 0] = 7.875 * math.log(2.0)
    qt = qt.to(DT[dtype])
    o = lv.cache4_attn(torch.as_tensor(cache).cuda(), qt.cuda(), dev([0, m]), dev([n]), m, n, softmax_scale=1.0)
    K, V = c4.decode(kc, ks), c4.decode(vc, vs)
    ref, _, A, size = c4.attention(qt.double().numpy(), [0, m], K, V, [n], 1.0)
    got = o.double().cpu().numpy()
    assert np.isfinite(got).all()
    rel = np.expm1(2 * size * (D + 4) * 2.0 ** -24)[..., None] + 2.0 ** -22
    u = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert (np.abs(got - ref) <= (u + rel + (n + 8) * 2.0 ** -24) * A + (u + 2.0 ** -23) * np.abs(ref)).all()


# ----------------------------------------------------------------------------- behind the framework's selection

def test_selected_rows_enter_the_cache_and_are_attended_like_a_decode():
    """The kept rows of the selection as they are packed, appended with their cu_seqlens;
    the next token behind them; its attention against the decode attention over the same
    rows read back. Both are within their own bounds of the 64-bit result."""
    case = synth.config_case(4, Tv=64, T=16, keep_ratio=0.5)
    q, k, v = (to_device(x, case.dtype) for x in (case.q, case.k, case.v))
    logit = torch.from_numpy(case.view_logit).cuda()
    _, keep, _ = lv.patch_select(logit, case.view_offsets, case.S, case.w_lexical, case.threshold)
    r = lv.token_score_topk(q, k, v, keep, case.keep_ratio, case.V_full)
    B, S, Hq, H, D = case.B, case.S, case.Hq, case.Hkv, case.D
    cu = r["cu_seqlens"]
    lens = (cu[1:] - cu[:-1]).cpu().numpy()
    log(f"selected rows {lens.tolist()} into the 4-bit cache")
    cap = (S + 1 + 31) // 32 * 32
    cache = lv.cache4_empty(B, H, D, cap)
    lv.cache4_append(cache, r["kc"], r["vc"], cu, dev([0] * B), S)
    rng = np.random.default_rng(960)
    q1, k1, v1 = (torch.as_tensor(rng.standard_normal((B, h, D))).to(torch.bfloat16).cuda() for h in (Hq, H, H))
    one = dev(np.arange(B + 1))
    lv.cache4_append(cache, k1, v1, one, dev(lens), 1)
    o = lv.cache4_attn(cache, q1, one, dev(lens + 1), 1, S + 1)
    check_attn(cache.cpu().numpy(), q1.double().cpu().numpy(), np.arange(B + 1), (lens + 1).tolist(), Hq, D, "bf16", 0, None,
               o.double().cpu().numpy(), None, "the next token")
    kr, vr = lv.cache4_read(cache, D, cu, dev([0] * B), S, rows=r["kc"].shape[0])
    k1r, v1r = lv.cache4_read(cache, D, one, dev(lens), 1)
    d = lv.decode_attn(q1, k1r, v1r, kr, vr, cu, S)
    kc, ks, vc, vs = c4.split_cache(cache.cpu().numpy(), D)
    _, _, A, _ = c4.attention(q1.double().cpu().numpy(), np.arange(B + 1), c4.decode(kc, ks), c4.decode(vc, vs), lens + 1,
                              1 / math.sqrt(D))
    # each call rounds its probabilities and its result to bf16: 2 * 2^-8 of sum p |V| a call
    assert (np.abs((o.double() - d.double()).cpu().numpy()) <= 4.1 * 2.0 ** -8 * A).all()
