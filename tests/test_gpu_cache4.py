"""GPU parity of the 4-bit cache's calls and of the draft verification against the
float64 oracle (oracle/cache4.py).

Tolerances, from the roundings that the calls make (u = 2^-8 for a rounding to
bf16, 2^-24 for one to fp32; half a step):
  stored rows, moved rows, kept positions, tokens, counts: exact.
  logits: a sum of D products that are exact in fp32, so within D * 2^-24 *
      sum |q_d K_d| * scale, and 2^-22 of their size for the scale and the
      exponent's argument: delta below. A probability is off by exp(2 delta) - 1
      and the exponential's own 2^-22.
  outputs: each probability rounded once to bf16 (bf16 queries only): u * A with
      A = sum p |V|; fp32 sums over n keys, n * 2^-24 * A; the result's rounding.
  weights: the probabilities' error on what is added, and fp32 sums.
  underflow: a probability below 2^-126 counts as 0, as the header says, so each of
      the n keys may lack 2^-126 |V|, and a result has no finer step than 2^-133
      (bf16) below 2^-126. This is what a row needs whose one heavy key has zeros
      where the others' probabilities, 2^-130 and less, multiply something: its
      result of 1e-47 has no fp32 value at all.
"""
import math

import numpy as np
import pytest
import torch

import paper_2506_07416_amd as lv
from oracle import cache4 as c4
from parity_util import log

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dtype).cuda()


def cumulate(lens):
    return np.concatenate(([0], np.cumsum(lens))).astype(np.int64)


def random_cache(rng, B, H, D, cap):
    """Bytes of a cache of random codes; scales around 1."""
    kc, vc = (rng.integers(0, 16, (B, H, cap, D)).astype(np.uint8) for _ in range(2))
    ks, vs = (rng.integers(122, 127, (B, H, cap, D // 32)).astype(np.uint8) for _ in range(2))
    return c4.join_cache(kc, ks, vc, vs)


def values(cache, D):
    kc, ks, vc, vs = c4.split_cache(cache, D)
    return c4.decode(kc, ks), c4.decode(vc, vs)


# ----------------------------------------------------------------------------- store

STORE = [
    # lens, start, H, D, cap, dtype
    ([1], [0], 1, 64, 32, "bf16"),
    ([1, 1, 1], [5, 31, 0], 2, 128, 32, "bf16"),
    ([0, 3, 65, 7], [4, 30, 1, 89], 2, 128, 96, "bf16"),
    ([64, 130, 0], [0, 3, 2], 3, 64, 160, "f32"),
    ([33, 2], [31, 0], 4, 128, 64, "f32"),
    ([10, 10, 10], [-3, 60, 64], 2, 64, 64, "bf16"),      # rows in front of and behind the cache are dropped
]


@pytest.mark.parametrize("lens,start,H,D,cap,dtype", STORE)
def test_append_and_read(lens, start, H, D, cap, dtype):
    log(f"store lens {lens} start {start} H {H} D {D} cap {cap} {dtype}")
    rng = np.random.default_rng(sum(lens) + D + cap)
    B, rows = len(lens), sum(lens)
    cu = cumulate(lens)
    x = [rng.standard_normal((rows + 2, H, D)) * np.exp2(rng.integers(-30, 30, (rows + 2, H, 1))) for _ in range(2)]
    x[0][0, 0, :32] = 0.0
    x[1][0, 0, 3] = np.nan
    x[1][rows - 1, H - 1, D - 1] = -np.inf
    x[0][rows // 2, 0, 32:64] = 1e-39
    x[0][rows // 3, H - 1, :4] = [3e38, -3.3e38, 1.0, 1e38]
    k, v = (torch.as_tensor(a).float().to(DT[dtype]).cuda() for a in x)
    before = rng.integers(0, 256, (B, H, cap * (D + D // 16))).astype(np.uint8)
    cache = torch.as_tensor(before).cuda()
    weight = torch.ones((B, H, cap), device="cuda")
    lv.cache4_append(cache, k, v, dev(cu), dev(start), max(lens), weight=weight)
    got = c4.split_cache(cache.cpu().numpy(), D)
    want = c4.split_cache(before, D)
    hit = np.ones((B, H, cap))
    kx, vx = k.double().cpu().numpy(), v.double().cpu().numpy()
    for b in range(B):
        for i in range(lens[b]):
            pos = start[b] + i
            if 0 <= pos < cap:
                r = cu[b] + i
                want[0][b, :, pos], want[1][b, :, pos] = c4.encode(kx[r])
                want[2][b, :, pos], want[3][b, :, pos] = c4.encode(vx[r])
                hit[b, :, pos] = 0
    for a, b, name in zip(got, want, ("K codes", "K scales", "V codes", "V scales")):
        assert np.array_equal(a, b), name
    assert np.array_equal(weight.cpu().numpy(), hit)
    # back, in either type, with rows behind the last one left alone
    for out in (torch.bfloat16, torch.float32):
        kr, vr = (torch.full((rows + 2, H, D), 7.0, dtype=out, device="cuda") for _ in range(2))
        lv.cache4_read(cache, D, dev(cu), dev(start), max(lens), out=(kr, vr))
        kd, vd = c4.decode(*got[:2]), c4.decode(*got[2:])
        for b in range(B):
            for i in range(lens[b]):
                pos = start[b] + i
                for t, ref in ((kr, kd), (vr, vd)):
                    row = t[cu[b] + i].double().cpu().numpy()
                    want_row = ref[b, :, pos] if 0 <= pos < cap else np.zeros((H, D))
                    np.testing.assert_array_equal(row, want_row)
        assert (kr[rows:] == 7).all() and (vr[rows:] == 7).all()


def test_append_and_read_of_nothing():
    cache = lv.cache4_empty(2, 1, 64, 32)
    k = torch.zeros((0, 1, 64), device="cuda")
    lv.cache4_append(cache, torch.zeros((1, 1, 64), device="cuda"), torch.zeros((1, 1, 64), device="cuda"),
                     dev([0, 0, 0]), dev([0, 0]), 0)
    # no rows at all, though some may come
    lv.cache4_append(cache, k, k, dev([0, 0, 0]), dev([3, 4]), 5)
    kr, vr = lv.cache4_read(cache, 64, dev([0, 0, 0]), dev([3, 4]), 5, rows=0)
    assert not cache.any() and kr.shape == vr.shape == (0, 1, 64)


def test_attention_of_nothing():
    """No queries: the weights pass through. No rows, or none that may be looked at: zeros."""
    cache = torch.full((2, 2, 32 * 68), 255, dtype=torch.uint8, device="cuda")
    w = torch.rand((2, 2, 32), device="cuda")
    out = torch.full_like(w, 9.0)
    q = torch.zeros((0, 4, 64), device="cuda")
    o = lv.cache4_attn(cache, q, dev([0, 0, 0]), dev([3, 32]), 2, 32, weight=w, weight_out=out, weight_rows=1)
    assert o.shape == q.shape and torch.equal(out[1], w[1]) and torch.equal(out[0, :, :3], w[0, :, :3])
    assert (out[0, :, 3:] == 9).all()
    q = torch.randn((3, 4, 64), device="cuda")
    for lengths, max_len in (([0, 0], 32), ([5, 5], 0), ([-4, 0], 7)):
        o = lv.cache4_attn(cache, q, dev([0, 1, 3]), dev(lengths), 2, max_len, weight=w, weight_out=out, weight_rows=2)
        assert not o.any()
    assert (out[0, :, 3:] == 9).all()


# ----------------------------------------------------------------------------- attention

def check_attn(cache, q, cu_q, lens, Hq, D, dtype, weight_rows, weight, o, w, what):
    """Outputs o and weights w (arrays) against the oracle, with the bounds above."""
    K, V = values(cache, D)
    scale = 1 / math.sqrt(D)
    ref, add, A, size = c4.attention(q, cu_q, K, V, lens, scale, weight_rows)
    n = max(1, max(lens))
    delta = size * (D + 4) * 2.0 ** -24
    rel = np.expm1(2 * delta) + 2.0 ** -22
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = (u if dtype == "bf16" else 0.0) * A + (rel[..., None] + (n + 8) * 2.0 ** -24) * A + (u + 2.0 ** -24) * np.abs(ref)
    tol = tol + 2.0 ** -126 * (n * np.nanmax(np.abs(V)) + 1)
    err = np.abs(o - ref)
    assert (err <= tol).all(), f"{what}: {(err > tol).sum()} outputs, worst {np.max(err / np.maximum(tol, 1e-300))}"
    if weight_rows:
        G = Hq // K.shape[1]
        want = weight + add
        wtol = (rel.max() + 2.0 ** -22 + (G * weight_rows + n) * 2.0 ** -24) * add + 2.0 ** -23 * np.abs(want) + G * weight_rows * 2.0 ** -126
        for b, m in enumerate(lens):
            e = np.abs(w[b, :, :m] - want[b, :, :m])
            assert (e <= wtol[b, :, :m]).all(), f"{what}: weights of sample {b}, worst {e.max()}"
            assert np.array_equal(w[b, :, m:], weight[b, :, m:]), f"{what}: weights behind the length of sample {b}"
    log(f"  {what}: {np.max(err / np.maximum(tol, 1e-300)):.3f} of the bound")


ATTN = [
    # lens, queries, Hq, H, D, cap, dtype, weight_rows, extra max_len
    ([1], [1], 1, 1, 64, 32, "bf16", 1, 0),
    ([1, 2, 31, 32, 33, 63, 64, 65], [1] * 8, 8, 2, 128, 96, "bf16", 1, 31),
    ([0, 1, 5, 40], [1, 3, 7, 2], 4, 4, 64, 64, "bf16", 7, 0),
    ([0, 1, 5, 40], [1, 3, 7, 0], 4, 4, 64, 64, "f32", 2, 20),
    ([300, 17, 511, 0, 129], [5, 4, 3, 2, 1], 32, 8, 128, 512, "bf16", 1, 0),
    ([300, 17, 255], [5, 4, 8], 28, 4, 128, 320, "bf16", 8, 5),
    ([127, 128, 129, 2], [1, 2, 1, 2], 16, 2, 128, 160, "f32", 2, 0),
    ([200, 90], [33, 40], 16, 16, 64, 224, "bf16", 40, 0),
    ([200, 90], [33, 40], 8, 1, 64, 224, "f32", 33, 0),
    ([700, 701], [2, 1], 128, 1, 128, 704, "bf16", 2, 0),
    ([2500, 1300], [1, 1], 32, 8, 128, 2528, "bf16", 1, 28),
    ([2500], [70], 8, 2, 128, 2528, "bf16", 3, 0),
    ([512, 1, 0, 77], [1, 2, 1, 0], 32, 8, 128, 512, "bf16", 2, 0),
    ([512, 300], [2, 1], 16, 4, 64, 544, "f32", 2, 1),
    ([513, 512], [7, 3], 16, 4, 128, 544, "bf16", 1, 0),
    ([1111, 900], [6, 1], 8, 4, 64, 1120, "f32", 6, 9),
]


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention_matches_oracle(case):
    lens, nq, Hq, H, D, cap, dtype, wr, extra = ATTN[case]
    what = f"attn lens {lens} queries {nq} heads {Hq}/{H} D {D} {dtype} weight rows {wr}"
    log(what)
    rng = np.random.default_rng(100 + case)
    B, cu = len(lens), cumulate(nq)
    cache = random_cache(rng, B, H, D, cap)
    qt = torch.as_tensor(rng.standard_normal((cu[-1] + 1, Hq, D)) * 2).to(DT[dtype])
    q = qt.double().numpy()[:cu[-1]]
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
    check_attn(cache, q, cu, lens, Hq, D, dtype, wr, weight.astype(np.float64), got[:cu[-1]], w, f"case {case}")
    # again: the same bits, with another workspace's contents, in place, and without weights
    ws.fill_(0x7F)
    o2 = lv.cache4_attn(*args, weight=wt, weight_rows=wr, workspace=ws)
    assert torch.equal(o2[:cu[-1]], o[:cu[-1]]) and torch.equal(wt, wo)
    odd = torch.zeros((B * H * cap + 1,), device="cuda")[1:].view(B, H, cap)
    odd.copy_(torch.as_tensor(weight))
    lv.cache4_attn(*args, weight=odd, weight_rows=wr)
    assert torch.equal(odd, wo)
    o3 = lv.cache4_attn(*args)
    assert torch.equal(o3[:cu[-1]], o[:cu[-1]])
    # weights from nothing, at an address not aligned to 16 bytes
    fresh = torch.zeros((B * H * cap + 1,), device="cuda")[1:].view(B, H, cap)
    lv.cache4_attn(*args, weight_out=fresh, weight_rows=wr)
    check_attn(cache, q, cu, lens, Hq, D, dtype, wr, np.zeros((B, H, cap)), got[:cu[-1]],
               fresh.double().cpu().numpy(), f"case {case}, from nothing")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_logits_and_scales(dtype):
    """One key far above the others, and rows of very different size."""
    rng = np.random.default_rng(7)
    B, Hq, H, D, cap, lens = 1, 4, 2, 128, 256, [250]
    cache = random_cache(rng, B, H, D, cap)
    kc, ks, vc, vs = c4.split_cache(cache, D)
    ks[0, :, 100] = 131
    vs[0, :, ::3] = 110
    cache = c4.join_cache(kc, ks, vc, vs)
    qt = torch.as_tensor(rng.standard_normal((3, Hq, D)) * 3).to(DT[dtype])
    o = lv.cache4_attn(torch.as_tensor(cache).cuda(), qt.cuda(), dev([0, 3]), dev(lens), 3, 250)
    check_attn(cache, qt.double().numpy(), np.array([0, 3]), lens, Hq, D, dtype, 0, None, o.double().cpu().numpy(), None,
               "large logits")


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_attention_nan_and_stale_rows(dtype, D):
    """NaN blocks reach the queries that see them and no other; rows behind the
    length may hold anything; a NaN query spoils its own row and its head's weights."""
    rng = np.random.default_rng(8)
    B, Hq, H, cap, n, m = 2, 4, 2, 96, 50, 4
    cache = random_cache(rng, B, H, D, cap)
    kc, ks, vc, vs = c4.split_cache(cache, D)
    clean = c4.join_cache(kc, ks, vc, vs)
    for a in (kc, vc):
        a[:, :, n:] = 15
    for s in (ks, vs):
        s[:, :, n:] = 255
    vs[0, 0, n - 2, 1] = 255          # queries 2 and 3 of sample 0 see it, in elements 32..63 of head 0's outputs
    ks[1, 1, n - 1, 0] = 255          # query 3 of sample 1, heads 2 and 3
    dirty = c4.join_cache(kc, ks, vc, vs)
    qt = torch.as_tensor(rng.standard_normal((B * m, Hq, D))).to(DT[dtype])
    cu, lens = np.array([0, m, 2 * m]), [n, n]
    outs, ws = [], []
    for c in (clean, dirty):
        w = torch.zeros((B, H, cap), device="cuda")
        o = lv.cache4_attn(torch.as_tensor(c).cuda(), qt.cuda(), dev(cu), dev(lens), m, cap, weight_out=w, weight_rows=m)
        outs.append(o.double().cpu().numpy())
        ws.append(w.cpu().numpy())
    bad = np.zeros((B * m, Hq, D), bool)
    bad[2:4, 0:2, 32:64] = True
    bad[m + 3, 2:4] = True
    assert np.array_equal(np.isnan(outs[1]), bad)
    assert np.array_equal(outs[0][~bad], outs[1][~bad])
    assert np.array_equal(ws[0][0], ws[1][0]) and np.array_equal(ws[0][1, 0], ws[1][1, 0])
    assert np.isnan(ws[1][1, 1, :n]).all() and (ws[1][:, :, n:] == 0).all()
    # visible to every query: the plain tiles
    vs[0, 1, 3, 0] = 255
    o = lv.cache4_attn(torch.as_tensor(c4.join_cache(kc, ks, vc, vs)).cuda(), qt.cuda(), dev(cu), dev(lens), m, cap)
    bad[0:4, 2:4, 0:32] = True
    assert np.array_equal(np.isnan(o.double().cpu().numpy()), bad)
    # a NaN and an infinite query
    qn = qt.clone()
    qn[1, 0, 5] = math.nan
    qn[m + 2, 3, 0] = math.inf
    w = torch.zeros((B, H, cap), device="cuda")
    o = lv.cache4_attn(torch.as_tensor(clean).cuda(), qn.cuda(), dev(cu), dev(lens), m, cap, weight_out=w, weight_rows=2)
    o = o.double().cpu().numpy()
    assert np.isnan(o[1, 0]).all() and np.isnan(o[m + 2, 3]).all()
    keep = np.ones((B * m, Hq), bool)
    keep[1, 0] = keep[m + 2, 3] = False
    assert np.array_equal(o[keep], outs[0][keep])
    assert np.isnan(w[0, 0, :n - 2].cpu().numpy()).all() and torch.isfinite(w[1]).all()


def test_attention_logits_of_minus_infinity():
    """Keys whose logit overflows to -inf have no weight; a row with nothing else is NaN."""
    D, cap = 64, 32
    kc = np.zeros((1, 1, cap, D), np.uint8)
    ks = np.full((1, 1, cap, 2), 127, np.uint8)
    rng = np.random.default_rng(9)
    vc = rng.integers(0, 16, (1, 1, cap, D)).astype(np.uint8)
    kc[0, 0, 0] = 7 | 8                    # -6 * 2^125 in every element
    ks[0, 0, 0] = 252
    cache = c4.join_cache(kc, ks, vc, ks * 0 + 127)
    q = torch.full((1, 1, D), 100.0, device="cuda")
    for n in (1, 3):
        w = torch.zeros((1, 1, cap), device="cuda")
        o = lv.cache4_attn(torch.as_tensor(cache).cuda(), q, dev([0, 1]), dev([n]), 1, n, weight_out=w, weight_rows=1)
        o = o.double().cpu().numpy()[0, 0]
        if n == 1:
            assert np.isnan(o).all() and math.isnan(float(w[0, 0, 0]))
        else:
            want = c4.E2M1[vc[0, 0, 1:3] & 7] * np.where(vc[0, 0, 1:3] & 8, -1, 1)
            assert np.abs(o - want.mean(0)).max() < 1e-6
            assert w[0, 0, :3].tolist() == [0.0, 0.5, 0.5]


def test_attention_in_a_cache_beyond_32_bit_offsets():
    """16777216 positions of two heads, 4.6 GB: one heavy key at the end of the last head."""
    cap, D = lv._abi.MAX_CACHE4, 128
    cache = torch.zeros((1, 2, cap * (D + D // 16)), dtype=torch.uint8, device="cuda")
    k = torch.zeros((1, 2, D), device="cuda")
    k[0, :, 0] = 4.0
    v = torch.ones((1, 2, D), device="cuda")
    v[0, 1] = 2.0
    lv.cache4_append(cache, k, v, dev([0, 1]), dev([cap - 1]), 1)
    q = torch.zeros((1, 2, D), device="cuda")
    q[0, :, 0] = 5.0
    w = torch.zeros((1, 2, cap), device="cuda")
    o = lv.cache4_attn(cache, q, dev([0, 1]), dev([cap]), 1, cap, softmax_scale=1.0, weight_out=w, weight_rows=1)
    p = math.exp(20.0) / (math.exp(20.0) + cap - 1)
    rest = 1 / (math.exp(20.0) + cap - 1)
    # sums of 2^24 equal terms in fp32: parts of at most 2^24 terms, each addition within 2^-24 of the running sum
    assert torch.allclose(o[0, 0].double(), torch.full((D,), p, dtype=torch.float64, device="cuda"), rtol=5e-3)
    assert torch.allclose(o[0, 1].double(), torch.full((D,), 2 * p, dtype=torch.float64, device="cuda"), rtol=5e-3)
    assert abs(float(w[0, 1, cap - 1]) / p - 1) < 5e-3 and abs(float(w[0, 1, 12345]) / rest - 1) < 5e-3
    kr, vr = lv.cache4_read(cache, D, dev([0, 2]), dev([cap - 1]), 2, dtype=torch.float32)
    assert torch.equal(kr[0], k[0]) and torch.equal(vr[0], v[0]) and not kr[1].any()


# ----------------------------------------------------------------------------- eviction

EVICT = [
    # lens, budget, recent, H, D, cap, cap_out, extra max_len
    ([1], 1, 0, 1, 64, 32, 32, 0),
    ([0, 1, 33, 64], 32, 32, 2, 128, 64, 32, 0),
    ([100, 37, 36, 99], 36, 5, 3, 64, 128, 64, 20),
    ([700, 513, 64], 63, 0, 2, 128, 704, 96, 0),
    ([3000, 2999, 1025], 1024, 100, 2, 64, 3008, 1024, 0),
    ([5000], 4999, 4998, 1, 128, 5024, 5024, 0),
    ([2048, 2047], 1, 1, 2, 64, 2048, 32, 0),
    ([40000, 16385, 32768], 9000, 77, 1, 64, 40000, 9024, 0),     # more keys than a workgroup holds at once
]


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_evict_matches_oracle(case, ties):
    lens, budget, recent, H, D, cap, cap_out, extra = EVICT[case]
    log(f"evict {EVICT[case]} ties {ties}")
    rng = np.random.default_rng(200 + case)
    B = len(lens)
    cache = rng.integers(0, 256, (B, H, cap * (D + D // 16))).astype(np.uint8)
    w = np.exp(3 * rng.standard_normal((B, H, cap))).astype(np.float32)
    if ties:
        w = rng.choice(np.array([0.0, -0.0, 1.0, 1e-40, np.nan, np.inf, -np.inf, -2.0], np.float32), (B, H, cap))
    co = rng.integers(0, 256, (B, H, cap_out * (D + D // 16))).astype(np.uint8)
    out = dict(cache=torch.as_tensor(co).cuda(), weight=torch.full((B, H, cap_out), 5.0, device="cuda"),
               kept_index=torch.full((B, H, budget), -7, dtype=torch.int32, device="cuda"))
    wt = torch.zeros((w.size + 1,), device="cuda")[1:].view(w.shape) if case % 2 else torch.zeros(w.shape, device="cuda")
    wt.copy_(torch.as_tensor(w))              # every other case: not aligned to 16 bytes
    r = lv.cache4_evict(torch.as_tensor(cache).cuda(), D, wt, dev(lens), budget, recent,
                        min(cap, max(lens) + extra), out=out)
    src, dst, old = (c4.split_cache(x, D) for x in (cache, r["cache"].cpu().numpy(), co))
    kept, wo = r["kept_index"].cpu().numpy(), r["weight"].cpu().numpy()
    assert r["lengths"].tolist() == [min(n, budget) for n in lens]
    for b in range(B):
        for g in range(H):
            want = c4.evict(w[b, g], lens[b], budget, recent)
            L = len(want)
            assert kept[b, g, :L].tolist() == want.tolist(), (b, g)
            assert (kept[b, g, L:] == -7).all()
            for a, s, o in zip(dst, src, old):
                assert np.array_equal(a[b, g, :L], s[b, g, want]), (b, g)
                assert np.array_equal(a[b, g, L:], o[b, g, L:]), (b, g)
            assert np.array_equal(wo[b, g, :L].view(np.int32), w[b, g, want].view(np.int32))
            assert (wo[b, g, L:] == 5).all()


# ----------------------------------------------------------------------------- verification

def run_verify(draft, n, p, q, u, r, dtype="f32", lengths=None):
    t = lambda x: None if x is None else torch.as_tensor(x).to(DT[dtype]).cuda()  # noqa: E731
    return lv.verify_draft(dev(draft), t(p), t(q), torch.as_tensor(u).float().cuda(), torch.as_tensor(r).float().cuda(),
                           n_draft=None if n is None else dev(n), lengths=None if lengths is None else dev(lengths))


VERIFY = [
    # B, m, V, dtype, proposal
    (1, 1, 1, "f32", True),
    (3, 1, 2, "bf16", False),
    (5, 4, 63, "f32", True),
    (4, 64, 129, "f32", False),
    (7, 3, 4096, "bf16", True),
    (2, 5, 4097, "f32", True),
    (5, 2, 8192, "f32", False),
    (5, 2, 8193, "bf16", True),
    (4, 3, 30001, "f32", True),
    (4, 3, 32768, "bf16", False),
    (4, 3, 32769, "f32", True),
    (6, 7, 50257, "bf16", True),
    (6, 2, 131072, "f32", True),
    (256, 2, 300, "f32", True),
    (2, 3, 1200001, "f32", False),
]


@pytest.mark.parametrize("case", range(len(VERIFY)))
def test_verify_matches_oracle(case):
    B, m, V, dtype, prop = VERIFY[case]
    log(f"verify {VERIFY[case]}")
    rng = np.random.default_rng(300 + case)

    def probs(n):
        x = np.exp(2.0 * rng.standard_normal((B, n, V)))
        return torch.as_tensor(x / x.sum(-1, keepdims=True)).to(DT[dtype])

    p = probs(m + 1)
    q = torch.as_tensor(0.5 * p[:, :m].float().numpy() + 0.5 * probs(m).float().numpy()).to(DT[dtype]) if prop else None
    draft = rng.integers(0, V, (B, m))
    top = p[:, :m].float().argmax(-1).numpy()
    draft = np.where(rng.random((B, m)) < 0.7, top, draft)
    n = rng.integers(0, m + 1, B)
    n[0] = m
    u, r = rng.random((B, m)).astype(np.float32) ** 2, rng.random(B).astype(np.float32)
    lengths = rng.integers(m, 1000, B)
    got = run_verify(draft, n, p, q, u, r, dtype, lengths)
    pf, qf = p.double().numpy(), None if q is None else q.double().numpy()
    for b in range(B):
        tokens, a = c4.verify(draft[b], n[b], pf[b], None if q is None else qf[b], u[b], r[b])
        assert int(got["n_accepted"][b]) == a, b
        assert got["tokens"][b].tolist() == tokens.tolist(), b
        assert int(got["lengths"][b]) == lengths[b] - (n[b] - a), b


def test_verify_lengths_in_place():
    """Without counts every draft counts; the cached lengths may be updated where they are."""
    B, m, V = 4, 3, 50
    p = torch.full((B, m + 1, V), 1 / V, device="cuda")
    draft = torch.randint(0, V, (B, m), device="cuda").to(torch.int32)
    u = torch.tensor([[0.0, 0.0, 0.0], [0.0, 0.9, 0.0], [0.9, 0.0, 0.0], [0.0, 0.0, 0.9]], device="cuda")
    lengths = dev([10, 11, 12, 13])
    r = lv.verify_draft(draft, p, None, u, torch.full((B,), 0.5, device="cuda"), lengths=lengths, out=dict(lengths=lengths))
    # u < 1 / V accepts: 3, 1, 0 and 2 of 3 drafts
    assert r["n_accepted"].tolist() == [3, 1, 0, 2]
    assert lengths.tolist() == [10, 9, 9, 12] and r["lengths"] is lengths


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 9001, 40001])
def test_verify_edges(dtype, V):
    """Ties and borders (all exact in 64 bits), empty rows, values that are no probabilities."""
    m = 2
    rows = []

    def add(draft, n, p, q, u, r):
        rows.append((draft, n, p, q, u, r))

    even = np.zeros(V)
    even[[0, V - 1]] = 0.5
    one = np.zeros(V)
    one[V // 2] = 1.0
    none = np.zeros(V)
    wild = np.full(V, np.nan)
    wild[1], wild[2], wild[3], wild[V - 1] = np.inf, -1.0, 0.25, 0.25
    big = np.full(V, 3e38)
    q = np.stack([one, even])
    add([V // 2, 0], 2, [one, even, even], q, [0.999, 0.999], 0.5)      # all accepted; r on the border: the second
    add([V // 2, 0], 2, [one, even, even], q, [0.999, 0.999], 0.4999)
    add([V // 2, 0], 2, [one, one, even], q, [0.5, 0.0], 0.0)           # 0 * 0.5 < 0 refuses
    add([V // 2, 0], 2, [one, even, even], q, [0.5, math.nan], 0.3)     # nothing left of p - q: p
    add([0, 0], 2, [one, even, even], q, [0.0, 0.5], 0.7)               # q(x) = 0 < p(x) fails for p(x) = 0
    add([-1, 0], 2, [even, even, even], q, [0.0, 0.0], 0.9)
    add([V, 0], 2, [even, even, even], q, [0.0, 0.0], 0.9)
    add([V // 2, 0], 1, [none, none, none], q, [0.0, 0.0], 0.5)         # empty rows give no token
    add([V // 2, 0], 0, [wild, one, one], q, [0.0, 0.0], 0.6)
    add([V // 2, 0], 0, [even, one, one], q, [0.0, 0.0], 1.0)
    add([V // 2, 0], 0, [even, one, one], q, [0.0, 0.0], math.nan)
    add([V // 2, 0], 0, [even, one, one], q, [0.0, 0.0], -1.0)
    add([V // 2, 0], -3, [even, one, one], q, [0.0, 0.0], 0.5)          # counts are clamped
    add([V // 2, 0], 99, [one, even, one], q, [0.9, 0.9], 0.5)
    add([V // 2, 0], 0, [big, one, one], q, [0.0, 0.0], 0.5)
    draft, n, p, qq, u, r = (np.array([x[i] for x in rows]) for i in range(6))
    for prop in (qq, None):
        got = run_verify(draft, n, p, prop, u, r, dtype)
        pd = torch.as_tensor(p).to(DT[dtype]).double().numpy()
        qd = None if prop is None else torch.as_tensor(prop).to(DT[dtype]).double().numpy()
        for b in range(len(rows)):
            tokens, a = c4.verify(draft[b], n[b], pd[b], None if prop is None else qd[b], np.float32(u[b]), np.float32(r[b]))
            assert got["tokens"][b].tolist() == tokens.tolist(), (b, prop is None)
            assert int(got["n_accepted"][b]) == a, (b, prop is None)


# ----------------------------------------------------------------------------- together

def generation_step(s):
    """One step of a generation: the last token and the drafts enter the cache, are
    attended to, and are verified; the caches' live rows follow."""
    lv.cache4_append(s["cache"], s["k"], s["v"], s["cu"], s["start"], s["m"] + 1, weight=s["w"])
    lv.cache4_attn(s["cache"], s["q"], s["cu"], s["n"], s["m"] + 1, s["cap"], weight=s["w"], weight_rows=1, out=s["o"],
                   workspace=s["ws"])
    lv.verify_draft(s["draft"], s["p"], s["qp"], s["u"], s["r"], lengths=s["n"], workspace=s["vws"],
                    out=dict(tokens=s["tokens"], n_accepted=s["acc"], lengths=s["left"]))


def step_state(rng, B, Hq, H, D, cap, m, V, lens):
    s = dict(m=m, cap=cap, cu=dev(np.arange(B + 1) * (m + 1)), start=dev(lens), n=dev(np.array(lens) + m + 1))
    rows = B * (m + 1)
    for name, heads in (("q", Hq), ("k", H), ("v", H)):
        s[name] = torch.as_tensor(rng.standard_normal((rows, heads, D))).to(torch.bfloat16).cuda()
    s["cache"] = torch.as_tensor(random_cache(rng, B, H, D, cap)).cuda()
    s["w"] = torch.as_tensor(rng.random((B, H, cap)).astype(np.float32)).cuda()
    s["o"] = torch.zeros((rows, Hq, D), dtype=torch.bfloat16, device="cuda")
    p = np.exp(2 * rng.standard_normal((B, m + 1, V)))
    s["p"] = torch.as_tensor(p / p.sum(-1, keepdims=True)).float().cuda()
    s["qp"] = s["p"][:, :m].roll(1, 0).contiguous()
    s["draft"] = dev(rng.integers(0, V, (B, m)))
    s["u"], s["r"] = torch.rand((B, m), device="cuda") * 0.6, torch.rand((B,), device="cuda")
    s["tokens"], s["acc"], s["left"] = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in ((B, m + 1), (B,), (B,)))
    s["ws"] = torch.empty((lv.cache4_attn_workspace_bytes(torch.bfloat16, B, Hq, H, D, m + 1, cap, 1),), dtype=torch.uint8,
                          device="cuda")
    s["vws"] = torch.empty((lv.verify_draft_workspace_bytes(B, m, V),), dtype=torch.uint8, device="cuda")
    return s


def test_generation_steps_and_eviction_together():
    """Three steps of four samples, then an eviction and a fourth step on what it left, each against the oracle."""
    rng = np.random.default_rng(400)
    B, Hq, H, D, cap, m, V = 4, 8, 2, 128, 160, 3, 900
    lens = np.array([120, 0, 33, 77])
    host = None
    for step in range(4):
        log(f"generation step {step}: cached rows {lens.tolist()}")
        s = step_state(rng, B, Hq, H, D, cap, m, V, lens)
        if host is not None:
            s["cache"], s["w"] = host
        before, w0 = s["cache"].cpu().numpy(), s["w"].double().cpu().numpy()
        generation_step(s)
        kc, ks, vc, vs = c4.split_cache(before, D)
        cu = np.arange(B + 1) * (m + 1)
        kx, vx = s["k"].double().cpu().numpy(), s["v"].double().cpu().numpy()
        for b in range(B):
            at = slice(lens[b], lens[b] + m + 1)
            for codes, scales, x in ((kc, ks, kx), (vc, vs, vx)):
                c, e = c4.encode(x[cu[b]:cu[b + 1]])
                codes[b, :, at], scales[b, :, at] = c.transpose(1, 0, 2), e.transpose(1, 0, 2)
            w0[b, :, at] = 0
        cache = c4.join_cache(kc, ks, vc, vs)
        assert np.array_equal(cache, s["cache"].cpu().numpy())
        check_attn(cache, s["q"].double().cpu().numpy(), cu, (lens + m + 1).tolist(), Hq, D, "bf16", 1, w0,
                   s["o"].double().cpu().numpy(), s["w"].double().cpu().numpy(), f"step {step}")
        p, qp = s["p"].double().cpu().numpy(), s["qp"].double().cpu().numpy()
        for b in range(B):
            tokens, a = c4.verify(s["draft"][b].tolist(), m, p[b], qp[b], s["u"][b].cpu().numpy(), float(s["r"][b]))
            assert s["tokens"][b].tolist() == tokens.tolist() and int(s["acc"][b]) == a
            assert int(s["left"][b]) == lens[b] + 1 + a
        lens = s["left"].cpu().numpy()
        host = s["cache"], s["w"]
        if step == 2:
            r = lv.cache4_evict(s["cache"], D, s["w"], s["left"], 64, 16, cap, cap_out=cap)
            wh = s["w"].cpu().numpy()
            for b in range(B):
                for g in range(H):
                    want = c4.evict(wh[b, g], int(lens[b]), 64, 16)
                    assert r["kept_index"][b, g, :len(want)].tolist() == want.tolist()
                    assert np.array_equal(r["weight"][b, g, :len(want)].cpu().numpy(), wh[b, g, want])
            moved = c4.split_cache(r["cache"].cpu().numpy(), D)
            for a, x in zip(moved, c4.split_cache(cache, D)):
                for b in range(B):
                    for g in range(H):
                        want = c4.evict(wh[b, g], int(lens[b]), 64, 16)
                        assert np.array_equal(a[b, g, :len(want)], x[b, g, want])
            lens = r["lengths"].cpu().numpy()
            host = r["cache"], r["weight"]


def test_generation_step_in_a_graph_and_on_another_stream():
    """The step and an eviction captured once: every replay, with other work and
    synchronisations between, gives the eager results; so does another stream."""
    rng = np.random.default_rng(500)
    B, Hq, H, D, cap, m, V = 3, 8, 4, 64, 1280, 2, 5000
    s = step_state(rng, B, Hq, H, D, cap, m, V, [1100, 40, 600])
    out = dict(cache=lv.cache4_empty(B, H, D, 512), weight=torch.zeros((B, H, 512), device="cuda"),
               lengths=torch.zeros((B,), dtype=torch.int32, device="cuda"),
               kept_index=torch.zeros((B, H, 500), dtype=torch.int32, device="cuda"))
    first = {k: s[k].clone() for k in ("cache", "w")}

    def whole():
        generation_step(s)
        lv.cache4_evict(s["cache"], D, s["w"], s["n"], 500, 20, cap, out=out)

    def reset():
        for k, x in first.items():
            s[k].copy_(x)
        for t in list(out.values()) + [s["o"], s["tokens"], s["left"]]:
            t.zero_()
        s["ws"].fill_(0x55)
        s["vws"].fill_(0x55)
        torch.cuda.synchronize()

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in [s["o"], s["w"], s["tokens"], s["acc"], s["left"], s["cache"], *out.values()]]

    reset()
    whole()
    want = results()
    side = torch.cuda.Stream()
    reset()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        whole()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(results(), want):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(g):
        whole()
    for rep in range(3):
        reset()
        g.replay()
        for a, b in zip(results(), want):
            assert torch.equal(a, b), f"replay {rep}"
        generation_step(s)
