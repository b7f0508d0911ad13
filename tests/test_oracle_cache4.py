"""The oracle of the 4-bit cache and of the draft verification, pinned without a
GPU: against the OCP number formats, closed forms, enumeration and the decode
attention's own oracle."""
import itertools
import math

import numpy as np
import pytest

import oracle
from oracle import cache4 as c4


def test_e2m1_values_follow_the_format():
    # sign, two exponent bits with bias 1, one mantissa bit, subnormals at exponent 0
    for code in range(16):
        e, m = (code >> 1) & 3, code & 1
        mag = 0.5 * m if e == 0 else (1 + 0.5 * m) * 2.0 ** (e - 1)
        want = -mag if code & 8 else mag
        got = c4.decode(np.full(32, code, np.uint8), np.array([127], np.uint8))
        assert (got == want).all()


def test_scale_is_the_least_that_covers_the_block():
    for top, E in [(7.0, 0), (np.nextafter(7.0, 8), 1), (6.0, 0), (3.5, -1), (3.51, 0), (1.0, -2), (0.0, -125),
                   (1e-45, -125), (7 * 2.0 ** -125, -125), (3.4e38, 125)]:
        x = np.zeros(32)
        x[5] = top
        _, s = c4.encode_block(x)
        assert s == E + 127, (top, s)


def test_ties_go_to_the_even_code_and_large_values_saturate():
    y = np.zeros(32)
    y[:9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, -0.75]
    codes, s = c4.encode_block(y)
    assert s == 127
    assert codes[:9].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 10]


def test_rounding_is_within_one_scale_and_values_survive():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 64)) * np.exp2(rng.integers(-20, 20, (50, 1)))
    codes, s = c4.encode(x)
    y = c4.decode(codes, s)
    step = np.repeat(2.0 ** (s.astype(float) - 127), 32, -1)
    assert (np.abs(x - y) <= step).all()
    # a value of the format decodes to itself, whatever scale it gets
    codes2, s2 = c4.encode(y)
    assert np.array_equal(c4.decode(codes2, s2), y)


def test_blocks_with_nan_or_infinity_read_as_nan():
    x = np.ones(64)
    x[3] = np.inf
    codes, s = c4.encode(x)
    y = c4.decode(codes, s)
    assert s.tolist() == [255, 125] and np.isnan(y[:32]).all() and (y[32:] == 1).all()


def test_cache_bytes_round_trip():
    rng = np.random.default_rng(4)
    kc, vc = (rng.integers(0, 16, (2, 3, 32, 64)).astype(np.uint8) for _ in range(2))
    ks, vs = (rng.integers(0, 256, (2, 3, 32, 2)).astype(np.uint8) for _ in range(2))
    cache = c4.join_cache(kc, ks, vc, vs)
    assert cache.shape == (2, 3, 32 * (64 + 4))
    for a, b in zip(c4.split_cache(cache, 64), (kc, ks, vc, vs)):
        assert np.array_equal(a, b)
    # the byte of elements 2c, 2c+1 of a row, and a scale's place
    assert cache[1, 2, 5 * 32 + 7] == kc[1, 2, 5, 14] | (kc[1, 2, 5, 15] << 4)
    assert cache[1, 2, 2 * 32 * 32 + 1 * 32 + 9] == ks[1, 2, 9, 1]


def test_attention_of_one_query_is_the_decode_attention():
    rng = np.random.default_rng(5)
    B, Hq, H, D, lens = 3, 4, 2, 64, [5, 1, 9]
    K, V = rng.standard_normal((2, B, H, 32, D))
    q = rng.standard_normal((B, Hq, D))
    o, w, _, _ = c4.attention(q, np.arange(B + 1), K, V, lens, 1 / math.sqrt(D), 1)
    cu = np.concatenate(([0], np.cumsum([n - 1 for n in lens])))
    kc = np.concatenate([K[b, :, :n - 1].transpose(1, 0, 2) for b, n in enumerate(lens)])
    vc = np.concatenate([V[b, :, :n - 1].transpose(1, 0, 2) for b, n in enumerate(lens)])
    k1 = np.stack([K[b, :, n - 1] for b, n in enumerate(lens)])
    v1 = np.stack([V[b, :, n - 1] for b, n in enumerate(lens)])
    ref = oracle.decode_attention(q, k1, v1, kc, vc, cu, Hq, H, 1 / math.sqrt(D))
    assert np.abs(o - ref).max() < 1e-12
    assert np.allclose(w.sum(-1), Hq // H)


def test_attention_is_causal_over_the_newest_tokens():
    rng = np.random.default_rng(6)
    K, V = rng.standard_normal((2, 1, 1, 32, 64))
    q = rng.standard_normal((4, 1, 64))
    o, _, _, _ = c4.attention(q, [0, 4], K, V, [3], 0.125)
    assert (o[0] == 0).all()                       # the first of 4 queries over 3 rows sees none
    for i in (1, 2, 3):
        one, _, _, _ = c4.attention(q[i:i + 1], [0, 1], K, V, [i], 0.125)
        assert np.abs(o[i] - one[0]).max() < 1e-14


def test_evict_keeps_recent_rows_and_the_heaviest():
    w = np.array([3.0, 1.0, 3.0, np.nan, 0.0, 9.0, 0.0])
    assert c4.evict(w, 7, 8, 2).tolist() == list(range(7))
    assert c4.evict(w, 7, 4, 2).tolist() == [0, 3, 5, 6]      # NaN first, then 3.0 at the lower position
    assert c4.evict(w, 7, 3, 3).tolist() == [4, 5, 6]
    assert c4.evict(w, 7, 2, 0).tolist() == [3, 5]


@pytest.mark.parametrize("proposal", [True, False])
def test_verification_draws_from_the_target(proposal):
    """Over all drafts and a fine grid of (u, r) the first token's distribution is the target's."""
    p = np.array([[0.5, 0.125, 0.25, 0.125], [0.25, 0.25, 0.25, 0.25]])
    q = np.array([[0.25, 0.25, 0.5, 0.0]])
    grid = (np.arange(64) + 0.5) / 64
    got = np.zeros(4)
    for x in range(4):
        share = q[0, x]
        for u, r in itertools.product(grid, grid):
            tokens, a = c4.verify([x], 1, p, q if proposal else None, [u], r)
            assert a == (tokens[1] >= 0)
            got[tokens[0]] += share / len(grid) ** 2
    # without a proposal the drafted token is accepted with p(x) and otherwise replaced in proportion
    want = p[0] if proposal else sum(q[0, x] * p[0] for x in range(4))
    assert np.abs(got - want).max() < 1 / 64


def test_verification_edges():
    p = np.array([[0.0, 1.0, 0.0], [0.5, 0.0, 0.5], [0.0, 0.0, 0.0]])
    q = np.array([[0.0, 1.0, 0.0], [1.0, 0.0, 0.0]])
    t, a = c4.verify([1, 0], 2, p, q, [0.0, 0.0], 0.0)        # both accepted, nothing to draw from
    assert a == 2 and t.tolist() == [1, 0, -1]
    t, a = c4.verify([1, 0], 2, p, q, [0.0, 0.9], 0.0)        # 0.9 * 1 < 0.5 fails: the rest is token 2
    assert a == 1 and t.tolist() == [1, 2, -1]
    t, a = c4.verify([1, 0], 1, p, q, [0.0, 0.9], 0.5)        # one draft: drawn from the target; 0.5 is not past r
    assert a == 1 and t.tolist() == [1, 2, -1]
    t, a = c4.verify([7, 0], 2, p, q, [0.0, 0.0], 0.0)        # a token that is none is refused
    assert a == 0 and t.tolist() == [1, -1, -1]               # p - q is empty: from the target
    t, a = c4.verify([0, 0], 0, p, q, [0.0, 0.0], 1.0)        # r = 1: the last there is
    assert a == 0 and t.tolist() == [1, -1, -1]
