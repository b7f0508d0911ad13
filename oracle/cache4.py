"""Plain float64 definitions of the 4-bit cache and of the draft verification
(test infrastructure only).

Paper: LiteVLM (arXiv 2506.07416), Results section (decoding against the cached
keys and values), Related Work (tokens ranked by the attention they receive),
Design section (drafted candidates verified by the target model).
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode_block(x: np.ndarray):
    """Codes (0..15) and scale byte of one block of 32 float64 values: the least E
    in [-125, 125] with max|x| <= 7 * 2^E, codes nearest to x * 2^-E, ties to the
    even code, values beyond 6 to 6; a block with a NaN or an infinity is byte 255."""
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    top, E = float(np.abs(x).max()), -125
    while E < 125 and top > 7.0 * 2.0 ** E:
        E += 1
    codes = np.zeros(32, np.uint8)
    for i, v in enumerate(np.abs(x) * 2.0 ** -E):
        dist = np.abs(E2M1 - v)
        near = np.nonzero(dist == dist.min())[0]
        codes[i] = near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]
    return codes + 8 * np.signbit(x).astype(np.uint8), E + 127


def encode(x: np.ndarray):
    """[..., D] to codes [..., D] and scale bytes [..., D/32]."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    out = [encode_block(b) for b in blocks]
    codes = np.array([c for c, _ in out], np.uint8).reshape(x.shape)
    return codes, np.array([s for _, s in out], np.uint8).reshape(x.shape[:-1] + (-1,))


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values of codes [..., D] with scale bytes [..., D/32]."""
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return v * np.repeat(s, 32, axis=-1)


def split_cache(cache: np.ndarray, D: int):
    """The K codes, K scales, V codes, V scales of a cache [B, H, bytes]: codes
    [B, H, cap, D] (unpacked) and scale bytes [B, H, cap, D/32]."""
    B, H, n = cache.shape
    cap = n // (D + D // 16)
    half, sc = cap * D // 2, cap * D // 32
    out = []
    for c0, s0 in ((0, 2 * half), (half, 2 * half + sc)):
        c = cache[:, :, c0:c0 + half].reshape(B, H, cap, D // 2)
        codes = np.stack((c & 15, c >> 4), -1).reshape(B, H, cap, D)
        scales = cache[:, :, s0:s0 + sc].reshape(B, H, D // 32, cap).transpose(0, 1, 3, 2)
        out += [codes, scales]
    return out


def join_cache(kc, ks, vc, vs) -> np.ndarray:
    """The cache bytes of unpacked codes [B, H, cap, D] and scales [B, H, cap, D/32]."""
    B, H = kc.shape[:2]
    packed = [(c[..., 0::2] | (c[..., 1::2] << 4)).reshape(B, H, -1) for c in (kc, vc)]
    scales = [s.transpose(0, 1, 3, 2).reshape(B, H, -1) for s in (ks, vs)]
    return np.concatenate(packed + scales, -1).astype(np.uint8)


def attention(q, cu_q, K, V, lengths, scale, weight_rows=0):
    """q [rows, Hq, D]; K, V [B, H, cap, D] (values); the queries of a sample are its
    newest tokens. Returns (o [rows, Hq, D], added weight [B, H, cap], and for the
    error bounds: A [rows, Hq, D] = sum_j p_j |V_j|, and [rows, Hq] the largest
    sum_d |q_d K_jd| * scale over the keys that the query sees)."""
    rows, Hq, D = q.shape
    B, H, cap, _ = K.shape
    G = Hq // H
    o, A, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    w = np.zeros((B, H, cap))
    for b in range(B):
        n, m = int(lengths[b]), int(cu_q[b + 1] - cu_q[b])
        for i in range(m):
            see = n - m + i + 1
            if see < 1:
                continue
            r = cu_q[b] + i
            for h in range(Hq):
                k, v = K[b, h // G, :see], V[b, h // G, :see]
                with np.errstate(all="ignore"):
                    x = k @ q[r, h] * scale
                    e = np.exp(x - x.max())
                    p = e / e.sum()
                    o[r, h] = p @ v
                    A[r, h] = p @ np.abs(v)
                    size[r, h] = (np.abs(k) @ np.abs(q[r, h])).max() * scale
                if i < weight_rows:
                    w[b, h // G, :see] += p
    return o, w, A, size


def evict(weight: np.ndarray, n: int, budget: int, recent: int) -> np.ndarray:
    """Positions kept of one head's n rows, ascending."""
    if n <= budget:
        return np.arange(n)
    old = n - recent
    ranked = sorted(range(old), key=lambda j: (0 if np.isnan(weight[j]) else 1,
                                               0.0 if np.isnan(weight[j]) else -float(weight[j]), j))
    return np.array(sorted(ranked[:budget - recent]) + list(range(old, n)), np.int64)


def verify(draft, n, target, proposal, u, r):
    """One sample: draft [m], n drafts, target [m+1, V], proposal [m, V] or None,
    u [m], r. Returns (tokens [m+1], accepted)."""
    m, V = len(draft), target.shape[1]
    n = min(max(int(n), 0), m)
    a = 0
    while a < n:
        x = int(draft[a])
        if not 0 <= x < V:
            break
        qx = 1.0 if proposal is None else float(proposal[a, x])
        if not float(u[a]) * qx < float(target[a, x]):
            break
        a += 1
    p = target[a].astype(np.float64)
    with np.errstate(invalid="ignore"):
        if a == n:
            w = p.copy()
        elif proposal is None:
            w = p - (np.arange(V) == int(draft[a]))
        else:
            w = p - proposal[a].astype(np.float64)
        w = np.where(np.isfinite(w) & (w > 0), w, 0.0)
        p = np.where(np.isfinite(p) & (p > 0), p, 0.0)
    if not w.any():
        w = p
    token, live = -1, np.nonzero(w)[0]
    if len(live):
        run = np.cumsum(w)
        hit = live[run[live] > float(r) * run[-1]]
        token = int(hit[0]) if len(hit) else int(live[-1])
    tokens = np.full(m + 1, -1, np.int64)
    tokens[:a] = draft[:a]
    tokens[a] = token
    return tokens, a
