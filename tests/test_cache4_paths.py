"""The forms of the attention over the 4-bit cache that the GPU tests reach, from the
rule that chooses them, written here a second time and checked against the library's
workspace query: a rule that changes fails here instead of leaving a form untested."""
import itertools

import pytest
import torch

import paper_2506_07416_amd as lv
import test_gpu_cache4 as base
import test_gpu_cache4_paths as paths

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ceil(a, b):
    return -(-a // b)


def form(dtype, B, Hq, H, D, max_q, max_len, weight_rows):
    """(row tiles, splits, what becomes of the logits, keys past the caches, workspace bytes)."""
    G = Hq // H
    rows, wrows, heads = max_q * G, weight_rows * G, B * H
    if rows <= 16:
        tiles = 1
    elif rows <= 32 and max_len <= 512:
        tiles = 2
    else:
        tiles = 1 if heads * ceil(rows, 16) * ceil(max_len, 128) <= 1536 else 2
    blocks = ceil(rows, 16 * tiles)
    groups, steps = max(heads * blocks, 1), max(ceil(max_len, 128), 1)
    want = ceil(512 if tiles == 1 or D == 64 else 256, groups)
    if tiles == 1:
        want = max(want, min(ceil(steps, 4), ceil(16384, groups)))
    want = min(want, steps)
    if max_len <= 512 and blocks == 1:
        want = 1
    splits = ceil(steps, ceil(steps, want))
    weights = weight_rows > 0 and max_len > 0
    kept = weights and wrows <= 8
    whole = kept and splits == 1 and blocks == 1 and max_len <= 512
    logits = "lds" if whole else "kept" if kept else "again" if weights else "none"
    once = logits != "again" and blocks == 1 and max_len * (D + D // 16) * heads > 128 << 20
    up = lambda x: (x + 255) & ~255  # noqa: E731
    total = up(heads * rows * splits * D * 4 if splits > 1 else 0)
    total += up(heads * rows * splits * 8 if splits > 1 or logits == "kept" else 0)
    total += up(heads * wrows * 8 if weights and not whole else 0)
    total += up(heads * wrows * ceil(max_len, 32) * 128 if logits == "kept" else 0)
    return tiles, splits, logits, once, max(total, 16)


def sizes():
    """Sizes of every parametrised attention call, as the tests make them."""
    for cases in (base.ATTN, paths.PATHS):
        for lens, nq, Hq, H, D, cap, dtype, wr, extra in cases:
            for w in (wr, 0):
                yield dtype, len(lens), Hq, H, D, max(nq), min(cap, max(lens) + extra), w
    for (B, Hq, H, D, cap, mq), dtype in itertools.product(paths.LONG, DT):
        for w in (0, 1, 3):
            yield dtype, B, Hq, H, D, mq, cap, w


def test_rule_is_the_library_s():
    for s in sizes():
        assert form(*s)[-1] == lv.cache4_attn_workspace_bytes(DT[s[0]], *s[1:]), s


@pytest.mark.parametrize("dtype,D", list(itertools.product(DT, (64, 128))))
def test_every_form_has_a_case(dtype, D):
    hit = set()
    for s in sizes():
        if s[0] == dtype and s[4] == D:
            tiles, splits, logits, once, _ = form(*s)
            hit.add((tiles, logits, once))
            hit.add((tiles, "unsplit" if splits == 1 else "few" if splits <= 4 else "many"))
    for tiles in (1, 2):
        want = {(tiles, x, False) for x in ("lds", "kept", "again", "none")}
        want |= {(tiles, x, True) for x in ("kept", "none")}
        want |= {(tiles, x) for x in ("unsplit", "few", "many")}
        assert want <= hit, sorted(want - hit, key=str)
