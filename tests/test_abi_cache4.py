"""Refusals of the 4-bit cache's calls and of the draft verification: every check
runs on the host, before any HIP call (fake, never-dereferenced addresses)."""
import os
import re

import pytest
import torch

import paper_2506_07416_amd as lv
from paper_2506_07416_amd import _abi

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "litevlm.h")
A = 0x7F0000000000


def at(i):
    """Fake buffers far apart."""
    return A + (i << 36)


def test_header_constants_match_binding():
    text = open(HEADER).read()
    assert int(re.search(r"LITEVLM_MAX_CACHE4 (\d+)", text).group(1)) == _abi.MAX_CACHE4
    assert int(re.search(r"LITEVLM_MAX_DRAFT (\d+)", text).group(1)) == _abi.MAX_DRAFT


def test_cache_bytes():
    f = lv.load().litevlm_cache4_bytes
    assert f(1, 1, 128, 32) == 32 * 136
    assert f(256, 128, 128, _abi.MAX_CACHE4) == 256 * 128 * 136 * _abi.MAX_CACHE4
    for bad in [(0, 1, 128, 32), (257, 1, 128, 32), (1, 0, 128, 32), (1, 129, 128, 32), (1, 1, 96, 32), (1, 1, 128, 0),
                (1, 1, 128, 48), (1, 1, 128, _abi.MAX_CACHE4 + 32), (1, 1, 128, -32)]:
        assert f(*bad) == 0, bad


def rows(call, dt=_abi.BF16, B=2, H=2, D=128, cap=64, most=8, k=at(0), v=at(1), cu=at(2), start=at(3), cache=at(4),
         weight=None):
    lib = lv.load()
    if call == "append":
        return lib.litevlm_cache4_append(dt, B, H, D, cap, most, k, v, cu, start, cache, weight, None)
    return lib.litevlm_cache4_read(dt, B, H, D, cap, most, cache, start, cu, k, v, None)


@pytest.mark.parametrize("call", ["append", "read"])
def test_rows_refusals(call):
    for name in ("k", "v", "cu", "start", "cache"):
        assert rows(call, **{name: None}) == _abi.ERR_NULL_POINTER
    assert rows(call, dt=_abi.FP8_E4M3) == _abi.ERR_UNSUPPORTED
    assert rows(call, dt=7) == _abi.ERR_UNSUPPORTED
    for bad in (dict(B=0), dict(B=257), dict(H=0), dict(D=32), dict(cap=33), dict(cap=0), dict(most=-1), dict(most=65),
                dict(B=256, cap=_abi.MAX_CACHE4, most=_abi.MAX_CACHE4)):
        assert rows(call, **bad) == _abi.ERR_BAD_SHAPE, bad
    for name in ("k", "v", "cache"):
        assert rows(call, **{name: A + 8}) == _abi.ERR_MISALIGNED
    for name in ("cu", "start"):
        assert rows(call, **{name: A + 2}) == _abi.ERR_MISALIGNED
    if call == "append":
        assert rows(call, weight=A + 1) == _abi.ERR_MISALIGNED


def attn(dt=_abi.BF16, B=2, Hq=8, H=2, D=128, cap=64, mq=4, ml=64, wr=1, q=at(0), cu=at(1), cache=at(2), ln=at(3),
         scale=0.1, o=at(4), wi=at(5), wo=at(5), ws=at(6), wsb=None):
    lib = lv.load()
    if wsb is None:
        wsb = lib.litevlm_cache4_attn_workspace(dt, B, Hq, H, D, mq, ml, wr)
    return lib.litevlm_cache4_attn(dt, B, Hq, H, D, cap, mq, ml, wr, q, cu, cache, ln, scale, o, wi, wo, ws, wsb, None)


def test_attn_refusals():
    for name in ("q", "cu", "cache", "ln", "o"):
        assert attn(**{name: None}) == _abi.ERR_NULL_POINTER
    assert attn(wo=None) == _abi.ERR_NULL_POINTER
    assert attn(dt=_abi.FP8_E4M3) == _abi.ERR_UNSUPPORTED
    for bad in (dict(B=0), dict(B=257), dict(Hq=0), dict(H=0), dict(Hq=9), dict(Hq=130), dict(D=96), dict(cap=40),
                dict(mq=-1), dict(ml=-1), dict(ml=65), dict(mq=_abi.MAX_CACHE4 + 1),
                dict(B=256, mq=_abi.MAX_CACHE4)):
        assert attn(**bad) == _abi.ERR_BAD_SHAPE, bad
    for bad in (dict(wr=-1), dict(wr=5), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(scale=-1.0), dict(o=at(0))):
        assert attn(**bad) == _abi.ERR_BAD_VALUE, bad
    for name in ("q", "cache", "o", "ws"):
        assert attn(**{name: A + 8}) == _abi.ERR_MISALIGNED
    for name in ("cu", "ln", "wi", "wo"):
        assert attn(**{name: A + 2}) == _abi.ERR_MISALIGNED
    big = dict(cap=2048, ml=2048)             # small calls need no workspace
    assert attn(ws=None, **big) == _abi.ERR_WORKSPACE
    assert attn(wsb=1, **big) == _abi.ERR_WORKSPACE
    lib = lv.load()
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 2, 128, 4, 2048, 1) > 16
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 2, 128, 4, 512, 1) == 16
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 2, 128, 4, 512, 4) > 16
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 2, 128, 4, 64, 1) > 0
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 3, 128, 4, 64, 1) == 0
    assert lib.litevlm_cache4_attn_workspace(_abi.BF16, 2, 8, 2, 128, 4, 64, 5) == 0


def evict(B=2, H=2, D=128, cap=64, cap_out=32, ml=64, budget=20, recent=4, c=at(0), w=at(1), ln=at(2), co=at(3),
          wo=at(4), lo=at(5), ki=at(6)):
    return lv.load().litevlm_cache4_evict(B, H, D, cap, cap_out, ml, budget, recent, c, w, ln, co, wo, lo, ki, None)


def test_evict_refusals():
    for name in ("c", "w", "ln", "co", "wo", "lo", "ki"):
        assert evict(**{name: None}) == _abi.ERR_NULL_POINTER
    for bad in (dict(B=0), dict(H=129), dict(D=48), dict(cap=65), dict(cap_out=31), dict(ml=65), dict(ml=-1),
                dict(budget=0), dict(budget=33)):
        assert evict(**bad) == _abi.ERR_BAD_SHAPE, bad
    assert evict(recent=21) == _abi.ERR_BAD_VALUE
    assert evict(recent=-1) == _abi.ERR_BAD_VALUE
    for name in ("c", "co"):
        assert evict(**{name: A + 8}) == _abi.ERR_MISALIGNED
    for name in ("w", "ln", "wo", "lo", "ki"):
        assert evict(**{name: A + 2}) == _abi.ERR_MISALIGNED
    # in place, or anywhere across an input or another output
    size = 2 * 2 * 64 * 136
    assert evict(co=at(0)) == _abi.ERR_BAD_VALUE
    assert evict(co=at(0) + size - 16) == _abi.ERR_BAD_VALUE
    assert evict(wo=at(1) + 16) == _abi.ERR_BAD_VALUE
    assert evict(lo=at(2)) == _abi.ERR_BAD_VALUE
    assert evict(ki=at(4)) == _abi.ERR_BAD_VALUE


def verify(dt=_abi.F32, B=2, m=3, V=40000, draft=at(0), nd=at(1), p=at(2), q=at(3), u=at(4), r=at(5), ln=at(6), tk=at(7),
           na=at(8), lo=at(9), ws=at(10), wsb=None):
    lib = lv.load()
    if wsb is None:
        wsb = lib.litevlm_verify_draft_workspace(B, m, V)
    return lib.litevlm_verify_draft(dt, B, m, V, draft, nd, p, q, u, r, ln, tk, na, lo, ws, wsb, None)


def test_verify_refusals():
    for name in ("draft", "p", "u", "r", "tk", "na", "lo"):
        assert verify(**{name: None}) == _abi.ERR_NULL_POINTER
    assert verify(dt=_abi.FP8_E4M3) == _abi.ERR_UNSUPPORTED
    for bad in (dict(B=0), dict(B=257), dict(m=0), dict(m=65), dict(V=0), dict(V=(1 << 24) + 1)):
        assert verify(**bad) == _abi.ERR_BAD_SHAPE, bad
    for name in ("p", "q", "ws"):
        assert verify(**{name: A + 8}) == _abi.ERR_MISALIGNED
    for name in ("draft", "nd", "u", "r", "ln", "tk", "na", "lo"):
        assert verify(**{name: A + 2}) == _abi.ERR_MISALIGNED
    assert verify(ws=None) == _abi.ERR_WORKSPACE
    assert verify(wsb=0) == _abi.ERR_WORKSPACE
    assert lv.load().litevlm_verify_draft_workspace(2, 3, 32768) == 16    # a small vocabulary needs none
    assert lv.load().litevlm_verify_draft_workspace(2, 3, 32769) > 16
    assert verify(nd=None, q=None, ln=None, lo=None, ws=None) == _abi.ERR_WORKSPACE   # optional arguments


def test_binding_refuses_tensors_that_do_not_fit():
    """Shapes, types, layouts and places are checked before any address is taken."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = torch.zeros((2, 2, 64 * 136), dtype=torch.uint8)
    k = torch.zeros((5, 2, 128))
    with pytest.raises(ValueError, match="GPU"):
        lv.cache4_append(cache, k, k, i32(3), i32(2), 4)
    with pytest.raises(ValueError, match="v"):
        lv.cache4_append(cache, k, k[:4], i32(3), i32(2), 4)
    with pytest.raises(ValueError, match="start"):
        lv.cache4_append(cache, k, k, i32(3), i32(3), 4)
    with pytest.raises(TypeError):
        lv.cache4_append(cache, k.half(), k.half(), i32(3), i32(2), 4)
    with pytest.raises(ValueError, match="bytes a position"):
        lv.cache4_append(cache[..., :-1].contiguous(), k, k, i32(3), i32(2), 4)
    q = torch.zeros((2, 4, 128))
    with pytest.raises(ValueError, match="lengths"):
        lv.cache4_attn(cache, q, i32(3), torch.zeros(2), 1, 64)
    with pytest.raises(ValueError, match="weight"):
        lv.cache4_attn(cache, q, i32(3), i32(2), 1, 64, weight_rows=1)
    with pytest.raises(ValueError, match="q"):
        lv.cache4_attn(cache, q.transpose(0, 1).contiguous().transpose(0, 1), i32(3), i32(2), 1, 64,
                       out=torch.zeros((2, 4, 128)))
    with pytest.raises(ValueError, match="weight"):
        lv.cache4_evict(cache, 128, torch.zeros((2, 2, 63)), i32(2), 10, 2, 64)
    p = torch.zeros((2, 4, 9))
    with pytest.raises(ValueError, match="proposal"):
        lv.verify_draft(i32(2, 3), p, p, torch.zeros((2, 3)), torch.zeros(2))
    with pytest.raises(ValueError, match="GPU"):
        lv.verify_draft(i32(2, 3), p, None, torch.zeros((2, 3)), torch.zeros(2))
