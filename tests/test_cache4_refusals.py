"""What the Python binding and the library refuse, beyond test_abi_cache4: on the host,
with stand-ins for tensors of the GPU. No call is enqueued."""
import pytest
import torch

import paper_2506_07416_amd as lv


class OnGpu(torch.Tensor):
    """A host tensor that says it is on a GPU: what the binding's checks look at."""
    index = 0

    def get_device(self):
        return self.index


def on_gpu(t, index=0):
    t = t.as_subclass(OnGpu)
    t.index = index
    return t


@pytest.fixture
def calls(monkeypatch):
    """The library calls that pass the binding's checks, in place of making them."""
    made = []
    monkeypatch.setattr(lv, "_enqueue", lambda call, dev, *args: made.append((call, dev, args)))
    return made


def evict_args(D=64, B=2, H=2, cap=64):
    cache = on_gpu(torch.zeros((B, H, cap * (D + D // 16)), dtype=torch.uint8))
    return cache, D, on_gpu(torch.zeros((B, H, cap))), on_gpu(torch.zeros((B,), dtype=torch.int32))


def evict_out(D=64, B=2, H=2, cap=32, budget=20):
    return dict(cache=on_gpu(torch.zeros((B, H, cap * (D + D // 16)), dtype=torch.uint8)),
                weight=on_gpu(torch.zeros((B, H, cap))), lengths=on_gpu(torch.zeros((B,), dtype=torch.int32)),
                kept_index=on_gpu(torch.zeros((B, H, budget), dtype=torch.int32)))


def test_evict_refuses_a_new_cache_elsewhere(calls):
    lv.cache4_evict(*evict_args(), 20, 4, 64, out=evict_out())
    assert len(calls) == 1
    for index in (-1, 1):                    # the host; another GPU
        for name in ("cache", "weight", "lengths", "kept_index"):
            out = evict_out()
            out[name].index = index
            with pytest.raises(ValueError, match="device"):
                lv.cache4_evict(*evict_args(), 20, 4, 64, out=out)
    assert len(calls) == 1


# ----------------------------------------------------------------------------- buffers that overlap

def at(i):
    """Fake buffers far apart: the library's checks read none of them."""
    return 0x7F0000000000 + (i << 36)


VERIFY_IN = dict(draft=at(0), nd=at(1), p=at(2), q=at(3), u=at(4), r=at(5), ln=at(6))
VERIFY_OUT = dict(tk=at(7), na=at(8), lo=at(9))


def verify(B=3, m=4, V=40000, dt=lv._abi.F32, ws=at(10), wsb=0, **a):
    a = {**VERIFY_IN, **VERIFY_OUT, **a}
    # too small a workspace: a call whose buffers are accepted ends there, on the host
    return lv.load().litevlm_verify_draft(dt, B, m, V, a["draft"], a["nd"], a["p"], a["q"], a["u"], a["r"], a["ln"], a["tk"],
                                          a["na"], a["lo"], ws, wsb, None)


def test_verify_refuses_outputs_over_inputs_and_each_other():
    B, m, V = 3, 4, 40000
    bad, fine = lv._abi.ERR_BAD_VALUE, lv._abi.ERR_WORKSPACE
    size = dict(draft=B * m, nd=B, p=B * (m + 1) * V, q=B * m * V, u=B * m, r=B, ln=B, tk=B * (m + 1), na=B, lo=B)
    assert verify() == fine
    for out in VERIFY_OUT:
        for other in list(VERIFY_IN) + list(VERIFY_OUT):
            if other == out:
                continue
            base = {**VERIFY_IN, **VERIFY_OUT}[other]
            n, own = 4 * size[other], 4 * size[out]
            same = fine if (out, other) in (("lo", "ln"), ("ln", "lo")) else bad
            assert verify(**{out: base}) == same, (out, other)
            for off in (4 - own, n - 4) if own > 4 else (n - 4,):
                if off:
                    assert verify(**{out: base + off}) == bad, (out, other, off)
            assert verify(**{out: base + n}) == fine and verify(**{out: base - own}) == fine, (out, other)
    half = dict(dt=lv._abi.BF16)              # two bytes a probability
    assert verify(**half, tk=at(2) + 2 * size["p"]) == fine and verify(**half, tk=at(2) + 2 * size["p"] - 4) == bad
    # what is not given is not looked at
    assert verify(nd=None, q=None, ln=None, lo=at(7)) == fine


def test_verify_refuses_a_workspace_over_its_buffers():
    wsb = lv.verify_draft_workspace_bytes(3, 4, 40000)
    for name in list(VERIFY_IN) + list(VERIFY_OUT):
        base = {**VERIFY_IN, **VERIFY_OUT}[name]
        assert verify(ws=base, wsb=wsb) == lv._abi.ERR_BAD_VALUE, name


def attn(dt=lv._abi.BF16, B=2, Hq=8, H=2, D=128, cap=2048, mq=4, ml=2048, wr=1, q=at(0), cu=at(1), cache=at(2), ln=at(3),
         scale=0.1, o=at(4), wi=at(5), wo=at(6), ws=at(7), wsb=0):
    return lv.load().litevlm_cache4_attn(dt, B, Hq, H, D, cap, mq, ml, wr, q, cu, cache, ln, scale, o, wi, wo, ws, wsb, None)


def test_attention_refuses_weights_over_its_inputs():
    bad, fine = lv._abi.ERR_BAD_VALUE, lv._abi.ERR_WORKSPACE
    n = 2 * 2 * 2048 * 4
    assert attn() == fine and attn(wi=at(6)) == fine            # in place
    for off in (4, -4, n - 4, 4 - n):
        assert attn(wo=at(5) + off) == bad, off
    assert attn(wo=at(5) + n) == fine and attn(wo=at(5) - n) == fine
    assert attn(wo=at(2)) == bad and attn(wo=at(2) + 4 * 2048 * 136 - 4) == bad and attn(wo=at(2) + 4 * 2048 * 136) == fine
    assert attn(wo=at(1) + 8) == bad and attn(wo=at(1) + 12) == fine and attn(wo=at(3) + 4) == bad
    # without weights neither address counts
    assert attn(wr=0, wo=at(5) + 4) == fine and attn(wr=0, wo=at(2)) == fine
    wsb = lv.cache4_attn_workspace_bytes(torch.bfloat16, 2, 8, 2, 128, 4, 2048, 1)
    for at_ws in (at(2), at(5), at(6), at(1) - 16, at(3) - wsb + 16):
        assert attn(ws=at_ws, wsb=wsb) == bad


# ----------------------------------------------------------------------------- the same in the binding

def attn_args(rows=5, Hq=4, D=64, B=2, H=2, cap=64, q=None):
    cache = on_gpu(torch.zeros((B, H, cap * (D + D // 16)), dtype=torch.uint8))
    q = on_gpu(torch.zeros((rows, Hq, D))) if q is None else q
    i32 = lambda n: on_gpu(torch.zeros((n,), dtype=torch.int32))  # noqa: E731
    return cache, q, i32(B + 1), i32(B), 3, cap


def part(buf, first, shape):
    n = 1
    for k in shape:
        n *= k
    return on_gpu(buf[first:first + n].view(shape))


def test_attention_refuses_an_output_over_what_it_reads(calls):
    buf = torch.zeros((3 * 5 * 4 * 64,))
    q, n = part(buf, 0, (5, 4, 64)), 5 * 4 * 64
    lv.cache4_attn(*attn_args(q=q), out=part(buf, n, (5, 4, 64)))
    assert len(calls) == 1
    for first in (0, 256, n - 4):
        with pytest.raises(ValueError, match="out"):
            lv.cache4_attn(*attn_args(q=q), out=part(buf, first, (5, 4, 64)))
    with pytest.raises(ValueError, match="out"):
        lv.cache4_attn(*attn_args(q=part(buf, 4, (5, 4, 64))), out=part(buf, 0, (5, 4, 64)))
    # over the cache
    a = attn_args(q=q)
    with pytest.raises(ValueError, match="out"):
        lv.cache4_attn(*a, out=on_gpu(a[0].view(-1)[64:64 + 4 * n].view(torch.float32).view(5, 4, 64)))
    # over the weights
    w = part(buf, n, (2, 2, 64))
    for kw in (dict(weight=w), dict(weight_out=w)):
        with pytest.raises(ValueError, match="out"):
            lv.cache4_attn(*attn_args(q=q), out=part(buf, n + 128, (5, 4, 64)), weight_rows=1, **kw)
    assert len(calls) == 1


def test_read_refuses_outputs_over_each_other_and_the_cache(calls):
    cache, i32 = on_gpu(torch.zeros((2, 2, 64 * 136), dtype=torch.uint8)), lambda n: on_gpu(torch.zeros((n,), dtype=torch.int32))
    buf = torch.zeros((2 * 5 * 2 * 128 + 4,))
    n, shape = 5 * 2 * 128, (5, 2, 128)
    read = lambda k, v: lv.cache4_read(cache, 128, i32(3), i32(2), 3, out=(k, v))  # noqa: E731
    read(part(buf, 0, shape), part(buf, n, shape))
    read(part(buf, n + 4, shape), part(buf, 4, shape))
    assert len(calls) == 2
    inside = on_gpu(cache.view(-1)[:4 * n].view(torch.float32).view(shape))
    for k, v in ((part(buf, 0, shape), part(buf, 0, shape)), (part(buf, 0, shape), part(buf, n - 4, shape)),
                 (part(buf, 4, shape), part(buf, 0, shape)), (inside, part(buf, 0, shape)), (part(buf, 0, shape), inside)):
        with pytest.raises(ValueError, match="overlap"):
            read(k, v)
    assert len(calls) == 2
    # without rows there is nothing to share
    none = torch.zeros((0, 2, 128))
    lv.cache4_read(cache, 128, i32(3), i32(2), 3, out=(on_gpu(none), on_gpu(none)))
    k, v = calls[-1][2][-2:]
    assert k != v and k % 16 == v % 16 == 0


def test_read_refuses_one_address_for_keys_and_values():
    read = lambda k, v, B=2: lv.load().litevlm_cache4_read(lv._abi.BF16, B, 2, 128, 64, 8, at(2), at(3), at(4), k, v,  # noqa: E731
                                                           None)
    assert read(at(0), at(0)) == lv._abi.ERR_BAD_VALUE
    assert read(at(0), at(0), B=0) == lv._abi.ERR_BAD_SHAPE


def test_attention_refuses_scales_beyond_fp32():
    """The kernels take logits to the base 2: softmax_scale * log2(e), which 2.4e38 carries past fp32."""
    for scale in (2.4e38, 3.4e38):
        assert attn(scale=scale) == lv._abi.ERR_BAD_VALUE
    for scale in (2.3e38, 1e-45):
        assert attn(scale=scale) == lv._abi.ERR_WORKSPACE


def test_append_refuses_weights_over_the_cache_and_either_over_its_counts():
    bad, nbytes = lv._abi.ERR_BAD_VALUE, 2 * 2 * 64 * 136

    def append(cu=at(2), start=at(3), cache=at(4), weight=at(5), B=2):
        # with refused arguments only: an accepted call would be enqueued
        return lv.load().litevlm_cache4_append(lv._abi.BF16, B, 2, 128, 64, 8, at(0), at(1), cu, start, cache, weight, None)

    assert append(B=0) == lv._abi.ERR_BAD_SHAPE
    for off in (0, nbytes - 4, 4 - 2 * 2 * 64 * 4):
        assert append(weight=at(4) + off) == bad, off
    assert append(weight=at(2)) == bad and append(weight=at(3) + 4) == bad
    assert append(cache=at(2) & ~15) == bad and append(start=at(4) + 32) == bad
