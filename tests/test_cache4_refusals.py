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
