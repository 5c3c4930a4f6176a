"""What the Python binding of include/otas_decode.h refuses before the library is called, without a GPU: objects are made without their memory, and the
library is one whose calls fail the test."""
import types

import pytest
import torch

from paper_2401_05031_amd import binding

H, KV, DH = 4, 2, 64


class NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


def context():
    ctx = binding.Context.__new__(binding.Context)
    ctx._lib, ctx._h, ctx.H, ctx.D, ctx.torch_dtype, ctx.device_index = NoLibrary(), None, H, H * DH, torch.bfloat16, 0
    ctx._need = lambda name, t, shape, dtype: 4096
    return ctx


def cache(cls, **more):
    c = cls.__new__(cls)
    c.slots, c.kv_heads, c.capacity, c.head_width, c.device_index, c.dtype, c.address = 2, KV, 32, DH, 0, torch.bfloat16, 8192
    for name, value in more.items():
        setattr(c, name, value)
    return c


def rows(n):
    return torch.empty((n, (H + 2 * KV) * DH), dtype=torch.bfloat16, device="meta")


def calls(ctx, c, four):
    """Every call with a cache, of one in 4 bits or of the others."""
    if four:
        yield lambda: ctx.otas_cache4_append(c, rows(2), [0, 2], None, [0], [0])
        yield lambda: ctx.otas_cache4_read(c, [0], [0], [0, 2], rows(2))
        yield lambda: ctx.otas_attention_cache4(c, rows(2), [0, 2], [0], [2], torch.empty(16, dtype=torch.uint8), rows(2), 5)
    else:
        yield lambda: ctx.otas_cache_append(c, rows(2), [0, 2], None, None, [0], [0])
        yield lambda: ctx.otas_attention_tree(c, rows(2), [0, 2], None, None, [0], [2], torch.empty(16, dtype=torch.uint8), rows(2))
        yield lambda: ctx.otas_cache_evict(c, [0], [2], [1], torch.empty(16, dtype=torch.uint8))
        yield lambda: ctx.otas_attention_recent(c, rows(2), [0, 2], [0], [2], torch.empty(16, dtype=torch.uint8), rows(2), 5)


@pytest.mark.parametrize("four", [False, True])
def test_a_cache_of_the_other_kind_is_refused(four):
    """Their descriptions are alike in memory (four addresses, three numbers): a call would take positions and mass for scales, and write past them."""
    ctx = context()
    right, wrong = (binding.KVCache4, binding.KVCache) if four else (binding.KVCache, binding.KVCache4)
    for call in calls(ctx, cache(right), four):
        with pytest.raises(AssertionError, match="was called"):
            call()
    for c in (cache(wrong, mass=torch.empty(2, 32, device="meta")), types.SimpleNamespace(**vars(cache(right))), None):
        for call in calls(ctx, c, four):
            with pytest.raises(ValueError, match="cache"):
                call()
