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


class Tensor:
    """As much of a tensor as the binding looks at."""

    def __init__(self, address, shape, dtype=torch.bfloat16, device=0):
        self.address, self.shape, self.dtype, self.device = address, torch.Size(shape), dtype, device

    def data_ptr(self):
        return self.address

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def __len__(self):
        return self.shape[0]


class Recorder:
    """A library that keeps the arguments of its last call and returns success."""
    last = None

    def __getattr__(self, name):
        def call(*args):
            self.last = name, args
            return 0
        return call


def recording():
    ctx = context()
    del ctx._need
    ctx._lib = Recorder()
    return ctx, Tensor(4096, (3, (H + 2 * KV) * DH)), Tensor(1 << 20, (3,), torch.int32)


def described(kind, address):
    return kind.from_address(address)


def test_the_gains_that_a_call_checks_are_those_that_it_passes():
    """Tensors assigned to a description after it was made."""
    ctx, qkv, pos = recording()
    norm, rope = binding.HeadNorm(Tensor(1 << 24, (DH,)), Tensor(2 << 24, (DH,))), binding.Rotary(DH)

    def passed():
        ctx.otas_norm_rotary(qkv, KV, norm, pos, rope, qkv)
        name, args = ctx._lib.last
        d = described(binding._HeadNormDesc, args[4])
        return d.q_gain, d.k_gain, d.eps, d.center, d.per_head
    first = passed()
    assert first[:2] == (1 << 24, 2 << 24) and first[4] == 0
    norm.q_gain, norm.k_gain, norm.per_head = Tensor(3 << 24, (H, DH)), None, True
    assert passed() == (3 << 24, None, *first[2:4], 1)
    norm.q_gain = Tensor(3 << 24, (DH,))
    with pytest.raises(ValueError):
        passed()


def test_the_slopes_that_a_call_checks_are_those_that_it_passes():
    ctx, qkv, _ = recording()
    score, o = binding.Score(0.5, 2.0, Tensor(1 << 24, (H,), torch.float32)), Tensor(8192, (3, H * DH))

    def passed():
        ctx.otas_attention_window(qkv, KV, [0, 3], o, 5, 0, score)
        name, args = ctx._lib.last
        return described(binding._ScoreDesc, args[7]).slopes
    assert passed() == 1 << 24
    score.slopes = Tensor(2 << 24, (H,), torch.float32)
    assert passed() == 2 << 24
    score.slopes = None
    assert passed() is None


def test_a_description_of_another_kind_is_refused():
    """The library reads as many bytes as the description that it expects has."""
    ctx, qkv, pos = recording()
    norm, rope, score, o = binding.HeadNorm(), binding.Rotary(DH), binding.Score(), Tensor(8192, (3, H * DH))
    four = cache(binding.KVCache4)
    for other in (norm, score, four, None):
        with pytest.raises(ValueError, match="rope"):
            ctx.otas_rotary(qkv, KV, pos, other, qkv)
        with pytest.raises(ValueError, match="rope"):
            ctx.otas_norm_rotary(qkv, KV, norm, pos, other, qkv)
    for other in (rope, score, four, None):
        with pytest.raises(ValueError, match="norm"):
            ctx.otas_norm_rotary(qkv, KV, other, pos, rope, qkv)
    for other in (rope, norm, four):
        with pytest.raises(ValueError, match="score"):
            ctx.otas_attention_window(qkv, KV, [0, 3], o, 5, 0, other)
    assert ctx._lib.last is None
