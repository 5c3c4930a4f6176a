"""Calls of the decoder's operators that their header allows and that lie at an edge of it, on the GPU."""
import numpy as np
import pytest

from tests.test_gpu_decode import _close, clone_cache, context, gen, new_cache  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,lengths,keep,lead,recent", [("f32", [300, 40, 9], [30, 7, 1], 0, 400), ("bf16", [300, 64], [299, 20], 4, 10000),
                                                            ("bf16", [33000, 500], [900, 499], 2, 20000), ("bf16", [130], [3], 8, None)])
def test_more_entries_protected_than_stay(lib, dtype, lengths, keep, lead, recent):
    """Protected entries are alike whatever their mass: the lowest of them stay, in a cache that is in no order, and nothing else does."""
    ctx, g, capacity = context(dtype, 2, 64), gen(len(lengths)), max(lengths) + 1
    cache = new_cache(lib, g, dtype, len(lengths), 1, capacity, 64)
    recent_from = None if recent is None else [2 * capacity - recent] * len(lengths)
    before = clone_cache(lib, cache)
    import torch
    ws = torch.empty(ctx.otas_cache_evict_workspace_bytes(lengths, keep), dtype=torch.uint8, device="cuda")
    slots = list(range(len(lengths)))
    ctx.otas_cache_evict(cache, slots, lengths, keep, ws, lead=lead, recent_from=recent_from)
    pos = before.positions.cpu().numpy()
    for q, (n, k) in enumerate(zip(lengths, keep)):
        first = np.flatnonzero((np.arange(n) < lead) | (pos[q, :n] >= recent_from[q] if recent is not None else False))
        if len(first) <= k:
            continue
        assert k < lead or recent is not None
        stay = first[:k]
        assert sorted(cache.positions[q, :k].tolist()) == sorted(pos[q, stay].tolist())
        below = stay[stay < k]                               # what stays below the cut does not move
        assert torch.equal(cache.k[q][:, below], before.k[q][:, below]) and torch.equal(cache.mass[q, below], before.mass[q, below])
        places, sources = np.setdiff1d(np.arange(k), stay), stay[stay >= k]
        for a, b in ((cache.k[q], before.k[q]), (cache.v[q], before.v[q])):
            assert torch.equal(a[:, places], b[:, sources])
        assert torch.equal(cache.mass[q, places], before.mass[q, sources])
        assert torch.equal(cache.k[q][:, k:], before.k[q][:, k:])
