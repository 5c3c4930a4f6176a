"""Calls of the decoder's operators that their header allows and that lie at an edge of it, on the GPU."""
import numpy as np
import pytest

from tests.test_gpu_decode import _close, clone_cache, context, gen, new_cache, normal  # noqa: F401

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


@pytest.mark.parametrize("dtype,H,KV,dh,nodes", [("f32", 2, 1, 64, 1), ("f32", 4, 2, 20, 3), ("bf16", 2, 1, 64, 1), ("bf16", 4, 1, 128, 2), ("bf16", 8, 1, 80, 6),
                                                 ("bf16", 8, 1, 64, 40), ("bf16", 2, 1, 40, 2)])
def test_a_key_that_is_not_a_number_behind_small_weights(lib, dtype, H, KV, dh, nodes):
    """Logits of -128 in the first chunks of a cache, one of them NaN, and +128 in the later ones, against which the first count
    exp(-256) = 0: the rows are NaN and so are the weights, as the formula says.  Another query of the call keeps its bits."""
    import torch
    ctx, g, n = context(dtype, H, dh), gen(nodes), 3000
    cache = new_cache(lib, g, dtype, 2, KV, n, dh)
    scale = 1.0 / 8
    cache.k[..., 0] = 32.0
    cache.k[:, :, :200, 0] = -32.0    # a whole chunk, joined together with some of the others
    qkv = normal(g, (2 * nodes, (H + 2 * KV) * dh), dtype, 0.01)
    qkv.view(2 * nodes, -1, dh)[:, :H, 0] = 32.0
    off, out, mass = [0, nodes, 2 * nodes], [], []
    start = cache.mass.clone()
    for bad in (False, True):
        if bad:
            cache.k[1, 0, 5, 3] = float("nan")
        cache.mass.copy_(start)
        ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, off, [n, n]), dtype=torch.uint8, device="cuda")
        out.append(torch.empty((2 * nodes, H * dh), dtype=qkv.dtype, device="cuda"))
        ctx.otas_attention_tree(cache, qkv, off, None, None, [0, 1], [n, n], ws, out[-1], score=lib.Score(scale=scale), add_mass=True)
        mass.append(cache.mass.clone())
    of_head = out[1][nodes:].view(nodes, H, dh)[:, :H // KV]
    assert bool(of_head.isnan().all()) and bool(mass[1][1].isnan().all())
    assert torch.equal(out[0][:nodes], out[1][:nodes]) and torch.equal(mass[0][0], mass[1][0]) and bool(out[0].isfinite().all())
