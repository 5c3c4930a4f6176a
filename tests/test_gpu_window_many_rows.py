"""Calls of attention over caches with very many rows x heads, on the GPU: what counts for a refusal is a launch's workgroups."""
import pytest

from tests.test_gpu_window import _close, context, gen, normal  # noqa: F401
from tests.test_gpu_window_edges import packed_cache, run_recent

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("dtype,dh", [("bf16", 8), ("f32", 8), ("bf16", 64)])
def test_more_than_2_to_the_26_rows_times_heads(lib, dtype, dh, four):
    """1025 queries of 2048 rows and 32 heads: 2.1 million workgroups of 32 rows, at width 64 524800 of 128.  The same rows in four calls give the same bits."""
    import torch
    H, KV, B, n, window, sinks = 32, 1, 1025, 2048, 3, 1
    ctx, g = context(dtype, H, dh), gen(dh)
    qkv = normal(g, (B * n, (H + 2 * KV) * dh), dtype)
    assert B * n * H > 2 ** 26
    k, v = normal(g, (2, KV, n, dh), dtype), normal(g, (2, KV, n, dh), dtype)
    cache = packed_cache(lib, k, v)[0] if four else lib.KVCache(k, v, torch.zeros((2, n), dtype=torch.int32, device="cuda"))

    def call(a, z):
        return run_recent(lib, ctx, four, cache, qkv[a * n:z * n], [n * q for q in range(z - a + 1)], [q % 2 for q in range(a, z)], [n] * (z - a), window, sinks)
    got = call(0, B)
    for a in range(0, B, 260):
        z = min(a + 260, B)
        assert torch.equal(got[a * n:z * n], call(a, z)), a
