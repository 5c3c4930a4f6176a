"""Attention through a window over values as large as the header takes, with logits that rise so slowly that the sums keep an old largest one: weights of up
to 2^8 meet them."""
import pytest

from tests import window_plain as plain
from tests.test_gpu_window import ALL, _close, context, gen, normal, offsets_of, within  # noqa: F401
from tests.test_gpu_window_edges import packed_cache, run_recent

pytestmark = pytest.mark.gpu
LARGEST = 1e30


def rising(H, KV, dh, dtype, n, rows, size):
    """Queries [rows], keys and values of n entries: entry j's logit is about 5.4 (7.8 for a base of 2) from entry 300 on and 0 before it; values of one
    sign, up to `size`."""
    import torch
    g = gen(n + dh)
    qkv = normal(g, (rows, (H + 2 * KV) * dh), dtype, 0.01)
    qkv.view(rows, -1, dh)[:, :H, 0] = 4.0
    k, v = normal(g, (1, KV, n, dh), dtype, 0.01), normal(g, (1, KV, n, dh), dtype)
    k[..., 0] = 0
    k[:, :, 300:, 0] = 1.35
    v.copy_((0.5 + 0.5 * torch.rand(v.shape, generator=g, device="cuda")) * size)
    return qkv, k, v


@pytest.mark.parametrize("over", ["rows", "cache", "four"])
@pytest.mark.parametrize("dtype,H,KV,dh,rows", [("f32", 2, 1, 64, 1), ("f32", 4, 1, 128, 20), ("bf16", 2, 1, 64, 1), ("bf16", 4, 1, 128, 40), ("bf16", 4, 2, 80, 200)])
def test_the_largest_values_of_the_header(lib, dtype, H, KV, dh, rows, over):
    import torch
    ctx, n = context(dtype, H, dh), 4000
    qkv, k, v = rising(H, KV, dh, dtype, n, rows, LARGEST)
    if over == "rows":
        x = torch.empty((n, (H + 2 * KV) * dh), dtype=qkv.dtype, device="cuda")
        y = x.view(n, H + 2 * KV, dh)
        y[:, :H] = qkv.view(rows, -1, dh)[:1, :H]
        y[:, H:H + KV], y[:, H + KV:] = k[0].transpose(0, 1), v[0].transpose(0, 1)
        o = torch.empty((n, H * dh), dtype=x.dtype, device="cuda")
        ctx.otas_attention_window(x, KV, [0, n], o, ALL, 0, lib.Score(1.0))
        within(o, *plain.window(x, H, KV, [0, n], ALL, 0, 1.0), "window")
    else:
        cache, (k, v) = packed_cache(lib, k, v) if over == "four" else (lib.KVCache(k, v, torch.zeros((1, n), dtype=torch.int32, device="cuda")), (k, v))
        o = run_recent(lib, ctx, over == "four", cache, qkv, [0, rows], [0], [n], ALL, 0, lib.Score(1.0))
        within(o, *plain.recent(qkv, H, k, v, [0, rows], [0], [n], ALL, 0, 1.0), "cached")
    assert bool(torch.isfinite(o).all())
