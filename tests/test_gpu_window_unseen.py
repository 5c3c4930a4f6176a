"""What no row sees does not change a bit of what attention through a window gives, on the GPU.  Capped scores take one of two forms by how large the
products of a tile are; both are within the header's bound, so that only a comparison of bits shows a choice that hung on something unseen."""
import pytest

from tests import window_plain as plain
from tests.test_gpu_window import ALL, _close, context, gen, normal, offsets_of  # noqa: F401
from tests.test_gpu_window_edges import run_recent

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", [30.0, 300.0])
@pytest.mark.parametrize("dtype,H,KV,dh,rows,lengths,window,sinks", [
    ("bf16", 8, 2, 128, [40, 1], [100, 33], ALL, 0), ("bf16", 8, 2, 64, [70], [225], 100, 4), ("bf16", 4, 1, 80, [60, 0, 12], [161, 5, 12], 64, 0),
    ("bf16", 4, 2, 96, [200], [200], ALL, 0), ("bf16", 8, 2, 128, [2, 3], [100, 33], ALL, 0), ("bf16", 2, 1, 72, [50], [97], 40, 3), ("f32", 4, 2, 64, [40], [100], ALL, 0)])
def test_what_lies_behind_the_entries_of_a_4_bit_cache(lib, dtype, H, KV, dh, rows, lengths, window, sinks, cap, slopes):
    """Four fillings behind the entries: nothing, elements in the thousands, the largest that there are, and groups that are no numbers beside any others."""
    import torch
    ctx, g, B = context(dtype, H, dh), gen(dh + sum(rows)), len(rows)
    off, capacity = offsets_of(rows), 256
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    sl = torch.full((H,), 0.05, device="cuda") if slopes else None
    enc = [plain.encode4(normal(g, (B, KV, capacity, dh), dtype)) for _ in range(2)]
    arrays = [plain.pack4(c) for c, _ in enc] + [s.transpose(-1, -2).contiguous().to(torch.uint8) for _, s in enc]
    out = []
    for filling in range(4):
        for t in arrays[:2]:
            for q, n in enumerate(lengths):
                t[q, :, n:] = [0, 0x77, 0x77, 0x77][filling]
        for t in arrays[2:]:
            for q, n in enumerate(lengths):
                rest = t[q, :, :, n:]
                rest.fill_([127, 137, 252, 255][filling])
                if filling == 3:
                    rest.random_(0, 256, generator=g)
                    rest[:, 0] = 255
        out.append(run_recent(lib, ctx, True, lib.KVCache4(*arrays), qkv, off, list(range(B)), lengths, window, sinks, lib.Score(0.0, cap, sl)))
    assert bool(torch.isfinite(out[0]).all())
    assert all(torch.equal(out[0], o) for o in out[1:])


@pytest.mark.parametrize("cap", [30.0, 300.0])
@pytest.mark.parametrize("over", ["rows", "cache", "four"])
@pytest.mark.parametrize("dtype,H,KV,dh", [("bf16", 4, 2, 64), ("bf16", 2, 2, 80), ("bf16", 2, 1, 96), ("bf16", 2, 2, 128), ("f32", 2, 2, 64)])
def test_keys_outside_the_windows_of_all_of_a_calls_rows(lib, dtype, H, KV, dh, over, cap):
    """300 entries, 8 in a window: large keys at some of them leave the rows that are 32 and more tokens away as they were (32 is what a wave has),
    those before and those after them."""
    import torch
    n, window, odd = 300, 8, [0, 45, 46, 130, 299]
    ctx, g = context(dtype, H, dh), gen(dh + 1)
    qkv = normal(g, (n, (H + 2 * KV) * dh), dtype)
    t = torch.arange(n, device="cuda")
    far = torch.stack([(t < j - 31) | (t >= j + window + 31) for j in odd]).all(dim=0)
    assert 60 < int(far.sum()) < 200
    out = []
    for size in (1.0, 300.0):
        x = qkv.clone()
        x.view(n, H + 2 * KV, dh)[odd, H:H + KV] *= size
        y = x.view(n, H + 2 * KV, dh)
        k, v = [y[:, a:a + KV].transpose(0, 1)[None] for a in (H, H + KV)]
        if over == "rows":
            o = torch.empty((n, H * dh), dtype=x.dtype, device="cuda")
            ctx.otas_attention_window(x, KV, [0, n], o, window, 0, lib.Score(0.0, cap))
        else:
            if over == "four":
                k, v = [torch.nn.functional.pad(t, (0, 0, 0, 20)) for t in (k, v)]
                enc = [plain.encode4(t) for t in (k, v)]
                cache = lib.KVCache4(*[plain.pack4(c) for c, _ in enc], *[s.transpose(-1, -2).contiguous().to(torch.uint8) for _, s in enc])
            else:
                cache = lib.KVCache(k.contiguous(), v.contiguous(), torch.zeros((1, n), dtype=torch.int32, device="cuda"))
            o = run_recent(lib, ctx, over == "four", cache, qkv, [0, n], [0], [n], window, 0, lib.Score(0.0, cap))
        out.append(o)
    assert torch.equal(out[0][far], out[1][far])
    assert not torch.equal(out[0], out[1])
