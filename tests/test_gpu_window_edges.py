"""Calls of the operators with norms of heads, windows and the cache in 4 bits that their header allows and that lie at an edge of it, and a
decoder's steps of them together, on the GPU."""
import math

import pytest

import otas_synth as synth
from tests import decode_plain
from tests import harness as hz
from tests import window_plain as plain
from tests.test_gpu_window import ALL, _close, context, gen, normal, offsets_of, within  # noqa: F401

pytestmark = pytest.mark.gpu


def packed_cache(lib, k, v):
    """A cache in 4 bits of k, v [slots, KV, capacity, dh] made on the CPU's terms, and the values it stands for."""
    import torch
    enc = [plain.encode4(t) for t in (k, v)]
    arrays = [plain.pack4(c) for c, _ in enc] + [s.transpose(-1, -2).contiguous().to(torch.uint8) for _, s in enc]
    return lib.KVCache4(*arrays), [plain.decode4(c, s) for c, s in enc]


def run_recent(lib, ctx, four, cache, qkv, off, slots, lengths, window, sinks, score=None):
    import torch
    H = ctx.H
    ws = torch.full((ctx.otas_attention_recent_workspace_bytes(cache.kv_heads, off, lengths, window, sinks),), 255, dtype=torch.uint8, device="cuda")
    o = torch.empty((off[-1], ctx.D), dtype=qkv.dtype, device="cuda")
    (ctx.otas_attention_cache4 if four else ctx.otas_attention_recent)(cache, qkv, off, slots, lengths, ws, o, window, sinks, score)
    assert H * cache.head_width == ctx.D
    return o


@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("dtype,H,KV,dh,rows,lengths,window,sinks", [
    ("bf16", 16, 8, 128, [1], [9001], ALL, 0), ("bf16", 4, 1, 64, [1, 1], [20000, 40], 15000, 70), ("f32", 4, 2, 64, [1], [9001], ALL, 0),
    ("f32", 2, 1, 80, [3, 1], [5003, 17], 4000, 5), ("bf16", 16, 2, 128, [256, 256, 1, 200], [4000, 3001, 900, 200], 2500, 4),
    ("bf16", 8, 4, 80, [300], [2049], ALL, 0), ("f32", 8, 2, 32, [600], [1500], 300, 33),
    ("bf16", 4, 2, 96, [150, 40], [1500, 700], 600, 40), ("bf16", 8, 2, 64, [100, 33, 1], [2500, 500, 64], ALL, 0), ("bf16", 6, 2, 128, [700, 3, 300], [3000, 2900, 2000], ALL, 0)])
def test_long_windows_in_parts(lib, dtype, H, KV, dh, rows, lengths, window, sinks, four):
    """Calls cut into several parts, of few rows and of many, joined by every form of the join."""
    ctx, g, B = context(dtype, H, dh), gen(lengths[0]), len(rows)
    off, capacity = offsets_of(rows), -(-max(lengths) // 32) * 32
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    k, v = normal(g, (B, KV, capacity, dh), dtype), normal(g, (B, KV, capacity, dh), dtype)
    import torch
    if four:
        cache, (k, v) = packed_cache(lib, k, v)
    else:
        cache = lib.KVCache(k, v, torch.zeros((B, capacity), dtype=torch.int32, device="cuda"))
    want, bound = plain.recent(qkv, H, k, v, off, range(B), lengths, window, sinks)
    first = run_recent(lib, ctx, four, cache, qkv, off, list(range(B)), lengths, window, sinks)
    within(first, want, bound, "parts")
    assert torch.equal(first, run_recent(lib, ctx, four, cache, qkv, off, list(range(B)), lengths, window, sinks))   # the same bits again


@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("dtype,H,KV,dh,rows", [("f32", 2, 1, 64, 1), ("bf16", 2, 1, 64, 1), ("bf16", 4, 1, 128, 2), ("bf16", 8, 1, 80, 20)])
def test_a_key_that_is_not_a_number_behind_small_weights(lib, dtype, H, KV, dh, rows, four):
    """Logits of -128 in the first entries, one of them NaN, and +128 in the later ones, against which the first count exp(-256) = 0: the rows are
    NaN all the same.  Another query of the call keeps its bits."""
    import torch
    ctx, g, n = context(dtype, H, dh), gen(rows), 3008
    k, v = normal(g, (2, KV, n, dh), dtype), normal(g, (2, KV, n, dh), dtype)
    k[..., 0] = 32.0
    k[:, :, :200, 0] = -32.0
    qkv = normal(g, (2 * rows, (H + 2 * KV) * dh), dtype, 0.01)
    qkv.view(2 * rows, -1, dh)[:, :H, 0] = 32.0
    off, out = [0, rows, 2 * rows], []
    for bad in (False, True):
        if bad:
            k[1, 0, 5, 3] = math.nan
        cache = packed_cache(lib, k, v)[0] if four else lib.KVCache(k, v, torch.zeros((2, n), dtype=torch.int32, device="cuda"))
        out.append(run_recent(lib, ctx, four, cache, qkv, off, [0, 1], [n, n], ALL, 0, lib.Score(0.125)))
    assert bool(torch.isnan(out[1][rows:].view(rows, H, dh)[:, :H // KV]).all())
    assert torch.equal(out[0][:rows], out[1][:rows]) and not bool(torch.isnan(out[0]).any())


@pytest.mark.parametrize("scale,cap", [(-0.3, 0.0), (-0.3, 5.0), (0.3, 1000.0), (1e-20, 0.0), (0.0, 0.01)])
@pytest.mark.parametrize("dtype,H,KV,dh,rows", [("f32", 4, 2, 64, 2), ("bf16", 4, 2, 64, 2), ("bf16", 8, 2, 128, 40)])
def test_scales_and_caps(lib, dtype, H, KV, dh, rows, scale, cap):
    import torch
    ctx, g, n = context(dtype, H, dh), gen(rows + int(10 * cap)), 160
    off, lengths, actual = [0, rows], [n], scale or dh ** -0.5
    qkv = normal(g, (rows, (H + 2 * KV) * dh), dtype)
    k, v = normal(g, (1, KV, n, dh), dtype), normal(g, (1, KV, n, dh), dtype)
    for four in (False, True):
        cache, (a, b) = packed_cache(lib, k, v) if four else (lib.KVCache(k, v, torch.zeros((1, n), dtype=torch.int32, device="cuda")), (k, v))
        want, bound = plain.recent(qkv, H, a, b, off, [0], lengths, 100, 3, actual, cap)
        if cap > 256 and dtype == "bf16":    # the header: up to 4e-6 of a logit, which here are below 20
            bound = bound + 20 * 4e-6 * plain.recent(qkv, H, a, b.abs(), off, [0], lengths, 100, 3, actual, cap)[0].abs()
        within(run_recent(lib, ctx, four, cache, qkv, off, [0], lengths, 100, 3, lib.Score(scale, cap)), want, bound, "cached")
    o = torch.empty((rows, H * dh), dtype=qkv.dtype, device="cuda")
    want, bound = plain.window(qkv, H, KV, off, 7, 2, actual, cap)
    if cap > 256 and dtype == "bf16":
        x = qkv.clone()
        x[:, (H + KV) * dh:] = x[:, (H + KV) * dh:].abs()
        bound = bound + 20 * 4e-6 * plain.window(x, H, KV, off, 7, 2, actual, cap)[0].abs()
    ctx.otas_attention_window(qkv, KV, off, o, 7, 2, lib.Score(scale, cap))
    within(o, want, bound, "window")


def test_rows_of_many_queries(lib):
    """More host numbers than the kernels' arguments hold: 1200 queries of 0 .. 2 rows, in every operator that has any."""
    import torch
    H, KV, dh, B, capacity = 4, 2, 64, 1200, 32
    ctx, g = context("bf16", H, dh), gen(1)
    rows = [q % 3 for q in range(B)]
    off = offsets_of(rows)
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), "bf16")
    o = torch.empty((off[-1], H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_window(qkv, KV, off, o, 1, 1)
    within(o, *plain.window(qkv, H, KV, off, 1, 1), "window")
    slots, before = [B - 1 - q for q in range(B)], [q % 7 for q in range(B)]
    cache = lib.KVCache4.empty(B, KV, capacity, dh)
    x = normal(g, (B, KV, capacity, dh), "bf16")
    fill = torch.cat([x.transpose(1, 2).reshape(B * capacity, KV * dh).new_zeros((B * capacity, H * dh)), x.transpose(1, 2).reshape(B * capacity, -1),
                      x.flip(0).transpose(1, 2).reshape(B * capacity, -1)], dim=1)
    for a in range(0, B, 400):   # 12800 rows: four a workgroup
        ctx.otas_cache4_append(cache, fill[a * capacity:(a + 400) * capacity], [capacity * q for q in range(401)], None, list(range(a, a + 400)), [0] * 400)
    lengths = ctx.otas_cache4_append(cache, qkv, off, None, slots, before)
    assert list(lengths) == [a + b for a, b in zip(before, rows)]
    k, v = x.clone(), x.flip(0).clone()
    y = qkv.view(off[-1], H + 2 * KV, dh)
    for q in range(B):
        for i in range(rows[q]):
            k[slots[q], :, before[q] + i], v[slots[q], :, before[q] + i] = y[off[q] + i, H:H + KV], y[off[q] + i, H + KV:]
    k, v = [plain.decode4(*plain.encode4(t)) for t in (k, v)]
    back = torch.empty((B * capacity, 2 * KV * dh), dtype=qkv.dtype, device="cuda")   # 38400 rows
    ctx.otas_cache4_read(cache, list(range(B)), [0] * B, [capacity * q for q in range(B + 1)], back)
    assert torch.equal(back.double(), torch.cat([t.transpose(1, 2).reshape(B * capacity, -1) for t in (k, v)], dim=1))
    got = run_recent(lib, ctx, True, cache, qkv, off, slots, [int(n) for n in lengths], 5, 1)
    within(got, *plain.recent(qkv, H, k, v, off, slots, lengths, 5, 1), "cache4")


@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
def test_a_slot_past_four_gigabytes(lib, four):
    """Offsets into the cache past 32 bits: the last slot of one of 4.8 GB (2.4 and its scales in 4 bits: past 2^31 and, of a head's rows, 2^32)."""
    import torch
    H, KV, dh, capacity = 16, 8, 128, 262144
    slots = 9 if not four else 17
    ctx, g, n, rows = context("bf16", H, dh), gen(7), 262100, 2
    qkv = normal(g, (rows, (H + 2 * KV) * dh), "bf16")
    slot, window, sinks = slots - 1, 3000, 10
    off = [0, rows]
    fill = normal(g, (4096, (H + 2 * KV) * dh), "bf16")
    shape = (slots, KV, capacity, dh)
    if four:
        cache = lib.KVCache4.empty(slots, KV, capacity, dh)
        assert cache.k.numel() > 2 ** 32 // 4 * 2
        ctx.otas_cache4_append(cache, fill, [0, 10], None, [slot], [0])
        ctx.otas_cache4_append(cache, fill, [0, 4096], None, [slot], [n - 4096])
    else:
        cache = lib.KVCache(torch.empty(shape, dtype=torch.bfloat16, device="cuda"), torch.empty(shape, dtype=torch.bfloat16, device="cuda"),
                            torch.empty((slots, capacity), dtype=torch.int32, device="cuda"))
        assert cache.k.numel() * 2 > 2 ** 32
        pos = torch.arange(4096, dtype=torch.int32, device="cuda")
        ctx.otas_cache_append(cache, fill, [0, 10], None, pos, [slot], [0])
        ctx.otas_cache_append(cache, fill, [0, 4096], None, pos, [slot], [n - 4096])
    got = run_recent(lib, ctx, four, cache, qkv, off, [slot], [n], window, sinks)
    # the same over a short cache: the sinks' entries, then the last 4096
    x = fill.view(4096, H + 2 * KV, dh)
    values = []
    for a in (H, H + KV):
        t = torch.cat([x[:10, a:a + KV], x[:, a:a + KV]]).transpose(0, 1)[None]
        values.append(plain.decode4(*plain.encode4(t)) if four else t)
    want, bound = plain.recent(qkv, H, values[0], values[1], off, [0], [4106], window, sinks)
    within(got, want, bound, "far slot")
    if four:
        back = torch.empty((3, 2 * KV * dh), dtype=torch.bfloat16, device="cuda")
        ctx.otas_cache4_read(cache, [slot], [n - 3], [0, 3], back)
        assert torch.equal(back.double(), torch.cat([t[0, :, -3:].transpose(0, 1).reshape(3, -1) for t in values], dim=1))


@pytest.mark.parametrize("dtype,H,KV,dh", [("bf16", 8, 2, 64), ("bf16", 4, 4, 80), ("bf16", 6, 2, 48), ("f32", 4, 1, 64)])
@pytest.mark.parametrize("singles", [5, 70, 340])
def test_a_long_run_among_single_rows(lib, dtype, H, KV, dh, singles):
    """Calls whose queries differ so much in rows that they are counted one by one (with 340 of them, over caches, in memory), also empty ones."""
    import torch
    ctx, g = context(dtype, H, dh), gen(singles)
    rows = [1] * (singles // 2) + [0, 700, 0] + [1] * (singles // 2) + [290, 0]
    off = offsets_of(rows)
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    o = torch.empty((off[-1], H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_window(qkv, KV, off, o, 100, 3)
    within(o, *plain.window(qkv, H, KV, off, 100, 3), "window")
    slots, lengths, capacity = [(7 * q) % 9 for q in range(len(rows))], [max(n, (13 * q) % 800) for q, n in enumerate(rows)], 800
    k, v = normal(g, (9, KV, capacity, dh), dtype), normal(g, (9, KV, capacity, dh), dtype)
    for four in (False, True):
        cache, (a, b) = packed_cache(lib, k, v) if four else (lib.KVCache(k, v, torch.zeros((9, capacity), dtype=torch.int32, device="cuda")), (k, v))
        for window, sinks in ((100, 3), (ALL, 0)):
            want, bound = plain.recent(qkv, H, a, b, off, slots, lengths, window, sinks)
            within(run_recent(lib, ctx, four, cache, qkv, off, slots, lengths, window, sinks), want, bound, "cached")


def decoder(lib, ctx, stream_tokens, H, KV, dh, dtype, window, sinks):
    """What a decoder's layer does with a token of each request, on buffers that it keeps."""
    import torch
    B, capacity = 3, 256
    st = {"qkv": torch.zeros((B, (H + 2 * KV) * dh), dtype=dtype, device="cuda"), "o": torch.zeros((B, H * dh), dtype=dtype, device="cuda"),
          "positions": torch.zeros(B, dtype=torch.int32, device="cuda"), "cache": lib.KVCache4.empty(B, KV, capacity, dh), "slots": [2, 0, 1]}
    g = gen(11)
    st["norm"] = lib.HeadNorm(1 + normal(g, (dh,), "bf16", 0.1).to(dtype), 1 + normal(g, (dh,), "bf16", 0.1).to(dtype), 1e-5)
    st["rope"] = lib.Rotary(dh // 2)
    st["workspace"] = torch.empty(ctx.otas_attention_recent_workspace_bytes(KV, [0, 1, 2, 3], [capacity] * B, window, sinks), dtype=torch.uint8, device="cuda")

    def step(lengths):
        ctx.otas_norm_rotary(st["qkv"], KV, st["norm"], st["positions"], st["rope"], st["qkv"])
        new = ctx.otas_cache4_append(st["cache"], st["qkv"], [0, 1, 2, 3], None, st["slots"], lengths)
        ctx.otas_attention_cache4(st["cache"], st["qkv"], [0, 1, 2, 3], st["slots"], [int(n) for n in new], st["workspace"], st["o"], window, sinks)
        return [int(n) for n in new]
    return st, step


def test_a_decoders_steps_together(lib):
    """Prompts through the window and into the cache, then tokens one by one: norms, rotation, append and attention as a layer uses them, against
    64 bits at every step (what each operator reads is what the one before it left)."""
    import torch
    H, KV, dh, window, sinks = 8, 2, 64, 40, 3
    for dtype in ("bf16", "f32"):
        ctx, g = context(dtype, H, dh), gen(5)
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        st, step = decoder(lib, ctx, None, H, KV, dh, tdt, window, sinks)
        prompts = [50, 1, 97]
        off = offsets_of(prompts)
        x = normal(g, (off[-1], (H + 2 * KV) * dh), dtype, 2.0)
        pos = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in prompts])
        y = torch.empty_like(x)
        ctx.otas_norm_rotary(x, KV, st["norm"], pos, st["rope"], y)
        freqs = decode_plain.frequencies(dh // 2)
        within(y, *plain.norm_rotary(x, H, KV, pos, dh // 2, False, freqs, st["norm"].q_gain, st["norm"].k_gain, 1e-5), "prompts' norms")
        o = torch.empty((off[-1], H * dh), dtype=tdt, device="cuda")
        ctx.otas_attention_window(y, KV, off, o, window, sinks)
        within(o, *plain.window(y, H, KV, off, window, sinks), "prompts")
        lengths = [int(n) for n in ctx.otas_cache4_append(st["cache"], y, off, None, st["slots"], [0, 0, 0])]
        held = [[list(plain.decode4(*plain.encode4(y[a:z].view(z - a, H + 2 * KV, dh)[:, p:p + KV]))) for p in (H, H + KV)] for a, z in zip(off, off[1:])]
        for n in range(6):
            new = normal(g, (3, (H + 2 * KV) * dh), dtype, 2.0)
            st["qkv"].copy_(new)
            st["positions"].copy_(torch.tensor(lengths, dtype=torch.int32))
            lengths = step(lengths)
            within(st["qkv"], *plain.norm_rotary(new, H, KV, st["positions"], dh // 2, False, freqs, st["norm"].q_gain, st["norm"].k_gain, 1e-5), "a step's norms")
            z = st["qkv"].view(3, H + 2 * KV, dh)
            for q in range(3):
                for i, p in enumerate((H, H + KV)):
                    held[q][i] += list(plain.decode4(*plain.encode4(z[q:q + 1, p:p + KV])))
                k, v = [torch.stack(t).transpose(0, 1)[None] for t in held[q]]
                want, bound = plain.recent(st["qkv"][q:q + 1], H, k, v, [0, 1], [0], [lengths[q]], window, sinks)
                within(st["o"][q:q + 1], want, bound, f"step {n} of query {q}")


def test_captured_steps_and_a_workspace_that_two_graphs_share(lib):
    """A step captured on the context's stream, and one of other lengths into a second graph with the same workspace: replayed in turn with eager work
    and synchronisations between them, every replay gives the eager call's bits.  Host numbers that do not fit the arguments are refused under capture."""
    import torch
    H, KV, dh, window, sinks = 8, 2, 64, 100, 3
    cfg = synth.Config("steps", L=1, D=H * dh, H=H, F=64, dtype="bf16", B=1, n0=4, strategies=[(0, 0)], seed=5)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = hz.make_context(cfg)[0]
        try:
            assert ctx.stream == stream.cuda_stream
            st, step = decoder(lib, ctx, stream, H, KV, dh, torch.bfloat16, window, sinks)
            g = gen(3)
            fill = normal(g, (600, (H + 2 * KV) * dh), "bf16")
            ctx.otas_cache4_append(st["cache"], fill, [0, 200, 400, 600], None, st["slots"], [0, 0, 0])
            kept = [t.clone() for t in (st["cache"].k, st["cache"].v, st["cache"].k_scales, st["cache"].v_scales)]
            new = normal(g, (3, (H + 2 * KV) * dh), "bf16")

            def restore(seed):
                for t, s in zip((st["cache"].k, st["cache"].v, st["cache"].k_scales, st["cache"].v_scales), kept):
                    t.copy_(s)
                st["qkv"].copy_(new * seed)
                st["positions"].fill_(77)
                st["workspace"].fill_(255)
                st["o"].zero_()
            calls = [[200, 200, 200], [30, 199, 1]]
            want = {}
            for i, lengths in enumerate(calls):
                for seed in (1, 2):
                    restore(seed)
                    step(lengths)
                    want[i, seed] = st["o"].clone()
            torch.cuda.synchronize()
            graphs = []
            for lengths in calls:
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1], stream=stream):
                    step(lengths)
            for i, seed in ((0, 1), (1, 1), (0, 2), (0, 1), (1, 2), (1, 1)):
                restore(seed)
                torch.cuda.synchronize()
                graphs[i].replay()
                torch.cuda.synchronize()
                assert torch.equal(st["o"], want[i, seed]), (i, seed)
                restore(seed)
                step(calls[i])
                torch.cuda.synchronize()
                assert torch.equal(st["o"], want[i, seed])
            B = 400   # 1201 numbers
            big = lib.KVCache4.empty(B, KV, 32, dh)
            many = normal(g, (B, (H + 2 * KV) * dh), "bf16")
            out = torch.empty((B, H * dh), dtype=torch.bfloat16, device="cuda")
            ws = torch.empty(ctx.otas_attention_recent_workspace_bytes(KV, list(range(B + 1)), [1] * B, 5), dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                for call in (lambda: ctx.otas_cache4_append(big, many, list(range(B + 1)), None, list(range(B)), [0] * B),
                             lambda: ctx.otas_attention_cache4(big, many, list(range(B + 1)), list(range(B)), [1] * B, ws, out, 5)):
                    with pytest.raises(lib.OtasError) as e:
                        call()
                    assert e.value.status == 5
                ctx.otas_norm_rotary(many, KV, st["norm"], None, lib.Rotary(0), many)
        finally:
            torch.cuda.synchronize()
            ctx.close()


def test_two_contexts_at_once(lib):
    """Two contexts on streams of their own, without a wait between their calls: each has its own plan (in memory: more numbers than arguments hold),
    workspace and results."""
    import torch
    H, KV, dh, B = 4, 2, 64, 400
    cfg = synth.Config("two", L=1, D=H * dh, H=H, F=64, dtype="bf16", B=1, n0=4, strategies=[(0, 0)], seed=5)
    state = []
    for seed in (1, 2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx, g = hz.make_context(cfg)[0], gen(seed)
            rows = [(q * seed) % 3 for q in range(B)]
            off, capacity = offsets_of(rows), 320
            qkv = normal(g, (off[-1], (H + 2 * KV) * dh), "bf16")
            cache, (k, v) = packed_cache(lib, normal(g, (B, KV, capacity, dh), "bf16"), normal(g, (B, KV, capacity, dh), "bf16"))
            lengths = [max(n, (q * 7 * seed) % capacity) for q, n in enumerate(rows)]
            ws = torch.empty(ctx.otas_attention_recent_workspace_bytes(KV, off, lengths, 50, 3), dtype=torch.uint8, device="cuda")
            state.append((stream, ctx, qkv, off, cache, lengths, ws, torch.empty((off[-1], H * dh), dtype=qkv.dtype, device="cuda"), k, v))
    torch.cuda.synchronize()
    for _ in range(4):
        for stream, ctx, qkv, off, cache, lengths, ws, o, k, v in state:
            with torch.cuda.stream(stream):
                ctx.otas_attention_cache4(cache, qkv, off, list(range(B)), lengths, ws, o, 50, 3)
    torch.cuda.synchronize()
    for stream, ctx, qkv, off, cache, lengths, ws, o, k, v in state:
        within(o, *plain.recent(qkv, H, k, v, off, range(B), lengths, 50, 3), "its own")
        ctx.close()


def test_rows_behind_the_last_entry_and_other_slots_stay(lib):
    """Neither attention writes anything but o and its workspace."""
    import torch
    H, KV, dh, n = 4, 2, 64, 300
    ctx, g = context("bf16", H, dh), gen(2)
    qkv = normal(g, (2, (H + 2 * KV) * dh), "bf16")
    k, v = normal(g, (3, KV, 320, dh), "bf16"), normal(g, (3, KV, 320, dh), "bf16")
    for four in (False, True):
        cache = packed_cache(lib, k, v)[0] if four else lib.KVCache(k, v, torch.zeros((3, 320), dtype=torch.int32, device="cuda"))
        arrays = (cache.k, cache.v) + ((cache.k_scales, cache.v_scales) if four else (cache.positions,))
        before = [t.clone() for t in arrays] + [qkv.clone()]
        run_recent(lib, ctx, four, cache, qkv, [0, 1, 2], [1, 1], [n, n - 5], 50, 2)
        assert all(torch.equal(a, b) for a, b in zip(arrays + (qkv,), before))


def test_wrong_tensors_are_refused_by_the_binding(lib):
    import torch
    H, KV, dh = 4, 2, 64
    ctx, g = context("bf16", H, dh), gen(1)
    qkv = normal(g, (3, (H + 2 * KV) * dh), "bf16")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    good = lib.KVCache4.empty(2, KV, 32, dh)
    o = torch.empty((3, H * dh), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1024, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        ctx.otas_norm_rotary(qkv, KV, lib.HeadNorm(torch.ones(dh - 1, dtype=torch.bfloat16, device="cuda")), pos, lib.Rotary(8), qkv)
    with pytest.raises(ValueError):
        ctx.otas_norm_rotary(qkv, KV, lib.HeadNorm(torch.ones(dh, dtype=torch.bfloat16, device="cuda"), per_head=True), pos, lib.Rotary(8), qkv)
    with pytest.raises(ValueError):
        ctx.otas_norm_rotary(qkv, KV, lib.HeadNorm(torch.ones(dh, device="cuda")), pos, lib.Rotary(8), qkv)
    with pytest.raises(ValueError):
        ctx.otas_attention_window(qkv, KV, [0, 2], o, 5)
    with pytest.raises(ValueError):
        lib.KVCache4(good.k, good.v, good.k_scales[..., :16], good.v_scales)
    with pytest.raises(ValueError):
        lib.KVCache4(good.k.float(), good.v, good.k_scales, good.v_scales)
    with pytest.raises(ValueError):
        lib.KVCache4(good.k.cpu(), good.v, good.k_scales, good.v_scales)
    with pytest.raises(ValueError):
        ctx.otas_attention_cache4(lib.KVCache4.empty(2, KV, 32, 32), qkv, [0, 1, 2, 3], [0, 1, 1], [5, 5, 5], ws, o, 4)
    with pytest.raises(lib.OtasError) as e:
        ctx.otas_attention_cache4(good, qkv, [0, 1, 2, 3], [0, 1, 1], [5, 5, 0], ws, o, 4)
    assert e.value.status == 1
    with pytest.raises(lib.OtasError):
        ctx.otas_attention_window(qkv, KV, [0, 3], o, 0)


@pytest.mark.parametrize("T", [4096, 180000])
def test_norms_of_many_rows(lib, T):
    """Row offsets past 2^32 bytes (180000 rows of 6144 elements in float32 are 4.4 GB), a few rows checked."""
    import torch
    H, KV, dh = 16, 16, 128
    ctx, g = context("f32", H, dh), gen(1)
    qkv = torch.empty((T, (H + 2 * KV) * dh), dtype=torch.float32, device="cuda")
    qkv.normal_(generator=g)
    pick = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rows = qkv[pick].clone()
    ctx.otas_norm_rotary(qkv, KV, lib.HeadNorm(), pos, lib.Rotary(128), qkv)
    want, bound = plain.norm_rotary(rows, H, KV, pos[pick], 128, False, decode_plain.frequencies(128))
    within(qkv[pick], want, bound, "norm")


def test_operator_cases_run_on_the_stream_that_is_current(lib):
    """The calls of perf/more_operators.py as a program on another stream makes them, and their outputs against the plain forms'."""
    import torch
    import perf.more_operators as ops
    before = ops.own
    cases = [{"op": "norm", "dtype": "bf16", "shape": "huge_g", "tokens": 33, "rot": 40, "layout": "half", "center": True, "per_head": True},
             {"op": "window", "dtype": "bf16", "shape": "base_g", "batch": 2, "tokens": 150, "ragged": 0.3, "window": 40, "sinks": 2, "cap": 30.0, "slopes": True},
             {"op": "recent", "dtype": "f32", "shape": "base_g", "batch": 2, "tokens": 2, "cached": 300, "ragged": 0.3, "window": 90, "sinks": 2, "cap": 0.0, "slopes": False},
             {"op": "append4", "dtype": "bf16", "shape": "narrow_g", "batch": 2, "tokens": 9, "ragged": 0.3, "taken": 2, "capacity": 64},
             {"op": "cache4", "dtype": "bf16", "shape": "wide_g8", "batch": 2, "tokens": 1, "cached": 300, "ragged": 0.3, "window": 0, "sinks": 0, "cap": 0.0, "slopes": False}]
    try:
        for case in cases:
            ops.own = False
            plain_out = [x.float() for x in ops.run(ops.prepare(case, 3)).values()]
            ops.own = True
            st = ops.prepare(case, 3)
            want = [x.clone() for x in ops.run(st).values()]
            for a, b in zip(want, plain_out):
                # both round to bf16 once (half a step each), weights once more: 4 half steps of the largest value
                assert float((a.float() - b).abs().max()) <= 4 * 2.0 ** -8 * float(b.abs().max()), case["op"]
            first = ops._context(st)[1]
            torch.cuda.synchronize()
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                ctx = ops._context(st)[1]
                assert ctx.stream == side.cuda_stream and ctx is not first
                got = [x.clone() for x in ops.run(st).values()]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), case["op"]
    finally:
        ops.own = before
        for c in ops._CONTEXTS.values():
            c.close()
        ops._CONTEXTS.clear()
