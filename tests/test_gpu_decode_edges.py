"""Calls of the decoder's operators that their header allows and that lie at an edge of it, on the GPU."""
import numpy as np
import pytest

from tests import decode_plain as plain
from tests.test_gpu_decode import _close, clone_cache, context, gen, new_cache, normal, slopes_of, within  # noqa: F401

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


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", [300.0, 1e4, 1e6, 1e9, 1e25, 2e38])
@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 2, 1, 64), ("bf16", 2, 1, 64), ("bf16", 2, 1, 80), ("bf16", 2, 2, 96), ("bf16", 4, 1, 128), ("bf16", 2, 1, 40)])
def test_caps_far_above_the_logits(lib, dtype, H, KV, dh, cap, slopes):
    """A cap that no logit comes near costs a logit 2^-18 of itself at most, however large the cap is: outputs are off by what they
    are without a cap, and by a mean of |v| times twice the largest change of a logit.
    At 300 logits past 3 / 32 of the cap stand beside small ones."""
    import torch
    ctx, g, off, std = context(dtype, H, dh), gen(int(np.log2(cap)) + dh), [0, 150, 331], 2.0
    qkv = normal(g, (331, (H + 2 * KV) * dh), dtype, std)
    qkv[[20, 200], :H * dh] *= 8                          # logits of a hundred among others
    sl = slopes_of(H) if slopes else None

    def more(q, k, v):   # twice what a logit may be off by for the cap (tanhf in float32: 8 half steps), times the largest value
        top = float((q.double() @ k.double().T.contiguous()).abs().max()) * dh ** -0.5
        return 2 * (2.0 ** -18 if dtype == "bf16" else 8 * plain.F32) * top * float(v.double().abs().max())
    score = lib.Score(cap=cap, slopes=sl)
    o = torch.empty((331, H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, KV, off, o, prefix=[3, 100], score=score)
    want = plain.masked(qkv, H, KV, off, True, [3, 100], None, None, None, cap, sl)[0]
    bound = plain.masked(qkv, H, KV, off, True, [3, 100], None, None, None, 0.0, sl)[1]
    x = qkv.view(331, H + 2 * KV, dh)
    q, k, v = x[:, :H].reshape(-1, dh), x[:, H:H + KV].reshape(-1, dh), x[:, H + KV:]
    within(o, want, bound + more(q, k, v), "masked")
    cache = new_cache(lib, g, dtype, 2, KV, 420, dh)
    before = clone_cache(lib, cache)
    for nodes in (1, 20, 40):                             # a few rows of a key head, and many
        rows, doff, cached = qkv[:2 * nodes].contiguous(), [0, nodes, 2 * nodes], [400, 129]
        pos = torch.arange(850, 850 + 2 * nodes, device="cuda", dtype=torch.int32)
        ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, doff, cached, add_mass=True), dtype=torch.uint8, device="cuda")
        o = torch.empty((2 * nodes, H * dh), dtype=qkv.dtype, device="cuda")
        cache.mass.copy_(before.mass)
        ctx.otas_attention_tree(cache, rows, doff, None, pos, [1, 0], cached, ws, o, score=score, add_mass=True)
        args = rows, H, cache.k, cache.v, cache.positions, before.mass, doff, None, pos, [1, 0], cached, None
        w, _, grown, _ = plain.tree(*args, cap, sl)
        _, b, _, gb = plain.tree(*args, 0.0, sl)
        extra = more(q, torch.cat([k, cache.k.reshape(-1, dh)]), torch.cat([v.reshape(-1, dh), cache.v.reshape(-1, dh)]))
        within(o, w, b + extra, "tree")
        for i, s in enumerate((1, 0)):                    # a weight is off by twice the change of itself
            grow = extra / float(torch.cat([v.reshape(-1, dh), cache.v.reshape(-1, dh)]).double().abs().max()) * (grown[s] - before.mass[s].double()).abs()
            within(cache.mass[s, :cached[i]], grown[s, :cached[i]], (gb[s] + grow)[:cached[i]] + 1e-30, "mass")


@pytest.mark.parametrize("dtype,H,KV,dh,nodes,cached", [("f32", 3, 3, 64, [1], [300]), ("f32", 3, 1, 8, [1, 0, 2], [900, 5, 300]), ("bf16", 3, 3, 64, [1], [600]),
                                                        ("bf16", 3, 1, 128, [1, 2], [0, 640]), ("bf16", 3, 1, 64, [15], [700]), ("bf16", 3, 1, 80, [41], [2000])])
def test_trees_of_an_odd_number_of_rows(lib, dtype, H, KV, dh, nodes, cached):
    """Rows times heads odd and several parts: the sums' place in the workspace is none that follows from the rows alone."""
    import torch
    ctx, g, B = context(dtype, H, dh), gen(dh + len(nodes)), len(nodes)
    cache = new_cache(lib, g, dtype, B, KV, max(cached), dh)
    before = clone_cache(lib, cache)
    off = [0, *np.cumsum(nodes).tolist()]
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    n = ctx.otas_attention_tree_workspace_bytes(KV, off, cached)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    o = torch.empty((off[-1], H * dh), dtype=qkv.dtype, device="cuda")
    assert off[-1] * H % 2 == 1
    ctx.otas_attention_tree(cache, qkv, off, None, None, list(range(B)), cached, ws[:n], o, add_mass=True)
    w, b, grown, gb = plain.tree(qkv, H, before.k, before.v, before.positions, before.mass, off, None, None, list(range(B)), cached)
    within(o, w, b, "tree")
    for q in range(B):
        within(cache.mass[q, :cached[q]], grown[q, :cached[q]], gb[q, :cached[q]] + 1e-30, "mass")
    assert bool((ws[n:] == 255).all())


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,H,KV,dh,T,rot,interleaved", [("f32", 2, 1, 64, 1, 64, False), ("f32", 4, 2, 20, 37, 10, True), ("f32", 4, 1, 128, 1101, 126, False),
                                                             ("bf16", 2, 1, 128, 8203, 128, False), ("bf16", 4, 2, 128, 8203, 122, False), ("bf16", 5, 5, 8, 70, 6, False),
                                                             ("bf16", 2, 1, 12, 65, 8, True), ("bf16", 4, 4, 80, 2051, 80, True), ("bf16", 2, 1, 100, 17, 98, False)])
def test_rotary_writes_its_rows_alone(lib, dtype, H, KV, dh, T, rot, interleaved, in_place):
    """Three rows on either side of the output keep their bits, in the kernels of whole and of odd halves."""
    import torch
    ctx, g, W = context(dtype, H, dh), gen(T + rot), (H + 2 * KV) * dh
    qkv = normal(g, (T, W), dtype)
    pos = torch.randint(0, 2 ** 17, (T,), generator=g, device="cuda", dtype=torch.int32)
    lead = 2 if W * qkv.element_size() % 16 else 3        # the output begins at a multiple of 16 bytes
    assert lead * W * qkv.element_size() % 16 == 0
    whole = torch.full((T + lead + 3, W), 7.0, dtype=qkv.dtype, device="cuda")
    out = whole[lead:lead + T]
    if in_place:
        out.copy_(qkv)
    ctx.otas_rotary(out if in_place else qkv, KV, pos, lib.Rotary(rot, layout=lib.OTAS_ROTARY_INTERLEAVED if interleaved else lib.OTAS_ROTARY_HALF), out)
    want, bound = plain.rotary(qkv, H, KV, pos, rot, interleaved, plain.frequencies(rot))
    within(out, want, bound + 1e-6 * (2.0 ** 17 * 2.0 ** -52 * 6.3), "rotary")
    assert bool((whole[:lead] == 7.0).all()) and bool((whole[lead + T:] == 7.0).all())


@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 4, 2, 64), ("bf16", 8, 2, 64), ("bf16", 12, 4, 80)])
def test_a_layer_of_the_librarys_operators(lib, dtype, H, KV, dh):
    """LayerNorm, a projection to grouped heads, rotation, masked attention, the cache, the next token over it, the projection back onto
    the float residual: every step against the 64-bit form on what the step before it gave."""
    import torch
    ctx, g, D = context(dtype, H, dh), gen(H * dh), H * dh
    off, T, W = [0, 130, 131, 200], 200, (H + 2 * KV) * dh
    half = plain.half_step(torch.float32 if dtype == "f32" else torch.bfloat16)
    x = normal(g, (T, D), dtype)
    gain, shift = normal(g, (D,), dtype, 0.1) + 1, normal(g, (D,), dtype, 0.1)
    w_in, b_in, w_out, b_out = normal(g, (W, D), dtype, D ** -0.5), normal(g, (W,), dtype), normal(g, (D, D), dtype, D ** -0.5), normal(g, (D,), dtype)

    def product(a, w, b):   # (result, what sums in float32 may be off by)
        p = a.double() @ w.double().T.contiguous() + b.double()
        return p, plain.F32 * (w.shape[1] + 2) * (a.double().abs() @ w.double().abs().T.contiguous() + b.double().abs())
    h = torch.empty_like(x)
    ctx.otas_layer_norm(x, gain, shift, T, h)
    z = x.double()
    s = (z - z.mean(1, keepdim=True)) / (z.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    want = s * gain.double() + shift.double()
    # the library's LayerNorm has tests of its own: mean and variance to within the sums' D half steps here
    within(h, want, half * want.abs() + plain.F32 * (D + 16) * (gain.double() * (1 + s.abs()) + want.abs()), "norm")
    qkv = torch.empty((T, W), dtype=x.dtype, device="cuda")
    ctx.otas_linear(h, w_in, b_in, None, T, W, D, 0, qkv)
    p, b = product(h, w_in, b_in)
    within(qkv, p, b + half * p.abs() * (1 + 2 ** -6), "projection")
    pos = torch.cat([torch.arange(z - a, device="cuda", dtype=torch.int32) for a, z in zip(off, off[1:])])
    rope = lib.Rotary(dh)
    p, b = plain.rotary(qkv, H, KV, pos, dh, False, plain.frequencies(dh))
    ctx.otas_rotary(qkv, KV, pos, rope, qkv)
    within(qkv, p, b, "rotary")
    o = torch.empty((T, D), dtype=x.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, KV, off, o)
    within(o, *plain.masked(qkv, H, KV, off, True), "attention")
    cache = new_cache(lib, g, dtype, 3, KV, 160, dh)
    rows = [i for a, z in zip(off, off[1:]) for i in range(a, z - 1)]   # all but every query's last row
    roff, slots = [0, 129, 129, 197], [2, 0, 1]
    filled = ctx.otas_cache_append(cache, qkv, roff, rows, pos, slots, [0, 0, 0]).tolist()
    last = qkv[[129, 130, 199]].contiguous()
    ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, [0, 1, 2, 3], filled), dtype=torch.uint8, device="cuda")
    o1 = torch.empty((3, D), dtype=x.dtype, device="cuda")
    ctx.otas_attention_tree(cache, last, [0, 1, 2, 3], None, None, slots, filled, ws, o1)
    p, b = plain.masked(qkv, H, KV, off, True)
    within(o1, p[[129, 130, 199]], b[[129, 130, 199]], "next token")
    res = x.float()
    p, b = product(o, w_out, b_out)
    want = p + res.double()
    ctx.otas_linear(o, w_out, b_out, res, T, D, D, 2, res)
    within(res, want, b + plain.F32 * (p.abs() + want.abs()) * 2, "residual")
