"""The decoder's operators on the GPU against their 64-bit forms (tests/decode_plain.py)."""
import numpy as np
import pytest

import otas_synth as synth
from tests import decode_plain as plain
from tests import harness as hz

pytestmark = pytest.mark.gpu

_CONTEXTS = {}


def context(dtype, H, dh):
    """One context per model shape for the whole module; otas_rotary and its like read no weights."""
    key = (dtype, H, dh)
    if key not in _CONTEXTS:
        cfg = synth.Config("decode", L=1, D=H * dh, H=H, F=64, dtype=dtype, B=1, n0=4, strategies=[(0, 0)], seed=5)
        _CONTEXTS[key] = hz.make_context(cfg)[0]
    return _CONTEXTS[key]


@pytest.fixture(scope="module", autouse=True)
def _close():
    yield
    for c in _CONTEXTS.values():
        c.close()
    _CONTEXTS.clear()


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, std=1.0):
    import torch
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(torch.float32 if dtype == "f32" else torch.bfloat16)


def within(got, want, bound, what=""):
    import torch
    bad = ~((got.double() - want).abs() <= bound)
    if bool(bad.any()):
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got {got[tuple(at)].item()}, want "
                             f"{want[tuple(at)].item()} within {bound[tuple(at)].item()}")


def slopes_of(H):
    import torch
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device="cuda")


# ------------------------------------------------------------------------------------------------------------ rotary
SCALINGS = {"plain": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0}, "parts": {"factor": 8.0, "original_length": 4096.0}}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,H,KV,dh,T,rot,interleaved,scaling,inverse", [
    ("f32", 3, 3, 64, 1, 64, False, "plain", False), ("f32", 4, 2, 20, 37, 10, False, "linear", False), ("f32", 4, 1, 20, 5, 18, True, "base", True),
    ("f32", 2, 1, 4, 3, 2, False, "plain", False), ("f32", 2, 2, 128, 1100, 128, True, "parts", False), ("f32", 2, 1, 36, 33, 24, False, "parts", True),
    ("bf16", 12, 4, 64, 197, 64, False, "parts", False), ("bf16", 4, 2, 80, 33, 40, False, "plain", False), ("bf16", 4, 4, 80, 7, 80, True, "linear", True),
    ("bf16", 8, 2, 96, 2049, 50, False, "base", False), ("bf16", 2, 1, 128, 8200, 128, False, "plain", False), ("bf16", 2, 1, 128, 9, 0, True, "plain", False),
    ("bf16", 2, 1, 12, 65, 12, True, "plain", False), ("bf16", 2, 1, 12, 65, 8, False, "plain", True), ("bf16", 2, 2, 64, 31, 6, True, "plain", False)])
def test_rotary(lib, dtype, H, KV, dh, T, rot, interleaved, scaling, inverse, in_place):
    import torch
    if H * dh % 8:
        pytest.skip("no such model width")
    ctx, g = context(dtype, H, dh), gen(T + rot)
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype)
    pos = torch.randint(-5, 2 ** 20, (T,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 2 ** 31 - 1
    kw = SCALINGS[scaling]
    codes = {"plain": lib.OTAS_ROTARY_PLAIN, "linear": lib.OTAS_ROTARY_LINEAR, "base": lib.OTAS_ROTARY_BASE, "parts": lib.OTAS_ROTARY_BY_PARTS}
    rope = lib.Rotary(rot, layout=lib.OTAS_ROTARY_INTERLEAVED if interleaved else lib.OTAS_ROTARY_HALF, base=5000.0, scaling=codes[scaling],
                      magnitude=0.75, inverse=inverse, **kw)
    want, bound = plain.rotary(qkv, H, KV, pos, rot, interleaved, plain.frequencies(rot, 5000.0, scaling, **kw) if rot else np.zeros(0), 0.75, inverse)
    whole = torch.full((T + 2, qkv.shape[1]), 7.0, dtype=qkv.dtype, device="cuda")   # rows on both sides stay as they were
    out = whole[1:T + 1] if (qkv.shape[1] * qkv.element_size()) % 16 == 0 else whole[:T]
    src = qkv
    if in_place:
        out.copy_(qkv)
        src = out
    ctx.otas_rotary(src, KV, pos, rope, out)
    # positions up to 2^31 in 64 bits: the oracle's own angle is good to 2^31 2^-53 turns x 2 pi, far below a float32 half step
    within(out, want, bound + 1e-6 * (2.0 ** 31 * 2.0 ** -52 * 6.3), "rotary")
    rest = whole.clone()
    rest[1:T + 1] = 7.0 if out.data_ptr() != whole.data_ptr() else rest[1:T + 1]
    assert bool((rest[-1] == 7.0).all())
    lo = torch.ones_like(want, dtype=torch.bool).view(T, H + 2 * KV, dh)
    lo[:, :H + KV, :rot] = False
    assert torch.equal(out[lo.view(T, -1)], qkv[lo.view(T, -1)])   # what does not turn keeps its bits


def test_rotary_and_its_inverse_are_gradients_of_each_other(lib):
    """The gradient of sum(w . rotary(x)) is the inverse rotation of w; against differences of the 64-bit form, and the magnitude once in each."""
    import torch
    H, KV, dh, T = 2, 1, 32, 5
    ctx, g = context("f32", H, dh), gen(3)
    x, w = normal(g, (T, (H + 2 * KV) * dh), "f32"), normal(g, (T, (H + 2 * KV) * dh), "f32")
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 100
    grad = torch.empty_like(w)
    ctx.otas_rotary(w, KV, pos, lib.Rotary(24, magnitude=1.25, inverse=True), grad)
    f = plain.frequencies(24)
    for row, col in [(0, 0), (1, 3), (2, 11), (3, 12), (4, 23), (4, 30), (3, 40), (2, 70), (1, 100)]:
        d = torch.zeros_like(x, dtype=torch.float64)
        d[row, col] = 1e-3

        def value(v):   # the 64-bit form is linear: differences are exact up to rounding
            out = v.clone().view(T, H + 2 * KV, dh)
            a = torch.from_numpy(pos.cpu().numpy()[:, None] * f[None, :]).to("cuda")[:, None, :]
            p, q = out[:, :H + KV, :12].clone(), out[:, :H + KV, 12:24].clone()
            out[:, :H + KV, :12], out[:, :H + KV, 12:24] = 1.25 * (p * a.cos() - q * a.sin()), 1.25 * (p * a.sin() + q * a.cos())
            return float((out.view(T, -1) * w.double()).sum())
        diff = (value(x.double() + d) - value(x.double() - d)) / 2e-3
        assert abs(diff - float(grad[row, col])) <= 20 * plain.F32 * 1.25 * 8, (row, col)


# ------------------------------------------------------------------------------------------------------ packed rows
MASKED = [
    # dtype, H, KV, dh, lengths, causal, prefix, documents, cap, slopes, positions
    ("f32", 3, 3, 64, [201, 1, 0, 33], True, None, False, 0.0, False, False),
    ("f32", 4, 2, 20, [65, 64, 7], True, [5, 64, 0], False, 5.0, True, False),
    ("f32", 2, 1, 128, [300, 31], False, None, True, 0.0, True, True),
    ("f32", 4, 1, 36, [129, 128, 127], True, [40, 0, 127], True, 2.0, False, False),
    ("bf16", 12, 4, 64, [197, 1, 64, 65, 0, 2, 128], True, None, False, 0.0, False, False),
    ("bf16", 12, 12, 64, [261, 33], True, [197, 33], False, 30.0, False, False),
    ("bf16", 4, 2, 80, [577, 100, 129], True, [16, 0, 129], True, 0.0, True, False),
    ("bf16", 2, 1, 96, [400, 31], False, [0, 31], True, 20.0, True, True),
    ("bf16", 4, 1, 128, [1000, 129, 3], True, None, False, 4.0, False, False),
    ("bf16", 2, 2, 128, [257, 512, 1], False, None, False, 0.0, False, False),
    ("bf16", 2, 1, 128, [1300], True, [700], True, 0.0, True, True),
    ("bf16", 2, 1, 32, [90, 5], True, [7, 0], True, 3.0, True, False),
]


def documents_of(g, lengths):
    """A few documents a query, in no order, padding among them; one query of padding alone where there are several."""
    import torch
    docs = [torch.randint(-1, 3, ((n + 15) // 16,), generator=g, device="cuda", dtype=torch.int32).repeat_interleave(16)[:n] for n in lengths]
    if len(lengths) > 1:
        docs[1].fill_(-3)
    return torch.cat(docs)


@pytest.mark.parametrize("dtype,H,KV,dh,lengths,causal,prefix,docs,cap,slopes,posit", MASKED)
def test_attention_masked(lib, dtype, H, KV, dh, lengths, causal, prefix, docs, cap, slopes, posit):
    import torch
    ctx, g = context(dtype, H, dh), gen(sum(lengths) + dh)
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    T = int(off[-1])
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype, 1.5)
    d = documents_of(g, lengths) if docs else None
    pos = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32) if posit else None
    sl = slopes_of(H) if slopes else None
    whole = torch.full((T + 64, H * dh), 5.0, dtype=qkv.dtype, device="cuda")
    o = whole[:T]
    ctx.otas_attention_masked(qkv, KV, off, o, causal=causal, prefix=prefix, documents=d, positions=pos, score=lib.Score(cap=cap, slopes=sl))
    want, bound = plain.masked(qkv, H, KV, off, causal, prefix, d, pos, None, cap, sl)
    within(o, want, bound, "masked")
    assert bool((whole[T:] == 5.0).all())
    if d is not None:
        assert bool((o[d < 0] == 0).all()) and bool((d < 0).any())
    again = torch.empty_like(o)
    ctx.otas_attention_masked(qkv, KV, off, again, causal=causal, prefix=prefix, documents=d, positions=pos, score=lib.Score(cap=cap, slopes=sl))
    assert torch.equal(o, again)


@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 2, 1, 64), ("bf16", 2, 1, 64), ("bf16", 2, 2, 128), ("bf16", 2, 1, 80), ("bf16", 2, 1, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(lib, dtype, H, KV, dh):
    """Infinities and NaN in later keys and values, in padding and in other documents; and those that a row does see do reach it."""
    import torch
    ctx, g, n = context(dtype, H, dh), gen(9), 200
    qkv = normal(g, (n, (H + 2 * KV) * dh), dtype)
    d = torch.zeros(n, dtype=torch.int32, device="cuda")
    d[150:] = 1
    d[60:70] = -1
    clean, dirty = torch.empty((n, H * dh), dtype=qkv.dtype, device="cuda"), torch.empty((n, H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, KV, [0, n], clean, documents=d)
    x = qkv.clone()
    k0 = H * dh
    x[60:70, k0:] = float("nan")                       # padding
    x[65, k0:] = float("inf")
    x[140, k0 + KV * dh + 3] = float("nan")            # a value: column 3 of the rows of document 0 from 140 on
    x[141, k0 + KV * dh + 5] = float("inf")            # column 5 from 141 on
    x[142, k0 + KV * dh + 5] = -float("inf")           # inf - inf from 142 on
    x[143, k0 + KV * dh + 6] = -float("inf")
    x[190, k0:] = float("nan")                         # a key: rows from 190 on
    ctx.otas_attention_masked(x, KV, [0, n], dirty, documents=d)
    free = torch.ones((n, H * dh), dtype=torch.bool, device="cuda")
    heads = [h for h in range(H) if h // (H // KV) == 0]
    for h in heads:
        free[140:150, h * dh + 3] = False
        free[141:150, h * dh + 5] = False
        free[143:150, h * dh + 6] = False
        assert bool(dirty[140:150, h * dh + 3].isnan().all())
        assert float(dirty[141, h * dh + 5]) == float("inf") and bool(dirty[142:150, h * dh + 5].isnan().all())
        assert bool((dirty[143:150, h * dh + 6] == -float("inf")).all())
    free[190:] = False
    assert bool(dirty[190:].isnan().all())
    assert torch.equal(clean[free], dirty[free])


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 64), ("bf16", 128)])
def test_masked_rows_of_extreme_logits(lib, dtype, dh):
    """Logits of +-3e4: the largest key takes all; logits of minus infinity everywhere: zero."""
    import torch
    ctx, n = context(dtype, 2, dh), 70
    qkv = torch.zeros((n, 4 * dh), dtype=ctx.torch_dtype, device="cuda")
    qkv[:, 0] = 512.0
    qkv[:, dh] = 512.0
    qkv[:, 2 * dh] = torch.where(torch.arange(n, device="cuda") % 64 == 33, 480.0, -480.0).to(qkv.dtype)
    qkv[:, 3 * dh:] = torch.arange(n, device="cuda")[:, None].to(qkv.dtype)
    o = torch.empty((n, 2 * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, 1, [0, n], o, causal=False)
    assert bool((o == 33.0).all())
    qkv[:, 2 * dh] = -float("inf")
    ctx.otas_attention_masked(qkv, 1, [0, n], o, causal=False)
    assert bool((o == 0.0).all())


def test_masked_agrees_with_the_encoders_attention(lib):
    """No mask, as many key heads as heads: what otas_attention computes."""
    import torch
    for dtype in ("f32", "bf16"):
        ctx, g = context(dtype, 3, 64), gen(4)
        off = [0, 197, 198, 300]
        qkv = normal(g, (300, 9 * 64), dtype)
        a, b = torch.empty((300, 192), dtype=qkv.dtype, device="cuda"), torch.empty((300, 192), dtype=qkv.dtype, device="cuda")
        ctx.otas_attention(qkv, None, off, 0, a)
        ctx.otas_attention_masked(qkv, 3, off, b, causal=False)
        want, bound = plain.masked(qkv, 3, 3, off, False)
        within(a, want, bound)
        within(b, want, bound)


# ---------------------------------------------------------------------------------------------------------- the cache
def new_cache(lib, g, dtype, slots, KV, capacity, dh, mass=True):
    import torch
    k, v = normal(g, (slots, KV, capacity, dh), dtype), normal(g, (slots, KV, capacity, dh), dtype)
    pos = torch.rand((slots, 2 * capacity), generator=g, device="cuda").argsort(dim=1)[:, :capacity].to(torch.int32).contiguous()
    m = torch.rand((slots, capacity), generator=g, device="cuda") if mass else None
    return lib.KVCache(k, v, pos, m)


def clone_cache(lib, c):
    return lib.KVCache(c.k.clone(), c.v.clone(), c.positions.clone(), None if c.mass is None else c.mass.clone())


def same_cache(a, b):
    import torch
    return all(x is None and y is None or torch.equal(x, y) for x, y in zip((a.k, a.v, a.positions, a.mass), (b.k, b.v, b.positions, b.mass)))


@pytest.mark.parametrize("dtype,H,KV,dh,counts,with_rows,mass", [
    ("f32", 3, 3, 64, [4, 0, 9], False, True), ("bf16", 4, 2, 80, [1], False, False), ("bf16", 2, 1, 12, [7, 3], True, True),
    ("bf16", 4, 1, 128, [30, 1, 12, 2], True, True), ("f32", 2, 2, 20, [500, 600], True, True), ("bf16", 2, 2, 64, [1] * 400, False, True)])
def test_cache_append(lib, dtype, H, KV, dh, counts, with_rows, mass):
    import torch
    if H * dh % 8:
        pytest.skip("no such model width")
    ctx, g, rng = context(dtype, H, dh), gen(len(counts)), np.random.default_rng(len(counts))
    B, capacity = len(counts), 700
    cache = new_cache(lib, g, dtype, B + 2, KV, capacity, dh, mass)
    want = clone_cache(lib, cache)
    off = np.concatenate([[0], np.cumsum(counts)])
    T = int(off[-1]) + 3
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype)
    pos = torch.randint(0, 9999, (T,), generator=g, device="cuda", dtype=torch.int32)
    slots = [int(s) for s in rng.permutation(B + 2)[:B]]
    lens = [int(rng.integers(0, capacity - c + 1)) for c in counts]
    lens[-1] = capacity - counts[-1]                    # to the brim
    rows = [int(r) for r in rng.integers(0, T, int(off[-1]))] if with_rows else None
    out = ctx.otas_cache_append(cache, qkv, off, rows, pos, slots, lens)
    assert out.tolist() == [l + c for l, c in zip(lens, counts)]
    x = qkv.view(T, H + 2 * KV, dh)
    for q in range(B):
        mine = list(range(int(off[q]), int(off[q + 1]))) if rows is None else rows[int(off[q]):int(off[q + 1])]
        to = slice(lens[q], lens[q] + counts[q])
        want.k[slots[q], :, to] = x[mine, H:H + KV].transpose(0, 1)
        want.v[slots[q], :, to] = x[mine, H + KV:].transpose(0, 1)
        want.positions[slots[q], to] = pos[mine]
        if mass:
            want.mass[slots[q], to] = 0
    assert same_cache(cache, want)


def tree_of(rng, n, kind):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "roots":
        return [-1 if i % 5 == 0 else int(rng.integers(0, i)) for i in range(n)]
    return [-1 if i == 0 else int(rng.integers(max(0, i - 4), i)) for i in range(n)]


TREES = [
    # dtype, H, KV, dh, nodes, cached, kind, cap, slopes, mass
    ("f32", 3, 3, 64, [1], [0], None, 0.0, False, False),
    ("f32", 4, 2, 20, [5, 1, 0, 64], [33, 0, 7, 129], "tree", 3.0, True, True),
    ("f32", 2, 1, 128, [9], [1500], "roots", 0.0, False, True),
    ("bf16", 4, 1, 128, [1], [1537], None, 0.0, True, False),
    ("bf16", 4, 1, 128, [1], [5000], None, 0.0, False, True),
    ("bf16", 12, 4, 64, [1, 1, 1, 1, 1], [0, 1, 31, 128, 700], None, 20.0, False, True),
    ("bf16", 8, 2, 64, [17, 64, 1, 33], [500, 129, 0, 2000], "tree", 0.0, True, True),
    ("bf16", 16, 2, 128, [48, 64], [4000, 63], "tree", 30.0, False, False),
    ("bf16", 4, 2, 80, [12, 7, 2], [300, 1, 64], "roots", 0.0, True, True),
    ("bf16", 8, 1, 96, [20, 40], [257, 256], "tree", 0.0, False, True),
    ("bf16", 2, 1, 32, [4, 10], [100, 0], "tree", 5.0, True, True),
    ("bf16", 16, 16, 64, [3, 2], [900, 64], None, 0.0, False, True),
]


@pytest.mark.parametrize("dtype,H,KV,dh,nodes,cached,kind,cap,slopes,mass", TREES)
def test_attention_tree(lib, dtype, H, KV, dh, nodes, cached, kind, cap, slopes, mass):
    import torch
    ctx, g, rng = context(dtype, H, dh), gen(sum(nodes) + dh), np.random.default_rng(sum(cached) + H)
    B = len(nodes)
    capacity = max(max(cached), 1) + 5
    cache = new_cache(lib, g, dtype, B + 1, KV, capacity, dh)
    slots = [int(s) for s in rng.permutation(B + 1)[:B]]
    for q in range(B):                                  # what is behind the entries may be anything
        cache.k[slots[q], :, cached[q]:] = float("nan")
        cache.v[slots[q], :, cached[q]:] = float("inf")
        cache.mass[slots[q], cached[q]:] = float("nan")
    off = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    T = int(off[-1])
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype, 1.5)
    parents = None if kind is None else sum([tree_of(rng, n, kind) for n in nodes], [])
    pos = torch.randint(2 * capacity, 2 * capacity + 50, (T,), generator=g, device="cuda", dtype=torch.int32)
    sl = slopes_of(H) if slopes else None
    before = clone_cache(lib, cache)
    ws = torch.full((ctx.otas_attention_tree_workspace_bytes(KV, off, cached),), 255, dtype=torch.uint8, device="cuda")
    whole = torch.full((T + 8, H * dh), 5.0, dtype=qkv.dtype, device="cuda")
    o = whole[:T]
    ctx.otas_attention_tree(cache, qkv, off, parents, pos, slots, cached, ws, o, score=lib.Score(cap=cap, slopes=sl), add_mass=mass)
    want, bound, grown, grown_bound = plain.tree(qkv, H, before.k, before.v, before.positions, before.mass if mass else None, off, parents, pos, slots, cached,
                                                 None, cap, sl)
    within(o, want, bound, "tree")
    assert bool((whole[T:] == 5.0).all())
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip((cache.k, cache.v), (before.k, before.v)))
    for q in range(B):
        n = cached[q]
        if mass:
            within(cache.mass[slots[q], :n], grown[slots[q], :n], grown_bound[slots[q], :n] + 1e-30, "mass")
        else:
            assert torch.equal(cache.mass[slots[q], :n], before.mass[slots[q], :n])
        assert bool(cache.mass[slots[q], n:].isnan().all())
    o2, c2 = torch.empty_like(o), before
    ctx.otas_attention_tree(c2, qkv, off, parents, pos, slots, cached, ws, o2, score=lib.Score(cap=cap, slopes=sl), add_mass=mass)
    assert torch.equal(o, o2) and torch.equal(cache.mass.nan_to_num(9.0), c2.mass.nan_to_num(9.0))


@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 2, 1, 64), ("bf16", 2, 1, 64), ("bf16", 4, 1, 128)])
def test_siblings_do_not_reach_each_other(lib, dtype, H, KV, dh):
    import torch
    ctx, g = context(dtype, H, dh), gen(2)
    cache = new_cache(lib, g, dtype, 1, KV, 40, dh)
    parents = [-1, 0, 0, 1, 2]
    qkv = normal(g, (5, (H + 2 * KV) * dh), dtype)
    ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, [0, 5], [40]), dtype=torch.uint8, device="cuda")
    clean, dirty = torch.empty((5, H * dh), dtype=qkv.dtype, device="cuda"), torch.empty((5, H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_tree(cache, qkv, [0, 5], parents, None, [0], [40], ws, clean)
    x = qkv.clone()
    x[1, H * dh:] = float("nan")
    x[4, H * dh:] = float("inf")
    ctx.otas_attention_tree(cache, x, [0, 5], parents, None, [0], [40], ws, dirty)
    assert torch.equal(clean[[0, 2]], dirty[[0, 2]]) and bool(dirty[[1, 3]].isnan().all()) and bool(dirty[4].isnan().all())


def test_queries_that_share_a_slot(lib):
    """Two queries may read one cache (a beam); the same rows then get the same answer as on their own."""
    import torch
    ctx, g = context("bf16", 4, 64), gen(6)
    cache = new_cache(lib, g, "bf16", 2, 2, 300, 64)
    qkv = normal(g, (2, 8 * 64), "bf16")
    ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(2, [0, 1, 2], [290, 250]), dtype=torch.uint8, device="cuda")
    o = torch.empty((2, 256), dtype=torch.bfloat16, device="cuda")
    ctx.otas_attention_tree(cache, qkv, [0, 1, 2], None, None, [1, 1], [290, 250], ws, o)
    want, bound, _, _ = plain.tree(qkv, 4, cache.k, cache.v, cache.positions, None, [0, 1, 2], None, None, [1, 1], [290, 250])
    within(o, want, bound)


@pytest.mark.parametrize("dtype,KV,dh,lengths,keep,lead,recent,kind", [
    ("f32", 3, 64, [100, 7, 0], [60, 7, 5], 4, 30, "random"), ("bf16", 2, 80, [1000, 999, 1], [10, 0, 1], 0, None, "random"),
    ("bf16", 1, 12, [300, 65], [299, 64], 1, 10, "ties"), ("bf16", 1, 128, [5000, 40], [3000, 1], 2, 100, "odd"),
    ("f32", 1, 20, [2000], [1999], 0, None, "ties"), ("f32", 1, 4, [20000], [9000], 4, 500, "odd"), ("bf16", 1, 64, [64] * 250, [40] * 250, 1, 3, "random"),
    ("bf16", 1, 64, [130], [20], 64, None, "random"), ("bf16", 1, 12, [40000, 3], [30000, 2], 3, 70, "odd"), ("bf16", 1, 12, [32768, 32767], [1, 32766], 0, None, "ties")])
def test_cache_evict(lib, dtype, KV, dh, lengths, keep, lead, recent, kind):
    import torch
    H = 2 if KV < 3 else 3
    if H * dh % 8:
        H *= 2
    ctx, g, rng = context(dtype, H, dh), gen(len(lengths)), np.random.default_rng(1)
    B, capacity = len(lengths), max(lengths) + 3
    cache = new_cache(lib, g, dtype, B + 1, KV, capacity, dh)
    if kind == "ties":
        cache.mass.copy_((cache.mass * 3).floor())
    if kind == "odd":
        cache.mass.sub_(0.5).mul_(1e-3)
        cache.mass[:, 5::11] = float("inf")
        cache.mass[:, 6::13] = -float("inf")
        cache.mass[:, 7::17] = float("nan")
        cache.mass[:, 8::19] = 0.0
        cache.mass[:, 9::19] = -0.0
        cache.mass[:, 10::23] = 1e-42
    slots = [int(s) for s in rng.permutation(B + 1)[:B]]
    recent_from = None if recent is None else [2 * capacity - recent] * B
    want = clone_cache(lib, cache)
    for q, (to, src) in enumerate(plain.evict(cache.mass, cache.positions, slots, lengths, keep, lead, recent_from)):
        assert len(to) == len(src)
        if to:
            s = slots[q]
            want.k[s][:, to], want.v[s][:, to] = want.k[s][:, src], want.v[s][:, src]
            want.positions[s][to], want.mass[s][to] = want.positions[s][src], want.mass[s][src]
    ws = torch.full((ctx.otas_cache_evict_workspace_bytes(lengths, keep),), 255, dtype=torch.uint8, device="cuda")
    out = ctx.otas_cache_evict(cache, slots, lengths, keep, ws, lead=lead, recent_from=recent_from)
    assert out.tolist() == [min(a, b) for a, b in zip(lengths, keep)]
    assert torch.equal(cache.k, want.k) and torch.equal(cache.v, want.v) and torch.equal(cache.positions, want.positions)
    assert torch.equal(cache.mass.view(torch.int32), want.mass.view(torch.int32))


# -------------------------------------------------------------------------------------------------------- as they are used
def test_a_decoders_layer_from_prompt_to_eviction(lib):
    """Pictures and text in, then drafts: rotate, attend under the prefix mask, fill the cache; a tree of drafts is verified, a path
    of it accepted and appended; the cache is cut, and the next token attends to what is left.  Every attention against the 64-bit
    form on the same rotated rows."""
    import torch
    H, KV, dh, capacity = 4, 2, 64, 256
    for dtype in ("f32", "bf16"):
        ctx, g, rng = context(dtype, H, dh), gen(77), np.random.default_rng(7)
        lens, prefix = [197, 60], [190, 0]
        off = [0, 197, 257]
        rope = lib.Rotary(48, layout=lib.OTAS_ROTARY_INTERLEAVED)
        qkv = normal(g, (257, (H + 2 * KV) * dh), dtype)
        pos = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in lens])
        want, bound = plain.rotary(qkv, H, KV, pos, 48, True, plain.frequencies(48))
        ctx.otas_rotary(qkv, KV, pos, rope, qkv)
        within(qkv, want, bound)
        o = torch.empty((257, H * dh), dtype=qkv.dtype, device="cuda")
        ctx.otas_attention_masked(qkv, KV, off, o, prefix=prefix)
        within(o, *plain.masked(qkv, H, KV, off, True, prefix))
        cache = new_cache(lib, g, dtype, 3, KV, capacity, dh)
        slots = [2, 0]
        filled = ctx.otas_cache_append(cache, qkv, off, None, pos, slots, [0, 0]).tolist()
        assert filled == lens
        # the whole prompt is in the cache: its last token, taken as a draft over the entries before it, gives the prompt's answer
        last = torch.stack([qkv[196], qkv[256]]).contiguous()
        ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
        o1 = torch.empty((2, H * dh), dtype=qkv.dtype, device="cuda")
        ctx.otas_attention_tree(cache, last, [0, 1, 2], None, None, slots, [196, 59], ws, o1)
        w, b = plain.masked(qkv, H, KV, off, True, prefix)
        within(o1, w[[196, 256]], b[[196, 256]])
        for step in range(3):
            nodes = [6, 9]
            doff = [0, 6, 15]
            parents = tree_of(rng, 6, "tree") + tree_of(rng, 9, "roots")
            x = normal(g, (15, (H + 2 * KV) * dh), dtype)
            dpos = torch.tensor([500 + 20 * step + i for i in range(15)], dtype=torch.int32, device="cuda")
            ctx.otas_rotary(x, KV, dpos, rope, x)
            before = clone_cache(lib, cache)
            od = torch.empty((15, H * dh), dtype=x.dtype, device="cuda")
            assert ctx.otas_attention_tree_workspace_bytes(KV, doff, filled) <= ws.numel()
            ctx.otas_attention_tree(cache, x, doff, parents, dpos, slots, filled, ws, od, add_mass=True)
            w, b, grown, gb = plain.tree(x, H, before.k, before.v, before.positions, before.mass, doff, parents, dpos, slots, filled)
            within(od, w, b)
            for q in range(2):
                within(cache.mass[slots[q], :filled[q]], grown[slots[q], :filled[q]], gb[slots[q], :filled[q]])
            rows = [0, 2, 6, 8, 9]
            filled = ctx.otas_cache_append(cache, x, [0, 2, 5], rows, dpos, slots, filled).tolist()
            keep = [filled[0] - 11, filled[1] - 2]
            moves = plain.evict(cache.mass, cache.positions, slots, filled, keep, 4, [490, 490])
            expect = clone_cache(lib, cache)
            for q, (to, src) in enumerate(moves):
                s = slots[q]
                expect.k[s][:, to], expect.v[s][:, to] = expect.k[s][:, src], expect.v[s][:, src]
                expect.positions[s][to], expect.mass[s][to] = expect.positions[s][src], expect.mass[s][src]
            filled = ctx.otas_cache_evict(cache, slots, filled, keep, ws, lead=4, recent_from=[490, 490]).tolist()
            assert filled == keep and same_cache(cache, expect)


def test_a_captured_step_on_a_stream_of_its_own(lib):
    """Rotation, tree, append and eviction captured into a graph on the context's stream and replayed between eager calls: every
    replay does what the eager calls do on the same memory."""
    import torch
    import paper_2401_05031_amd as otas
    H, KV, dh, capacity = 4, 2, 64, 640
    stream = torch.cuda.Stream()
    cfg = synth.Config("graph", L=1, D=H * dh, H=H, F=64, dtype="bf16", B=1, n0=4, strategies=[(0, 0)], seed=5)
    layers = synth.all_weights(cfg)
    ctx = otas.Context.from_host_weights(1, H * dh, H, 64, otas.OTAS_BF16, 1e-6, 1, layers, stream=stream.cuda_stream)
    g = gen(12)
    cache = new_cache(lib, g, "bf16", 2, KV, capacity, dh)
    qkv = normal(g, (7, (H + 2 * KV) * dh), "bf16")
    pos = torch.tensor([900, 901, 901, 902, 50, 51, 52], dtype=torch.int32, device="cuda")
    x, o = torch.empty_like(qkv), torch.empty((7, H * dh), dtype=qkv.dtype, device="cuda")
    off, parents, slots, lens = [0, 4, 7], [-1, 0, 0, 1, -1, 0, 1], [1, 0], [600, 40]
    rope, score = lib.Rotary(64), lib.Score(cap=20.0, slopes=slopes_of(H))
    ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, off, lens), dtype=torch.uint8, device="cuda")
    we = torch.empty(ctx.otas_cache_evict_workspace_bytes([603, 42], [500, 42]), dtype=torch.uint8, device="cuda")

    def step():
        ctx.otas_rotary(qkv, KV, pos, rope, x)
        ctx.otas_attention_tree(cache, x, off, parents, pos, slots, lens, ws, o, score=score, add_mass=True)
        ctx.otas_cache_append(cache, x, [0, 3, 5], [0, 1, 3, 4, 5], pos, slots, lens)
        ctx.otas_cache_evict(cache, slots, [603, 42], [500, 42], we, lead=1, recent_from=[890, 890])

    first = clone_cache(lib, cache)
    inputs = [normal(g, (7, (H + 2 * KV) * dh), "bf16") for _ in range(3)]

    def restore(i):
        for a, b in zip((cache.k, cache.v, cache.positions, cache.mass), (first.k, first.v, first.positions, first.mass)):
            a.copy_(b)
        qkv.copy_(inputs[i])
        o.fill_(3.0)

    torch.cuda.synchronize()
    want = []
    for i in range(3):
        restore(i)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want.append((o.clone(), clone_cache(lib, cache)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in (2, 0, 1, 0):
        restore(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[i][0]) and same_cache(cache, want[i][1]), i
        other = torch.empty_like(x)
        ctx.otas_rotary(x, KV, pos, rope, other)
        torch.cuda.synchronize()
    # host numbers that do not fit the kernels' arguments are refused under capture, and work outside
    many = list(range(400))
    big = new_cache(lib, g, "bf16", 400, 1, 4, 64)
    rows = normal(g, (400, (H + 2) * dh), "bf16")
    p400 = torch.zeros(400, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2, stream=stream):
        with pytest.raises(lib.OtasError) as e:
            ctx.otas_cache_append(big, rows, list(range(401)), None, p400, many, [0] * 400)
        assert e.value.status == 5
        ctx.otas_rotary(qkv, KV, pos, rope, x)
    ctx.otas_cache_append(big, rows, list(range(401)), None, p400, many, [0] * 400)
    torch.cuda.synchronize()
    assert torch.equal(big.k[:, 0, 0], rows.view(400, H + 2, dh)[:, H])
    ctx.close()


def test_calls_that_the_binding_refuses(lib):
    """Wrong shapes, types and places of tensors raise before the library is called; wrong numbers come back as statuses."""
    import torch
    H, KV, dh = 4, 2, 64
    ctx, g = context("bf16", H, dh), gen(1)
    qkv = normal(g, (6, (H + 2 * KV) * dh), "bf16")
    pos = torch.zeros(6, dtype=torch.int32, device="cuda")
    o = torch.empty((6, H * dh), dtype=torch.bfloat16, device="cuda")
    cache = new_cache(lib, g, "bf16", 2, KV, 50, dh)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rope = lib.Rotary(64)
    for call in (lambda: ctx.otas_rotary(qkv.float(), KV, pos, rope, qkv), lambda: ctx.otas_rotary(qkv, 4, pos, rope, qkv),
                 lambda: ctx.otas_rotary(qkv, KV, pos.long(), rope, qkv), lambda: ctx.otas_rotary(qkv, KV, pos[:5], rope, qkv),
                 lambda: ctx.otas_rotary(qkv, KV, pos, rope, qkv[:5]), lambda: ctx.otas_rotary(qkv.cpu(), KV, pos, rope, qkv),
                 lambda: ctx.otas_rotary(qkv.t().contiguous().t(), KV, pos, rope, qkv),
                 lambda: ctx.otas_attention_masked(qkv, KV, [0, 5], o), lambda: ctx.otas_attention_masked(qkv, KV, [0, 6], o, prefix=[1, 2]),
                 lambda: ctx.otas_attention_masked(qkv, KV, [0, 6], o, documents=pos.float()),
                 lambda: ctx.otas_attention_masked(qkv, KV, [0, 6], o, score=lib.Score(slopes=slopes_of(5))),
                 lambda: ctx.otas_attention_tree(cache, qkv, [0, 6], [-1] * 5, pos, [0], [3], ws, o),
                 lambda: ctx.otas_attention_tree(cache, qkv, [0, 6], None, pos, [0, 1], [3], ws, o),
                 lambda: ctx.otas_cache_append(cache, qkv, [0, 6], [0], pos, [0], [3]),
                 lambda: lib.KVCache(cache.k, cache.v[:1], cache.positions), lambda: lib.KVCache(cache.k, cache.v, cache.positions[:, :4])):
        with pytest.raises(ValueError):
            call()
    tree = lambda **kw: ctx.otas_attention_tree(cache, qkv, kw.get("off", [0, 6]), kw.get("par"), kw.get("pos", pos), kw.get("slot", [0]),  # noqa: E731
                                                kw.get("len", [3]), kw.get("ws", ws), o, score=kw.get("score"), add_mass=kw.get("mass", False))
    for status, call in ((1, lambda: tree(par=[0, 0, 0, 0, 0, 0])), (1, lambda: tree(par=[-1, 0, 0, 0, 0, -2])), (1, lambda: tree(slot=[2])),
                         (1, lambda: tree(slot=[-1])), (1, lambda: tree(len=[51])), (1, lambda: tree(off=[0, 3, 6], slot=[1, 1], len=[3, 4], mass=True)),
                         (1, lambda: tree(pos=None, score=lib.Score(slopes=slopes_of(H)))), (1, lambda: tree(score=lib.Score(cap=-1.0))),
                         (3, lambda: tree(ws=ws[:128])), (1, lambda: tree(ws=ws[8:])),
                         (1, lambda: ctx.otas_cache_append(cache, qkv, [0, 6], None, pos, [0], [45])),
                         (1, lambda: ctx.otas_cache_append(cache, qkv, [0, 3, 6], None, pos, [0, 0], [4, 4])),
                         (1, lambda: ctx.otas_cache_append(cache, qkv, [0, 2], [0, 6], pos, [0], [4])),
                         (1, lambda: ctx.otas_cache_evict(cache, [0, 0], [9, 9], [4, 4], ws)),
                         (3, lambda: ctx.otas_cache_evict(cache, [0, 1], [50, 50], [25, 25], ws[:256])),
                         (1, lambda: ctx.otas_cache_evict(lib.KVCache(cache.k, cache.v, cache.positions), [0], [9], [4], ws)),
                         (1, lambda: ctx.otas_attention_masked(qkv, KV, [0, 6], o, prefix=[7])),
                         (1, lambda: ctx.otas_rotary(qkv, KV, pos, lib.Rotary(63), qkv)), (1, lambda: ctx.otas_rotary(qkv, KV, pos, lib.Rotary(66), qkv))):
        with pytest.raises(lib.OtasError) as e:
            call()
        assert e.value.status == status, call


# ------------------------------------------------------------------------------------- calls at the edges of the header
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,H,KV,dh,T,rot", [("bf16", 4, 2, 128, 8203, 122), ("bf16", 3, 1, 64, 300, 58), ("bf16", 2, 2, 80, 1030, 2), ("bf16", 5, 5, 8, 70, 6),
                                                 ("bf16", 2, 1, 100, 17, 98), ("bf16", 4, 4, 96, 2050, 72), ("f32", 4, 1, 128, 8200, 126), ("f32", 2, 2, 68, 9, 66),
                                                 ("f32", 4, 2, 4, 1100, 2)])
def test_rotary_halves_that_no_chunk_divides(lib, dtype, H, KV, dh, T, rot, in_place):
    import torch
    ctx, g = context(dtype, H, dh), gen(T + rot)
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype)
    pos = torch.randint(0, 2 ** 17, (T,), generator=g, device="cuda", dtype=torch.int32)
    want, bound = plain.rotary(qkv, H, KV, pos, rot, False, plain.frequencies(rot))
    src = qkv.clone()
    out = src if in_place else torch.empty_like(qkv)
    ctx.otas_rotary(src, KV, pos, lib.Rotary(rot), out)
    within(out, want, bound + 1e-6 * (2.0 ** 17 * 2.0 ** -52 * 6.3), "rotary")
    assert in_place or torch.equal(src, qkv)
    kept = torch.ones((H + 2 * KV, dh), dtype=torch.bool, device="cuda")
    kept[:H + KV, :rot] = False
    assert torch.equal(out.view(T, -1, dh)[:, kept], qkv.view(T, -1, dh)[:, kept])


@pytest.mark.parametrize("scale", [-0.25, 0.03125, 1.5])
@pytest.mark.parametrize("dtype,H,KV,dh,cap,slopes", [("f32", 2, 1, 64, 0.0, True), ("f32", 2, 1, 36, 3.0, False), ("bf16", 2, 1, 64, 0.0, False), ("bf16", 2, 2, 80, 0.0, True),
                                                      ("bf16", 4, 1, 128, 20.0, False), ("bf16", 2, 1, 96, 5.0, True)])
def test_scales_of_either_sign(lib, dtype, H, KV, dh, cap, slopes, scale):
    import torch
    ctx, g, off = context(dtype, H, dh), gen(int(scale * 64) + dh), [0, 150, 331]
    qkv = normal(g, (331, (H + 2 * KV) * dh), dtype)
    sl = slopes_of(H) if slopes else None
    score = lib.Score(scale=scale, cap=cap, slopes=sl)
    o = torch.empty((331, H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, KV, off, o, prefix=[3, 100], score=score)
    within(o, *plain.masked(qkv, H, KV, off, True, [3, 100], None, None, scale, cap, sl), "masked")
    cache = new_cache(lib, g, dtype, 2, KV, 420, dh)
    before = clone_cache(lib, cache)
    for nodes in (1, 20):                               # a few rows of a key head, and many
        rows, doff, cached = qkv[:2 * nodes].contiguous(), [0, nodes, 2 * nodes], [400, 129]
        pos = torch.arange(850, 850 + 2 * nodes, device="cuda", dtype=torch.int32)
        ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, doff, cached, add_mass=True), dtype=torch.uint8, device="cuda")
        o = torch.empty((2 * nodes, H * dh), dtype=qkv.dtype, device="cuda")
        cache.mass.copy_(before.mass)
        ctx.otas_attention_tree(cache, rows, doff, None, pos, [1, 0], cached, ws, o, score=score, add_mass=True)
        w, b, grown, gb = plain.tree(rows, H, cache.k, cache.v, cache.positions, before.mass, doff, None, pos, [1, 0], cached, scale, cap, sl)
        within(o, w, b, "tree")
        for q, s in enumerate((1, 0)):
            within(cache.mass[s, :cached[q]], grown[s, :cached[q]], gb[s, :cached[q]] + 1e-30, "mass")


@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 2, 1, 64), ("bf16", 8, 2, 64), ("bf16", 3, 3, 80)])
def test_more_queries_than_the_arguments_hold(lib, dtype, H, KV, dh):
    """Their numbers go through the plan buffer: lengths of zero to a few, in one call of each operator."""
    import torch
    ctx, g, rng = context(dtype, H, dh), gen(31), np.random.default_rng(31)
    B, capacity = 1001, 90
    lens = [int(x) for x in rng.integers(0, 6, B)]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(off[-1])
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype)
    prefix = [int(rng.integers(0, n + 1)) for n in lens]
    o = torch.empty((T, H * dh), dtype=qkv.dtype, device="cuda")
    ctx.otas_attention_masked(qkv, KV, off, o, prefix=prefix)
    within(o, *plain.masked(qkv, H, KV, off, True, prefix), "masked")
    cache = new_cache(lib, g, dtype, B, KV, capacity, dh)
    slots, cached = [int(s) for s in rng.permutation(B)], [int(x) for x in rng.integers(0, capacity - 6, B)]
    parents = sum([tree_of(rng, n, "roots") for n in lens], [])
    before = clone_cache(lib, cache)
    ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, off, cached, add_mass=True), dtype=torch.uint8, device="cuda")
    ctx.otas_attention_tree(cache, qkv, off, parents, None, slots, cached, ws, o, add_mass=True)
    w, b, grown, gb = plain.tree(qkv, H, before.k, before.v, before.positions, before.mass, off, parents, None, slots, cached)
    within(o, w, b, "tree")
    filled = torch.zeros((B, capacity), dtype=torch.bool, device="cuda")
    for q in range(B):
        filled[slots[q], :cached[q]] = True
    within(cache.mass[filled], grown[filled], gb[filled] + 1e-30, "mass")
    assert torch.equal(cache.mass[~filled], before.mass[~filled])
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    now = ctx.otas_cache_append(cache, qkv, off, None, pos, slots, cached).tolist()
    q = int(np.argmax(lens))
    assert torch.equal(cache.v[slots[q], KV - 1, cached[q]:now[q]], qkv.view(T, H + 2 * KV, dh)[off[q]:off[q + 1], H + 2 * KV - 1])
    keep = [n // 2 for n in now]
    want = clone_cache(lib, cache)
    for q, (to, src) in enumerate(plain.evict(cache.mass, cache.positions, slots, now, keep, 1, None)):
        s = slots[q]
        want.k[s][:, to], want.v[s][:, to] = want.k[s][:, src], want.v[s][:, src]
        want.positions[s][to], want.mass[s][to] = want.positions[s][src], want.mass[s][src]
    ws = torch.empty(ctx.otas_cache_evict_workspace_bytes(now, keep), dtype=torch.uint8, device="cuda")
    assert ctx.otas_cache_evict(cache, slots, now, keep, ws, lead=1).tolist() == keep and same_cache(cache, want)


@pytest.mark.parametrize("dtype,dh,slopes,cap,n", [("bf16", 64, True, 0.0, 4500), ("bf16", 80, False, 20.0, 4200), ("f32", 64, False, 0.0, 1900)])
def test_long_rows_of_documents(lib, dtype, dh, slopes, cap, n):
    """More tiles than a wave looks at at once; documents that come back, that end inside a wave's rows and that no row of a wave
    has; a prefix that ends inside a tile; padding in the middle and behind the last."""
    import torch
    ctx, g = context(dtype, 2, dh), gen(n)
    d = torch.cat([torch.full((k,), i, dtype=torch.int32) for k, i in ((700, 5), (301, 2), (17, -1), (500, 5), (n - 1518 - 133, 9), (133, -7))]).cuda()
    off, prefix = [0, n, n + 70], [77, 0]
    d = torch.cat([d, torch.zeros(70, dtype=torch.int32, device="cuda")])
    qkv = normal(g, (n + 70, 4 * dh), dtype)
    sl = slopes_of(2) if slopes else None
    for causal in (True, False):
        o = torch.empty((n + 70, 2 * dh), dtype=qkv.dtype, device="cuda")
        ctx.otas_attention_masked(qkv, 1, off, o, causal=causal, prefix=prefix, documents=d, score=lib.Score(cap=cap, slopes=sl))
        want, bound = plain.masked(qkv, 2, 1, off, causal, prefix, d, None, None, cap, sl)
        within(o, want, bound, "documents")
        assert bool((o[d < 0] == 0).all())


def test_offsets_beyond_32_bits(lib):
    """Slots and rows more than 2^31 elements into their arrays: what the same numbers give at the front."""
    import torch
    H, KV, dh, capacity, slots = 4, 2, 128, 1 << 20, 9
    ctx, g = context("bf16", H, dh), gen(3)
    assert (slots - 1) * KV * capacity * dh >= 2 ** 31
    far = lib.KVCache(*(torch.empty((slots, KV, capacity, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                      torch.empty((slots, capacity), dtype=torch.int32, device="cuda"), torch.zeros((slots, capacity), device="cuda"))
    n, W = 3000, (H + 2 * KV) * dh
    T = 2 ** 31 // W + 40
    qkv = torch.empty((T, W), dtype=torch.bfloat16, device="cuda")
    rows = normal(g, (40, W), "bf16")
    qkv[-40:] = rows
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    out = torch.empty_like(rows)
    ctx.otas_rotary(rows, KV, pos[-40:].contiguous(), lib.Rotary(122), out)
    ctx.otas_rotary(qkv, KV, pos, lib.Rotary(122), qkv)
    assert torch.equal(qkv[-40:], out)
    near = lib.KVCache(normal(g, (1, KV, n + 40, dh), "bf16"), normal(g, (1, KV, n + 40, dh), "bf16"), pos[:n + 40].view(1, -1).clone(),
                       torch.rand((1, n + 40), generator=g, device="cuda"))
    base = capacity - n - 40                            # entries up to the last one that a slot holds
    for a, b in ((far.k, near.k), (far.v, near.v)):
        a[8, :, :n + 40] = b[0]
    far.positions[8, :n + 40], far.mass[8, :n + 40] = near.positions[0], near.mass[0]
    r = list(range(T - 40, T))
    assert ctx.otas_cache_append(far, qkv, [0, 40], r, pos, [8], [n]).tolist() == [n + 40]
    ctx.otas_cache_append(near, out, [0, 40], None, pos[-40:].contiguous(), [0], [n])
    assert torch.equal(far.k[8, :, :n + 40], near.k[0]) and torch.equal(far.positions[8, :n + 40], near.positions[0])
    ctx.otas_cache_append(far, qkv, [0, 40], r, pos, [8], [base + n])
    assert torch.equal(far.v[8, :, -40:], near.v[0, :, n:])
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    o = [torch.empty((12, H * dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for i, (c, s) in enumerate(((far, 8), (near, 0))):
        ctx.otas_attention_tree(c, out[:12].contiguous(), [0, 12], None, None, [s], [n + 40], ws, o[i], add_mass=True)
        assert ctx.otas_cache_evict(c, [s], [n + 40], [n - 500], ws, lead=4).tolist() == [n - 500]
    assert torch.equal(o[0], o[1]) and torch.equal(far.mass[8, :n - 500], near.mass[0, :n - 500])
    assert torch.equal(far.k[8, :, :n - 500], near.k[0, :, :n - 500]) and torch.equal(far.v[8, :, :n - 500], near.v[0, :, :n - 500])


def test_graphs_that_share_a_workspace(lib):
    """Two captured trees of different shapes with one workspace, replayed in turn with an eager call between them."""
    import torch
    import paper_2401_05031_amd as otas
    H, KV, dh = 4, 2, 64
    stream = torch.cuda.Stream()
    cfg = synth.Config("graphs", L=1, D=H * dh, H=H, F=64, dtype="bf16", B=1, n0=4, strategies=[(0, 0)], seed=5)
    ctx = otas.Context.from_host_weights(1, H * dh, H, 64, otas.OTAS_BF16, 1e-6, 1, synth.all_weights(cfg), stream=stream.cuda_stream)
    g = gen(21)
    cache = new_cache(lib, g, "bf16", 3, KV, 2000, dh)
    mass = cache.mass.clone()
    calls = []
    for off, slots, cached in (([0, 1, 2], [0, 2], [2000, 900]), ([0, 33, 40], [1, 0], [700, 1999]), ([0, 4], [2], [0])):
        qkv = normal(g, (off[-1], (H + 2 * KV) * dh), "bf16")
        calls.append((off, slots, cached, qkv, torch.empty((off[-1], H * dh), dtype=qkv.dtype, device="cuda")))
    ws = torch.empty(max(ctx.otas_attention_tree_workspace_bytes(KV, c[0], c[2], add_mass=True) for c in calls), dtype=torch.uint8, device="cuda")

    def run(c):
        ctx.otas_attention_tree(cache, c[3], c[0], None, None, c[1], c[2], ws, c[4], add_mass=True)
    want = []
    for c in calls:
        cache.mass.copy_(mass)
        torch.cuda.synchronize()
        run(c)
        torch.cuda.synchronize()
        want.append((c[4].clone(), cache.mass.clone()))
    graphs = []
    for c in calls[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            run(c)
    for turn in range(3):
        for i, go in ((0, graphs[0].replay), (1, graphs[1].replay), (2, lambda: run(calls[2])), (1, graphs[1].replay)):
            cache.mass.copy_(mass)
            calls[i][4].fill_(9.0)
            ws.fill_(255)
            torch.cuda.synchronize()
            go()
            torch.cuda.synchronize()
            assert torch.equal(calls[i][4], want[i][0]) and torch.equal(cache.mass, want[i][1]), (turn, i)
    ctx.close()


def test_refusals_of_very_wide_calls(lib):
    import torch
    ctx = context("bf16", 16, 64)
    n = 300000
    qkv, o = torch.empty((n, 18 * 64), dtype=torch.bfloat16, device="cuda"), torch.empty((n, 1024), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lib.OtasError) as e:             # 900 x 16 x 2344 row blocks of 128, nearly all of them empty
        ctx.otas_attention_masked(qkv, 1, [0] + [n] * 900, o)
    assert e.value.status == 5
    ctx.otas_attention_masked(qkv[:5].contiguous(), 1, [0] + [5] * 900, o[:5].contiguous())


@pytest.mark.parametrize("dtype,H,KV,dh", [("f32", 2, 1, 64), ("f32", 2, 2, 20), ("bf16", 4, 2, 64), ("bf16", 2, 1, 80), ("bf16", 2, 1, 128), ("bf16", 2, 1, 40)])
def test_a_query_that_is_not_a_number(lib, dtype, H, KV, dh):
    """Its row is NaN, as the formula says, however the keys are split; no other row changes."""
    import torch
    ctx, g = context(dtype, H, dh), gen(8)
    qkv = normal(g, (200, (H + 2 * KV) * dh), dtype)
    bad = qkv.clone()
    bad[[3, 150], :H * dh] = float("nan")
    ok = torch.ones(200, dtype=torch.bool, device="cuda")
    ok[[3, 150]] = False
    for cap in (0.0, 20.0):
        a, b = (torch.empty((200, H * dh), dtype=qkv.dtype, device="cuda") for _ in range(2))
        ctx.otas_attention_masked(qkv, KV, [0, 200], a, score=lib.Score(cap=cap))
        ctx.otas_attention_masked(bad, KV, [0, 200], b, score=lib.Score(cap=cap))
        assert torch.equal(a[ok], b[ok]) and bool(b[~ok].isnan().all())
        cache = new_cache(lib, g, dtype, 1, KV, 3000, dh)
        for nodes in (5, 20, 40):
            for cached in (0, 100, 3000):
                ws = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, [0, nodes], [cached]), dtype=torch.uint8, device="cuda")
                x, o = qkv[:nodes].contiguous(), [torch.empty((nodes, H * dh), dtype=qkv.dtype, device="cuda") for _ in range(2)]
                for out in o:
                    ctx.otas_attention_tree(cache, x, [0, nodes], None, None, [0], [cached], ws, out, score=lib.Score(cap=cap))
                    x = bad[:nodes].contiguous()
                assert torch.equal(o[0][ok[:nodes]], o[1][ok[:nodes]]) and bool(o[1][3].isnan().all()), (nodes, cached)


@pytest.mark.parametrize("dtype,H,KV,dh,B,nodes,longest", [("bf16", 16, 16, 128, 20, 1, 2600), ("bf16", 16, 8, 64, 24, 3, 1900), ("bf16", 8, 8, 96, 40, 2, 900),
                                                           ("f32", 8, 4, 64, 24, 2, 700)])
def test_many_queries_over_long_caches_of_all_lengths(lib, dtype, H, KV, dh, B, nodes, longest):
    """A full chip: lengths from none to the longest, cut by every query's own length, the nodes behind the first chunk or apart."""
    import torch
    ctx, g, rng = context(dtype, H, dh), gen(B + longest), np.random.default_rng(B)
    cache = new_cache(lib, g, dtype, B, KV, longest, dh)
    cached = [int(x) for x in rng.integers(0, longest, B)]
    cached[:4] = [longest, 0, 384, 385]
    slots = [int(s) for s in rng.permutation(B)]
    off = [nodes * q for q in range(B + 1)]
    qkv = normal(g, (nodes * B, (H + 2 * KV) * dh), dtype, 1.5)
    before = clone_cache(lib, cache)
    ws = torch.full((ctx.otas_attention_tree_workspace_bytes(KV, off, cached),), 255, dtype=torch.uint8, device="cuda")
    for mass in (True, False):
        o = torch.empty((nodes * B, H * dh), dtype=qkv.dtype, device="cuda")
        cache.mass.copy_(before.mass)
        ctx.otas_attention_tree(cache, qkv, off, [-1, 0, 0][:nodes] * B, None, slots, cached, ws, o, add_mass=mass)
        w, b, grown, gb = plain.tree(qkv, H, before.k, before.v, before.positions, before.mass, off, [-1, 0, 0][:nodes] * B, None, slots, cached)
        within(o, w, b, "tree")
        for q in range(B if mass else 0):
            within(cache.mass[slots[q], :cached[q]], grown[slots[q], :cached[q]], gb[slots[q], :cached[q]] + 1e-30, "mass")
    assert same_cache(cache, before)
