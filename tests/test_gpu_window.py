"""The operators with norms of heads, windows and the cache in 4 bits on the GPU against their 64-bit forms (tests/window_plain.py)."""
import math

import numpy as np
import pytest

import otas_synth as synth
from tests import decode_plain
from tests import harness as hz
from tests import window_plain as plain

pytestmark = pytest.mark.gpu

_CONTEXTS = {}
ALL = 2 ** 31 - 1


def context(dtype, H, dh):
    key = (dtype, H, dh)
    if key not in _CONTEXTS:
        cfg = synth.Config("window", L=1, D=H * dh, H=H, F=64, dtype=dtype, B=1, n0=4, strategies=[(0, 0)], seed=5)
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
    """Within the bound; NaN in `want`: no finite number."""
    import torch
    nan = torch.isnan(want)
    bad = torch.where(nan, torch.isfinite(got), ~((got.double() - want).abs() <= bound))
    if bool(bad.any()):
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got {got[tuple(at)].item()}, want "
                             f"{want[tuple(at)].item()} within {bound[tuple(at)].item()}")


def slopes_of(H):
    import torch
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device="cuda")


def offsets_of(lengths):
    return [0] + [int(x) for x in np.cumsum(lengths)]


class Fenced:
    """A tensor with rows of sevens on both sides, which a call has to leave."""

    def __init__(self, rows, width, dtype):
        import torch
        pad = 8
        self.whole = torch.full((rows + 2 * pad, width), 7.0, dtype=dtype, device="cuda")
        self.t = self.whole[pad:pad + rows]

    def check(self):
        assert bool((self.whole[:8] == 7.0).all()) and bool((self.whole[len(self.whole) - 8:] == 7.0).all())


def workspace_of(bytes_):
    """Exactly the bytes asked for, full of NaN, with a fence behind."""
    import torch
    whole = torch.full((bytes_ + 256,), 255, dtype=torch.uint8, device="cuda")
    return whole, whole[:bytes_]


# -------------------------------------------------------------------------------------------------- norms and rotation
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,H,KV,dh,T,rot,interleaved,center,per_head,gains", [
    ("f32", 3, 3, 64, 1, 64, False, False, False, True), ("f32", 4, 2, 20, 37, 10, False, True, True, True), ("f32", 4, 1, 20, 5, 18, True, False, False, False),
    ("f32", 2, 1, 4, 3, 2, False, False, True, True), ("f32", 2, 2, 128, 1100, 128, True, True, False, True), ("f32", 2, 1, 36, 33, 24, False, False, False, True),
    ("bf16", 12, 4, 64, 197, 64, False, False, False, True), ("bf16", 4, 2, 80, 33, 40, False, True, False, True), ("bf16", 4, 4, 80, 7, 80, True, False, True, True),
    ("bf16", 8, 2, 96, 2049, 50, False, False, False, False), ("bf16", 2, 1, 128, 8200, 128, False, False, False, True), ("bf16", 2, 1, 128, 9, 0, True, False, False, True),
    ("bf16", 2, 1, 12, 65, 12, True, True, False, True), ("bf16", 2, 1, 12, 65, 8, False, False, False, True), ("bf16", 2, 2, 64, 31, 6, True, False, True, True),
    ("bf16", 2, 1, 8, 3, 8, False, True, False, True), ("bf16", 2, 1, 128, 300, 122, False, False, False, True), ("f32", 2, 1, 8, 70, 6, False, False, False, True)])
def test_norm_rotary(lib, dtype, H, KV, dh, T, rot, interleaved, center, per_head, gains, in_place):
    import torch
    ctx, g = context(dtype, H, dh), gen(T + rot + dh)
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype, 3.0)
    qkv[0] *= 1e-4                                   # the squares' mean is smaller than eps
    if T > 2:
        qkv[1] = 0
    pos = torch.randint(-5, 2 ** 20, (T,), generator=g, device="cuda", dtype=torch.int32)
    shape = (lambda n: (n, dh)) if per_head else (lambda n: (dh,))
    q_gain, k_gain = (normal(g, shape(H), dtype), normal(g, shape(KV), dtype)) if gains else (None, None)
    want, bound = plain.norm_rotary(qkv, H, KV, pos, rot, interleaved, decode_plain.frequencies(rot, 5000.0) if rot else np.zeros(0),
                                    q_gain, k_gain, 1e-5, center, 0.75)
    fenced = Fenced(T, qkv.shape[1], qkv.dtype)
    src = qkv
    if in_place:
        fenced.t.copy_(qkv)
        src = fenced.t
    rope = lib.Rotary(rot, layout=lib.OTAS_ROTARY_INTERLEAVED if interleaved else lib.OTAS_ROTARY_HALF, base=5000.0, magnitude=0.75)
    ctx.otas_norm_rotary(src, KV, lib.HeadNorm(q_gain, k_gain, 1e-5, center, per_head), pos if rot else None, rope, fenced.t)
    within(fenced.t, want, bound + 1e-6 * (2.0 ** 20 * 2.0 ** -52 * 6.3), "norm")
    fenced.check()
    values = (H + KV) * dh
    assert torch.equal(fenced.t[:, values:], qkv[:, values:])


# ------------------------------------------------------------------------------------------------------ packed rows
WINDOW = [
    # dtype, H, KV, dh, lengths, window, sinks, cap, slopes
    ("f32", 3, 3, 64, [201, 1, 0, 33], 40, 0, 0.0, False),
    ("f32", 4, 2, 20, [65, 64, 7], 1, 3, 5.0, True),
    ("f32", 2, 1, 128, [300, 31], 64, 70, 0.0, True),
    ("f32", 4, 1, 36, [129, 128, 127], 500, 0, 2.0, False),
    ("f32", 2, 1, 4, [97], 32, 33, 0.0, False),
    ("bf16", 12, 4, 64, [197, 1, 64, 65, 0, 2, 128], 64, 1, 0.0, False),
    ("bf16", 12, 12, 64, [261, 33], 1, 0, 30.0, False),
    ("bf16", 4, 2, 80, [577, 100, 129], 100, 4, 0.0, True),
    ("bf16", 2, 1, 96, [400, 31], 65, 200, 20.0, True),
    ("bf16", 8, 2, 96, [700, 31, 3], 130, 64, 0.0, False),
    ("bf16", 4, 1, 128, [1000, 129, 3], 256, 4, 4.0, False),
    ("bf16", 2, 2, 128, [257, 512, 1], 31, 65, 0.0, False),
    ("bf16", 8, 1, 128, [1300], 63, 1, 300.0, False),
    ("bf16", 2, 1, 128, [500], ALL, 0, 0.0, False),
    ("bf16", 2, 1, 128, [500], ALL, ALL, 0.0, False),
    ("bf16", 2, 1, 32, [90, 5], 17, 2, 3.0, True),
    ("bf16", 2, 1, 72, [140, 64], 33, 40, 0.0, False),
]


@pytest.mark.parametrize("poison", [False, True])
@pytest.mark.parametrize("case", WINDOW, ids=lambda c: "-".join(str(x) for x in c[:4]) + f"-{c[5]}-{c[6]}")
def test_window(lib, case, poison):
    import torch
    dtype, H, KV, dh, lengths, window, sinks, cap, slopes = case
    ctx, g = context(dtype, H, dh), gen(sum(lengths) + dh)
    off = offsets_of(lengths)
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    if poison:   # keys and values of some rows are no numbers: those that see them have none, the others theirs
        x = qkv.view(off[-1], H + 2 * KV, dh)
        for n, row in enumerate(range(5, off[-1], 53)):
            x[row, H + (n % 2) * KV + n % KV, n % dh] = [math.inf, -math.inf, math.nan][n % 3] if n % 2 else math.nan
    sl = slopes_of(H) if slopes else None
    want, bound = plain.window(qkv, H, KV, off, window, sinks, 0.3, cap, sl)
    fenced = Fenced(off[-1], H * dh, qkv.dtype)
    ctx.otas_attention_window(qkv, KV, off, fenced.t, window, sinks, lib.Score(0.3, cap, sl))
    within(fenced.t, want, bound, "window")
    fenced.check()


# ------------------------------------------------------------------------------------------- the last tokens of a cache
RECENT = [
    # dtype, H, KV, dh, rows, lengths, capacity, window, sinks, cap, slopes
    ("f32", 3, 3, 64, [1, 1, 0, 1], [201, 1, 5, 33], 224, ALL, 0, 0.0, False),
    ("f32", 4, 2, 24, [3, 7, 64], [65, 7, 64], 96, 9, 3, 5.0, True),
    ("f32", 2, 1, 128, [40, 31], [300, 31], 320, 64, 70, 0.0, True),
    ("f32", 8, 1, 40, [2, 9], [500, 77], 512, 100, 0, 2.0, False),
    ("f32", 4, 4, 96, [1], [1500], 1504, 1400, 4, 0.0, False),
    ("f32", 2, 1, 8, [1, 20], [97, 97], 128, 32, 33, 0.0, False),
    ("bf16", 12, 4, 64, [1, 1, 1, 1, 0, 2, 5], [197, 1, 64, 65, 0, 2, 128], 224, 64, 1, 0.0, False),
    ("bf16", 12, 12, 64, [1, 33], [261, 33], 288, 1, 0, 30.0, False),
    ("bf16", 4, 2, 80, [77, 1, 16], [577, 100, 129], 608, 100, 4, 0.0, True),
    ("bf16", 2, 1, 96, [400, 31], [400, 60], 416, 65, 200, 20.0, True),
    ("bf16", 16, 2, 128, [1, 1, 1], [3000, 129, 3], 3008, ALL, 0, 4.0, False),
    ("bf16", 16, 2, 128, [8, 300, 3], [3000, 1029, 3], 3008, 700, 4, 0.0, False),
    ("bf16", 2, 2, 128, [1, 1, 1], [257, 512, 1], 512, 31, 65, 0.0, False),
    ("bf16", 8, 1, 128, [2], [1300], 1312, 63, 1, 300.0, False),
    ("bf16", 32, 1, 64, [3, 1], [5000, 700], 5024, 4500, 40, 0.0, False),
    ("bf16", 2, 1, 32, [9, 5], [90, 5], 96, 17, 2, 3.0, True),
    ("bf16", 2, 1, 72, [14, 64], [140, 64], 160, 33, 40, 0.0, False),
    ("bf16", 2, 1, 8, [4, 1], [140, 64], 160, 33, 40, 0.0, True),
    ("bf16", 4, 1, 112, [1, 1], [64, 1024], 1024, ALL, ALL, 0.0, False),
]


def recent_ids(c):
    return "-".join(str(x) for x in c[:4]) + f"-{max(c[4])}-{max(c[5])}-{c[7]}-{c[8]}"


@pytest.mark.parametrize("poison", [False, True])
@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("case", RECENT, ids=recent_ids)
def test_recent(lib, case, four, poison):
    import torch
    dtype, H, KV, dh, rows, lengths, capacity, window, sinks, cap, slopes = case
    ctx, g = context(dtype, H, dh), gen(sum(lengths) + dh)
    off, B = offsets_of(rows), len(rows)
    if not four:
        capacity = max(lengths) + 3                 # any number, and the last tile ends past it
    qkv = normal(g, (off[-1], (H + 2 * KV) * dh), dtype)
    qkv[:, H * dh:] = math.nan                      # not read
    k, v = normal(g, (B + 1, KV, capacity, dh), dtype), normal(g, (B + 1, KV, capacity, dh), dtype)
    slots = [(2 * q + 1) % (B + 1) if B % 2 else q for q in range(B)]
    if poison:
        for q in range(B):
            for n, e in enumerate(range(3, lengths[q], 41)):
                t = (v, k)[n % 2]
                t[slots[q], n % KV, e, (7 * n) % dh] = [math.inf, -math.inf, math.nan][n % 3] if t is v else math.nan
    ends = {slot: max(n for s, n in zip(slots, lengths) if s == slot) for slot in slots}   # queries may share a slot
    for slot, end in ends.items():                  # behind the entries lies anything
        k[slot, :, end:] = math.nan
        v[slot, :, end:] = math.inf
    if four:
        enc = [plain.encode4(t) for t in (k, v)]
        k, v = [plain.decode4(c, s) for c, s in enc]
        packed = [plain.pack4(c) for c, _ in enc] + [s.transpose(-1, -2).contiguous().to(torch.uint8) for _, s in enc]
        for slot, end in ends.items():
            for t in packed[2:]:
                t[slot, :, :, end:] = torch.randint(0, 256, t[slot, :, :, end:].shape, generator=g, device="cuda", dtype=torch.uint8)
            for t in packed[:2]:
                t[slot, :, end:] = 0x77
        cache = lib.KVCache4(*packed)
    else:
        cache = lib.KVCache(k, v, torch.zeros((B + 1, capacity), dtype=torch.int32, device="cuda"))
    sl = slopes_of(H) if slopes else None
    want, bound = plain.recent(qkv, H, k, v, off, slots, lengths, window, sinks, 0.3, cap, sl)
    fenced = Fenced(off[-1], H * dh, qkv.dtype)
    need = ctx.otas_attention_recent_workspace_bytes(KV, off, lengths, window, sinks)
    whole, ws = workspace_of(need)
    call = ctx.otas_attention_cache4 if four else ctx.otas_attention_recent
    call(cache, qkv, off, slots, lengths, ws, fenced.t, window, sinks, lib.Score(0.3, cap, sl))
    within(fenced.t, want, bound, "recent")
    fenced.check()
    assert bool((whole[need:] == 255).all())


# ------------------------------------------------------------------------------------------------------- rows in 4 bits
def every_value(dtype, count):
    """`count` values: all bf16 bit patterns in order for bf16, for f32 those and their neighbours."""
    import torch
    bits = torch.arange(65536, device="cuda", dtype=torch.int64).to(torch.int32) << 16
    x = bits.view(torch.float32)
    if dtype == "f32":
        x = torch.stack([x, (bits + 1).view(torch.float32), (bits + 0x7FFF).view(torch.float32), (bits + 0xFFFF).view(torch.float32)], dim=1).flatten()
        return x[:count]
    return x.to(torch.bfloat16)[:count]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cache4_holds_every_value_as_the_header_says(lib, dtype):
    """Every bf16 value (and floats beside them) under group maxima of its own size and larger: codes, scales and what is read back."""
    import torch
    H = KV = 2
    dh = 64
    ctx = context(dtype, H, dh)
    base = every_value(dtype, 65536 if dtype == "bf16" else 262144).view(-1, 32)
    # a group's elements are neighbours; then the same with one that is 1, 7/4 and 6 powers of two larger in the last place
    grown = [base]
    for f in (1.0, 1.75, 1.7578125, 5.0, 64.0):
        t = base.clone()
        t[:, 31] = (base[:, :31].float().abs().amax(dim=1) * f).to(base.dtype)
        grown.append(t)
    x = torch.cat(grown)
    rows = len(x) // 8
    x = x[:rows * 8].view(rows, 2 * KV * dh)
    qkv = torch.cat([torch.zeros((rows, H * dh), dtype=x.dtype, device="cuda"), x], dim=1).contiguous()
    capacity = -(-rows // 32) * 32
    cache = lib.KVCache4.empty(1, KV, capacity, dh)
    assert list(ctx.otas_cache4_append(cache, qkv, [0, rows], None, [0], [0])) == [rows]
    code, scale = plain.encode4(x.view(rows, 2 * KV, dh))
    for got, sc, want_c, want_s in ((cache.k, cache.k_scales, code[:, :KV], scale[:, :KV]), (cache.v, cache.v_scales, code[:, KV:], scale[:, KV:])):
        s = sc[0, :, :, :rows].permute(2, 0, 1).long()
        assert torch.equal(s, want_s)
        c = plain.unpack4(got[0, :, :rows].transpose(0, 1))
        wrong = (c != want_c).nonzero()
        assert len(wrong) == 0, (len(wrong), wrong[0].tolist(), x.view(rows, 2, KV, dh)[wrong[0][0], :, wrong[0][1], wrong[0][2]].tolist(),
                                 int(c[tuple(wrong[0])]), int(want_c[tuple(wrong[0])]))
    back = torch.empty_like(x)
    ctx.otas_cache4_read(cache, [0], [0], [0, rows], back)
    want = plain.decode4(code, scale).view(rows, -1)
    assert torch.equal(torch.isnan(back), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(back.double()), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype,H,KV,dh,counts,lengths,picked", [
    ("f32", 3, 3, 64, [5, 0, 33], [7, 3, 0], False), ("bf16", 4, 2, 80, [1, 1, 1, 1], [0, 95, 31, 32], False), ("bf16", 16, 8, 128, [40, 2], [20, 94], True),
    ("bf16", 2, 1, 8, [64, 3], [0, 33], True), ("f32", 4, 1, 96, [17], [79], False), ("bf16", 4, 1, 40, [9, 9], [1, 2], False)])
def test_cache4_append_and_read(lib, dtype, H, KV, dh, counts, lengths, picked):
    import torch
    ctx, g = context(dtype, H, dh), gen(sum(counts) + dh)
    off, B, capacity = offsets_of(counts), len(counts), 96
    T = off[-1] + (5 if picked else 0)
    rows = [int(r) for r in torch.randint(0, T, (off[-1],), generator=g, device="cuda").tolist()] if picked else None   # one of them twice
    qkv = normal(g, (T, (H + 2 * KV) * dh), dtype, 10.0)
    cache = lib.KVCache4.empty(B + 1, KV, capacity, dh)
    arrays = (cache.k, cache.v, cache.k_scales, cache.v_scales)
    for t in arrays:
        t.random_(0, 256, generator=g)
    before = [t.clone() for t in arrays]
    slots = [B - q for q in range(B)]
    new = ctx.otas_cache4_append(cache, qkv, off, rows, slots, lengths)
    assert list(new) == [a + b for a, b in zip(lengths, counts)]
    x = qkv.view(T, H + 2 * KV, dh)[torch.tensor(rows if picked else list(range(T)), device="cuda", dtype=torch.int64), H:]
    code, scale = plain.encode4(x)
    for q, (slot, n) in enumerate(zip(slots, lengths)):
        a, z = off[q], off[q + 1]
        before[0][slot, :, n:n + z - a] = plain.pack4(code[a:z, :KV]).transpose(0, 1)
        before[1][slot, :, n:n + z - a] = plain.pack4(code[a:z, KV:]).transpose(0, 1)
        before[2][slot, :, :, n:n + z - a] = scale[a:z, :KV].permute(1, 2, 0).to(torch.uint8)
        before[3][slot, :, :, n:n + z - a] = scale[a:z, KV:].permute(1, 2, 0).to(torch.uint8)
    assert all(torch.equal(a, b) for a, b in zip(arrays, before))     # and nothing else has changed
    fenced = Fenced(off[-1], 2 * KV * dh, qkv.dtype)
    ctx.otas_cache4_read(cache, slots, lengths, off, fenced.t)
    assert torch.equal(fenced.t.double(), plain.decode4(code, scale).view(off[-1], -1))
    fenced.check()
