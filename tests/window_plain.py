"""The operators with norms of heads, windows and the cache in 4 bits (include/otas_decode.h) in 64 bits, query by query and head by head,
with bounds on what a correct implementation in the operands' type may be off by.  Used by the tests only."""
import math

import torch

from tests.decode_plain import BF16, F32

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def norm_rotary(qkv, H, KV, positions, rot, interleaved, freqs, q_gain=None, k_gain=None, eps=1e-6, center=False, magnitude=1.0):
    """(result, bound).  The mean and the mean of squares are sums of d_h terms, each addition off by F32 of the sum of sizes; root, reciprocal,
    gain and their products add 8; the rotation is bounded as otas_rotary's; one rounding to qkv's type."""
    T = qkv.shape[0]
    dh = qkv.shape[1] // (H + 2 * KV)
    x = qkv.double().view(T, H + 2 * KV, dh).clone()
    off = torch.zeros_like(x)
    for a, b, gain in ((0, H, q_gain), (H, H + KV, k_gain)):
        z = x[:, a:b]
        lost = torch.zeros_like(z[..., :1])
        if center:
            lost = (dh + 2) * F32 * z.abs().mean(dim=-1, keepdim=True)
            z = z - z.mean(dim=-1, keepdim=True)
        square = (z * z).mean(dim=-1, keepdim=True) + eps
        g = torch.ones((b - a, dh), dtype=torch.float64, device=x.device) if gain is None else gain.double().expand(b - a, dh)
        r = square.rsqrt()
        y = z * r * g
        # of the squares' mean: a lost mean moves it by 2 lost mean|z| at most
        rel = (dh / 2 + 8) * F32 + lost * z.abs().mean(dim=-1, keepdim=True) / square
        off[:, a:b] = y.abs() * rel + lost * r * g.abs()
        x[:, a:b] = y
    if rot:
        angle = positions.double()[:, None] * torch.from_numpy(freqs).to(x.device)[None, :]
        c, s = angle.cos()[:, None, :], angle.sin()[:, None, :]
        first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
        second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
        p, q = x[:, :H + KV, first].clone(), x[:, :H + KV, second].clone()
        e, f = off[:, :H + KV, first].clone(), off[:, :H + KV, second].clone()
        x[:, :H + KV, first], x[:, :H + KV, second] = magnitude * (p * c - q * s), magnitude * (p * s + q * c)
        more = abs(magnitude) * (p.abs() + q.abs()) * 9 * F32
        off[:, :H + KV, first] = abs(magnitude) * (e * c.abs() + f * s.abs()) + more
        off[:, :H + KV, second] = abs(magnitude) * (e * s.abs() + f * c.abs()) + more
    if qkv.dtype != torch.float32:
        off[:, :H + KV] += BF16 * x[:, :H + KV].abs() * (1 + 2 ** -6)
    else:
        off[:, :H + KV] += F32 * x[:, :H + KV].abs()
    return x.view(T, -1), off.view(T, -1)


def attend(q, k, v, visible, dtype, cut, scale, cap=0.0, slope=0.0, distance=None):
    """One head: q [m, dh], k, v [n, dh], visible [m, n] -> (o, bound of o), 64 bits; what a row does not see may hold anything.

    As tests/decode_plain.py: attend.  cut: operands in three pieces, whose products are eight additions an element where there is one
    otherwise: roundings of N additions in a row add up to 4 sqrt(N) of the sum of sizes, which for short heads is more than the dh + 4 of
    the worst case of one each."""
    q, k, v = q.double(), k.double(), v.double()
    n, dh = k.shape
    m = q.shape[0]
    clean_k, clean_v = torch.where(torch.isfinite(k), k, 0.0), torch.where(torch.isfinite(v), v, 0.0)
    bad_k = ~torch.isfinite(k).all(dim=1)
    s = (q @ clean_k.T.contiguous()) * scale
    terms = max(dh + 4, 4 * math.sqrt(8 * dh) + 4) if cut else dh + 4
    off = F32 * (terms * abs(scale) * (q.abs() @ clean_k.abs().T.contiguous()) + 2 * s.abs())
    if cap:
        s = cap * torch.tanh(s / cap)
        off = off + (8 * F32 if dtype == torch.float32 else 2.0 ** -20) * cap
    if slope:
        s = s - slope * distance.abs()
        off = off + F32 * (2 * slope * distance.abs() + s.abs())
    s = s.masked_fill(~visible, -math.inf)
    top = s.amax(dim=1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(total > 0, e / total.clamp_min(1e-300), 0.0)
    o = p @ clean_v
    off = torch.where(visible, off + F32 * (2 * (s - top).abs() + 16), 0.0)
    off = torch.where(torch.isfinite(off), off, 0.0)
    rel = off + (p * off).sum(dim=1, keepdim=True)
    bound = (p * rel) @ clean_v.abs() + 4 * F32 * math.sqrt((8 if cut else 1) * n) * (p @ clean_v.abs()) + F32 * o.abs()
    if dtype != torch.float32:
        bound = bound + BF16 * ((p @ clean_v.abs()) + o.abs()) * (1 + 2 ** -6)
    # NaN marks what has to come out as no finite number
    seen_bad = (visible.double() @ (~torch.isfinite(v)).double()) > 0
    o = o.masked_fill(seen_bad | (visible & bad_k[None, :]).any(dim=1)[:, None], math.nan)
    return o, bound + 1e-30


def visible(places, n, window, sinks, device):
    t, j = places.view(-1, 1), torch.arange(n, device=device).view(1, -1)
    return (j <= t) & ((t - j < window) | (j < sinks))


def window(qkv, H, KV, offsets, window_, sinks, scale=None, cap=0.0, slopes=None):
    dh = qkv.shape[1] // (H + 2 * KV)
    scale = dh ** -0.5 if scale is None else scale
    o = torch.zeros((qkv.shape[0], H * dh), dtype=torch.float64, device=qkv.device)
    bound = torch.zeros_like(o)
    for a, z in zip(offsets, offsets[1:]):
        if a == z:
            continue
        x = qkv[a:z].view(z - a, H + 2 * KV, dh)
        i = torch.arange(z - a, device=qkv.device)
        vis = visible(i, z - a, window_, sinks, qkv.device)
        for h in range(H):
            kh = h // (H // KV)
            o[a:z, h * dh:(h + 1) * dh], bound[a:z, h * dh:(h + 1) * dh] = attend(
                x[:, h], x[:, H + kh], x[:, H + KV + kh], vis, qkv.dtype, False, scale, cap, 0.0 if slopes is None else float(slopes[h]),
                (i.view(-1, 1) - i.view(1, -1)).double())
    return o, bound


def recent(qkv, H, k, v, offsets, slots, lengths, window_, sinks, scale=None, cap=0.0, slopes=None):
    """k, v [slots, KV, capacity, dh], any type."""
    KV, dh = k.shape[1], k.shape[3]
    scale = dh ** -0.5 if scale is None else scale
    o = torch.zeros((qkv.shape[0], H * dh), dtype=torch.float64, device=qkv.device)
    bound = torch.zeros_like(o)
    for q, (a, z) in enumerate(zip(offsets, offsets[1:])):
        if a == z:
            continue
        n, slot = int(lengths[q]), int(slots[q])
        x = qkv[a:z].view(z - a, H + 2 * KV, dh)
        t = torch.arange(n - (z - a), n, device=qkv.device)
        vis = visible(t, n, window_, sinks, qkv.device)
        dist = (t.view(-1, 1) - torch.arange(n, device=qkv.device).view(1, -1)).double()
        for h in range(H):
            kh = h // (H // KV)
            o[a:z, h * dh:(h + 1) * dh], bound[a:z, h * dh:(h + 1) * dh] = attend(
                x[:, h], k[slot, kh, :n], v[slot, kh, :n], vis, qkv.dtype, qkv.dtype == torch.float32, scale, cap,
                0.0 if slopes is None else float(slopes[h]), dist)
    return o, bound


def power_of_two(e):
    """2^e for whole numbers |e| <= 128, exactly (a library's pow may be off in the last place)."""
    return torch.tensor([2.0 ** t for t in range(-128, 129)], dtype=torch.float64, device=e.device)[e.long() + 128]


def encode4(x):
    """x [..., dh] -> (codes [..., dh], scale bytes [..., groups]) by trying all exponents and all values, 64 bits."""
    dh = x.shape[-1]
    pad = torch.nn.functional.pad(x.double(), (0, -dh % 32)).unflatten(-1, (-1, 32))
    finite = torch.isfinite(pad).all(dim=-1)
    pad = torch.where(finite[..., None], pad, 0.0)
    top = pad.abs().amax(dim=-1)
    e = torch.full_like(top, 125.0)
    for t in range(124, -126, -1):
        e = torch.where(top <= 7 * 2.0 ** t, float(t), e)
    y = pad.abs() / power_of_two(e)[..., None]
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    gap = (y[..., None] - grid).abs()
    best = gap.amin(dim=-1, keepdim=True)
    near = gap == best                      # one, or two neighbours, of which one has an even place
    place = torch.arange(8, device=x.device)
    cost = torch.where(near, place + 8 * (place % 2) * (near.sum(dim=-1, keepdim=True) - 1), 99)
    code = cost.argmin(dim=-1) + 8 * torch.signbit(pad).long()
    code = torch.where(finite[..., None], code, 0).flatten(-2)[..., :dh]
    return code, torch.where(finite, e + 127, 255.0).long()


def decode4(codes, scales):
    """codes [..., dh], scale bytes [..., groups] -> 64-bit values."""
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64, device=codes.device)
    s = torch.where(scales == 255, math.nan, power_of_two(scales - 127))
    return grid[codes] * s.repeat_interleave(32, dim=-1)[..., :codes.shape[-1]]


def unpack4(bytes_):
    return torch.stack([bytes_ & 15, bytes_ >> 4], dim=-1).flatten(-2).long()


def pack4(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).to(torch.uint8)
