"""The decoder's operators (include/otas_decode.h) in 64 bits, query by query and head by head, with bounds on what a correct
implementation in the operands' type may be off by.  Used by the tests only."""
import math

import numpy as np
import torch

F32 = 2.0 ** -24     # half a step of float32, relative
BF16 = 2.0 ** -8     # of bfloat16


def half_step(dtype):
    return F32 if dtype == torch.float32 else BF16


def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, original_length=8192.0, fast_turns=32.0, slow_turns=1.0):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        w = np.clip((original_length * f / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns), 0, 1)
        f = w * f + (1 - w) * f / factor
    return f


def rotary(qkv, H, KV, positions, rot, interleaved, freqs, magnitude=1.0, inverse=False):
    """(result, bound): |error| <= bound for products, sums and sines in float32 and one rounding to qkv's type."""
    T = qkv.shape[0]
    dh = qkv.shape[1] // (H + 2 * KV)
    x = qkv.double().view(T, H + 2 * KV, dh).clone()
    # float32: the angle as a fraction of a half turn 1.6, sine and cosine 4, magnitude, product and sum 3, each times what it goes with
    off = torch.zeros_like(x)
    a = torch.from_numpy(positions.cpu().numpy().astype(np.float64)[:, None] * freqs[None, :]).to(x.device)[:, None, :]
    a = -a if inverse else a
    first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    p, q = x[:, :H + KV, first].clone(), x[:, :H + KV, second].clone()
    x[:, :H + KV, first] = magnitude * (p * a.cos() - q * a.sin())
    x[:, :H + KV, second] = magnitude * (p * a.sin() + q * a.cos())
    size = abs(magnitude) * (p.abs() + q.abs()) * 9 * F32
    off[:, :H + KV, first] = size
    off[:, :H + KV, second] = size
    if qkv.dtype != torch.float32:
        off[:, :H + KV, :rot] += BF16 * x[:, :H + KV, :rot].abs() * (1 + 2 ** -6)
    return x.view(T, -1), off.view(T, -1)


def attend(q, k, v, visible, dtype, scale, cap=0.0, slope=0.0, distance=None):
    """One head: q [m, dh], k, v [n, dh], visible [m, n] -> (o, bound of o, weights, bound of the weights), 64 bits.

    Logits: dh products and sums, scale, cap (tanh good to 4 half steps, in bfloat16 to 2^-20, times cap), slope and distance,
    each rounded in float32.  Weights of a logit that is off by d are off by d of themselves and by the mean of d over the row; exponential,
    running sum and its factors add 16 half steps.  In bfloat16 the weight is rounded once before it meets the value, and the output
    once."""
    q, k, v = q.double(), k.double(), v.double()
    m, n, dh = q.shape[0], k.shape[0], q.shape[1]
    if n == 0:
        z = torch.zeros((m, v.shape[1]), dtype=torch.float64, device=q.device)
        e = torch.zeros((m, 0), dtype=torch.float64, device=q.device)
        return z, z, e, e
    seen = visible.any(dim=0)      # what no row sees may hold anything
    k, v = torch.where(seen[:, None], k, 0.0), torch.where(seen[:, None], v, 0.0)
    s = (q @ k.T.contiguous()) * scale
    off = F32 * ((dh + 4) * abs(scale) * (q.abs() @ k.abs().T.contiguous()) + 2 * s.abs())
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
    o = p @ v
    off = torch.where(visible, off + F32 * (2 * (s - top).abs() + 16), 0.0)
    off = torch.where(torch.isfinite(off), off, 0.0)
    rel = off + (p * off).sum(dim=1, keepdim=True)
    po = p * rel
    bound = po @ v.abs() + 4 * F32 * math.sqrt(n) * (p @ v.abs()) + F32 * o.abs()
    if dtype != torch.float32:
        bound = bound + BF16 * ((p @ v.abs()) + o.abs()) * (1 + 2 ** -6)
    return o, bound + 1e-30, p, po


def masked(qkv, H, KV, offsets, causal, prefix=None, documents=None, positions=None, scale=None, cap=0.0, slopes=None):
    dh = qkv.shape[1] // (H + 2 * KV)
    scale = dh ** -0.5 if scale is None else scale
    o = torch.zeros((qkv.shape[0], H * dh), dtype=torch.float64, device=qkv.device)
    b = torch.zeros_like(o)
    for q in range(len(offsets) - 1):
        a, z = int(offsets[q]), int(offsets[q + 1])
        n = z - a
        if n == 0:
            continue
        x = qkv[a:z].view(n, H + 2 * KV, dh)
        i = torch.arange(n, device=qkv.device)
        doc = torch.zeros(n, dtype=torch.int64, device=qkv.device) if documents is None else documents[a:z].long()
        pos = i if positions is None else positions[a:z].long()
        vis = doc[:, None] == doc[None, :]
        if causal:
            vis &= i[None, :] <= i[:, None]
        if prefix is not None:
            vis |= i[None, :] < int(prefix[q])
        vis &= (doc[:, None] >= 0) & (doc[None, :] >= 0)
        dist = (pos[:, None] - pos[None, :]).double()
        for h in range(H):
            kh = h // (H // KV)
            # rows are taken apart by what they see, so that a value that some of them do not see cannot reach them
            r, e, _, _ = attend(x[:, h], x[:, H + kh], x[:, H + KV + kh], vis, qkv.dtype, scale, cap,
                                0.0 if slopes is None else float(slopes[h]), dist)
            o[a:z, h * dh:(h + 1) * dh], b[a:z, h * dh:(h + 1) * dh] = r, e
    return o, b


def lines(parents):
    n = len(parents)
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        at = i
        while at >= 0:
            see[i, at] = True
            at = parents[at]
    return see


def tree(qkv, H, k, v, kpos, mass, offsets, parents, positions, slots, lengths, scale=None, cap=0.0, slopes=None):
    """(o, bound, mass, bound): mass is None or grows."""
    KV, dh = k.shape[1], k.shape[3]
    scale = dh ** -0.5 if scale is None else scale
    o = torch.zeros((qkv.shape[0], H * dh), dtype=torch.float64, device=qkv.device)
    b = torch.zeros_like(o)
    got = None if mass is None else mass.double().clone()
    got_b = None if mass is None else torch.zeros_like(got)
    for q in range(len(offsets) - 1):
        a, z, slot, n = int(offsets[q]), int(offsets[q + 1]), int(slots[q]), int(lengths[q])
        m = z - a
        if m == 0:
            continue
        x = qkv[a:z].view(m, H + 2 * KV, dh)
        mine = [i - 1 for i in range(m)] if parents is None else [int(p) for p in parents[a:z]]
        vis = torch.cat([torch.ones((m, n), dtype=torch.bool), torch.from_numpy(lines(mine))], dim=1).to(qkv.device)
        dist = None
        if slopes is not None:
            pos = torch.cat([kpos[slot, :n], positions[a:z]]).double()
            dist = positions[a:z].double()[:, None] - pos[None, :]
        add = torch.zeros(n, dtype=torch.float64, device=qkv.device)
        add_b = torch.zeros_like(add)
        for h in range(H):
            kh = h // (H // KV)
            r, e, p, pb = attend(x[:, h], torch.cat([k[slot, kh, :n], x[:, H + kh]]), torch.cat([v[slot, kh, :n], x[:, H + KV + kh]]), vis,
                                 qkv.dtype, scale, cap, 0.0 if slopes is None else float(slopes[h]), dist)
            o[a:z, h * dh:(h + 1) * dh], b[a:z, h * dh:(h + 1) * dh] = r, e
            add += p[:, :n].sum(dim=0)
            add_b += pb[:, :n].sum(dim=0)
        if got is not None:
            got[slot, :n] += add
            got_b[slot, :n] = add_b + F32 * (m * H * add + got[slot, :n].abs() + add)   # one rounding per addend, one of the sum
    return o, b, got, got_b


def evict(mass, positions, slots, lengths, keep, lead, recent_from):
    """Per query the (places, sources) of its moves, by sorting."""
    out = []
    m, p = mass.cpu().numpy(), positions.cpu().numpy()
    for q, (slot, n, kp) in enumerate(zip(slots, lengths, keep)):
        if kp >= n:
            out.append(([], []))
            continue
        score = m[slot, :n].astype(np.float64)
        first = np.arange(n) < lead
        if recent_from is not None:
            first |= p[slot, :n] >= recent_from[q]
        nan = np.isnan(score)
        order = sorted(range(n), key=lambda j: (not first[j], nan[j], 0.0 if nan[j] or first[j] else -score[j], j))
        stays = set(order[:kp])
        out.append(([j for j in range(kp) if j not in stays], [j for j in range(kp, n) if j in stays]))
    return out
