"""More operators of a decoder's layer, as cases that a performance measurement can run.

  norm     otas_norm_rotary        norms of query and key heads with rotary positions in the same pass
  window   otas_attention_window   attention over packed rows through a sliding window, with first tokens that stay visible
  recent   otas_attention_recent   the same for the last tokens of a key/value cache
  append4  otas_cache4_append      keys and values of packed rows into a cache of 4 bits an element, and back out of it
           otas_cache4_read
  cache4   otas_attention_cache4   attention of the last tokens over that cache

Where `own` is false, `run` computes the same in elementary torch operations.  `exact` computes it in 64 bits.

Packed rows are [T, (H + 2 Hkv) dh]: the query heads, the key heads, the value heads.  The cache is [slots, Hkv, capacity, dh], twice.
In 4 bits it is [slots, Hkv, capacity, dh / 2] bytes, the even element in the low half, and [slots, Hkv, ceil(dh / 32), capacity] bytes
of scale, 127 more than a power of two for 32 elements.
"""
import math

import numpy as np
import torch

own = False

# heads, key heads, head width.  base, huge: the encoder shapes of the repository's workloads; wide: 2048 columns.
SHAPES = {"base": (12, 12, 64), "base_g": (12, 4, 64), "huge": (16, 16, 80), "huge_g": (16, 4, 80), "narrow_g": (8, 2, 96),
          "wide": (16, 16, 128), "wide_g2": (16, 8, 128), "wide_g8": (16, 2, 128)}
GROUP = 32
EPS = 1e-6
ALL = 2 ** 31 - 1


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a step of a few requests, part of each head rotated, float32
        {"name": "norm_step_f32", "op": "norm", "dtype": "f32", "shape": "base", "tokens": 9, "rot": 24, "layout": "interleaved", "center": False, "per_head": False},
        # the prompts of a batch on their way from the QKV projection to attention
        {"name": "norm_prompts", "op": "norm", "dtype": "bf16", "shape": "wide_g2", "tokens": 16384, "rot": 128, "layout": "half", "center": False, "per_head": False},
        # three short prompts, float32
        {"name": "window_small_f32", "op": "window", "dtype": "f32", "shape": "base_g", "batch": 3, "tokens": 260, "ragged": 0.3, "window": 64, "sinks": 1, "cap": 0.0, "slopes": False},
        # a ragged batch of prompts through a narrow window, scores capped, the first twenty tokens stay
        {"name": "window_batch_cap", "op": "window", "dtype": "bf16", "shape": "base_g", "batch": 12, "tokens": 1500, "ragged": 0.6, "window": 300, "sinks": 20, "cap": 30.0, "slopes": False},
        # one long prompt
        {"name": "window_long", "op": "window", "dtype": "bf16", "shape": "wide_g8", "batch": 1, "tokens": 8192, "ragged": 0.0, "window": 1024, "sinks": 4, "cap": 0.0, "slopes": False},
        # drafted runs of two requests, float32
        {"name": "recent_drafts_f32", "op": "recent", "dtype": "f32", "shape": "base_g", "batch": 2, "tokens": 5, "cached": 700, "ragged": 0.2, "window": 256, "sinks": 4, "cap": 0.0, "slopes": True},
        # one token of each of 32 requests, long caches of which the window shows a part
        {"name": "recent_step", "op": "recent", "dtype": "bf16", "shape": "wide_g2", "batch": 32, "tokens": 1, "cached": 8192, "ragged": 0.3, "window": 2048, "sinks": 4, "cap": 0.0, "slopes": False},
        # the new tokens of a step into the cache
        {"name": "append4_step", "op": "append4", "dtype": "bf16", "shape": "wide_g2", "batch": 32, "tokens": 1, "ragged": 0.0, "taken": 0, "capacity": 2048},
        # prompts into the cache
        {"name": "append4_prompts", "op": "append4", "dtype": "bf16", "shape": "wide_g2", "batch": 24, "tokens": 700, "ragged": 0.5, "taken": 0, "capacity": 2048},
        # a single request, float32
        {"name": "cache4_one_f32", "op": "cache4", "dtype": "f32", "shape": "huge_g", "batch": 1, "tokens": 1, "cached": 3001, "ragged": 0.0, "window": 0, "sinks": 0, "cap": 0.0, "slopes": False},
        # one token of each of 32 requests over all of their caches
        {"name": "cache4_step", "op": "cache4", "dtype": "bf16", "shape": "wide_g2", "batch": 32, "tokens": 1, "cached": 8192, "ragged": 0.3, "window": 0, "sinks": 0, "cap": 0.0, "slopes": False},
        # a prompt in pieces: 256 rows of each of four requests, scores capped, a window over the cache
        {"name": "cache4_pieces", "op": "cache4", "dtype": "bf16", "shape": "wide_g8", "batch": 4, "tokens": 256, "cached": 4000, "ragged": 0.5, "window": 2500, "sinks": 4, "cap": 50.0, "slopes": False},
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op, dtype = rng.choice(["norm", "window", "window", "recent", "recent", "append4", "cache4", "cache4"]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    shape = rng.choice(sorted(SHAPES))
    dh = SHAPES[shape][2]
    c = {"op": op, "dtype": dtype, "shape": shape}
    if op == "norm":
        c |= {"tokens": log(1, 16384), "rot": 2 * rng.randint(0, dh // 2), "layout": rng.choice(["half", "interleaved"]),
              "center": rng.random() < 0.3, "per_head": rng.random() < 0.3}
    elif op == "append4":
        c |= {"batch": log(1, 24), "tokens": log(1, 700), "ragged": rng.choice([0.0, 0.3, 0.9]), "taken": rng.choice([0, 0, 1, 2]), "capacity": 2048}
    elif op == "window":
        n = log(1, 2500 if dtype == "f32" else 6000)
        c |= {"batch": max(1, min(24, log(1, 24), 9000000 // (n * n) + 1)), "tokens": n, "ragged": rng.choice([0.0, 0.3, 0.95]), "window": log(1, 2 * n),
              "sinks": rng.choice([0, 1, 4, rng.randint(1, 200)]), "cap": rng.choice([0.0, 0.0, 30.0]), "slopes": rng.random() < 0.3}
    else:
        batch, cached, rows = log(1, 32), log(1, 8000), rng.choice([1, 1, 1, rng.randint(2, 8), log(9, 300)])
        rows = max(1, min(rows, cached, 3000000 // (batch * cached)))
        c |= {"batch": batch, "tokens": rows, "cached": cached, "ragged": rng.choice([0.0, 0.3, 0.95]),
              "window": log(1, 8000) if op == "recent" or rng.random() < 0.4 else 0,
              "sinks": rng.choice([0, 1, 4, rng.randint(1, 200)]), "cap": rng.choice([0.0, 0.0, 50.0]), "slopes": rng.random() < 0.3}
    return c


def _ragged(most, batch, ragged):
    """`batch` lengths spread over [(1 - ragged) most, most]."""
    return [max(1, int(most * (1.0 - ragged * (q * 0.618034 % 1.0)))) for q in range(batch)]


def _lengths(case):
    """Filled entries of every query, its own rows' among them."""
    return [max(n, case["tokens"]) for n in _ragged(case["cached"], case["batch"], case["ragged"])]


def _window(case):
    return case["window"] or ALL


def _seen(places, window, sinks):
    """How many tokens those at `places` see."""
    near = np.minimum(places + 1, window)
    return int((near + np.minimum(np.maximum(places + 1 - near, 0), sinks)).sum())


def work(case):
    H, KV, dh = SHAPES[case["shape"]]
    e, op = 4 if case["dtype"] == "f32" else 2, case["op"]
    if op == "norm":
        return {"bytes": case["tokens"] * (2 * (H + 2 * KV) * dh * e + 4), "flops": case["tokens"] * (H + KV) * (4 * dh + 3 * case["rot"])}
    held = dh // 2 + -(-dh // GROUP)  # bytes of a head of an entry in 4 bits
    if op == "append4":
        rows = sum(_ragged(case["tokens"], case["batch"], case["ragged"])) if not case["taken"] else case["taken"] * case["batch"]
        return {"bytes": rows * 2 * KV * (2 * dh * e + 2 * held), "flops": rows * 2 * KV * dh * 4}
    window, sinks = _window(case), case["sinks"]
    if op == "window":
        n = _ragged(case["tokens"], case["batch"], case["ragged"])
        return {"bytes": sum(n) * (2 * H + 2 * KV) * dh * e, "flops": 4 * dh * H * sum(_seen(np.arange(m), window, sinks) for m in n)}
    m, entries, pairs = case["tokens"], 0, 0
    for n in _lengths(case):
        first = max(0, n - m + 1 - window)  # of the window of the query's first row
        entries += n - first + min(first, sinks)
        pairs += _seen(np.arange(n - m, n), window, sinks)
    return {"bytes": entries * 2 * KV * (held if op == "cache4" else dh * e) + 2 * m * case["batch"] * H * dh * e, "flops": 4 * dh * H * pairs}


# ----------------------------------------------------------------------------------------------------------- inputs
def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device="cuda")


def prepare(case, seed):
    """What a serving program holds before the call: packed rows, the cache, the requests' lengths and slots as host
    integers (the scheduler's own) and, for the plain form, the same numbers on the device."""
    H, KV, dh = SHAPES[case["shape"]]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 32))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dt)

    st, op = {"case": dict(case), "heads": (H, KV, dh), "dt": dt}, case["op"]
    if op == "norm":
        T = case["tokens"]
        st["qkv"], st["out"] = normal(T, (H + 2 * KV) * dh, std=3.0), torch.empty((T, (H + 2 * KV) * dh), dtype=dt, device="cuda")
        st["positions"] = torch.randint(0, 131072, (T,), generator=g, device="cuda", dtype=torch.int32)
        gains = (lambda n: (n, dh)) if case["per_head"] else (lambda n: (dh,))
        st["q_gain"], st["k_gain"] = normal(*gains(H), std=0.2) + 1, normal(*gains(KV), std=0.2) + 1
        return st
    B = case["batch"]
    n = _ragged(case["tokens"], B, case["ragged"]) if op in ("window", "append4") else [case["tokens"]] * B
    st["offsets"] = [0] + [int(x) for x in np.cumsum(n)]
    st["offsets_dev"] = torch.tensor(st["offsets"], device="cuda")
    T = st["offsets"][-1]
    st["qkv"] = normal(T, (H + 2 * KV) * dh)
    if op != "append4":
        st["o"] = torch.empty((T, H * dh), dtype=dt, device="cuda")
        st["slopes"] = _slopes(H) if case["slopes"] else None
    if op == "window":
        return st
    # the slots of a call are in no order, and one of the cache's is another request's
    st["slots"] = [(q * 7 + 3) % (B + 1) if (B + 1) % 7 else (q + 3) % (B + 1) for q in range(B)]
    st["slots_dev"] = torch.tensor(st["slots"], device="cuda")
    if op == "append4":
        capacity = case["capacity"]
        st["lengths"] = [int(x) for x in rng.randint(0, capacity - max(n) + 1, B)]
        st["rows"], st["row_offsets"] = None, st["offsets"]
        if case["taken"]:  # accepted drafts: rows of a request in rising order
            take = min(case["taken"], min(n))
            st["rows"] = [int(a + r) for a, m in zip(st["offsets"], n) for r in np.sort(rng.choice(m, take, replace=False))]
            st["row_offsets"] = [take * q for q in range(B + 1)]
        m = np.diff(st["row_offsets"])
        st["rows_dev"] = torch.tensor(st["rows"] if st["rows"] is not None else range(T), device="cuda")
        st["entry_dev"] = torch.tensor(np.concatenate([l + np.arange(k) for l, k in zip(st["lengths"], m)]), device="cuda")
        st["query_dev"] = torch.tensor(np.repeat(np.arange(B), m), device="cuda")
        st["back"] = torch.empty((st["row_offsets"][-1], 2 * KV * dh), dtype=dt, device="cuda")
    else:
        st["lengths"] = _lengths(case)
        st["lengths_dev"] = torch.tensor(st["lengths"], device="cuda")
        capacity = -(-max(st["lengths"]) // 64) * 64
    if op == "recent":
        st["k"], st["v"] = normal(B + 1, KV, capacity, dh), normal(B + 1, KV, capacity, dh)
        st["positions_cache"] = torch.arange(capacity, dtype=torch.int32, device="cuda").repeat(B + 1, 1)
        return st
    for name in ("k", "v"):
        codes = torch.empty((B + 1, KV, capacity, dh // 2), dtype=torch.uint8, device="cuda")
        scales = torch.empty((B + 1, KV, -(-dh // GROUP), capacity), dtype=torch.uint8, device="cuda")
        for s in range(B + 1):
            c, e = _encode(normal(KV, capacity, dh))
            codes[s], scales[s] = c, e.transpose(-1, -2)
        st[name], st[name + "_scales"] = codes, scales
    return st


# ------------------------------------------------------------------------------------------------------- plain form
def _encode(x):
    """x [..., dh] in 4 bits: bytes [..., dh / 2] and scales [..., groups]."""
    dh = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -dh % GROUP)).unflatten(-1, (-1, GROUP))
    fraction, exponent = torch.frexp(x.abs().amax(dim=-1))  # fraction in [1/2, 1): 7 2^e is 7/8 of 2^(e + 3)
    e = exponent - torch.where(fraction > 0.875, 2, 3)
    e = torch.where(fraction == 0.0, -125, e).clamp(-125, 125).to(torch.int32)
    y = x.abs() * ((127 - e) << 23).view(torch.float32)[..., None]
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8) + 8 * (x < 0).to(torch.uint8)
    code = code.flatten(-2)[..., :dh]
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """The float32 values of bytes [..., dh / 2] with scales [..., groups]."""
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    x = torch.stack([values[(codes & 15).int()], values[(codes >> 4).int()]], dim=-1).flatten(-2)
    size = (scales.int() << 23).view(torch.float32).repeat_interleave(GROUP, dim=-1)
    return x * size[..., :x.shape[-1]]


def _plain_norm(st):
    case, (H, KV, dh) = st["case"], st["heads"]
    rot = case["rot"]
    x = st["qkv"].view(-1, H + 2 * KV, dh)
    y = x.to(torch.float32, copy=True)
    for heads, gain in ((slice(0, H), st["q_gain"]), (slice(H, H + KV), st["k_gain"])):
        z = y[:, heads]
        if case["center"]:
            z = z - z.mean(dim=-1, keepdim=True)
        y[:, heads] = z / torch.sqrt((z * z).mean(dim=-1, keepdim=True) + EPS) * gain.float()
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    angle = st["positions"].double()[:, None] * f
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    z = y[:, :H + KV, :rot]
    if case["layout"] == "half":
        a, b = z[..., :rot // 2], z[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = z[..., 0::2], z[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    y[:, :H + KV, :rot] = turned
    return {"qkv": y.to(st["dt"]).view_as(st["qkv"])}


def _weights(s, visible):
    """Softmax over the visible keys; rows without any are zero."""
    s = torch.where(visible, s, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    return p / torch.where(total == 0.0, 1.0, total)


def _attend(st, q, k, v, row, key):
    """q [B, H, m, dh] of tokens row [B, m], k, v [B, KV, n, dh] of tokens key [n]; float32."""
    case, (H, KV, dh) = st["case"], st["heads"]
    B, m, n = q.shape[0], q.shape[2], k.shape[2]
    s = torch.matmul(q.reshape(B, KV, H // KV * m, dh), k.transpose(-1, -2).contiguous()) * dh ** -0.5
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    s = s.view(B, H, m, n)
    behind = row[:, :, None] - key[None, None, :]
    if st["slopes"] is not None:
        s = s - st["slopes"][:, None, None] * behind[:, None].abs()
    visible = (behind >= 0) & ((behind < _window(case)) | (key < case["sinks"])[None, None, :])
    return torch.matmul(_weights(s, visible[:, None]).view(B, KV, H // KV * m, n), v).view(B, H, m, dh)


def _plain_window(st):
    H, KV, dh = st["heads"]
    off = st["offsets_dev"]
    at = torch.arange(int(max(np.diff(st["offsets"]))), device="cuda")
    inside = at[None, :] < (off[1:] - off[:-1])[:, None]
    x = st["qkv"][torch.where(inside, off[:-1, None] + at[None, :], 0)].float().view(len(off) - 1, -1, H + 2 * KV, dh).transpose(1, 2)
    o = _attend(st, x[:, :H], x[:, H:H + KV].contiguous(), x[:, H + KV:].contiguous(), at.expand(len(off) - 1, -1), at)
    return {"o": o.transpose(1, 2)[inside].reshape(-1, H * dh).to(st["dt"])}


def _plain_cached(st, k, v):
    (H, KV, dh), m, B = st["heads"], st["case"]["tokens"], st["case"]["batch"]
    q = st["qkv"].float().view(B, m, H + 2 * KV, dh).transpose(1, 2)[:, :H]
    row = st["lengths_dev"][:, None] - m + torch.arange(m, device="cuda")[None, :]
    o = _attend(st, q, k, v, row, torch.arange(k.shape[2], device="cuda"))
    return {"o": o.transpose(1, 2).reshape(B * m, H * dh).to(st["dt"])}


def _plain_recent(st):
    longest = max(st["lengths"])
    return _plain_cached(st, st["k"][st["slots_dev"], :, :longest].float(), st["v"][st["slots_dev"], :, :longest].float())


def _plain_cache4(st):
    longest = max(st["lengths"])
    k, v = [_decode(st[name][st["slots_dev"], :, :longest], st[name + "_scales"][st["slots_dev"], :, :, :longest].transpose(-1, -2)) for name in ("k", "v")]
    return _plain_cached(st, k, v)


def _plain_append4(st):
    H, KV, dh = st["heads"]
    x = st["qkv"].view(-1, H + 2 * KV, dh)[st["rows_dev"]]
    slot, entry = st["slots_dev"][st["query_dev"]], st["entry_dev"]
    back = []
    for name, rows in (("k", x[:, H:H + KV]), ("v", x[:, H + KV:])):
        codes, scales = _encode(rows)
        st[name][slot, :, entry] = codes
        st[name + "_scales"][slot, :, :, entry] = scales
        back.append(_decode(st[name][slot, :, entry], st[name + "_scales"][slot, :, :, entry]))
    return {"kv": torch.cat(back, dim=1).to(st["dt"]).view(len(slot), -1)}


PLAIN = {"norm": _plain_norm, "window": _plain_window, "recent": _plain_recent, "append4": _plain_append4, "cache4": _plain_cache4}


# ----------------------------------------------------------------------------------------------- the framework's calls
_CONTEXTS = {}


def _context(st):
    """The program's context for this model shape on the current device and stream, to which a context is bound."""
    import paper_2401_05031_amd as otas
    H, KV, dh = st["heads"]
    device = torch.cuda.current_device()
    # torch.cuda.current_stream() makes an object, 2.7 us; its number alone takes 0.1
    key = (H, dh, st["dt"], device, torch._C._cuda_getCurrentRawStream(device))
    if key not in _CONTEXTS:
        D = H * dh
        sizes = {"ln1_g": (D,), "ln1_b": (D,), "w_qkv": (3 * D, D), "b_qkv": (3 * D,), "w_proj": (D, D), "b_proj": (D,), "ln2_g": (D,), "ln2_b": (D,),
                 "w_fc1": (2 * D, D), "b_fc1": (2 * D,), "w_fc2": (D, 2 * D), "b_fc2": (D,)}
        layer = {name: torch.zeros(size, dtype=st["dt"], device="cuda") for name, size in sizes.items()}
        _CONTEXTS[key] = otas.Context(1, D, H, 2 * D, otas.OTAS_F32 if st["dt"] == torch.float32 else otas.OTAS_BF16, 1e-6, 1, [layer])
    return otas, _CONTEXTS[key]


def _own(st):
    otas, ctx = _context(st)
    case, (H, KV, dh), op = st["case"], st["heads"], st["case"]["op"]
    if op == "norm":
        if "rope" not in st:
            st["rope"] = otas.Rotary(rot_dim=case["rot"], layout={"half": otas.OTAS_ROTARY_HALF, "interleaved": otas.OTAS_ROTARY_INTERLEAVED}[case["layout"]], base=10000.0)
            st["norm"] = otas.HeadNorm(st["q_gain"], st["k_gain"], eps=EPS, center=case["center"], per_head=case["per_head"])
        ctx.otas_norm_rotary(st["qkv"], KV, st["norm"], st["positions"], st["rope"], st["out"])
        return {"qkv": st["out"]}
    if op == "append4":
        cache = otas.KVCache4(st["k"], st["v"], st["k_scales"], st["v_scales"])
        ctx.otas_cache4_append(cache, st["qkv"], st["row_offsets"], st["rows"], st["slots"], st["lengths"])
        ctx.otas_cache4_read(cache, st["slots"], st["lengths"], st["row_offsets"], st["back"])
        return {"kv": st["back"]}
    score, window, sinks = otas.Score(cap=case["cap"], slopes=st["slopes"]), _window(case), case["sinks"]
    if op == "window":
        ctx.otas_attention_window(st["qkv"], KV, st["offsets"], st["o"], window, sinks=sinks, score=score)
        return {"o": st["o"]}
    if "workspace" not in st:
        st["workspace"] = torch.empty(ctx.otas_attention_recent_workspace_bytes(KV, st["offsets"], st["lengths"], window, sinks), dtype=torch.uint8, device="cuda")
    if op == "recent":
        cache = otas.KVCache(st["k"], st["v"], st["positions_cache"])
        ctx.otas_attention_recent(cache, st["qkv"], st["offsets"], st["slots"], st["lengths"], st["workspace"], st["o"], window, sinks=sinks, score=score)
    else:
        cache = otas.KVCache4(st["k"], st["v"], st["k_scales"], st["v_scales"])
        ctx.otas_attention_cache4(cache, st["qkv"], st["offsets"], st["slots"], st["lengths"], st["workspace"], st["o"], window, sinks=sinks, score=score)
    return {"o": st["o"]}


def run(st):
    return _own(st) if own else PLAIN[st["case"]["op"]](st)


# ------------------------------------------------------------------------------------------------------------ 64 bits
def _exact_norm(case, st, H, KV, dh):
    rot = case["rot"]
    x = st["qkv"].double().view(-1, H + 2 * KV, dh)
    gain = torch.ones((H + 2 * KV, dh), dtype=torch.float64, device="cuda")
    gain[:H], gain[H:H + KV] = st["q_gain"].double(), st["k_gain"].double()
    heads = x[:, :H + KV]
    if case["center"]:
        heads = heads - heads.sum(dim=2, keepdim=True) / dh
    x[:, :H + KV] = heads * torch.rsqrt(heads.pow(2).sum(dim=2, keepdim=True) / dh + EPS) * gain[:H + KV]
    if rot:
        f = np.exp(-np.log(10000.0) * 2 * np.arange(rot // 2, dtype=np.float64) / rot)
        turn = torch.from_numpy(np.exp(1j * st["positions"].cpu().numpy().astype(np.float64)[:, None] * f[None, :])).to("cuda")[:, None, :]
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[:, :H + KV, first].contiguous(), x[:, :H + KV, second].contiguous()) * turn
        x[:, :H + KV, first], x[:, :H + KV, second] = z.real, z.imag
    return {"qkv": x.view_as(st["qkv"])}


def _exact_rows(case, st, q, k, v, first):
    """q [m, H, dh] of the tokens from `first` on over k, v [n, KV, dh], 64 bits."""
    m, H, dh = q.shape
    out = torch.zeros_like(q)
    group = H // k.shape[1]
    for a in range(0, m, 2048):
        token = torch.arange(first + a, first + min(m, a + 2048), device="cuda").view(-1, 1)
        key = torch.arange(k.shape[0], device="cuda").view(1, -1)
        hidden = (key > token) | ((key <= token - _window(case)) & (key >= case["sinks"]))
        for h in range(H):
            s = (q[a:a + 2048, h] / math.sqrt(dh)) @ k[:, h // group].T.contiguous()
            if case["cap"]:
                s = case["cap"] * (s / case["cap"]).tanh()
            if st["slopes"] is not None:
                s -= float(st["slopes"][h]) * (token - key)
            s[hidden] = -1e300
            e = (s - s.max(dim=1, keepdim=True).values).exp()
            out[a:a + 2048, h] = e @ v[:, h // group] / e.sum(dim=1, keepdim=True)  # a row always sees itself
    return out


def _exact_window(case, st, H, KV, dh):
    out = []
    for a, b in zip(st["offsets"], st["offsets"][1:]):
        x = st["qkv"][a:b].double().view(b - a, H + 2 * KV, dh)
        out.append(_exact_rows(case, st, x[:, :H], x[:, H:H + KV], x[:, H + KV:], 0))
    return {"o": torch.cat(out).view(-1, H * dh)}


def _exact_value(codes, scales):
    """Bytes [n, KV, dh / 2] and scales [KV, groups, n] as 64-bit values [n, KV, dh], from the bits of the two-bit exponent and the one of
    the mantissa."""
    bits = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).long()
    exponent, mantissa = bits // 2 % 4, bits % 2
    size = torch.where(exponent == 0, mantissa * 0.5, (1 + 0.5 * mantissa) * torch.pow(2.0, (exponent - 1).double()))
    group = torch.arange(bits.shape[-1], device="cuda") // GROUP
    return torch.where(bits >= 8, -size, size) * torch.pow(2.0, scales.permute(2, 0, 1)[..., group].double() - 127.0)


def _exact_cached(case, st, H, KV, dh):
    m, out = case["tokens"], []
    for q, (slot, n) in enumerate(zip(st["slots"], st["lengths"])):
        x = st["qkv"][q * m:(q + 1) * m].double().view(m, H + 2 * KV, dh)
        if case["op"] == "recent":
            k, v = st["k"][slot, :, :n].double().transpose(0, 1), st["v"][slot, :, :n].double().transpose(0, 1)
        else:
            k, v = [_exact_value(st[name][slot, :, :n].transpose(0, 1), st[name + "_scales"][slot, :, :, :n]) for name in ("k", "v")]
        out.append(_exact_rows(case, st, x[:, :H], k.contiguous(), v.contiguous(), n - m))
    return {"o": torch.cat(out).view(-1, H * dh)}


def _exact_append4(case, st, H, KV, dh):
    rows = st["rows"] if st["rows"] is not None else list(range(st["offsets"][-1]))
    grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device="cuda")  # those of even codes first
    later = torch.tensor([0.0] * 4 + [1e-9] * 4, dtype=torch.float64, device="cuda")  # which a value between two goes to
    out = torch.empty((len(rows), 2 * KV, dh), dtype=torch.float64, device="cuda")
    for a in range(0, len(rows), 1024):
        x = st["qkv"][rows[a:a + 1024]].double().view(-1, H + 2 * KV, dh)[:, H:]
        for d in range(0, dh, GROUP):
            y = x[..., d:d + GROUP]
            top = y.abs().max(dim=-1, keepdim=True).values
            e = torch.floor(torch.log2(top.clamp_min(1e-300))) - 4  # then up to the first that holds the largest to half a step
            for _ in range(4):
                e += top > 7.0 * torch.pow(2.0, e)
            scale = torch.pow(2.0, e.clamp(-125, 125))
            nearest = grid[((y.abs() / scale)[..., None] - grid).abs().add(later).argmin(dim=-1)]
            out[a:a + 1024, :, d:d + GROUP] = torch.sign(y) * nearest * scale
    return {"kv": out.view(len(rows), -1)}


def exact(case, seed):
    if case["op"] in ("recent", "cache4") and case["batch"] * case["cached"] > 400000:
        return None
    st = prepare(case, seed)
    H, KV, dh = st["heads"]
    return {"norm": _exact_norm, "window": _exact_window, "recent": _exact_cached, "cache4": _exact_cached, "append4": _exact_append4}[case["op"]](case, st, H, KV, dh)
