"""The operators of a decoder's attention around its key/value cache, as cases that a performance measurement can run.

  rotary   otas_rotary            rotary positions on packed query and key heads
  append   otas_cache_append      rotated keys and values of packed rows, or of accepted drafts, into the cache
  masked   otas_attention_masked  attention over packed rows: causal, a prefix that all see, documents, capped scores,
                                  a bias by distance
  tree     otas_attention_tree    attention of drafted tokens (a tree; one node when nothing is drafted) over the cache
  evict    otas_cache_evict       the cache cut down to the tokens that got the most attention

Where `own` is false, `run` computes the same in elementary torch operations.  `exact` computes it in 64 bits.

Packed rows are [T, (H + 2 Hkv) dh]: the query heads, the key heads, the value heads.  The cache is [slots, Hkv,
capacity, dh], twice, with a position and an accumulated attention weight per slot and entry.
"""
import math

import numpy as np
import torch

own = False

# heads, key heads, head width.  base, huge: the encoder shapes of the repository's workloads; wide: 2048 columns.
SHAPES = {"base": (12, 12, 64), "base_g": (12, 4, 64), "huge": (16, 16, 80), "huge_g": (16, 4, 80), "narrow_g": (8, 2, 96),
          "wide": (16, 16, 128), "wide_g2": (16, 8, 128), "wide_g8": (16, 2, 128)}
TWO_PI = 2 * math.pi


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a step of a few requests, part of each head rotated, float32
        {"name": "rotary_step_f32", "op": "rotary", "dtype": "f32", "shape": "base", "tokens": 37, "rot": 24, "layout": "interleaved", "scaling": "plain"},
        # the prompts of a batch on their way from the QKV projection to attention, positions scaled for long contexts
        {"name": "rotary_prompts", "op": "rotary", "dtype": "bf16", "shape": "wide_g2", "tokens": 16384, "rot": 128, "layout": "half", "scaling": "parts"},
        # the accepted drafts of eight requests: four rows of each one's twelve
        {"name": "append_accepted_f32", "op": "append", "dtype": "f32", "shape": "base", "batch": 8, "tokens": 12, "taken": 4, "ragged": 0.0, "capacity": 1024},
        # the prompts of a batch into the cache
        {"name": "append_prompts", "op": "append", "dtype": "bf16", "shape": "wide_g2", "batch": 8, "tokens": 2000, "taken": 0, "ragged": 0.5, "capacity": 4096},
        # pictures of 197 tokens in front of short texts, float32
        {"name": "masked_pictures_f32", "op": "masked", "dtype": "f32", "shape": "base", "batch": 8, "tokens": 261, "ragged": 0.2, "causal": True, "prefix": 197, "documents": 0, "cap": 0.0, "slopes": False},
        # documents packed into long rows with padding behind the last, weights falling off with the distance
        {"name": "masked_documents", "op": "masked", "dtype": "bf16", "shape": "huge", "batch": 3, "tokens": 4000, "ragged": 0.1, "causal": True, "prefix": 16, "documents": 7, "cap": 0.0, "slopes": True},
        # one long prompt, capped scores
        {"name": "masked_long_cap", "op": "masked", "dtype": "bf16", "shape": "wide_g8", "batch": 1, "tokens": 8192, "ragged": 0.0, "causal": True, "prefix": 0, "documents": 0, "cap": 30.0, "slopes": False},
        # the next token of one request: latency
        {"name": "tree_one_token", "op": "tree", "dtype": "bf16", "shape": "wide_g8", "batch": 1, "nodes": 1, "cached": 1537, "ragged": 0.0, "cap": 0.0, "slopes": True, "mass": False},
        # the next token of 32 requests with long caches that count the attention they get
        {"name": "tree_batch_mass", "op": "tree", "dtype": "bf16", "shape": "wide_g2", "batch": 32, "nodes": 1, "cached": 8192, "ragged": 0.3, "cap": 0.0, "slopes": False, "mass": True},
        # trees of drafts to be verified
        {"name": "tree_drafts_cap", "op": "tree", "dtype": "bf16", "shape": "wide_g2", "batch": 8, "nodes": 48, "cached": 4000, "ragged": 0.5, "cap": 50.0, "slopes": False, "mass": False},
        # two small float32 caches cut to three quarters
        {"name": "evict_small_f32", "op": "evict", "dtype": "f32", "shape": "base_g", "batch": 2, "cached": 1000, "ragged": 0.1, "keep": 0.75, "lead": 4, "recent": 64},
        # long caches of a batch cut by a quarter
        {"name": "evict_batch", "op": "evict", "dtype": "bf16", "shape": "wide_g2", "batch": 16, "cached": 16000, "ragged": 0.2, "keep": 0.75, "lead": 4, "recent": 256},
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op, dtype = rng.choice(["rotary", "append", "masked", "masked", "tree", "tree", "evict"]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    shape = rng.choice(sorted(SHAPES))
    H, KV, dh = SHAPES[shape]
    c = {"op": op, "dtype": dtype, "shape": shape}
    if op == "rotary":
        c |= {"tokens": log(1, 16384), "rot": 2 * rng.randint(1, dh // 2), "layout": rng.choice(["half", "interleaved"]),
              "scaling": rng.choice(["plain", "linear", "base", "parts"])}
        if c["rot"] < 4:
            c["scaling"] = "plain"
    elif op == "append":
        c |= {"batch": log(1, 32), "tokens": log(2, 900), "taken": rng.choice([0, 0, 1, 2]), "ragged": rng.choice([0.0, 0.3, 0.9]), "capacity": 2048}
    elif op == "masked":
        n = log(20, 2500 if dtype == "f32" else 5500)
        c |= {"batch": max(1, min(24, log(1, 24), 9000000 // (n * n) + 1)), "tokens": n, "ragged": rng.choice([0.0, 0.3, 0.95]), "causal": rng.random() < 0.75,
              "prefix": rng.choice([0, 0, rng.randint(1, n)]), "documents": rng.choice([0, 0, 3, 11]), "cap": rng.choice([0.0, 0.0, 30.0, 50.0]), "slopes": rng.random() < 0.4}
    elif op == "tree":
        c |= {"batch": log(1, 24), "nodes": rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 64)]), "cached": log(1, 8000), "ragged": rng.choice([0.0, 0.3, 0.95]),
              "cap": rng.choice([0.0, 0.0, 50.0]), "slopes": rng.random() < 0.3, "mass": rng.random() < 0.4}
    else:
        c |= {"batch": log(1, 16), "cached": log(64, 16000), "ragged": rng.choice([0.0, 0.2, 0.8]), "keep": round(rng.uniform(0.05, 0.98), 3), "lead": rng.choice([0, 1, 4]),
              "recent": log(1, 300)}
    return c


def _ragged(most, batch, ragged):
    """`batch` lengths spread over [(1 - ragged) most, most]."""
    return [max(1, int(most * (1.0 - ragged * (q * 0.618034 % 1.0)))) for q in range(batch)]


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def _kept(case):
    return [max(1, int(n * case["keep"])) for n in _ragged(case["cached"], case["batch"], case["ragged"])]


def _documents(n, count):
    """The edges of `count` documents of unequal length in n rows, a fiftieth of which is padding behind them."""
    return [int((n - n // 50) * (k / count) ** 1.3) for k in range(count + 1)]


def _visible_pairs(case):
    total = 0
    for n in _ragged(case["tokens"], case["batch"], case["ragged"]):
        p = min(case["prefix"], n)
        edges = _documents(n, case["documents"]) if case["documents"] else [0, n]
        if not case["causal"]:
            total += sum((b - a) * ((b - a) + p - (min(p, b) - min(p, a))) for a, b in zip(edges, edges[1:]))
            continue
        for a, b in zip(edges, edges[1:]):  # row i of [a, b) sees the prefix, and of its document [a, i]
            inside = np.arange(a, b)
            total += int((p + np.maximum(0, inside + 1 - np.maximum(a, p))).sum())
    return total


def work(case):
    H, KV, dh = SHAPES[case["shape"]]
    e, op = _element(case), case["op"]
    if op == "rotary":
        return {"bytes": case["tokens"] * (2 * (H + 2 * KV) * dh * e + 4), "flops": case["tokens"] * (H + KV) * case["rot"] * 3}
    if op == "append":
        rows = sum(_ragged(case["tokens"], case["batch"], case["ragged"])) if not case["taken"] else case["taken"] * case["batch"]
        return {"bytes": rows * (4 * KV * dh * e + 12), "flops": 0}
    if op == "masked":
        T = sum(_ragged(case["tokens"], case["batch"], case["ragged"]))
        return {"bytes": T * (2 * H + 2 * KV) * dh * e, "flops": 4 * dh * H * _visible_pairs(case)}
    if op == "tree":
        n = sum(_ragged(case["cached"], case["batch"], case["ragged"]))
        T = case["nodes"] * case["batch"]
        return {"bytes": n * (2 * KV * dh * e + (4 if case["slopes"] else 0) + (8 if case["mass"] else 0)) + T * (2 * H + 2 * KV) * dh * e, "flops": 4 * dh * H * case["nodes"] * n}
    n, m = _ragged(case["cached"], case["batch"], case["ragged"]), _kept(case)
    moved = sum(min(b, a - b) * b // a for a, b in zip(n, m))  # about so many of the kept entries lie behind the cut
    return {"bytes": 8 * sum(n) + moved * (4 * KV * dh * e + 16), "flops": sum(n)}


# ----------------------------------------------------------------------------------------------------------- inputs
def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device="cuda")


def _cache(case, st, normal, g, slots, capacity):
    H, KV, dh = SHAPES[case["shape"]]
    st["k"], st["v"] = normal(slots, KV, capacity, dh), normal(slots, KV, capacity, dh)
    # positions and weights side by side, as a program that saves and restores them in one go keeps them
    st["meta"] = torch.empty((2, slots, capacity), dtype=torch.int32, device="cuda")
    st["positions_cache"], st["mass"] = st["meta"][0], st["meta"][1].view(torch.float32)
    # entries are in no order once some were evicted: every position below twice the capacity at most once
    st["positions_cache"].copy_(torch.rand((slots, 2 * capacity), generator=g, device="cuda").argsort(dim=1)[:, :capacity])
    st["mass"].copy_(torch.rand((slots, capacity), generator=g, device="cuda").pow_(4))
    st["slots"] = [(q * 7 + 3) % slots if slots % 7 else (q + 3) % slots for q in range(case["batch"])]
    st["slots_dev"] = torch.tensor(st["slots"], device="cuda")


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
    if op == "rotary":
        T = case["tokens"]
        st["qkv"], st["out"] = normal(T, (H + 2 * KV) * dh), torch.empty((T, (H + 2 * KV) * dh), dtype=dt, device="cuda")
        st["positions"] = torch.randint(0, 131072, (T,), generator=g, device="cuda", dtype=torch.int32)
        return st
    B = case["batch"]
    if op in ("append", "masked"):
        n = _ragged(case["tokens"], B, case["ragged"])
    else:
        n = [case["nodes"]] * B if op == "tree" else []
    st["offsets"] = [0] + [int(x) for x in np.cumsum(n)]
    T = st["offsets"][-1]
    if op != "evict":
        st["qkv"] = normal(T, (H + 2 * KV) * dh)
        st["offsets_dev"] = torch.tensor(st["offsets"], device="cuda")
    if op == "append":
        capacity = case["capacity"]
        _cache(case, st, normal, g, B + 1, capacity)
        st["lengths"] = [int(x) for x in rng.randint(0, capacity - max(n) + 1, B)]
        st["positions"] = torch.cat([torch.arange(m, device="cuda", dtype=torch.int32) + 5 for m in n])
        st["rows"] = None
        st["row_offsets"] = st["offsets"]
        if case["taken"]:  # an accepted path: rows of a request in rising order
            take = min(case["taken"], min(n))
            st["rows"] = [int(a + r) for a, m in zip(st["offsets"], n) for r in np.sort(rng.choice(m, take, replace=False))]
            st["row_offsets"] = [take * q for q in range(B + 1)]
        m = np.diff(st["row_offsets"])
        st["rows_dev"] = torch.tensor(st["rows"] if st["rows"] is not None else range(T), device="cuda")
        st["entry_dev"] = torch.tensor(np.concatenate([l + np.arange(k) for l, k in zip(st["lengths"], m)]), device="cuda")
        st["query_dev"] = torch.tensor(np.repeat(np.arange(B), m), device="cuda")
    elif op == "masked":
        st["o"] = torch.empty((T, H * dh), dtype=dt, device="cuda")
        st["prefix"] = [min(case["prefix"], m) for m in n] if case["prefix"] else None
        st["prefix_dev"] = torch.tensor(st["prefix"] or [0] * B, device="cuda")
        st["documents"] = None
        if case["documents"]:
            docs = [np.full(m, -1, dtype=np.int32) for m in n]
            for d, m in zip(docs, n):
                edges = _documents(m, case["documents"])
                for k, (a, b) in enumerate(zip(edges, edges[1:])):
                    d[a:b] = k
            st["documents"] = torch.from_numpy(np.concatenate(docs)).to("cuda")
        st["slopes"] = _slopes(H) if case["slopes"] else None
    elif op == "tree":
        st["lengths"] = _ragged(case["cached"], B, case["ragged"])
        capacity = -(-max(st["lengths"]) // 64) * 64
        _cache(case, st, normal, g, B + 1, capacity)
        st["parents"], depth = [], []
        for q in range(B):  # every node hangs on one of the six before it
            d = []
            for i in range(case["nodes"]):
                p = int(rng.randint(max(0, i - 6), i)) if i else -1
                st["parents"].append(p)
                d.append(d[p] + 1 if i else 0)
            depth += d
        st["positions"] = torch.tensor([2 * capacity + d for d in depth], dtype=torch.int32, device="cuda")
        sees = np.zeros((B, case["nodes"], case["nodes"]), dtype=bool)
        for q in range(B):
            for i in range(case["nodes"]):
                p = st["parents"][q * case["nodes"] + i]
                if p >= 0:
                    sees[q, i] = sees[q, p]
                sees[q, i, i] = True
        st["sees"] = torch.from_numpy(sees).to("cuda")
        st["lengths_dev"] = torch.tensor(st["lengths"], device="cuda")
        st["o"] = torch.empty((T, H * dh), dtype=dt, device="cuda")
        st["slopes"] = _slopes(H) if case["slopes"] else None
    else:
        st["lengths"], st["keep"] = _ragged(case["cached"], B, case["ragged"]), _kept(case)
        capacity = -(-max(st["lengths"]) // 64) * 64
        _cache(case, st, normal, g, B + 1, capacity)
        st["recent_from"] = [2 * capacity - case["recent"]] * B
        st["meta0"] = st["meta"].clone()
        st["lengths_dev"], st["keep_dev"] = torch.tensor(st["lengths"], device="cuda"), torch.tensor(st["keep"], device="cuda")
        st["recent_dev"] = torch.tensor(st["recent_from"], device="cuda")
    return st


# ------------------------------------------------------------------------------------------------------- plain form
def _rotary_frequencies(case):
    rot, base, factor = case["rot"], 10000.0, 8.0
    if case["scaling"] == "base":
        base *= factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        w = ((8192.0 * f / TWO_PI - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = w * f + (1.0 - w) * f / factor
    return f


def _plain_rotary(st):
    case, (H, KV, dh) = st["case"], st["heads"]
    rot = case["rot"]
    angle = st["positions"].double()[:, None] * _rotary_frequencies(case)
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    x = st["qkv"].view(-1, H + 2 * KV, dh)
    y = x.to(torch.float32, copy=True)
    z = y[:, :H + KV, :rot]
    if case["layout"] == "half":
        a, b = z[..., :rot // 2], z[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = z[..., 0::2], z[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    y[:, :H + KV, :rot] = turned
    return {"qkv": y.to(st["dt"]).view_as(st["qkv"])}


def _plain_append(st):
    H, KV, dh = st["heads"]
    x = st["qkv"].view(-1, H + 2 * KV, dh)[st["rows_dev"]]
    slot = st["slots_dev"][st["query_dev"]]
    st["k"][slot, :, st["entry_dev"]] = x[:, H:H + KV]
    st["v"][slot, :, st["entry_dev"]] = x[:, H + KV:]
    st["positions_cache"][slot, st["entry_dev"]] = st["positions"][st["rows_dev"]]
    st["mass"][slot, st["entry_dev"]] = 0.0
    return {"k": st["k"], "v": st["v"], "positions": st["positions_cache"], "mass": st["mass"]}


def _capped(s, cap):
    return cap * torch.tanh(s / cap) if cap else s


def _weights(s, visible):
    """Softmax over the visible keys; rows without any are zero."""
    s = torch.where(visible, s, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    return p / torch.where(total == 0.0, 1.0, total)


def _plain_masked(st):
    case, (H, KV, dh) = st["case"], st["heads"]
    off = st["offsets_dev"]
    n = off[1:] - off[:-1]
    at = torch.arange(int(max(np.diff(st["offsets"]))), device="cuda")
    inside = at[None, :] < n[:, None]
    row = torch.where(inside, off[:-1, None] + at[None, :], 0)
    x = st["qkv"][row].float().view(len(n), -1, H + 2 * KV, dh).transpose(1, 2)
    q, k, v = x[:, :H], x[:, H:H + KV].repeat_interleave(H // KV, dim=1), x[:, H + KV:].repeat_interleave(H // KV, dim=1)
    s = _capped(torch.matmul(q, k.transpose(-1, -2).contiguous()) * dh ** -0.5, case["cap"])
    if st["slopes"] is not None:
        s = s - st["slopes"][:, None, None] * (at[:, None] - at[None, :]).abs()
    d = st["documents"][row] if st["documents"] is not None else torch.zeros_like(row)
    alive = inside & (d >= 0)
    same = d[:, :, None] == d[:, None, :]
    if case["causal"]:
        same = same & (at[None, :, None] >= at[None, None, :])
    visible = (same | (at[None, None, :] < st["prefix_dev"][:, None, None])) & alive[:, :, None] & alive[:, None, :]
    o = torch.matmul(_weights(s, visible[:, None]), v)
    return {"o": o.transpose(1, 2)[inside].reshape(-1, H * dh).to(st["dt"])}


def _plain_tree(st):
    case, (H, KV, dh) = st["case"], st["heads"]
    B, m, G = case["batch"], case["nodes"], H // KV
    longest = max(st["lengths"])
    x = st["qkv"].float().view(B, m, H + 2 * KV, dh).transpose(1, 2)
    k = torch.cat([st["k"][st["slots_dev"], :, :longest].float(), x[:, H:H + KV]], dim=2)
    v = torch.cat([st["v"][st["slots_dev"], :, :longest].float(), x[:, H + KV:]], dim=2)
    q = x[:, :H].reshape(B, KV, G * m, dh)
    s = _capped(torch.matmul(q, k.transpose(-1, -2).contiguous()) * dh ** -0.5, case["cap"]).view(B, H, m, longest + m)
    live = torch.arange(longest, device="cuda")[None, :] < st["lengths_dev"][:, None]
    if st["slopes"] is not None:
        pos = st["positions"].view(B, m)
        key = torch.cat([st["positions_cache"][st["slots_dev"], :longest], pos], dim=1)
        s = s - st["slopes"][:, None, None] * (pos[:, None, :, None] - key[:, None, None, :]).abs()
    visible = torch.cat([live[:, None, :].expand(B, m, longest), st["sees"]], dim=2)
    p = _weights(s, visible[:, None])
    o = torch.matmul(p.view(B, KV, G * m, longest + m), v)
    out = {"o": o.view(B, H, m, dh).transpose(1, 2).reshape(B * m, H * dh).to(st["dt"])}
    if case["mass"]:
        st["mass"][st["slots_dev"], :longest] += p[..., :longest].sum(dim=(1, 2))
        out["mass"] = st["mass"]
    return out


def _plain_evict(st):
    case = st["case"]
    longest = max(st["lengths"])
    slot = st["slots_dev"]
    at = torch.arange(longest, device="cuda")[None, :]
    live = at < st["lengths_dev"][:, None]
    first = live & ((at < case["lead"]) | (st["positions_cache"][slot, :longest] >= st["recent_dev"][:, None]))
    rank = torch.where(first, math.inf, torch.where(live, st["mass"][slot, :longest], -math.inf))
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    kept = torch.zeros_like(live)
    kept.scatter_(1, order, at < st["keep_dev"][:, None])
    free = ~kept & (at < st["keep_dev"][:, None])
    moves = kept & (at >= st["keep_dev"][:, None])
    q, to = free.nonzero(as_tuple=True)
    src = moves.nonzero(as_tuple=True)[1]
    s = slot[q]
    st["k"][s, :, to] = st["k"][s, :, src]
    st["v"][s, :, to] = st["v"][s, :, src]
    st["meta"][:, s, to] = st["meta"][:, s, src]
    return {"k": st["k"], "v": st["v"], "positions": st["positions_cache"], "mass": st["mass"]}


PLAIN = {"rotary": _plain_rotary, "append": _plain_append, "masked": _plain_masked, "tree": _plain_tree, "evict": _plain_evict}


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
    if op == "rotary":
        if "rope" not in st:
            st["rope"] = otas.Rotary(rot_dim=case["rot"], layout={"half": otas.OTAS_ROTARY_HALF, "interleaved": otas.OTAS_ROTARY_INTERLEAVED}[case["layout"]], base=10000.0,
                                     scaling={"plain": otas.OTAS_ROTARY_PLAIN, "linear": otas.OTAS_ROTARY_LINEAR, "base": otas.OTAS_ROTARY_BASE, "parts": otas.OTAS_ROTARY_BY_PARTS}[case["scaling"]],
                                     factor=8.0, original_length=8192.0, fast_turns=32.0, slow_turns=1.0)
        ctx.otas_rotary(st["qkv"], KV, st["positions"], st["rope"], st["out"])
        return {"qkv": st["out"]}
    if op == "masked":
        score = otas.Score(cap=case["cap"], slopes=st["slopes"])
        ctx.otas_attention_masked(st["qkv"], KV, st["offsets"], st["o"], causal=case["causal"], prefix=st["prefix"], documents=st["documents"], score=score)
        return {"o": st["o"]}
    cache = otas.KVCache(st["k"], st["v"], st["positions_cache"], st["mass"])
    if op == "append":
        ctx.otas_cache_append(cache, st["qkv"], st["row_offsets"], st["rows"], st["positions"], st["slots"], st["lengths"])
    elif op == "tree":
        if "workspace" not in st:
            st["workspace"] = torch.empty(ctx.otas_attention_tree_workspace_bytes(KV, st["offsets"], st["lengths"]), dtype=torch.uint8, device="cuda")
        score = otas.Score(cap=case["cap"], slopes=st["slopes"])
        ctx.otas_attention_tree(cache, st["qkv"], st["offsets"], st["parents"], st["positions"], st["slots"], st["lengths"], st["workspace"], st["o"], score=score, add_mass=case["mass"])
        return {"o": st["o"], "mass": st["mass"]} if case["mass"] else {"o": st["o"]}
    else:
        if "workspace" not in st:
            st["workspace"] = torch.empty(ctx.otas_cache_evict_workspace_bytes(st["lengths"], st["keep"]), dtype=torch.uint8, device="cuda")
        ctx.otas_cache_evict(cache, st["slots"], st["lengths"], st["keep"], st["workspace"], lead=case["lead"], recent_from=st["recent_from"])
    return {"k": st["k"], "v": st["v"], "positions": st["positions_cache"], "mass": st["mass"]}


def run(st):
    if st["case"]["op"] == "evict":
        st["meta"].copy_(st["meta0"])  # positions and weights as the steps before left them, so that every pass has its work to do
    if own:
        return _own(st)
    return PLAIN[st["case"]["op"]](st)


# ------------------------------------------------------------------------------------------------------------ 64 bits
def _exact_softmax(logits, mask):
    """Weights of one head's rows over the keys that `mask` lets them see, 64 bits."""
    shown = logits.masked_fill(~mask, -1e300)
    e = (shown - shown.max(dim=1, keepdim=True).values).exp() * mask
    return e / e.sum(dim=1, keepdim=True).clamp_min(1e-300)


def _exact_rotary(case, st, H, KV, dh):
    rot = case["rot"]
    i = np.arange(rot // 2, dtype=np.float64)
    base = 10000.0 * (8.0 ** (rot / (rot - 2.0)) if case["scaling"] == "base" else 1.0)
    f = np.exp(-np.log(base) * 2 * i / rot)
    if case["scaling"] == "linear":
        f /= 8.0
    if case["scaling"] == "parts":
        keep = np.clip((8192.0 / (2 * np.pi / f) - 1.0) / 31.0, 0, 1)
        f = f * keep + f / 8.0 * (1 - keep)
    t = st["positions"].cpu().numpy().astype(np.float64)[:, None] * f[None, :]
    turn = torch.from_numpy(np.exp(1j * t)).to("cuda")[:, None, :]
    x = st["qkv"].double().view(-1, H + 2 * KV, dh)
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(x[:, :H + KV, first].contiguous(), x[:, :H + KV, second].contiguous()) * turn
    x[:, :H + KV, first], x[:, :H + KV, second] = z.real, z.imag
    return {"qkv": x.view_as(st["qkv"])}


def _exact_append(case, st, H, KV, dh):
    k, v, pos, mass = st["k"].double(), st["v"].double(), st["positions_cache"].clone(), st["mass"].double()
    rows = st["rows"] if st["rows"] is not None else list(range(st["offsets"][-1]))
    for q, (slot, length) in enumerate(zip(st["slots"], st["lengths"])):
        mine = rows[st["row_offsets"][q]:st["row_offsets"][q + 1]]
        to = slice(length, length + len(mine))
        x = st["qkv"][mine].double().view(len(mine), H + 2 * KV, dh)
        k[slot, :, to], v[slot, :, to] = x[:, H:H + KV].transpose(0, 1), x[:, H + KV:].transpose(0, 1)
        pos[slot, to], mass[slot, to] = st["positions"][mine], 0
    return {"k": k, "v": v, "positions": None, "mass": mass}


def _exact_masked(case, st, H, KV, dh):
    out = torch.zeros((st["offsets"][-1], H, dh), dtype=torch.float64, device="cuda")
    for q, (a, b) in enumerate(zip(st["offsets"], st["offsets"][1:])):
        n = b - a
        x = st["qkv"][a:b].double().view(n, H + 2 * KV, dh)
        doc = st["documents"][a:b] if st["documents"] is not None else torch.zeros(n, dtype=torch.int32, device="cuda")
        ids = torch.arange(n, device="cuda")
        mask = doc.view(-1, 1) == doc.view(1, -1)
        if case["causal"]:
            mask = mask.tril()
        if st["prefix"]:
            mask[:, :st["prefix"][q]] = True
        mask &= (doc >= 0).view(-1, 1) & (doc >= 0).view(1, -1)
        for h in range(H):
            s = (x[:, h] / math.sqrt(dh)) @ x[:, H + h // (H // KV)].T.contiguous()
            if case["cap"]:
                s = case["cap"] * (s / case["cap"]).tanh()
            if st["slopes"] is not None:
                s -= float(st["slopes"][h]) * (ids.view(-1, 1) - ids.view(1, -1)).abs()
            out[a:b, h] = _exact_softmax(s, mask) @ x[:, H + KV + h // (H // KV)]
    return {"o": out.view(-1, H * dh)}


def _exact_tree(case, st, H, KV, dh):
    m = case["nodes"]
    out = torch.zeros((m * case["batch"], H, dh), dtype=torch.float64, device="cuda")
    mass = st["mass"].double()
    for q in range(case["batch"]):
        n, slot, rows = st["lengths"][q], st["slots"][q], slice(q * m, (q + 1) * m)
        x = st["qkv"][rows].double().view(m, H + 2 * KV, dh)
        mask = torch.ones((m, n + m), dtype=torch.bool)
        mask[:, n:] = False
        for i in range(m):  # a node, its parent, its parent's parent ...
            at = i
            while at >= 0:
                mask[i, n + at] = True
                at = st["parents"][q * m + at]
        mask = mask.to("cuda")
        where = torch.cat([st["positions_cache"][slot, :n], st["positions"][rows]]).double()
        for h in range(H):
            keys = torch.cat([st["k"][slot, h // (H // KV), :n].double(), x[:, H + h // (H // KV)]])
            vals = torch.cat([st["v"][slot, h // (H // KV), :n].double(), x[:, H + KV + h // (H // KV)]])
            s = (x[:, h] / math.sqrt(dh)) @ keys.T.contiguous()
            if case["cap"]:
                s = case["cap"] * (s / case["cap"]).tanh()
            if st["slopes"] is not None:
                s -= float(st["slopes"][h]) * (where[n:].view(-1, 1) - where.view(1, -1)).abs()
            p = _exact_softmax(s, mask)
            out[rows, h] = p @ vals
            mass[slot, :n] += p[:, :n].sum(dim=0)
    return {"o": out.view(-1, H * dh), "mass": mass} if case["mass"] else {"o": out.view(-1, H * dh)}


def _exact_evict(case, st, H, KV, dh):
    k, v, mass = st["k"].double(), st["v"].double(), st["mass"].double()
    pos, weight = st["positions_cache"].cpu().numpy(), st["mass"].cpu().numpy()
    for q, (slot, n, keep) in enumerate(zip(st["slots"], st["lengths"], st["keep"])):
        first = (np.arange(n) < case["lead"]) | (pos[slot, :n] >= st["recent_from"][q])
        best = np.lexsort((np.arange(n), -weight[slot, :n].astype(np.float64), ~first))[:keep]
        to = np.setdiff1d(np.arange(min(n, keep)), best)
        src = np.sort(best[best >= keep])
        to, src = torch.from_numpy(to).to("cuda"), torch.from_numpy(src).to("cuda")
        k[slot][:, to], v[slot][:, to], mass[slot][to] = k[slot][:, src], v[slot][:, src], mass[slot][src]
    return {"k": k, "v": v, "positions": None, "mass": mass}


def exact(case, seed):
    if case["op"] == "tree" and case["batch"] * case["cached"] > 400000:
        return None
    st = prepare(case, seed)
    H, KV, dh = st["heads"]
    return {"rotary": _exact_rotary, "append": _exact_append, "masked": _exact_masked, "tree": _exact_tree, "evict": _exact_evict}[case["op"]](case, st, H, KV, dh)
