"""The three operators of one decode step around the K/V cache, as measured work.

    append   queries and keys normalised per head and turned to their cache positions, and the
             new K/V rows written behind the live slots of a layer's planes
    attend   one new token per stream over the slots of a layer's planes
    head     Token Entropy of the round's tokens straight from the hidden states and the LM
             head's weight, the vocabulary taken in pieces, no logits kept

``run`` computes them in elementary torch operations (``own`` false) or through the package's
calls (``own`` true); ``exact`` computes the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6


# --------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------

def _append(name, streams, max_new, least, heads, kv_heads, dim, capacity, first, norm, pairing, base, dtype):
    """``least`` .. ``max_new`` new tokens per stream, behind up to ``first`` live slots."""
    return {"name": name, "op": "append", "streams": streams, "max_new": max_new, "least": least,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "capacity": capacity, "first": first,
            "norm": norm, "pairing": pairing, "base": base, "dtype": dtype}


def _attend(name, streams, heads, kv_heads, dim, capacity, shortest, longest, dtype):
    """Streams of ``shortest`` .. ``longest`` slots (0: a stream without a token this step)."""
    return {"name": name, "op": "attend", "streams": streams, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "capacity": capacity, "shortest": shortest, "longest": longest, "dtype": dtype}


def _head(name, streams, max_new, least, width, vocab, dtype):
    """``least`` .. ``max_new`` tokens per stream, hidden states of ``width`` elements."""
    return {"name": name, "op": "head", "streams": streams, "max_new": max_new, "least": least,
            "width": width, "vocab": vocab, "dtype": dtype}


def listed():
    return [
        # one token of one dialogue, far into a long cache: the smallest call, bound by latency
        _append("append_1_token", 1, 1, 1, 32, 8, 128, 16384, 12001, False, "half", 500000.0, "bf16"),
        # a decode step of 64 dialogues, some of them idle, all heads their own K/V
        _append("append_64_streams", 64, 1, 0, 32, 32, 128, 2048, 1500, False, "half", 10000.0, "bf16"),
        # short ragged turns of a few dialogues, narrow heads, interleaved pairs, normalised
        _append("append_short_turns", 5, 120, 0, 12, 4, 80, 640, 512, True, "interleaved", 10000.0, "f16"),
        # a user's turn of 4096 tokens, with per-head norms
        _append("append_4096_tokens", 1, 4096, 4096, 32, 8, 128, 16384, 8192, True, "half", 500000.0, "bf16"),
        # one token over a small cache, narrow heads: latency
        _attend("attend_small_cache", 1, 8, 8, 64, 1024, 257, 257, "f16"),
        # one token over a long cache with grouped heads, an odd length
        _attend("attend_long_cache", 1, 32, 8, 128, 16384, 12287, 12287, "bf16"),
        # seven dialogues of very different lengths, one of them idle, groups of six heads
        _attend("attend_ragged", 7, 48, 8, 96, 8192, 0, 8191, "bf16"),
        # a decode step of 64 dialogues, all heads their own K/V
        _attend("attend_64_streams", 64, 32, 32, 128, 2048, 900, 1280, "bf16"),
        # the score of one generated token
        _head("head_1_token", 1, 1, 1, 4096, 32000, "bf16"),
        # a decode step of 64 dialogues over a large vocabulary
        _head("head_64_streams", 64, 1, 0, 4096, 128256, "bf16"),
        # short ragged turns, odd vocabulary, a width that is no multiple of a tile
        _head("head_short_turns", 5, 120, 7, 1000, 50257, "f16"),
        # a user's turn of 4096 tokens over a large vocabulary
        _head("head_4096_tokens", 1, 4096, 4096, 4096, 128256, "bf16"),
    ]


def _spread(rng, low, high):
    """A whole number in [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "head"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "append":
        streams = _spread(rng, 1, 64)
        max_new = _spread(rng, 1, max(1, 4096 // streams))
        kv_heads = rng.choice([1, 2, 4, 5, 8, 16])
        heads = kv_heads * rng.randint(1, max(1, 32 // kv_heads))
        first = rng.randint(0, 2048)
        return _append("append", streams, max_new, rng.choice([0, max_new]), heads, kv_heads,
                       16 * rng.randint(1, 8 if heads > 16 else 16), first + max_new + rng.randint(0, 100), first,
                       rng.random() < 0.5, rng.choice(["half", "interleaved"]),
                       rng.choice([10000.0, 500000.0, 1000000.0]), dtype)
    if op == "attend":
        streams = _spread(rng, 1, 64)
        kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8] + ([17, 32] if kv_heads < 4 else []))
        dim = 8 * rng.choice([2, 5, 8, 8, 10, 12, 16, 16, 24, 32])
        # at most the slots x heads x elements of the largest listed case
        most = min(16384, (64 * 32 * 1280 * 128) // (streams * kv_heads * dim))
        longest = _spread(rng, 1, most)
        shortest = rng.choice([0, 1, longest, rng.randint(1, longest)])
        return _attend("attend", streams, heads, kv_heads, dim, longest + rng.randint(0, 64), min(shortest, longest),
                       longest, dtype)
    streams = _spread(rng, 1, 64)
    max_new = _spread(rng, 1, max(1, 2048 // streams))
    vocab = _spread(rng, 500, 130000)
    return _head("head", streams, max_new, rng.choice([0, max_new]), 8 * _spread(rng, 8, 512), vocab, dtype)


# --------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------

def _lengths(low, high, n):
    """n whole numbers spread evenly from low to high."""
    return [high] if n == 1 else [low + (high - low) * i // (n - 1) for i in range(n)]


def _ints(values, gen, device):
    t = torch.tensor(values, dtype=torch.int32, device=device)
    return t[torch.randperm(len(values), generator=gen, device=device)]


def _normal(shape, gen, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device=gen.device)
    out.normal_(0.0, scale, generator=gen)
    return out


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = _DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "append":
        S, M, H, KH, D = c["streams"], c["max_new"], c["heads"], c["kv_heads"], c["dim"]
        # one fused projection's output: queries, keys and values side by side in every row
        qkv = _normal((S * M, (H + 2 * KH), D), gen, dt)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
        s["q_weight"] = s["k_weight"] = None
        if c["norm"]:
            s["q_weight"] = 1.0 + _normal((D,), gen, dt, 0.2)
            s["k_weight"] = 1.0 + _normal((D,), gen, dt, 0.2)
        s["first_slot"] = _ints(_lengths(c["first"] // 2 if S > 1 else c["first"], c["first"], S), gen, "cuda")
        s["n_new"] = _ints(_lengths(c["least"], M, S), gen, "cuda")
        s["q_out"] = torch.zeros(S * M, H, D, dtype=dt, device="cuda")
        # two layers of planes [stream][layer][kv head][slot][element]; the call fills layer 1
        s["k"] = _normal((S, 2, KH, c["capacity"], D), gen, dt)
        s["v"] = _normal((S, 2, KH, c["capacity"], D), gen, dt)
        s["layer"] = 1
    elif c["op"] == "attend":
        S, H, KH, D = c["streams"], c["heads"], c["kv_heads"], c["dim"]
        s["q"] = _normal((S, H, D), gen, dt)
        s["k"] = _normal((S, 1, KH, c["capacity"], D), gen, dt)
        s["v"] = _normal((S, 1, KH, c["capacity"], D), gen, dt)
        s["kv_len"] = _ints(_lengths(c["shortest"], c["longest"], S), gen, "cuda")
        s["out"] = torch.zeros(S, H, D, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(S, H, dtype=torch.float32, device="cuda")
        s["layer"] = 0
    else:
        S, M, W, V = c["streams"], c["max_new"], c["width"], c["vocab"]
        rows = S * M
        s["weight"] = _normal((V, W), gen, dt, 2.0 / math.sqrt(W))
        s["hidden"] = _normal((rows, W), gen, dt)
        s["token_ids"] = torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        # half of the tokens are predictable: their hidden state leans towards their weight row
        lean = (torch.rand(rows, 1, generator=gen, device="cuda") < 0.5).to(dt) * 2.0
        s["hidden"] += lean * s["weight"][s["token_ids"].long()]
        # no prediction for a stream's first token now and then
        s["token_ids"][torch.rand(rows, generator=gen, device="cuda") < 0.01] = -1
        s["n_new"] = _ints(_lengths(c["least"], M, S), gen, "cuda")
        s["entropy"] = torch.zeros(rows, dtype=torch.float32, device="cuda")
    return s


# --------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------

def _config(c):
    """The package's configuration of a case."""
    from paper_2405_12528_b200 import binding as sir
    cap = c.get("capacity", max(c.get("max_new", 1), 1))
    return sir.make_config(n_streams=c["streams"], n_layers=2 if c["op"] == "append" else 1,
                           n_kv_heads=c.get("kv_heads", 1), head_dim=c.get("dim", 8), capacity=cap,
                           budget=cap, n_sink=0, n_recent=0, max_new=c.get("max_new", 1),
                           vocab=c.get("vocab", 1), logits_dtype="f32", kv_dtype=c["dtype"])


def _calls(s):
    """The step's calls, checked and marshalled once as a decode loop keeps them."""
    from paper_2405_12528_b200 import binding as sir
    c = s["case"]
    cfg = _config(c)
    if c["op"] == "append":
        pairing = sir.ROPE_HALF if c["pairing"] == "half" else sir.ROPE_INTERLEAVED
        ws = sir.new_workspace(cfg)
        return [sir.prepared(sir.sirllm_append_kv, cfg, s["layer"], s["q"], s["k_new"], s["v_new"], s["q_weight"],
                             s["k_weight"], _EPS, c["base"], pairing, s["first_slot"], s["n_new"], s["q_out"],
                             s["k"], s["v"], ws)]
    if c["op"] == "attend":
        ws = sir.new_attend_workspace(cfg)
        return [sir.prepared(sir.sirllm_attend, cfg, s["layer"], s["q"], s["k"], s["v"], s["kv_len"],
                             1.0 / math.sqrt(c["dim"]), s["out"], s["lse"], ws)]
    ws = sir.new_workspace(cfg)
    rows = c["streams"] * c["max_new"]
    pairs = torch.empty(rows, sir.sirllm_head_tiles(cfg, c["vocab"]), 2, dtype=torch.float32, device="cuda")
    target = torch.empty(rows, dtype=torch.float32, device="cuda")
    return [sir.prepared(sir.sirllm_head_pairs, cfg, s["hidden"], s["weight"], 0, s["token_ids"], s["n_new"],
                         pairs, target, ws),
            sir.prepared(sir.sirllm_score_pairs, cfg, pairs, target, s["token_ids"], s["n_new"], s["entropy"], ws)]


def _positions(s):
    """Per row of a case: its stream, its place among the stream's new rows, whether it is used."""
    c = s["case"]
    row = torch.arange(c["streams"] * c["max_new"], device="cuda")
    stream, t = row // c["max_new"], row % c["max_new"]
    return stream, t, t < s["n_new"].long()[stream]


def _norm_and_turn(x, weight, cos, sin, pairing):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * weight.float()
    half = y.shape[-1] // 2
    a, b = (y[..., :half], y[..., half:]) if pairing == "half" else (y[..., 0::2], y[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat([u, v], -1) if pairing == "half" else torch.stack([u, v], -1).flatten(-2)


def _plain_append(s):
    c = s["case"]
    dt, D = _DTYPES[c["dtype"]], c["dim"]
    stream, t, used = _positions(s)
    slot = s["first_slot"].long()[stream] + t
    # positions reach tens of thousands of turns: the angles are taken in 64 bits
    theta = torch.pow(torch.tensor(c["base"], dtype=torch.float64, device="cuda"),
                      -torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    angle = slot.double()[:, None] * theta
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    q = _norm_and_turn(s["q"], s["q_weight"], cos, sin, c["pairing"]).to(dt)
    k = _norm_and_turn(s["k_new"], s["k_weight"], cos, sin, c["pairing"]).to(dt)
    use = used[:, None, None]
    s["q_out"].copy_(torch.where(use, q, s["q_out"]))
    kc, vc = s["k"][:, s["layer"]], s["v"][:, s["layer"]]
    kc[stream, :, slot] = torch.where(use, k, kc[stream, :, slot])   # a row that is not used writes back what is there
    vc[stream, :, slot] = torch.where(use, s["v_new"], vc[stream, :, slot])
    return s["q_out"], s["k"], s["v"]


def _plain_attend(s):
    c = s["case"]
    S, H, KH, D = c["streams"], c["heads"], c["kv_heads"], c["dim"]
    k, v = s["k"][:, s["layer"]].float(), s["v"][:, s["layer"]].float()
    q = s["q"].float().view(S, KH, H // KH, D)
    z = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    seen = (torch.arange(c["capacity"], device="cuda") < s["kv_len"].long()[:, None])[:, None, None]
    z = torch.where(seen, z, float("-inf"))
    some = (s["kv_len"] > 0)[:, None, None, None]
    m = torch.where(some, z.amax(-1, keepdim=True), 0.0)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    out = torch.where(some, torch.matmul(p, v) / torch.where(some, total, 1.0), 0.0)
    s["out"].copy_(out.view(S, H, D).to(_DTYPES[c["dtype"]]))
    s["lse"].copy_((m + torch.log(total)).view(S, H))
    return s["out"], s["lse"]


def _plain_head(s):
    stream, t, used = _positions(s)
    z = torch.matmul(s["hidden"].float(), s["weight"].float().t())
    m = z.amax(-1)
    lse = m + torch.log(torch.exp(z - m[:, None]).sum(-1))
    ids = s["token_ids"].long()
    e = lse - z.gather(1, ids.clamp(min=0)[:, None])[:, 0]
    e = torch.where(ids < 0, 0.0, e)
    s["entropy"].copy_(torch.where(used, e, s["entropy"]))
    return s["entropy"]


def run(state):
    op = state["case"]["op"]
    if own:
        if "calls" not in state:
            state["calls"] = _calls(state)
        for call in state["calls"]:
            call()
        if op == "append":
            return state["q_out"], state["k"], state["v"]
        return (state["out"], state["lse"]) if op == "attend" else state["entropy"]
    return {"append": _plain_append, "attend": _plain_attend, "head": _plain_head}[op](state)


# --------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------

def work(case):
    c = case
    S = c["streams"]
    if c["op"] == "append":
        n = sum(_lengths(c["least"], c["max_new"], S))
        elems = n * (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": 4 * elems + 8 * S, "flops": 8 * elems}
    if c["op"] == "attend":
        n = sum(_lengths(c["shortest"], c["longest"], S))
        return {"bytes": 4 * n * c["kv_heads"] * c["dim"] + S * c["heads"] * (4 * c["dim"] + 4) + 4 * S,
                "flops": 4 * n * c["heads"] * c["dim"]}
    n = sum(_lengths(c["least"], c["max_new"], S))
    return {"bytes": 2 * c["vocab"] * c["width"] + n * (2 * c["width"] + 8) + 4 * S,
            "flops": 2 * n * c["vocab"] * c["width"]}


# --------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------

def _exact_rotated(vec, weight, pos, base, pairing):
    """One token's heads [heads, D] (fp64): root-mean-square norm, then pair i as a complex
    number times exp(1j * pos * base**(-2i/D))."""
    if weight is not None:
        vec = vec / (vec.square().sum(-1, keepdim=True) / vec.shape[-1] + _EPS).sqrt() * weight.double()
    D = vec.shape[-1]
    i = torch.arange(D // 2, dtype=torch.float64, device=vec.device)
    turn = torch.polar(torch.ones_like(i), pos * base ** (-2.0 * i / D))
    first, second = (i.long(), i.long() + D // 2) if pairing == "half" else (2 * i.long(), 2 * i.long() + 1)
    z = torch.complex(vec[..., first], vec[..., second]) * turn
    out = torch.empty_like(vec)
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "append":
        M = c["max_new"]
        q_out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
        n_new, first = s["n_new"].tolist(), s["first_slot"].tolist()
        for st in range(c["streams"]):
            n, f = n_new[st], first[st]
            r = slice(st * M, st * M + n)
            pos = torch.arange(f, f + n, dtype=torch.float64, device="cuda")[:, None, None]
            q_out[r] = _exact_rotated(s["q"][r].double(), s["q_weight"], pos, c["base"], c["pairing"])
            turned = _exact_rotated(s["k_new"][r].double(), s["k_weight"], pos, c["base"], c["pairing"])
            k[st, s["layer"], :, f:f + n] = turned.transpose(0, 1)
            v[st, s["layer"], :, f:f + n] = s["v_new"][r].double().transpose(0, 1)
        return q_out, k, v
    if c["op"] == "attend":
        H, G = c["heads"], c["heads"] // c["kv_heads"]
        out = torch.zeros(c["streams"], H, c["dim"], dtype=torch.float64, device="cuda")
        lse = torch.full((c["streams"], H), float("-inf"), dtype=torch.float64, device="cuda")
        for st, n in enumerate(s["kv_len"].tolist()):
            if n == 0:
                continue
            for g in range(c["kv_heads"]):
                rows = slice(g * G, g * G + G)
                z = s["q"][st, rows].double() @ s["k"][st, s["layer"], g, :n].double().T / math.sqrt(c["dim"])
                lse[st, rows] = torch.logsumexp(z, -1)
                out[st, rows] = torch.softmax(z, -1) @ s["v"][st, s["layer"], g, :n].double()
        return out, lse
    e = s["entropy"].double()
    w = s["weight"].double()
    for st, n in enumerate(s["n_new"].tolist()):
        for a in range(0, n, 512):
            r = slice(st * c["max_new"] + a, st * c["max_new"] + min(n, a + 512))
            ids = s["token_ids"][r].long()
            logp = torch.log_softmax(s["hidden"][r].double() @ w.T, -1)
            e[r] = torch.where(ids < 0, 0.0, -logp[torch.arange(ids.numel(), device="cuda"), ids.clamp(min=0)])
    return e
