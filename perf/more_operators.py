"""Operators for streams that have a past in common, as measured work: the beams of one prompt, or
dialogues behind one system prompt.

    select   the best continuations of every group of beams, from the beams' logits and running totals
    reorder  the surviving beams' state (K/V rows of every layer, entropy scores, tags, lengths) moved
             in place to the streams that continue them
    attend   one new token per stream over slots of which the first ones are held once per group

``run`` computes them in elementary torch operations (``own`` false) or through the package's
calls (``own`` true); ``exact`` computes the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_END = 2   # the token that ends a text


# --------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------

def _select(name, groups, group, n_out, vocab, pad, ended, places, dtype):
    """``groups`` prompts of ``group`` beams each; rows ``vocab + pad`` elements apart; a share
    ``ended`` of the beams has ended, as many hold no beam."""
    return {"name": name, "op": "select", "groups": groups, "group": group, "n_out": n_out, "vocab": vocab,
            "pad": pad, "ended": ended, "places": places, "dtype": dtype}


def _reorder(name, groups, group, layers, kv_heads, dim, shared, longest, spread, survivors, tags, dtype):
    """Streams of ``longest - spread`` .. ``longest`` slots, the first ``shared`` the same within a
    group; ``survivors`` of each group's streams go on, the others continue one of them."""
    return {"name": name, "op": "reorder", "groups": groups, "group": group, "layers": layers,
            "kv_heads": kv_heads, "dim": dim, "shared": shared, "longest": longest, "spread": spread,
            "survivors": survivors, "tags": tags, "dtype": dtype}


def _attend(name, groups, group, heads, kv_heads, dim, shortest, shared, least, suffix, dtype):
    """Groups that share ``shortest`` .. ``shared`` slots; ``least`` .. ``suffix`` slots of a stream's own."""
    return {"name": name, "op": "attend", "groups": groups, "group": group, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "shortest": shortest, "shared": shared, "least": least, "suffix": suffix, "dtype": dtype}


def listed():
    return [
        # one dialogue, four beams: the smallest call, bound by latency
        _select("select_4_beams", 1, 4, 4, 32000, 0, 0.0, True, "bf16"),
        # five prompts of three beams, odd vocabulary, fp32, some beams ended; twice as many candidates as beams
        _select("select_odd", 5, 3, 6, 50257, 0, 0.2, False, "f32"),
        # a serving batch: 16 prompts of 8 beams over a large vocabulary, a pool of 16 candidates
        _select("select_16_prompts", 16, 8, 16, 128256, 0, 0.1, False, "bf16"),
        # the largest batch: 64 prompts of 8 beams
        _select("select_64_prompts", 64, 8, 8, 128256, 0, 0.1, True, "bf16"),
        # a few tokens behind a short prompt, a small model: latency
        _reorder("reorder_small", 1, 4, 4, 8, 64, 200, 230, 0, 2, True, "f16"),
        # five prompts of three beams, narrow odd heads, lengths that differ
        _reorder("reorder_odd", 5, 3, 6, 3, 80, 77, 403, 50, 2, False, "bf16"),
        # a prompt's cache handed to all of its eight beams: one stream goes on as all
        _reorder("reorder_fork", 1, 8, 32, 8, 128, 0, 1023, 0, 1, True, "bf16"),
        # four prompts of four beams, several hundred tokens into the answer
        _reorder("reorder_4_prompts", 4, 4, 32, 8, 128, 256, 903, 100, 2, True, "bf16"),
        # four beams of a short prompt, narrow heads: latency
        _attend("attend_4_beams", 1, 4, 8, 8, 64, 257, 257, 1, 20, "f16"),
        # eight beams of a long prompt with grouped heads, odd lengths
        _attend("attend_8_beams", 1, 8, 32, 8, 128, 12001, 12001, 3, 202, "bf16"),
        # sixteen prompts of four beams, lengths that differ, all heads their own K/V
        _attend("attend_16_prompts", 16, 4, 32, 32, 128, 200, 1100, 1, 150, "bf16"),
        # 64 dialogues behind one long system prompt
        _attend("attend_64_dialogues", 1, 64, 32, 8, 128, 15873, 15873, 1, 500, "bf16"),
    ]


def _spread(rng, low, high):
    """A whole number in [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["select", "reorder", "attend"])
    if op == "select":
        group = rng.choice([1, 2, 3, 4, 5, 8, 8, 12, 16, 31, 64])
        groups = _spread(rng, 1, max(1, 512 // group))
        places = rng.random() < 0.5
        n_out = group if places else rng.randint(1, min(64, 2 * group))
        dtype = rng.choice(["bf16", "f32"])
        vocab = _spread(rng, 300, 128256 if dtype == "bf16" else 64128)
        return _select("select", groups, group, n_out, vocab, rng.choice([0, 0, 1, 8, 64]),
                       rng.choice([0.0, 0.1, 0.3]), places, dtype)
    dtype = rng.choice(["bf16", "f16"])
    if op == "reorder":
        group = rng.choice([2, 3, 4, 5, 8, 16])
        groups = _spread(rng, 1, max(1, 32 // group))
        layers, kv_heads = _spread(rng, 1, 32), rng.choice([1, 2, 3, 5, 8])
        dim = 8 * rng.choice([1, 5, 8, 10, 12, 16, 16, 32])
        # at most the slots x heads x elements of the largest listed case
        most = max(8, min(4096, (16 * 32 * 8 * 1024 * 128) // (groups * group * layers * kv_heads * dim)))
        longest = _spread(rng, 2, most)
        shared = rng.choice([0, rng.randint(0, longest)])
        return _reorder("reorder", groups, group, layers, kv_heads, dim, shared, longest,
                        rng.randint(0, longest - shared), rng.randint(1, group), rng.random() < 0.5, dtype)
    group = rng.choice([2, 3, 4, 5, 8, 13, 16, 32, 64])
    groups = _spread(rng, 1, max(1, 64 // group))
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16, 32])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 5, 7, 8] + ([17, 32] if kv_heads < 3 else []))
    dim = 8 * rng.choice([2, 5, 8, 8, 10, 12, 16, 16, 16, 24, 32])
    # at most the slots x heads x elements held, and the products, of the largest listed case
    most = min(16384, (64 * 8 * 16384 * 128) // (groups * group * kv_heads * dim),
               (64 * 32 * 16384 * 128) // (groups * group * heads * dim))
    shared = _spread(rng, 16, max(17, most * 7 // 8))
    suffix = _spread(rng, 1, max(1, min(1500, most - shared)))
    return _attend("attend", groups, group, heads, kv_heads, dim, rng.choice([shared, rng.randint(0, shared)]),
                   shared, rng.choice([0, 1, suffix]), suffix, dtype)


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


def _rand(n, gen):
    return torch.rand(n, generator=gen, device=gen.device)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = _DTYPES[c["dtype"]]
    S = c["groups"] * c["group"]
    s = {"case": c}
    if c["op"] == "select":
        V = c["vocab"]
        wide = _normal((S, V + c["pad"]), gen, dt, 2.0)
        s["logits"] = wide[:, :V]
        # a few likely tokens per row stand out
        likely = torch.randint(0, V, (S, 12), generator=gen, device="cuda")
        s["logits"].scatter_add_(1, likely, (4.0 + 5.0 * torch.rand(S, 12, generator=gen, device="cuda")).to(dt))
        s["totals"] = -5.0 - 6.0 * _rand(S, gen)
        fate = _rand(S, gen)
        s["ended"] = (fate < c["ended"]).to(torch.int32)
        s["totals"][(fate >= c["ended"]) & (fate < 2 * c["ended"])] = float("-inf")
        n = c["groups"] * c["n_out"]
        s["totals_out"] = torch.zeros(n, dtype=torch.float32, device="cuda")
        s["entropy"] = torch.zeros(n, dtype=torch.float32, device="cuda")
        for name in ("source", "token_ids", "ended_out"):
            s[name] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif c["op"] == "reorder":
        cap = c["longest"] + 8
        s["k"] = _normal((S, c["layers"] * c["kv_heads"], cap, c["dim"]), gen, dt)
        s["v"] = _normal((S, c["layers"] * c["kv_heads"], cap, c["dim"]), gen, dt)
        s["scores"] = 12.0 * _rand(S * cap, gen).view(S, cap)
        s["serial"] = torch.randint(0, 1 << 40, (S, cap), generator=gen, device="cuda") if c["tags"] else None
        s["live_len"] = _ints(_lengths(c["longest"] - c["spread"], c["longest"], S), gen, "cuda")
        s["shared_len"] = torch.full((c["groups"],), c["shared"], dtype=torch.int32, device="cuda") \
            if c["shared"] else None
        # a survivor goes on in its own place; every other stream continues one of its group's survivors
        source = torch.arange(S, dtype=torch.int32, device="cuda").view(c["groups"], c["group"])
        for g in range(c["groups"]):
            order = torch.randperm(c["group"], generator=gen, device="cuda")
            alive, gone = order[:c["survivors"]], order[c["survivors"]:]
            pick = torch.randint(0, c["survivors"], (gone.numel(),), generator=gen, device="cuda")
            source[g, gone] = source[g, alive[pick]].clone()
        s["source"] = source.view(S)
    else:
        H, KH, D = c["heads"], c["kv_heads"], c["dim"]
        cap = c["shared"] + c["suffix"]
        s["q"] = _normal((S, H, D), gen, dt)
        # [stream][layer][kv head][slot][element]; a group's shared slots are those of its first stream
        s["k"] = _normal((S, 1, KH, cap, D), gen, dt)
        s["v"] = _normal((S, 1, KH, cap, D), gen, dt)
        s["shared_len"] = _ints(_lengths(c["shortest"], c["shared"], c["groups"]), gen, "cuda")
        s["kv_len"] = s["shared_len"].repeat_interleave(c["group"]) + \
            _ints(_lengths(c["least"], c["suffix"], S), gen, "cuda")
        s["out"] = torch.zeros(S, H, D, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(S, H, dtype=torch.float32, device="cuda")
    return s


# --------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------

def _config(c):
    """The package's configuration of a case."""
    from paper_2405_12528_b200 import binding as sir
    cap = c["longest"] + 8 if c["op"] == "reorder" else c["shared"] + c["suffix"] if c["op"] == "attend" else 1
    vocab = c.get("vocab", 1)
    return sir.make_config(n_streams=c["groups"] * c["group"], n_layers=c.get("layers", 1),
                           n_kv_heads=c.get("kv_heads", 1), head_dim=c.get("dim", 8), capacity=cap, budget=cap,
                           n_sink=0, n_recent=0, max_new=1, vocab=vocab,
                           logits_dtype=c["dtype"] if c["op"] == "select" else "f32",
                           kv_dtype="bf16" if c["op"] == "select" else c["dtype"],
                           logits_row_stride=vocab + c.get("pad", 0))


def _call(s):
    """The step's call, checked and marshalled once as a decode loop keeps it."""
    from paper_2405_12528_b200 import binding as sir
    c = s["case"]
    cfg = _config(c)
    if c["op"] == "select":
        return sir.prepared(sir.sirllm_beam_select, cfg, s["logits"], c["group"], c["n_out"], s["totals"], s["ended"],
                            _END, c["places"], s["totals_out"], s["source"], s["token_ids"], s["entropy"],
                            s["ended_out"], sir.new_beam_workspace(cfg))
    if c["op"] == "reorder":
        return sir.prepared(sir.sirllm_reorder_streams, cfg, c["group"], s["source"], s["shared_len"], s["scores"],
                            s["serial"], s["live_len"], s["k"], s["v"], sir.new_workspace(cfg))
    return sir.prepared(sir.sirllm_attend_shared, cfg, 0, c["group"], s["shared_len"], s["q"], s["k"], s["v"],
                        s["kv_len"], 1.0 / math.sqrt(c["dim"]), s["out"], s["lse"],
                        sir.new_attend_shared_workspace(cfg, c["group"], c["heads"]))


def _plain_select(s):
    c = s["case"]
    B, G, N, V = c["groups"], c["group"], c["n_out"], c["vocab"]
    dev = s["logits"].device
    # 64 bits: the order of candidates hangs on small differences between beams
    z = s["logits"].double()
    m = z.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))
    logp = z - lse
    totals = s["totals"].double()[:, None]
    stopped = (s["ended"] != 0)[:, None]
    token = torch.arange(V, device=dev)
    # an ended beam goes on as one candidate, which stands at token 0 here
    score = torch.where(stopped, torch.where(token == 0, totals, float("-inf")), totals + logp).view(B, G * V)
    surprise = torch.where(stopped, 0.0, -logp).view(B, G * V)
    flat = torch.arange(G * V, device=dev)
    base = torch.arange(B, device=dev)[:, None] * G
    best, src, tok, ent = [], [], [], []
    for _ in range(N):
        top = score.amax(-1, keepdim=True)
        at = torch.where(score == top, flat, G * V).amin(-1, keepdim=True)
        real = top > float("-inf")
        best.append(top)
        src.append(torch.where(real, base + at // V, -1))
        tok.append(torch.where(real, at % V, -1))
        ent.append(torch.where(real, surprise.gather(1, at), 0.0))
        score.scatter_(1, at, float("-inf"))
    best, src, tok, ent = (torch.cat(x, 1) for x in (best, src, tok, ent))
    was_ended = (src >= 0) & (s["ended"].long()[src.clamp(min=0)] != 0)
    tok = torch.where(was_ended, _END, tok)
    if c["places"]:
        # a stream's best continuation stays in the stream's place, the others fill the free ones in order
        j = torch.arange(N, device=dev)
        same = (src[:, :, None] == src[:, None, :]) & (j[None, :, None] > j[None, None, :])
        first = ~same.any(-1) & (src >= 0)
        own_place = torch.where(first, src - base, N)
        taken = (own_place[:, :, None] == j).any(1)
        free = torch.argsort(torch.where(taken, N + j, j.expand(B, N)), 1)
        rank = torch.cumsum((~first).long(), 1) - 1
        place = torch.where(first, own_place, free.gather(1, rank.clamp(min=0)))
        order = torch.empty_like(place).scatter_(1, place, j.expand(B, N))
        best, src, tok, ent, was_ended = (x.gather(1, order) for x in (best, src, tok, ent, was_ended))
    s["totals_out"].copy_(best.view(-1))
    s["source"].copy_(src.view(-1))
    s["token_ids"].copy_(tok.view(-1))
    s["entropy"].copy_(ent.view(-1))
    s["ended_out"].copy_((was_ended | (tok == _END)).view(-1))
    return s["totals_out"], s["source"], s["token_ids"], s["entropy"], s["ended_out"]


def _plain_reorder(s):
    c = s["case"]
    src = s["source"].long()
    slot = torch.arange(s["scores"].shape[1], device=src.device)
    first = s["shared_len"].long().repeat_interleave(c["group"])[:, None] if s["shared_len"] is not None else 0
    moves = (slot >= first) & (slot < s["live_len"].long()[src][:, None]) & \
        (src != torch.arange(src.numel(), device=src.device))[:, None]
    for name in ("k", "v"):
        for plane in range(s[name].shape[1]):   # one plane of all streams at a time
            x = s[name][:, plane]
            x.copy_(torch.where(moves[:, :, None], x[src], x))
    for name in ("scores", "serial"):
        if s[name] is not None:
            s[name].copy_(torch.where(moves, s[name][src], s[name]))
    s["live_len"].copy_(s["live_len"][src])
    return _reorder_state(s)


def _reorder_state(s):
    return {n: s[n] for n in ("k", "v", "scores", "serial", "live_len") if s[n] is not None}


def _plain_attend(s):
    c = s["case"]
    B, G, H, KH, D = c["groups"], c["group"], c["heads"], c["kv_heads"], c["dim"]
    cap = s["k"].shape[3]
    slot = torch.arange(cap, device="cuda")
    for g in range(B):
        mine = slice(g * G, g * G + G)
        shared = (slot < s["shared_len"][g].long())[:, None]
        q = s["q"][mine].float().view(G, KH, H // KH, D)
        n = s["kv_len"][mine].long()
        seen = (slot < n[:, None])[:, None, :]
        some = (n > 0)[:, None, None]
        for h in range(KH):
            k = torch.where(shared, s["k"][g * G, 0, h], s["k"][mine, 0, h]).float()
            v = torch.where(shared, s["v"][g * G, 0, h], s["v"][mine, 0, h]).float()
            z = torch.matmul(q[:, h], k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
            z = torch.where(seen, z, float("-inf"))
            m = torch.where(some, z.amax(-1, keepdim=True), 0.0)
            p = torch.exp(z - m)
            total = p.sum(-1, keepdim=True)
            out = torch.where(some, torch.matmul(p, v) / torch.where(some, total, 1.0), 0.0)
            heads = slice(h * (H // KH), (h + 1) * (H // KH))
            s["out"][mine, heads] = out.to(s["out"].dtype)
            s["lse"][mine, heads] = (m + torch.log(total))[..., 0]
    return s["out"], s["lse"]


def run(state):
    op = state["case"]["op"]
    if own:
        if "call" not in state:
            state["call"] = _call(state)
        state["call"]()
        if op == "select":
            return state["totals_out"], state["source"], state["token_ids"], state["entropy"], state["ended_out"]
        return _reorder_state(state) if op == "reorder" else (state["out"], state["lse"])
    return {"select": _plain_select, "reorder": _plain_reorder, "attend": _plain_attend}[op](state)


# --------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------

def work(case):
    c = case
    S = c["groups"] * c["group"]
    if c["op"] == "select":
        n = int(S * (1.0 - 2.0 * c["ended"]))
        size = 4 if c["dtype"] == "f32" else 2
        return {"bytes": n * c["vocab"] * size + 8 * S + 20 * c["groups"] * c["n_out"], "flops": 4 * n * c["vocab"]}
    if c["op"] == "reorder":
        rows = c["longest"] - c["spread"] // 2 - c["shared"]
        gone = c["group"] - c["survivors"]
        copied = c["groups"] * gone * rows
        sources = c["groups"] * min(gone, c["survivors"]) * rows
        row = 4 * c["layers"] * c["kv_heads"] * c["dim"] + (12 if c["tags"] else 4)
        return {"bytes": (copied + sources) * row + 12 * S, "flops": 0}
    shared = _lengths(c["shortest"], c["shared"], c["groups"])
    suffix = sum(_lengths(c["least"], c["suffix"], S))
    row = 4 * c["kv_heads"] * c["dim"]
    return {"bytes": (sum(shared) + suffix) * row + S * c["heads"] * (4 * c["dim"] + 4) + 4 * S,
            "flops": 4 * (sum(shared) * c["group"] + suffix) * c["heads"] * c["dim"]}


# --------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------

def _exact_select(c, s):
    G, N = c["group"], c["n_out"]
    out = {"totals": [], "source": [], "token": [], "entropy": [], "ended": []}
    ended, totals = s["ended"].tolist(), s["totals"].double().tolist()
    for g in range(c["groups"]):
        found = []   # (-score, stream, token, entropy, has ended)
        for st in range(g * G, g * G + G):
            if ended[st]:
                found.append((-totals[st], st, _END, 0.0, True))
            elif totals[st] > float("-inf"):
                logp = torch.log_softmax(s["logits"][st].double(), -1)
                top = torch.sort(logp, descending=True, stable=True)
                for lp, v in zip(top.values[:N].tolist(), top.indices[:N].tolist()):
                    if lp > float("-inf"):
                        found.append((-(totals[st] + lp), st, v, -lp, v == _END))
        found = [f for f in found if f[0] < float("inf")]
        # of an ended beam there is one candidate, so (score, stream, token) orders them all
        found = sorted(found, key=lambda f: f[:3])[:N]
        found += [(float("inf"), -1, -1, 0.0, False)] * (N - len(found))
        if c["places"]:
            at = [None] * N
            rest = []
            for f in found:
                if f[1] >= 0 and at[f[1] - g * G] is None:
                    at[f[1] - g * G] = f
                else:
                    rest.append(f)
            found = [f if f is not None else rest.pop(0) for f in at]
        for name, column in zip(out, zip(*[(-f[0], f[1], f[2], f[3], int(f[4])) for f in found])):
            out[name] += column
    real = lambda x: torch.tensor(x, dtype=torch.float64, device="cuda")
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return real(out["totals"]), whole(out["source"]), whole(out["token"]), real(out["entropy"]), whole(out["ended"])


def exact(case, seed):
    c, s = case, prepare(case, seed)
    G = c["group"]
    if c["op"] == "select":
        return _exact_select(c, s)
    if c["op"] == "reorder":
        new = {n: t.clone() for n, t in _reorder_state(s).items()}
        length = s["live_len"].tolist()
        for st, src in enumerate(s["source"].tolist()):
            if src == st:
                continue
            rows = slice(c["shared"], length[src])
            new["k"][st][:, rows] = s["k"][src][:, rows]
            new["v"][st][:, rows] = s["v"][src][:, rows]
            new["scores"][st, rows] = s["scores"][src, rows]
            if c["tags"]:
                new["serial"][st, rows] = s["serial"][src, rows]
            new["live_len"][st] = length[src]
        return new
    H, KH = c["heads"], c["kv_heads"]
    out = torch.zeros(G * c["groups"], H, c["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((G * c["groups"], H), float("-inf"), dtype=torch.float64, device="cuda")
    shared = s["shared_len"].tolist()
    for st, n in enumerate(s["kv_len"].tolist()):
        if n == 0:
            continue
        first, common = st // G * G, min(n, shared[st // G])
        k = torch.cat([s["k"][first, 0, :, :common], s["k"][st, 0, :, common:n]], 1).double()
        v = torch.cat([s["v"][first, 0, :, :common], s["v"][st, 0, :, common:n]], 1).double()
        q = s["q"][st].double().view(KH, H // KH, -1)
        z = torch.einsum("hqd,hnd->hqn", q, k) / math.sqrt(c["dim"])
        lse[st] = torch.logsumexp(z, -1).view(H)
        out[st] = torch.einsum("hqn,hnd->hqd", torch.softmax(z, -1), v).reshape(H, -1)
    return out, lse
