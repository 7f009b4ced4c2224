"""Streams with a past in common, on the GPU, where a call's answer hangs on the last bits or on the ends of
the number range: equal streams at every alignment, totals and logits of the lowest value, segments of
many trips, a retention round between two tokens."""
import math

import pytest
import torch

from paper_2405_12528_b200 import binding as B
from test_gpu_beams import beams, check_select, select
from test_gpu_decode import gen, ref_attend

pytestmark = pytest.mark.gpu


def at_skew(z, skew, stride):
    """The same rows, the first one ``skew`` elements behind a 16-byte boundary, ``stride`` elements apart."""
    S, V = z.shape
    buf = torch.full((skew + S * stride + 16,), 50.0, dtype=z.dtype, device="cuda")
    view = buf[skew:skew + S * stride].view(S, stride)[:, :V]
    view.copy_(z)
    return view


# --------------------------------------------------------------------------------------
# equal streams: the lower one wins, wherever the rows begin
# --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 9, 300, 1029, 5003, 50257])
def test_select_equal_streams_tie_at_every_alignment(dtype, V):
    z, _ = beams(V, 1, V, dtype)
    N = min(40, 8 * V)
    order = torch.sort(z[0].double(), descending=True, stable=True).indices.tolist()
    # the eight streams of a group are the same: token by token (equal logits: token behind token in a stream)
    want, i = [], 0
    while len(want) < N:
        run = [v for v in order[i:] if z[0, v] == z[0, order[i]]]
        want += [(s, v) for s in range(8) for v in run]
        i += len(run)
    want = want[:N]
    rows = z.expand(8, V)
    for skew in range(0, 16 // z.element_size()):
        for stride in (V, V + 1, V + 3):
            tot, src, tok, ent, _ = select(at_skew(rows, skew, stride), 8, N, torch.full((8,), -3.0, device="cuda"), end=-1)
            assert list(zip(src.tolist(), tok.tolist())) == want, (skew, stride)
            for v in set(tok.tolist()):
                assert tot[tok == v].unique().numel() == 1 and ent[tok == v].unique().numel() == 1, (skew, stride, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3, 513, 4099, 50257])
def test_select_same_bits_at_every_alignment(dtype, V):
    z, totals = beams(V + 1, 6, V, dtype)
    per = 16 // z.element_size()
    want = select(at_skew(z, 0, (V + per - 1) // per * per), 3, 7, totals, end=-1)
    for skew in range(per):
        for stride in range(V, V + per, 1 if V < 5000 else 3):
            got = select(at_skew(z, skew, stride), 3, 7, totals, end=-1)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (skew, stride)


# --------------------------------------------------------------------------------------
# totals and logits at the ends of the number range: only -inf says that there is no candidate
# --------------------------------------------------------------------------------------

LOWEST = torch.finfo(torch.float32).min


def check_first_stream(z, G, N, totals, alive=None):
    """All totals so low that no logit shows beside them: the lowest live stream's best logits, in order."""
    tot, src, tok, ent, fin = select(z, G, N, totals, end=-1)
    for g in range(z.shape[0] // G):
        s = g * G + (0 if alive is None else alive)
        order = torch.sort(z[s].double(), descending=True, stable=True).indices[:N]
        out = slice(g * N, g * N + N)
        assert src[out].tolist() == [s] * N
        assert torch.equal(tok[out].long(), order)
        assert (tot[out] == LOWEST).all() and (fin[out] == 0).all()
        want = -torch.log_softmax(z[s].double(), -1)[order]
        assert ((ent[out].double() - want).abs() <= 2.0 ** -18 + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [40, 300, 3000, 5003, 128256])
@pytest.mark.parametrize("G,N", [(1, 1), (4, 4), (4, 33), (16, 16)])
def test_select_all_totals_of_the_lowest_value(dtype, V, G, N):
    z, _ = beams(V, 2 * G, V, dtype)
    totals = torch.full((2 * G,), LOWEST, device="cuda")
    check_first_stream(z, G, N, totals)
    if G > 1:
        totals.view(2, G)[:, 0] = -math.inf          # and a stream without a beam in front
        check_first_stream(z, G, N, totals, alive=1)


def test_select_lowest_totals_beside_ended_beams():
    z, _ = beams(3, 8, 9001, torch.float32)
    totals = torch.full((8,), LOWEST, device="cuda")
    ended = torch.tensor([0, 1, 0, 0, 1, 1, 1, 1], dtype=torch.int32, device="cuda")
    tot, src, tok, _, fin = select(z, 4, 4, totals, ended)
    order = torch.sort(z[0], descending=True, stable=True).indices[:4].tolist()
    assert src.tolist() == [0, 0, 0, 0, 4, 5, 6, 7] and tok.tolist() == order + [2] * 4
    assert (tot == LOWEST).all() and fin.tolist() == [int(t == 2) for t in order] + [1] * 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [5, 300, 5003, 128256])
def test_select_logits_further_apart_than_fp32_reaches(dtype, V):
    # 3e38 and -3e38: a difference that only fp64 holds; such tokens are candidates, their totals round to -inf
    z = torch.full((4, V), -3e38, dtype=dtype, device="cuda")
    z[:, V // 2] = 3e38
    z[3, :V // 2 - 1] = -math.inf
    totals = torch.tensor([0.0, -1.0, -math.inf, -3.0], device="cuda")
    tot, src, tok, ent, _ = select(z, 2, 5, totals, end=-1)
    low = [v for v in range(V) if v != V // 2]
    behind = [v for v in range(V // 2 - 1, V) if v != V // 2]
    n = min(4, len(behind))
    assert src.tolist() == [0, 1, 0, 0, 0, 3] + [3] * n + [-1] * (4 - n)
    assert tok.tolist() == [V // 2, V // 2] + low[:3] + [V // 2] + behind[:n] + [-1] * (4 - n)
    assert tot.tolist() == [0.0, -1.0] + [-math.inf] * 3 + [-3.0] + [-math.inf] * 4
    assert ent.tolist() == [0.0, 0.0] + [math.inf] * 3 + [0.0] + [math.inf] * n + [0.0] * (4 - n)


@pytest.mark.parametrize("V", [300, 128256])
def test_select_lowest_totals_and_rows_masked_by_the_lowest_value(V):
    z, _ = beams(V, 4, V, torch.float32)
    z[:, 20:] = LOWEST
    tot, src, tok, _, _ = select(z, 4, 30, torch.full((4,), LOWEST, device="cuda"), end=-1)
    best = torch.sort(z[:, :20], descending=True, stable=True).indices
    # total + logit rounds to the lowest value in all streams where the logit counts: 20 and 10 of them
    assert src.tolist() == [0] * 20 + [1] * 10 and (tot == LOWEST).all()
    assert tok.tolist() == best[0].tolist() + best[1, :10].tolist()
    tot, src, tok, _, _ = select(z[:1], 1, 30, torch.full((1,), LOWEST, device="cuda"), end=-1)
    assert src.tolist() == [0] * 30 and tok.tolist() == best[0].tolist() + list(range(20, 30))
    assert tot.tolist() == [LOWEST] * 20 + [-math.inf] * 10


# --------------------------------------------------------------------------------------
# long segments: what a lane adds up in fp32
# --------------------------------------------------------------------------------------

def log_sum_bound(trips, V):
    """What lse may be off by, u = 2^-24.  A term: exp to 4u, its argument (a difference, a product, a sum: 3u of
    it, and the arguments' mean, weighted by the terms, is at most ln V).  A trip of a lane: 8 additions in each of
    four sums, 2 to join them, 1 onto the lane's sum, which a new maximum multiplies by an exp first (6u a trip; the
    arguments of all these together weigh little: T e^-T).  Lanes and segments: another exp and 5 additions, another
    exp, the rest in fp64."""
    return (6 * trips + 10 + 4 + 3 * math.log(V) + 10 + 6) * 2.0 ** -24


@pytest.mark.parametrize("ascending", [False, True])
@pytest.mark.parametrize("rows,V,dtype,trips", [
    (2600, 131071, torch.bfloat16, 64),     # more than 64 trips would bring a segment per warp: two segments a row
    (1200, 70001, torch.float32, 35),
    (640, 40001, torch.bfloat16, 6),
])
def test_select_segments_of_many_trips(rows, V, dtype, trips, ascending):
    size = 2 if dtype == torch.bfloat16 else 4
    whole = -(-V * size // 2048)
    assert min(64, whole, -(-whole * rows // (148 * 32))) == trips
    if ascending:   # every trip brings a new maximum
        z = torch.linspace(-4, 14, V, device="cuda").to(dtype).expand(rows, V).contiguous()
        z += torch.linspace(0, 3, rows, device="cuda").to(dtype)[:, None]
        totals = torch.linspace(-9, -1, rows, device="cuda")
    else:
        z, totals = beams(V, rows, V, dtype)
    N = 4
    tot, src, tok, ent, _ = select(z, 1, N, totals, end=-1)
    assert torch.equal(src, torch.arange(rows, dtype=torch.int32, device="cuda").repeat_interleave(N))
    tol = log_sum_bound(trips, V)
    for r in range(0, rows, 100):
        x = z[r:r + 100].double()
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :N]
        out = slice(r * N, min(rows, r + 100) * N)
        assert torch.equal(tok[out].view(-1, N).long(), order)
        e = torch.logsumexp(x, -1, keepdim=True) - x.gather(1, order)
        t = totals[r:r + 100].double()[:, None] - e
        for got, want in ((ent, e), (tot, t)):
            d = (got[out].view(-1, N).double() - want).abs()
            assert (d <= tol + 2.0 ** -24 * want.abs()).all(), float(d.max())


# --------------------------------------------------------------------------------------
# retention rounds between tokens: sinks that cover the shared slots leave them in place
# --------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,C,layout", [(3, 160, None), (3, 160, B.ROPE_HALF), (40, 6000, None)])
@pytest.mark.parametrize("shared", [[64, 40], [1, 64], [384, 301]])
def test_rounds_between_tokens_of_streams_that_share_their_sinks(G, C, layout, shared):
    """A cache whose followers hold nothing below shared_len (NaN) against one with the shared slots copied to every
    stream, round for round: the same slots stay, and attention over them is the same."""
    S, H, KH, D, V, new, sink = 2 * G, 4, 2, 64, 500, 5, max(shared)
    C = max(C, sink + 60)
    cfg = B.make_config(n_streams=S, n_layers=1, n_kv_heads=KH, head_dim=D, capacity=C, budget=sink + 36, n_sink=sink,
                        n_recent=8, threshold=sink + 46, max_new=new, vocab=V, logits_dtype="f32", kv_dtype="bf16")
    g = gen(G + C)
    ws, wa, wp = B.new_workspace(cfg), B.new_attend_shared_workspace(cfg, G, H), B.new_attend_workspace(cfg)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    live = [sink + 6 + 7 * (s % 5) for s in range(S)]
    plain = [torch.randn(S, 1, KH, C, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    for s in range(S):
        for x in plain:
            x[s, :, :, :shared[s // G]] = x[s // G * G, :, :, :shared[s // G]]
    held = [x.clone() for x in plain]
    for s in range(S):
        for x in held:
            if s % G:
                x[s, :, :, :shared[s // G]] = math.nan
    E = torch.rand(S, C, generator=g, device="cuda") * 9
    E_held = E.clone()
    for s in range(S):
        if s % G:
            E_held[s, :shared[s // G]] = 1e30       # whatever stands there
    lens, lens_held = i32(*live), i32(*live)
    keeps = [torch.zeros(S, cfg.threshold, dtype=torch.int32, device="cuda") for _ in range(2)]
    n_keep = [torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2)]
    decay = torch.full((S,), 0.9, device="cuda")
    evicted = False
    for rnd in range(12):
        n_new = i32(*[1 + (s + rnd) % new for s in range(S)])
        logits = torch.randn(S * new, V, generator=g, device="cuda") * 2
        ids = torch.randint(0, V, (S * new,), generator=g, device="cuda", dtype=torch.int32)
        rows = [torch.randn(S, KH, new, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        for s, n in enumerate(lens.tolist()):
            for x, y, r in zip(plain, held, rows):
                x[s, 0, :, n:n + new] = y[s, 0, :, n:n + new] = r[s]
        for i, (kv, e, n) in enumerate(((plain, E, lens), (held, E_held, lens_held))):
            B.sirllm_step(cfg, logits, ids, n_new, e, None, n, decay, *kv, keeps[i], n_keep[i], None, ws)
            if layout is not None:
                B.sirllm_rerotate_keys(cfg, kv[0], keeps[i], n_keep[i], 1e4, layout)
        assert torch.equal(lens, lens_held) and torch.equal(n_keep[0], n_keep[1])
        evicted |= bool((n_keep[0] == cfg.budget).any())
        q = torch.randn(S, H, D, generator=g, device="cuda").to(torch.bfloat16)
        out, want = torch.empty_like(q), torch.empty_like(q)
        B.sirllm_attend_shared(cfg, 0, G, i32(*shared), q, *held, lens_held, None, out, None, wa)
        B.sirllm_attend(cfg, 0, q, *plain, lens, None, want, None, wp)
        for s, n in enumerate(lens.tolist()):
            assert torch.equal(keeps[0][s, :n], keeps[1][s, :n])
            lo = shared[s // G]
            for x, y in zip(plain, held):
                assert torch.equal(x[s, 0, :, lo:n], y[s, 0, :, lo:n])
                assert torch.equal(x[s, 0, :, :lo], y[s // G * G, 0, :, :lo])
            # both are within the tolerance of the same formula
            tol = ref_attend(q[s], plain[0][s, 0], plain[1][s, 0], n, D ** -0.5)[2]
            assert ((out[s].double() - want[s].double()).abs() <= 2 * tol).all()
    assert evicted and B.sirllm_status(ws) == 0 and B.sirllm_status(wa) == 0


def test_shared_slots_handed_out_make_plain_streams():
    G, S, H, KH, D, C = 4, 8, 4, 2, 64, 300
    shared, lens = [200, 37], [205, 290, 200, 231, 40, 37, 300, 99]
    cfg = B.make_config(n_streams=S, n_layers=1, n_kv_heads=KH, head_dim=D, capacity=C, budget=C, n_sink=0, n_recent=0,
                        max_new=1, vocab=1, logits_dtype="f32", kv_dtype="bf16")
    g = gen(77)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(S, 1, KH, C, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    E = torch.rand(S, C, generator=g, device="cuda")
    was = [x.clone() for x in (k, v, E)]
    q = torch.randn(S, H, D, generator=g, device="cuda").to(torch.bfloat16)
    out, want = torch.empty_like(q), torch.empty_like(q)
    B.sirllm_attend_shared(cfg, 0, G, i32(*shared), q, k, v, i32(*lens), None, want, None, B.new_attend_shared_workspace(cfg, G, H))
    ws, held = B.new_workspace(cfg), i32(*[shared[s // G] for s in range(S)])
    B.sirllm_reorder_streams(cfg, G, i32(*[s // G * G for s in range(S)]), None, E, None, held, k, v, ws)
    assert B.sirllm_status(ws) == 0 and held.tolist() == [shared[s // G] for s in range(S)]
    for s in range(S):
        lo = shared[s // G]
        for x, y in zip((k[:, 0], v[:, 0]), (was[0][:, 0], was[1][:, 0])):
            assert torch.equal(x[s, :, :lo], y[s // G * G, :, :lo]) and torch.equal(x[s, :, lo:], y[s, :, lo:])
        assert torch.equal(E[s, :lo], was[2][s // G * G, :lo]) and torch.equal(E[s, lo:], was[2][s, lo:])
    B.sirllm_attend(cfg, 0, q, k, v, i32(*lens), None, out, None, B.new_attend_workspace(cfg))
    for s in range(S):
        tol = ref_attend(q[s], k[s, 0], v[s, 0], lens[s], D ** -0.5)[2]
        assert ((out[s].double() - want[s].double()).abs() <= 2 * tol).all()


def test_select_totals_that_are_no_numbers():
    z, _ = beams(21, 8, 20001, torch.float32)
    totals = torch.tensor([0.0, math.inf, math.nan, -1.0, math.nan, math.nan, -math.inf, math.nan], device="cuda")
    tot, src, tok, _, _ = select(z, 4, 40, totals, end=-1)      # +inf: ahead of all; NaN: no beam
    assert src[:40].tolist() == [1] * 40 and (tot[:40] == math.inf).all()
    assert tok[:40].tolist() == torch.sort(z[1], descending=True, stable=True).indices[:40].tolist()
    assert (src[40:] == -1).all() and (tok[40:] == -1).all() and (tot[40:] == -math.inf).all()


# --------------------------------------------------------------------------------------
# the largest vocabulary; calls captured first, and behind other streams
# --------------------------------------------------------------------------------------

@pytest.mark.parametrize("skew", [0, 3])
def test_select_largest_vocabulary(skew):
    V = B.MAX_BEAM_VOCAB
    z = at_skew(torch.zeros(2, V, dtype=torch.bfloat16, device="cuda"), skew, V + 8)
    for s, (at, value) in enumerate(((V - 1, 3.0), (V // 2 + 7, 2.0))):
        z[s, at] = value
    z[0, 0] = 1.0
    totals = torch.tensor([-1.0, -1.5], device="cuda")
    tot, src, tok, ent, _ = select(z, 2, 8, totals, end=V - 1)
    assert src.tolist() == [0, 1, 0] + [0] * 5 and tok.tolist() == [V - 1, V // 2 + 7, 0, 1, 2, 3, 4, 5]
    lse = [math.log(math.fsum([V - 2, math.exp(3.0), math.e])), math.log(math.fsum([V - 1, math.exp(2.0)]))]
    want = [lse[0] - 3.0, lse[1] - 2.0, lse[0] - 1.0] + [lse[0]] * 5
    for e, t, s, w in zip(ent.tolist(), tot.tolist(), src.tolist(), want):
        tol = log_sum_bound(64, V) + 2.0 ** -24 * 20
        assert abs(e - w) <= tol and abs(t - (totals[s].item() - w)) <= tol


FIRST_CALLS = """
import torch
from paper_2405_12528_b200 import binding as B
G, H, KH, D, C, V = {G}, {H}, 2, {D}, {C}, 40001
cfg = B.make_config(G, 1, KH, D, C, C, 0, 0, 1, V, "f32", "bf16")
i32 = dict(dtype=torch.int32, device="cuda")
ws, wb, wa = B.new_workspace(cfg), B.new_beam_workspace(cfg), B.new_attend_shared_workspace(cfg, G, H)
k, v = (torch.randn(G, KH, C, D, device="cuda").to(torch.bfloat16) for _ in range(2))
q = torch.randn(G, H, D, device="cuda").to(torch.bfloat16)
out, logits = torch.zeros_like(q), torch.randn(G, V, device="cuda")
shared, live = torch.full((1,), 500, **i32), torch.full((G,), 520, **i32)
totals, source, tokens = torch.zeros(G, device="cuda"), torch.zeros(G, **i32), torch.zeros(G, **i32)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    B.sirllm_attend_shared(cfg, 0, G, shared, q, k, v, live, None, out, None, wa)
    B.sirllm_beam_select(cfg, logits, G, G, totals, None, -1, True, totals, source, tokens, None, None, wb)
    B.sirllm_reorder_streams(cfg, G, source, shared, None, None, live, k, v, ws)
g.replay()
torch.cuda.synchronize()
assert float(out[0].abs().sum()) > 0 and float(totals.max()) < 0 and int(source.min()) >= 0
assert all(B.sirllm_status(w) == 0 for w in (ws, wb, wa))
print("captured")
"""


@pytest.mark.parametrize("G,H,D,C", [(4, 4, 64, 600), (4, 8, 128, 45000), (40, 4, 64, 9000), (16, 8, 256, 3000)])
def test_the_process_first_calls_may_be_captured_ones(G, H, D, C):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(G=G, H=H, D=D, C=C)], capture_output=True, text=True,
                         cwd=root, timeout=300)
    assert run.returncode == 0 and "captured" in run.stdout, run.stderr[-2000:]


@pytest.mark.parametrize("G,C", [(4, 600), (4, 45000), (40, 9000)])
def test_shared_calls_behind_a_join_of_two_captured_streams(G, C):
    # lengths, queries, rows and sources that another stream writes just before each call
    H, KH, D, V = 4, 2, 64, 3001
    cfg = B.make_config(G, 1, KH, D, C, C, 0, 0, 1, V, "f32", "bf16")
    g = gen(C)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    ws, wb, wa = B.new_workspace(cfg), B.new_beam_workspace(cfg), B.new_attend_shared_workspace(cfg, G, H)
    k, v = (torch.randn(G, 1, KH, C, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    was = k.clone(), v.clone()
    q_from = torch.randn(G, H, D, generator=g, device="cuda").to(torch.bfloat16)
    z_from, totals = torch.randn(G, V, generator=g, device="cuda") * 3, -torch.rand(G, generator=g, device="cuda")
    q, z, out = torch.zeros_like(q_from), torch.zeros_like(z_from), torch.zeros_like(q_from)
    shared, live = i32(0), i32(*[0] * G)
    tot, src, tok = torch.zeros(G, device="cuda"), i32(*[0] * G), i32(*[0] * G)
    lens = [512 + 2 * s for s in range(G)]
    lens_from = i32(*lens)
    main, other = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        other.wait_stream(main)
        with torch.cuda.stream(other):
            shared.fill_(512)
            live.copy_(lens_from)
            q.copy_(q_from)
            k.copy_(was[0])
        v.copy_(was[1])
        main.wait_stream(other)
        B.sirllm_attend_shared(cfg, 0, G, shared, q, k, v, live, None, out, None, wa)
        other.wait_stream(main)
        with torch.cuda.stream(other):
            z.copy_(z_from)
        main.wait_stream(other)
        B.sirllm_beam_select(cfg, z, G, G, totals, None, -1, True, tot, src, tok, None, None, wb)
        B.sirllm_reorder_streams(cfg, G, src, shared, None, None, live, k, v, ws)
    want = select(z_from, G, G, totals, end=-1, places=True, cfg=cfg)
    for _ in range(4):
        for x in (shared, live, q, z, k, v, out, tot, src, tok):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tot, want[0]) and torch.equal(src, want[1]) and torch.equal(tok, want[2])
        for s, f in enumerate(src.tolist()):
            ks, vs = (torch.cat([x[0, 0, :, :512], x[s, 0, :, 512:]], 1) for x in was)
            o, _, to, _ = ref_attend(q_from[s], ks, vs, lens[s], D ** -0.5)
            assert ((out[s].double() - o).abs() <= to).all()
            assert int(live[s]) == lens[f] and torch.equal(k[s, 0, :, 512:lens[f]], was[0][f, 0, :, 512:lens[f]])
