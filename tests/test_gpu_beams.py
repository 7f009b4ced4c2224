"""Streams with a past in common, on the GPU, against plain forms in 64 bits: ``sirllm_beam_select``,
``sirllm_reorder_streams``, ``sirllm_attend_shared``, and a beam search made of them.

Tolerances.  select: a chunk's sum is fp32 (at most 64 terms per thread, then a tree: 2^-20 of the sum
at the very most, terms' own errors included), joined in fp64, and totals and entropies are rounded once:
2^-20 + 2^-24 |value|; whole numbers are equal.  The inputs keep candidates that are not equal apart
by more than that.  reorder: bit equal.  attend: those of the calls of one decode step."""
import math

import pytest
import torch

from paper_2405_12528_b200 import binding as B
from test_gpu_decode import DT, F64, gen, i32, randn, ref_attend, same_bits

pytestmark = pytest.mark.gpu

END = 2


def config(S=1, L=1, KH=1, D=64, C=256, V=16, kv="bf16", logits="f32", stride=None, M=1):
    return B.make_config(n_streams=S, n_layers=L, n_kv_heads=KH, head_dim=D, capacity=C, budget=C, n_sink=0,
                         n_recent=0, max_new=M, vocab=V, logits_dtype=logits, kv_dtype=kv, logits_row_stride=stride)


# --------------------------------------------------------------------------------------
# select
# --------------------------------------------------------------------------------------

def ref_select(logits, G, N, totals, ended, end, places):
    """Lists of (stream, token, total, entropy, ended) per group, from the definition, on the host."""
    z = logits.double().cpu()
    e_all = -torch.log_softmax(z, -1)     # (logits - maximum) - log sum: exact for rows of lowest values too
    groups = []
    for g0 in range(0, z.shape[0], G):
        found = []
        for s in range(g0, g0 + G):
            t = float(totals[s])
            if not t > -math.inf:
                continue
            if ended is not None and int(ended[s]):
                found.append((t, s, end, 0.0, 1))
                continue
            e = e_all[s]
            order = torch.sort(z[s], descending=True, stable=True).indices[:N].tolist()
            found += [(t - float(e[v]), s, v, float(e[v]), int(v == end)) for v in order if z[s, v] > -math.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2] if f[4] == 0 or ended is None or not int(ended[f[1]]) else 0))
        found = found[:N]
        found += [(-math.inf, -1, -1, 0.0, 0)] * (N - len(found))
        if places:
            at, rest = [None] * N, []
            for f in found:
                if f[1] >= 0 and at[f[1] - g0] is None:
                    at[f[1] - g0] = f
                else:
                    rest.append(f)
            found = [f or rest.pop(0) for f in at]
        groups += found
    return groups


def select(logits, G, N, totals, ended=None, end=END, places=False, ws=None, cfg=None, in_place=False):
    S, V = logits.shape
    cfg = cfg or config(S=S, V=V, logits="bf16" if logits.dtype == torch.bfloat16 else "f32",
                        stride=logits.stride(0) if S > 1 else V)
    ws = B.new_beam_workspace(cfg) if ws is None else ws
    n = S // G * N
    tot = totals.clone() if in_place else torch.full((n,), 7.0, device="cuda")
    end_out = ended.clone() if in_place and ended is not None else torch.full((n,), 7, dtype=torch.int32, device="cuda")
    src, tok = (torch.full((n,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    ent = torch.full((n,), 7.0, device="cuda")
    B.sirllm_beam_select(cfg, logits, G, N, tot if in_place else totals, end_out if in_place and ended is not None else ended,
                         end, places, tot, src, tok, ent, end_out, ws)
    return tot, src, tok, ent, end_out


def check_select(logits, G, N, totals, ended=None, end=END, places=False, **kw):
    got = select(logits, G, N, totals, ended, end, places, **kw)
    want = ref_select(logits, G, N, totals, ended, end, places)
    tot, src, tok, ent, fin = (x.tolist() for x in got)
    assert src == [f[1] for f in want]
    assert tok == [f[2] for f in want]
    assert fin == [f[4] for f in want]
    for a, e, f in zip(tot, ent, want):
        assert a == f[0] or abs(a - f[0]) <= 2.0 ** -20 + 2.0 ** -24 * abs(f[0]), (a, f)
        assert abs(e - f[3]) <= 2.0 ** -20 + 2.0 ** -24 * abs(f[3]), (e, f)


def beams(seed, S, V, dtype, pad=0):
    g = gen(seed)
    wide = randn(g, S, V + pad, dtype=dtype, scale=2.0)
    z = wide[:, :V]
    n = min(V, 10)
    at = torch.rand(S, V, generator=g, device="cuda").argsort(-1)[:, :n]
    z.scatter_add_(1, at, (3 + 5 * torch.rand(S, n, generator=g, device="cuda")).to(dtype))
    return z, -4 - 6 * torch.rand(S, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 255, 2047, 2048, 2049, 4097, 16383, 50257])
@pytest.mark.parametrize("G,N,groups", [(1, 1, 1), (4, 4, 1), (3, 6, 5), (8, 16, 2)])
def test_select_sizes(dtype, V, G, N, groups):
    z, totals = beams(V + G, G * groups, V, dtype)
    check_select(z, G, N, totals, end=END if V > END else -1, places=N == G)


@pytest.mark.parametrize("pad", [1, 3, 8, 61])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select_rows_at_any_distance_and_alignment(pad, dtype):
    z, totals = beams(pad, 12, 5003, dtype, pad)
    check_select(z, 4, 8, totals)
    # a first row off its 16 bytes
    wide = torch.empty(13, 5003 + pad, dtype=dtype, device="cuda")
    view = wide.view(-1)[1:1 + 12 * (5003 + pad)].view(12, 5003 + pad)[:, :5003]
    view.copy_(z)
    check_select(view, 4, 8, totals)


@pytest.mark.parametrize("rows", [1, 37, 300, 640])   # chunks of 4 to 32 KB
def test_select_chunks_of_every_size(rows):
    z, totals = beams(rows, rows, 40001, torch.bfloat16)
    check_select(z, 1, 5, totals)


def test_select_64_beams_and_64_candidates():
    z, totals = beams(5, 128, 3001, torch.float32)
    check_select(z, 64, 64, totals, places=True)
    check_select(z, 64, 33, totals)
    check_select(z[:64], 1, 64, totals[:64])


@pytest.mark.parametrize("places", [False, True])
def test_select_ended_and_absent_beams(places):
    z, totals = beams(9, 24, 1000, torch.float32)
    ended = i32(*[(s % 3 == 1) * 5 for s in range(24)])
    totals[::4] = -math.inf
    totals[16:24] = -math.inf                    # a group without beams
    check_select(z, 8, 8, totals, ended, places=places)
    check_select(z, 8, 8, totals, ended, places=places, in_place=True)
    check_select(z, 8, 8, totals, ended, end=-1, places=places)
    check_select(z, 8, 8, totals, torch.ones_like(ended), places=places)   # all have ended
    z[:, END] = 40.0                             # and all end
    check_select(z, 8, 8, totals, ended, places=places)


def test_select_starts_from_one_beam():
    z, _ = beams(10, 8, 777, torch.bfloat16)
    totals = torch.full((8,), -math.inf, device="cuda")
    totals[0] = totals[4] = 0.0
    check_select(z, 4, 4, totals, places=True)


def test_select_fewer_candidates_than_asked_for_and_masked_logits():
    z, totals = beams(11, 6, 500, torch.float32)
    z[0] = -math.inf                             # a row that is masked whole
    z[1, 3:] = -math.inf
    z[2:, 10:490] = -math.inf
    z[3:5] = -math.inf
    z[4, 499] = -300.0                           # one token left
    check_select(z, 3, 6, totals)
    check_select(z, 3, 64, totals)
    check_select(z, 2, 2, totals, places=True)
    # masked by the type's lowest value: such tokens are candidates
    for dt in (torch.float32, torch.bfloat16):
        low = z.to(dt).clone()
        low[low == -math.inf] = torch.finfo(dt).min
        check_select(low, 3, 6, totals)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select_rows_masked_with_infinities_beside_rows_masked_with_lowest_values(dtype):
    lowest = torch.finfo(dtype).min
    z = torch.full((4, 128256), -math.inf, dtype=dtype, device="cuda")
    z[0, [5, 100000]] = torch.tensor([1.0, 2.0], dtype=dtype, device="cuda")
    z[1, 77] = 0.5
    z[2] = lowest
    z[2, [3000, 90001]] = torch.tensor([0.25, 3.0], dtype=dtype, device="cuda")
    totals = torch.tensor([-1.0, -2.0, -3.0, -math.inf], device="cuda")
    check_select(z, 4, 16, totals)
    z = torch.full((1, 600001), -math.inf, dtype=dtype, device="cuda")
    z[0, 300007:] = lowest
    z[0, [9, 500000]] = torch.tensor([1.0, 0.5], dtype=dtype, device="cuda")
    check_select(z, 1, 8, totals[:1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [5, 3000, 70000])
def test_select_ties_go_to_the_lower_stream_and_token(dtype, V):
    z = torch.zeros(8, V, dtype=dtype, device="cuda")
    totals = torch.full((8,), -1.0, device="cuda")
    N = min(64, 2 * V)
    check_select(z, 4, N, totals)                # every candidate the same: long lists of equal ones
    check_select(z, 8, 8, totals, places=True)
    z[:, V // 2:] = 1.0
    check_select(z, 4, N, totals)
    g = gen(3)
    z = torch.randint(-3, 3, (8, V), generator=g, device="cuda").to(dtype)
    z[5] = z[4]
    check_select(z, 2, min(33, V), torch.full((8,), -2.0, device="cuda"))


def test_select_sorted_logits_fill_one_threads_share():
    # the best logits side by side, so that single threads hold more of them than others in all
    for V, descending in ((40000, True), (40000, False), (4096, True)):
        z = torch.linspace(-9, 9, V, device="cuda").flip(0 if descending else ()).expand(4, V).contiguous()
        z[1:] -= torch.tensor([0.0101, 0.0207, 0.0303], device="cuda")[:, None]
        z[:, 5] += torch.tensor([0.3, 0.1, 0.2, 0.7], device="cuda")
        check_select(z, 4, 64, torch.tensor([-3.0, -3.001, -3.0003, -2.9007], device="cuda"))


def test_select_extreme_totals_and_logits():
    z, totals = beams(12, 4, 300, torch.float32)
    totals = torch.tensor([-1e30, -1000.0, -1e-3, 0.0], device="cuda")
    check_select(z, 4, 8, totals)
    check_select(z * 1e4, 2, 4, totals)
    check_select(z - 1e6, 1, 1, totals)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select_negative_zero_is_zero(dtype):
    z = torch.full((2, 600), -3.0, dtype=dtype, device="cuda")
    z[:, 50:400:7] = 0.0
    z[:, 57] = -0.0                              # equal to its neighbours, ahead of all but one of them
    z[1, 43] = -0.0
    check_select(z, 1, 20, torch.tensor([-1.0, -1.0], device="cuda"))
    check_select(z, 2, 40, torch.tensor([-1.0, -1.0], device="cuda"))


@pytest.mark.parametrize("G,N", [(8, 8), (4, 16), (64, 64)])
def test_select_wide_rows_masked_but_for_a_few_tokens(G, N):
    g = gen(16)
    z, totals = beams(16, G, 128256, torch.bfloat16)
    keep = torch.rand(G, 128256, generator=g, device="cuda") < 0.0005
    z[~keep] = -math.inf
    check_select(z, G, N, totals)
    z[:, 64000:64300] = 1.0                      # and a run of equal ones
    check_select(z, G, N, totals)


def test_select_reads_one_row_per_stream_whatever_max_new_is():
    z, totals = beams(13, 6, 800, torch.float32)
    check_select(z, 3, 3, totals, cfg=config(S=6, V=800, M=64))


def test_select_outputs_that_may_be_left_out():
    z, totals = beams(14, 4, 900, torch.bfloat16)
    cfg = config(S=4, V=900, logits="bf16")
    ws = B.new_beam_workspace(cfg)
    tot, src, tok, _, _ = select(z, 4, 4, totals)
    tot2, src2, tok2 = torch.zeros_like(tot), torch.zeros_like(src), torch.zeros_like(tok)
    B.sirllm_beam_select(cfg, z, 4, 4, totals, None, END, False, tot2, src2, tok2, None, None, ws)
    assert torch.equal(tot, tot2) and torch.equal(src, src2) and torch.equal(tok, tok2)
    assert B.sirllm_status(ws) == 0


def test_select_graph_replays_and_repeats_are_the_same_bits():
    z, totals = beams(15, 24, 20011, torch.bfloat16)
    cfg = config(S=24, V=20011, logits="bf16")
    ws = B.new_beam_workspace(cfg)
    want = select(z, 8, 8, totals, places=True, ws=ws, cfg=cfg)
    out = [torch.zeros_like(x) for x in want]
    call = B.prepared(B.sirllm_beam_select, cfg, z, 8, 8, totals, None, END, True, *out, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
        call()
    for _ in range(20):
        for x in out:
            x.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


# --------------------------------------------------------------------------------------
# reorder
# --------------------------------------------------------------------------------------

def reorder_case(S, G, source, lens, shared=None, L=2, KH=2, D=64, C=100, kv="bf16", tags=True, scores=True, seed=0,
                 keys=True, values=True, want_status=0):
    g = gen(seed)
    cfg = config(S=S, L=L, KH=KH, D=D, C=C, kv=kv)
    k, v = (randn(g, S, L * KH, C, D, dtype=DT[kv]) for _ in range(2))
    E = torch.rand(S, C, generator=g, device="cuda") if scores else None
    T = torch.randint(-2**62, 2**62, (S, C), generator=g, device="cuda") if tags else None
    live = i32(*lens)
    ws = B.new_workspace(cfg)
    was = [x.clone() if x is not None else None for x in (k, v, E, T)]
    want = [x.clone() if x is not None else None for x in was]
    want_len = list(lens)
    for s, f in enumerate(source):
        lo = shared[s // G] if shared is not None else 0
        if f in (-1, s) or f // G != s // G or f < 0 or not 0 <= lens[f] <= C or not 0 <= lo <= C:
            continue
        n = lens[f]
        for i, x in enumerate(want):
            if x is None or (i == 0 and not keys) or (i == 1 and not values):
                continue
            if i < 2:
                x[s, :, lo:n] = was[i][f, :, lo:n]
            else:
                x[s, lo:n] = was[i][f, lo:n]
        want_len[s] = n
    B.sirllm_reorder_streams(cfg, G, i32(*source), i32(*shared) if shared is not None else None, E, T, live,
                             k if keys else None, v if values else None, ws)
    assert B.sirllm_status(ws) == want_status
    assert live.tolist() == want_len
    assert same_bits(k, want[0]) and same_bits(v, want[1])
    assert E is None or torch.equal(E, want[2])
    assert T is None or torch.equal(T, want[3])


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("D", [8, 40, 64, 128, 256, 512])
@pytest.mark.parametrize("source", [[0, 0, 2, 2], [0, 0, 0, 0], [1, 0, 3, 2], [1, 2, 3, 0], [3, 3, 0, 0], [0, 1, 2, 3],
                                    [-1, 0, -1, 2], [2, -1, 1, 1]])
def test_reorder_forks_swaps_and_cycles(kv, D, source):
    reorder_case(4, 4, source, [100, 37, 64, 1], D=D, kv=kv, seed=D)
    reorder_case(4, 4, source, [90, 90, 91, 90], shared=[33], D=D, kv=kv, seed=D)


@pytest.mark.parametrize("C,lens", [(1, [1, 0, 1]), (2, [0, 0, 0]), (1000, [999, 1000, 3]), (4001, [4001, 17, 2048])])
@pytest.mark.parametrize("source", [[1, 2, 0], [0, 0, 0], [2, 2, 2]])
def test_reorder_lengths(C, lens, source):
    reorder_case(3, 3, source, lens, C=C, L=1, KH=3, D=80, seed=C)


@pytest.mark.parametrize("shared", [[0, 50, 100, 7], [100, 100, 100, 100], [1, 99, 64, 33]])
def test_reorder_shared_slots_stay(shared):
    lens = [100, 80, 60, 99, 50, 51, 100, 1, 8, 7, 6, 100]
    reorder_case(12, 3, [0, 0, 1, 4, 3, 5, 8, 8, 8, 10, 11, 9], lens, shared=shared)


def test_reorder_many_groups_and_big_groups():
    g = torch.Generator()
    g.manual_seed(4)
    for S, G in ((1200, 2), (256, 256), (512, 128), (70, 35)):
        source = [s // G * G + int(torch.randint(0, G, (1,), generator=g)) for s in range(S)]
        lens = torch.randint(0, 41, (S,), generator=g).tolist()
        reorder_case(S, G, source, lens, C=40, L=1, KH=1, D=64, seed=S)
    perm = torch.randperm(256, generator=g).tolist()
    reorder_case(256, 256, perm, [40] * 256, C=40, L=1, KH=2, D=128, seed=1)


def test_reorder_parts_left_out():
    for kw in (dict(keys=False), dict(values=False), dict(keys=False, values=False), dict(tags=False),
               dict(scores=False), dict(tags=False, scores=False)):
        reorder_case(4, 2, [1, 0, 2, 2], [100, 50, 60, 70], **kw)


def test_reorder_bad_sources_and_lengths_leave_their_streams_alone():
    lens = [100, 50, 60, 70, 20, 30]
    reorder_case(6, 3, [0, 3, 0, 4, 3, 5], lens, want_status=B.STATUS_BAD_SOURCE)
    reorder_case(6, 3, [-2, 6, 2**31 - 1, -2**31, 3, 3], lens, want_status=B.STATUS_BAD_SOURCE)
    reorder_case(6, 3, [0, 0, 0, 4, 3, 3], [-1, 50, 60, 101, 20, 30], want_status=B.STATUS_OVERFLOW)
    reorder_case(6, 3, [1, 1, 1, 4, 4, 4], lens, shared=[-1, 10], want_status=B.STATUS_OVERFLOW)
    reorder_case(6, 3, [1, 1, 1, 4, 4, 4], lens, shared=[10, 101], want_status=B.STATUS_OVERFLOW)


def test_reorder_repeated_from_a_graph_follows_the_device():
    # lengths and sources travel through device memory: a cycle of four brings everything back
    S, C, D = 4, 600, 128
    cfg = config(S=S, L=3, KH=4, D=D, C=C)
    g = gen(8)
    k, v = (randn(g, S, 12, C, D, dtype=torch.bfloat16) for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    E = torch.rand(S, C, generator=g, device="cuda")
    E0, live, source = E.clone(), i32(600, 600, 600, 600), i32(1, 2, 3, 0)
    call = B.prepared(B.sirllm_reorder_streams, cfg, S, source, None, E, None, live, k, v, B.new_workspace(cfg))
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        graph.replay()
        if i == 0:
            assert same_bits(k, k0[[2, 3, 0, 1]]) and torch.equal(E, E0[[2, 3, 0, 1]])
    assert same_bits(k, k0) and same_bits(v, v0) and torch.equal(E, E0)
    live.copy_(i32(10, 20, 30, 40))
    graph.replay()
    assert live.tolist() == [20, 30, 40, 10]
    assert same_bits(k[0, :, :20], k0[1, :, :20]) and same_bits(k[0, :, 20:], k0[0, :, 20:])
    assert same_bits(k[3, :, :10], k0[0, :, :10]) and same_bits(k[3, :, 10:], k0[3, :, 10:])


def test_reorder_past_32_bits():
    # planes whose elements are counted beyond 2^31
    S, L, KH, D, C = 2, 64, 8, 512, 4800
    cfg = config(S=S, L=L, KH=KH, D=D, C=C)
    k = torch.zeros(S, L * KH, C, D, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2**31
    k[1, -1] = randn(gen(2), C, D, dtype=torch.bfloat16)
    k[1, :, 4799, 511] = torch.arange(L * KH, device="cuda").to(torch.bfloat16)
    live = i32(5, 4800)
    B.sirllm_reorder_streams(cfg, 2, i32(1, 1), i32(4000), None, None, live, k, None, B.new_workspace(cfg))
    assert live.tolist() == [4800, 4800]
    assert same_bits(k[0, :, 4000:], k[1, :, 4000:]) and not k[0, :, :4000].any()


# --------------------------------------------------------------------------------------
# attend
# --------------------------------------------------------------------------------------

PARTS_FROM = 160 * 2**20    # bytes of K and V of a layer from which on shared slots are computed once at any group


def capacities(S, KH, D, C):
    """The capacity as it is, and one that takes the other way through the call, where there is one."""
    need = PARTS_FROM // (S * KH * D * 4) + 1
    return [C] + ([need] if C < need <= B.MAX_CAPACITY else [])


def shared_case(S, G, H, KH, D, C, shared, lens, **kw):
    for c in capacities(S, KH, D, C):
        result = shared_once(S, G, H, KH, D, c, shared, lens, **kw)
    return result


def shared_once(S, G, H, KH, D, C, shared, lens, kv="bf16", L=1, layer=0, seed=0, scale=None, fill=None, some=None):
    g = gen(seed)
    dt = DT[kv]
    cfg = config(S=S, L=L, KH=KH, D=D, C=C, kv=kv)
    wide = randn(g, S, H + 3, D, dtype=dt)
    q = wide[:, 1:1 + H]
    k, v = randn(g, S, L, KH, C, D, dtype=dt), randn(g, S, L, KH, C, D, dtype=dt)
    if fill is not None:   # what is not to be read: behind a stream's slots, and in front of a follower's own
        for s, n in enumerate(lens):
            lo = shared[s // G]
            end = max(n, lo) if s % G == 0 else n
            for x in (k, v):
                x[s, :, :, end:] = fill
                if s % G:
                    x[s, :, :, :lo] = fill
    o_wide = torch.full((S, H + 2, D), 7.0, dtype=dt, device="cuda")
    out = o_wide[:, 2:]
    lse = torch.full((S, H), 7.0, device="cuda")
    ws = B.new_attend_shared_workspace(cfg, G, H)
    B.sirllm_attend_shared(cfg, layer, G, i32(*shared), q, k, v, i32(*lens), scale, out, lse, ws)
    assert B.sirllm_status(ws) == 0
    assert (o_wide[:, :2] == 7).all()
    scale = D ** -0.5 if scale is None else scale
    for s in range(S) if some is None else some:
        n, lo, first = lens[s], shared[s // G], s // G * G
        ks = torch.cat([k[first, layer, :, :min(lo, n)], k[s, layer, :, min(lo, n):n]], 1)
        vs = torch.cat([v[first, layer, :, :min(lo, n)], v[s, layer, :, min(lo, n):n]], 1)
        o, l, to, tl = ref_attend(q[s], ks, vs, n, scale)
        if n == 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            continue
        d = (out[s].double() - o).abs()
        assert (d <= to).all(), f"stream {s} ({n} slots, {lo} shared): worst {float((d / to).max()):.2f} x tol"
        d = (lse[s].double() - l).abs()
        assert (d <= tl).all(), f"stream {s} ({n} slots, {lo} shared): lse off by {float(d.max()):.3g}"
    return cfg, q, k, v, out, lse, ws


SHARED = [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 300, 511, 640]


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("D", [8, 40, 64, 80, 96, 128, 200, 256])
@pytest.mark.parametrize("G,group", [(2, 1), (3, 3), (4, 8), (16, 4), (5, 11), (33, 2)])
def test_shared_head_sizes_and_groups(kv, D, G, group):
    groups = 4 if G > 8 else len(SHARED)
    shared = (SHARED if groups > 4 else [300, 128, 0, 640])[:groups]
    S = G * groups
    lens = [shared[s // G] + (7 * s) % 90 for s in range(S)]
    shared_case(S, G, 2 * group, 2, D, 740, shared, lens, kv=kv, seed=D + G, fill=math.nan)


@pytest.mark.parametrize("H,KH", [(32, 8), (32, 32), (71, 1), (48, 8), (17, 1), (5, 5), (130, 1)])
@pytest.mark.parametrize("G", [2, 8, 40])
def test_shared_head_layouts(H, KH, G):
    lens = [2001 + (13 * s) % 300 for s in range(G)]
    shared_case(G, G, H, KH, 128, 2400, [2001], lens, L=2, layer=1, seed=H)


@pytest.mark.parametrize("G,group", [(4, 1), (16, 8), (64, 4)])
def test_shared_streams_shorter_than_the_shared_slots(G, group):
    # idle streams, streams that see a part of the shared slots only, and the shared slots alone
    shared = [700, 384]
    lens = [(0, 1, 100, 383, 384, 385, 699, 700, 701, 900)[s % 10] for s in range(2 * G)]
    shared_case(2 * G, G, 2 * group, 2, 128, 1000, shared, lens, seed=G)
    shared_case(2 * G, G, 2 * group, 2, 64, 1000, shared, [n if s % 3 else 0 for s, n in enumerate(lens)], kv="f16", seed=G)


@pytest.mark.parametrize("D", [64, 192])
@pytest.mark.parametrize("G,group", [(2, 4), (16, 4)])
def test_shared_streams_without_slots_of_their_own(D, G, group):
    # the shared slots are all that most streams see, whole tiles of them or not, or all that all do
    shared = [512, 777, 40]
    lens = [shared[s // G] + (s % 5 == 4) for s in range(3 * G)]
    shared_case(3 * G, G, 4 * group, 4, D, 800, shared, lens, seed=D + G, fill=math.nan)
    shared_case(3 * G, G, 4 * group, 4, D, 800, shared, [shared[s // G] for s in range(3 * G)], seed=D, fill=math.nan)


@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("G,group,KH", [(2, 16, 2), (2, 16, 16), (3, 10, 16), (8, 8, 16)])
def test_shared_groups_of_many_heads(D, G, group, KH):
    # units of one and of several blocks, with heads of a stream that two blocks share
    lens = [900 + 31 * s for s in range(2 * G)]
    shared_case(2 * G, G, group * KH, KH, D, 1400, [900, 333], lens, seed=D + group, fill=math.nan)


@pytest.mark.parametrize("G,C", [(8, 600), (4, 45000), (40, 6000)])
def test_shared_without_log_sums(G, C):
    cfg, q, k, v, out, lse, ws = shared_once(G, G, 4, 2, 64, C, [400], [401 + s for s in range(G)], seed=9)
    again = torch.zeros_like(out)
    B.sirllm_attend_shared(cfg, 0, G, i32(400), q, k, v, i32(*[401 + s for s in range(G)]), None, again, None, ws)
    assert same_bits(again, out)


@pytest.mark.parametrize("n,D", [(16384, 128), (48990, 64), (30011, 128)])
@pytest.mark.parametrize("G,H,KH", [(4, 8, 2), (64, 16, 2)])
def test_shared_long_prefixes(n, D, G, H, KH):
    lens = [n + (5 * s) % 150 for s in range(G)]
    shared_case(G, G, H, KH, D, n + 160, [n], lens, seed=n + G, some=range(0, G, 7))


def test_shared_ragged_groups_of_very_different_prefixes():
    shared = [0, 5000, 130, 20, 3333, 1, 1024, 2047]
    G = 24
    lens = [shared[s // G] + (11 * s) % 40 for s in range(8 * G)]
    shared_case(8 * G, G, 8, 2, 128, 5100, shared, lens, seed=3, some=range(0, 8 * G, 5), fill=math.inf)


def test_shared_one_stream_per_group_is_attend():
    S, H, KH, D, C = 6, 8, 2, 128, 700
    shared = [0, 10, 128, 300, 512, 700]
    cfg, q, k, v, out, lse, ws = shared_once(S, 1, H, KH, D, C, shared, [700] * 6, seed=5)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    B.sirllm_attend(cfg, 0, q, k, v, i32(*[700] * 6), None, o2, l2, B.new_attend_workspace(cfg))
    tol = ref_attend(q[0], k[0, 0], v[0, 0], 700, D ** -0.5)[2]
    assert (out.double() - o2.double()).abs().max() <= 2 * tol.max()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 30.0])
@pytest.mark.parametrize("kv", ["bf16", "f16"])
def test_shared_scales(scale, kv):
    shared_case(32, 32, 8, 2, 64, 700, [500], [500 + s for s in range(32)], kv=kv, scale=scale, seed=11)


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("cap", [4000, 24000])
def test_shared_scores_that_keep_rising_and_falling(kv, order, cap):
    g = gen(12)
    S, H, KH, D, C, n = 32, 8, 1, 64, cap, 3900
    cfg = config(S=S, KH=KH, D=D, C=C, kv=kv)
    q = torch.zeros(S, H, D, dtype=DT[kv], device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(S, 1, KH, C, D, dtype=DT[kv], device="cuda")
    k[..., :4000, 0] = torch.linspace(-2000, 2000, 4000, device="cuda") * order
    v = randn(g, S, 1, KH, C, D, dtype=DT[kv])
    out, lse = torch.empty_like(q), torch.empty(S, H, device="cuda")
    B.sirllm_attend_shared(cfg, 0, S, i32(n), q, k, v, i32(*[4000] * S), 1.0, out, lse,
                           B.new_attend_shared_workspace(cfg, S, H))
    for s in (0, 5, 31):
        ks, vs = torch.cat([k[0, 0, :, :n], k[s, 0, :, n:]], 1), torch.cat([v[0, 0, :, :n], v[s, 0, :, n:]], 1)
        o, l, to, tl = ref_attend(q[s], ks, vs, 4000, 1.0)
        assert ((out[s].double() - o).abs() <= to).all() and ((lse[s].double() - l).abs() <= tl).all()


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("G,H,at", [(2, 1, 5), (64, 4, 5), (64, 4, 16000), (64, 4, 16500)])
@pytest.mark.parametrize("faint", [22.0, 25.5, 30.0])
@pytest.mark.parametrize("KH", [1, 2, 19])
def test_shared_one_dominant_slot_and_many_faint_ones(kv, G, H, at, KH, faint):
    # as for sirllm_attend: an fp16 weight is off by u of itself or by 2^-36 of the maximum
    g = gen(17)
    n, C, D, dt = 16384, 16600, 64, DT[kv]
    H = H * KH
    cfg = config(S=G, KH=KH, D=D, C=C, kv=kv)
    q = torch.zeros(G, H, D, dtype=dt, device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(G, 1, KH, C, D, dtype=dt, device="cuda")
    k[..., at, 0] = 1.0
    v = (1 + randn(g, 1, 1, 1, C, D, scale=0.2)).to(dt).expand(G, 1, KH, C, D).contiguous()
    v[..., at, :] = 0.0
    scale = faint * math.log(2)
    out, lse = torch.empty_like(q), torch.empty(G, H, device="cuda")
    B.sirllm_attend_shared(cfg, 0, G, i32(n), q, k, v, i32(*[C] * G), scale, out, lse,
                           B.new_attend_shared_workspace(cfg, G, H))
    want, l, tol, tol_l = ref_attend(q[0], k[0, 0], v[0, 0], C, scale)
    tol = tol + 2.0 ** -36 * v[0, 0, 0].double().abs().sum(-2).amax()
    d = (out.double() - want).abs()
    assert (d <= tol).all(), f"worst {float((d / tol).max()):.2f} x tol"
    assert ((lse.double() - l).abs() <= tol_l).all()


@pytest.mark.parametrize("G,cap", [(2, 300), (16, 45000), (64, 300), (64, 12000)])
def test_shared_infinite_scores_follow_the_formula(G, cap):
    n, C = 256, 300
    cfg = config(S=G, D=64, C=cap)
    ws = B.new_attend_shared_workspace(cfg, G, 1)
    q = torch.ones(G, 1, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(G, 1, 1, cap, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.arange(cap, device="cuda").view(1, 1, 1, cap, 1).expand(G, 1, 1, cap, 64).to(torch.bfloat16).contiguous()
    out, lse = torch.empty_like(q), torch.empty(G, 1, device="cuda")
    shared = i32(n)
    k[0, 0, 0, 5:, 0] = -math.inf          # of the shared slots only the first five weigh
    k[1:, 0, 0, n:, 0] = -math.inf
    B.sirllm_attend_shared(cfg, 0, G, shared, q, k, v, i32(*[C] * G), 1.0, out, lse, ws)
    assert (out == 2.0).all() and ((lse - math.log(5)).abs() < 1e-6).all()
    k[0, 0, 0, :n, 0] = -math.inf          # none of them: the stream's own slots alone
    k[1:, 0, 0, 256, 0] = 0.0
    B.sirllm_attend_shared(cfg, 0, G, shared, q, k, v, i32(*[C] * G), 1.0, out, lse, ws)
    assert (out[1:] == 256.0).all() and (lse[1:].abs() < 1e-6).all()
    k[0, 0, 0, 200, 0] = math.nan
    B.sirllm_attend_shared(cfg, 0, G, shared, q, k, v, i32(*[C] * G), 1.0, out, lse, ws)
    assert out.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("G,group,C", [(2, 2, 200), (32, 2, 200), (32, 1, 5200), (32, 2, 5200)])
def test_shared_lengths_outside_the_planes_leave_their_rows_alone(G, group, C):
    S, H, KH, D = 2 * G, 2 * group, 2, 64
    cfg, q, k, v, out, lse, ws = shared_once(S, G, H, KH, D, C, [150, 130], [200] * S, seed=4)
    want, want_l = out.clone(), lse.clone()
    lens = [200] * S
    lens[1], lens[G] = C + 1, -1
    out.fill_(3.0), lse.fill_(3.0)
    B.sirllm_attend_shared(cfg, 0, G, i32(150, 130), q, k, v, i32(*lens), None, out, lse, ws)
    assert B.sirllm_status(ws, clear=True) == B.STATUS_OVERFLOW
    for s in range(S):
        if s in (1, G):
            assert (out[s] == 3).all() and (lse[s] == 3).all()
        else:
            assert same_bits(out[s], want[s]) and torch.equal(lse[s], want_l[s])
    for bad in (-1, C + 1, 2**31 - 1, -2**31):
        out.fill_(3.0), lse.fill_(3.0)
        B.sirllm_attend_shared(cfg, 0, G, i32(bad, 130), q, k, v, i32(*[200] * S), None, out, lse, ws)
        assert B.sirllm_status(ws, clear=True) == B.STATUS_OVERFLOW
        assert (out[:G] == 3).all() and (lse[:G] == 3).all()
        assert (out[G:].double() - want[G:].double()).abs().max() <= 2 ** -7


@pytest.mark.parametrize("G,KH,C", [(3, 2, 1500), (6, 8, 3600), (48, 2, 1500), (48, 2, 1800)])
def test_shared_graph_replays_follow_the_device_and_repeat_bits(G, KH, C):
    S, H, D = 2 * G, 4 * KH, 128
    shared, lens = i32(1000, 600), i32(*[1000 + s % 400 if s < G else 600 + s % 99 for s in range(S)])
    cfg, q, k, v, out, lse, ws = shared_once(S, G, H, KH, D, C, shared.tolist(), lens.tolist(), seed=6)
    want, want_l = out.clone(), lse.clone()
    call = B.prepared(B.sirllm_attend_shared, cfg, 0, G, shared, q, k, v, lens, None, out, lse, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for _ in range(10):
        out.zero_(), lse.zero_()
        graph.replay()
        assert same_bits(out, want) and torch.equal(lse, want_l)
    shared.copy_(i32(100, 1400)), lens.fill_(1450)
    graph.replay()
    eager, eager_l = torch.empty_like(out), torch.empty_like(lse)
    B.sirllm_attend_shared(cfg, 0, G, i32(100, 1400), q, k, v, i32(*[1450] * S), None, eager, eager_l,
                           B.new_attend_shared_workspace(cfg, G, H))
    assert same_bits(out, eager) and torch.equal(lse, eager_l)


@pytest.mark.parametrize("C", [2600, 10500])
def test_shared_on_two_streams_at_once(C):
    S = G = 32
    a = shared_once(S, G, 8, 2, 128, C, [2500], [2501 + s for s in range(S)], seed=21)
    b = shared_once(S, G, 8, 2, 64, C, [2300], [2301 + s for s in range(S)], kv="f16", seed=22)
    calls, wants = [], []
    for (cfg, q, k, v, out, lse, ws), n in ((a, 2500), (b, 2300)):
        wants.append((out.clone(), lse.clone()))
        calls.append(B.prepared(B.sirllm_attend_shared, cfg, 0, G, i32(n), q, k, v, i32(*[n + 1 + s for s in range(S)]),
                                None, out, lse, ws))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(50):
        for st, call in zip(streams, calls):
            with torch.cuda.stream(st):
                call()
    torch.cuda.synchronize()
    for x, (o, l) in zip((a, b), wants):
        assert same_bits(x[4], o) and torch.equal(x[5], l)


# --------------------------------------------------------------------------------------
# together
# --------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,prompt", [(4, 37), (12, 300)])
def test_a_beam_search_step_by_step(G, prompt):
    """Two prompts, one layer of a toy model: append, attend over the shared prompt, logits, selection,
    reordering; against the same search that keeps every beam's tokens and recomputes its attention from the
    whole history."""
    S, H, KH, D, C, V, steps = 2 * G, 8, 2, 64, prompt + 16, 211, 9
    g = gen(31)
    dt = torch.float16
    cfg = config(S=S, KH=KH, D=D, C=C, V=V, kv="f16")
    ws, bws, aws = B.new_workspace(cfg), B.new_beam_workspace(cfg), B.new_attend_shared_workspace(cfg, G, H)
    emb = randn(g, V, (H + 2 * KH) * D, scale=0.5)
    head = randn(g, V, H * D, scale=0.25)
    k, v = (torch.zeros(S, 1, KH, C, D, dtype=dt, device="cuda") for _ in range(2))
    E = torch.zeros(S, C, device="cuda")
    tags = torch.full((S, C), -1, dtype=torch.int64, device="cuda")
    past = torch.randint(0, V, (2, prompt), generator=g, device="cuda")
    shared = i32(prompt - 1, prompt - 1)          # the prompt's last token is each beam's first query
    pcfg = config(S=2, KH=KH, D=D, C=C, V=V, kv="f16", M=prompt)
    rows = emb[past].view(2 * prompt, H + 2 * KH, D).to(dt)
    pk, pv = (torch.zeros(2, 1, KH, C, D, dtype=dt, device="cuda") for _ in range(2))
    B.sirllm_append_kv(pcfg, 0, None, rows[:, H:H + KH], rows[:, H + KH:], None, None, 0.0, 1e4, B.ROPE_HALF, i32(0, 0),
                       i32(prompt - 1, prompt - 1), None, pk, pv, B.new_workspace(pcfg))
    k[::G], v[::G] = pk, pv
    live = i32(*[prompt - 1] * S)
    tokens = past[:, -1].repeat_interleave(G).to(torch.int32)
    totals = torch.full((S,), -math.inf, device="cuda")
    totals[::G] = 0.0
    ended = torch.zeros(S, dtype=torch.int32, device="cuda")
    history = [[past[s // G, -1].item()] for s in range(S)]
    src, tok, fin = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(3))
    ent, out = torch.zeros(S, device="cuda"), torch.zeros(S, H, D, dtype=dt, device="cuda")
    q_out = torch.zeros_like(out)
    for step in range(steps):
        qkv = emb[tokens.long().clamp(min=0)].view(S, H + 2 * KH, D).to(dt)
        B.sirllm_append_kv(cfg, 0, qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:], None, None, 0.0, 1e4, B.ROPE_HALF, live,
                           None, q_out, k, v, ws)
        E.scatter_(1, live.long()[:, None], ent[:, None])
        tags.scatter_(1, live.long()[:, None], tokens.long()[:, None])
        live += 1
        B.sirllm_attend_shared(cfg, 0, G, shared, q_out, k, v, live, None, out, None, aws)
        # the same from the tokens alone: whole histories, rotated and attended in a cache of one's own
        fcfg = config(S=S, KH=KH, D=D, C=C, V=V, kv="f16", M=prompt + step)
        whole = torch.stack([torch.cat([past[s // G, :-1], torch.tensor(history[s], device="cuda")]) for s in range(S)])
        frows = emb[whole.clamp(min=0)].view(-1, H + 2 * KH, D).to(dt)
        fk, fv = (torch.zeros(S, 1, KH, C, D, dtype=dt, device="cuda") for _ in range(2))
        B.sirllm_append_kv(fcfg, 0, None, frows[:, H:H + KH], frows[:, H + KH:], None, None, 0.0, 1e4, B.ROPE_HALF,
                           i32(*[0] * S), None, None, fk, fv, B.new_workspace(fcfg))
        for s in range(S):
            if totals[s] > -math.inf:
                o, _, to, _ = ref_attend(q_out[s], fk[s, 0], fv[s, 0], prompt + step, D ** -0.5)
                assert ((out[s].double() - o).abs() <= to).all(), (step, s)
        logits = (out.view(S, -1).float() @ head.t()).contiguous()
        want = ref_select(logits, G, G, totals, ended, END, True)
        B.sirllm_beam_select(cfg, logits, G, G, totals, ended, END, True, totals, src, tok, ent, ended, bws)
        assert src.tolist() == [f[1] for f in want] and tok.tolist() == [f[2] for f in want]
        assert ended.tolist() == [f[4] for f in want]
        B.sirllm_reorder_streams(cfg, G, src, shared, E, tags, live, k, v, ws)
        history = [history[max(f, 0)] + [t] for f, t in zip(src.tolist(), tok.tolist())]
        tokens.copy_(tok)
        for s in range(S):   # tags and entropies followed their beams
            assert tags[s, prompt - 1:prompt + step].tolist() == history[s][:-1]
    assert B.sirllm_status(ws) == 0 and B.sirllm_status(aws) == 0 and B.sirllm_status(bws) == 0
    # the winner goes back to the stream that holds the prompt: a plain cache again
    best = [int(totals[i * G:(i + 1) * G].argmax()) + i * G for i in range(2)]
    B.sirllm_reorder_streams(cfg, G, i32(*[best[s // G] if s % G == 0 else -1 for s in range(S)]), shared, E, tags, live, k,
                             v, ws)
    for i in range(2):
        assert tags[i * G, prompt - 1:prompt + steps - 1].tolist() == history[best[i]][:-1]
        assert int(live[i * G]) == prompt - 1 + steps
