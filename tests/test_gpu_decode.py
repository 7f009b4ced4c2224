"""The calls of a decode step around the cache, on the GPU, against plain forms in 64 bits:
``sirllm_append_kv``, ``sirllm_attend``, ``sirllm_head_pairs``, and a run of them together.

Tolerances.  ``u`` is half a step of the 16-bit type.  append: fp32 arithmetic and one rounding:
u * |want| plus 2e-6 of the pair's length (a dozen fp32 roundings of 2^-24, 7.2e-7, and sine and
cosine off by 5.5e-7 together in their fast forms and 3e-7 for the angle in fp32).  attend: the weights of the second product are rounded to 16 bits (u of
sum p|V|), the result once more (u of |out|), and an error dz of the scores moves the weights by
2 dz; dz is D products and sums in fp32, 2^-23 D sum|q k| scale at the very most.  head: the
framework's bound for scores, plus the random walk of d fp32 roundings."""
import math

import pytest
import torch

from paper_2405_12528_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
F64 = torch.float64


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def config(S=1, L=1, KH=1, D=64, C=256, M=1, V=16, kv="bf16"):
    return B.make_config(n_streams=S, n_layers=L, n_kv_heads=KH, head_dim=D, capacity=C, budget=C, n_sink=0,
                         n_recent=0, max_new=M, vocab=V, logits_dtype="f32", kv_dtype=kv)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


# --------------------------------------------------------------------------------------
# append
# --------------------------------------------------------------------------------------

def ref_rope(x, w, pos, eps, base, layout):
    """[T, heads, D] fp64, positions [T] -> normalised and turned, and each element's pair length."""
    if w is not None:
        x = x * w.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    D = x.shape[-1]
    i = torch.arange(D // 2, device=x.device)
    a, b = (i, i + D // 2) if layout == B.ROPE_HALF else (2 * i, 2 * i + 1)
    ang = pos.to(F64)[:, None, None] * torch.pow(torch.tensor(base, dtype=F64, device=x.device), -2.0 * i.to(F64) / D)
    out, length = torch.empty_like(x), torch.empty_like(x)
    out[..., a] = x[..., a] * torch.cos(ang) - x[..., b] * torch.sin(ang)
    out[..., b] = x[..., a] * torch.sin(ang) + x[..., b] * torch.cos(ang)
    length[..., a] = length[..., b] = torch.hypot(x[..., a], x[..., b])
    return out, length


def assert_turned(got, want, length):
    u = half_step(got.dtype)
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps / 2    # half a subnormal step
    tol = u * want.abs() + 2e-6 * length + tiny
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} off, worst {float(((got.double() - want).abs() / tol).max()):.2f} x tol"


APPEND = [  # S, M, H, KH, D, first, capacity
    (1, 1, 1, 1, 16, [0], 1),
    (1, 1, 32, 8, 128, [12001], 16384),
    (1, 1, 4, 4, 256, [49151], 49152),
    (3, 7, 6, 2, 80, [0, 100, 249], 256),
    (5, 33, 12, 4, 48, [3, 0, 17, 200, 31], 256),
    (2, 300, 8, 1, 64, [40000, 5], 40300),
    (2, 3, 2, 2, 512, [11, 0], 14),
    (4, 5, 3, 3, 112, [0, 1, 2, 3], 9),
    (2, 200, 40, 3, 512, [0, 7], 210),       # more heads than one block takes
    (300, 1, 5, 5, 32, [17] * 300, 20),
]


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("layout", [B.ROPE_HALF, B.ROPE_INTERLEAVED])
@pytest.mark.parametrize("norms", ["none", "both", "q", "k"])
@pytest.mark.parametrize("shape", APPEND)
def test_append_against_64_bits(kv, layout, norms, shape):
    S, M, H, KH, D, first, C = shape
    dt, g = DT[kv], gen(sum(first) + D)
    cfg = config(S=S, L=2, KH=KH, D=D, C=C, M=M, kv=kv)
    qkv = randn(g, S * M, H + 2 * KH, D, dtype=dt)
    q, kn, vn = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
    wq = randn(g, D, dtype=dt) if norms in ("both", "q") else None
    wk = randn(g, D, dtype=dt) if norms in ("both", "k") else None
    k, v = randn(g, S, 2, KH, C, D, dtype=dt), randn(g, S, 2, KH, C, D, dtype=dt)
    q_out = randn(g, S * M, H, D, dtype=dt)
    k0, v0, q0 = k.clone(), v.clone(), q_out.clone()
    n_new = [M - (s % 3) if M > 3 else (M if s == 0 else s % (M + 1)) for s in range(S)]
    ws = B.new_workspace(cfg)
    B.sirllm_append_kv(cfg, 1, q, kn, vn, wq, wk, 1e-5, 500000.0, layout, i32(*first), i32(*n_new), q_out, k, v, ws)
    assert B.sirllm_status(ws) == 0
    for s in range(S):
        n, f = n_new[s], first[s]
        r = slice(s * M, s * M + n)
        pos = torch.arange(f, f + n, device="cuda")
        assert_turned(q_out[r], *ref_rope(q[r].double(), wq, pos, 1e-5, 500000.0, layout))
        want, length = ref_rope(kn[r].double(), wk, pos, 1e-5, 500000.0, layout)
        assert_turned(k[s, 1, :, f:f + n], want.transpose(0, 1), length.transpose(0, 1))
        assert same_bits(v[s, 1, :, f:f + n], vn[r].transpose(0, 1))
        # nothing else moved: rows behind the stream's last, other slots, the other layer
        assert same_bits(q_out[s * M + n:(s + 1) * M], q0[s * M + n:(s + 1) * M])
        k[s, 1, :, f:f + n] = k0[s, 1, :, f:f + n]
        v[s, 1, :, f:f + n] = v0[s, 1, :, f:f + n]
    assert same_bits(k, k0) and same_bits(v, v0)


def test_append_without_lengths_without_queries_and_in_place():
    g = gen(3)
    S, M, H, KH, D, C = 2, 4, 6, 3, 64, 16
    cfg = config(S=S, KH=KH, D=D, C=C, M=M)
    ws = B.new_workspace(cfg)
    q, kn, vn = (randn(g, S * M, h, D, dtype=torch.bfloat16) for h in (H, KH, KH))
    k, v = (torch.zeros(S, 1, KH, C, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty_like(q)
    first = i32(12, 0)
    B.sirllm_append_kv(cfg, 0, q, kn, vn, None, None, 0.0, 1e4, B.ROPE_HALF, first, None, out, k, v, ws)
    k2, v2, q2 = torch.zeros_like(k), torch.zeros_like(v), q.clone()
    B.sirllm_append_kv(cfg, 0, None, kn, vn, None, None, 0.0, 1e4, B.ROPE_HALF, first, None, None, k2, v2, ws)
    assert same_bits(k, k2) and same_bits(v, v2)
    B.sirllm_append_kv(cfg, 0, q2, kn, vn, None, None, 0.0, 1e4, B.ROPE_HALF, first, None, q2, k2, v2, ws)
    assert same_bits(q2, out) and B.sirllm_status(ws) == 0
    assert k[0, 0, :, 12:].abs().sum() > 0 and k[0, 0, :, :12].abs().sum() == 0


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("S,M,H,KH,D", [(1, 1, 32, 8, 128), (3, 5, 6, 2, 80), (2, 300, 5, 1, 512)])
def test_append_rows_of_every_tensor_at_a_distance_of_their_own(kv, norms, S, M, H, KH, D):
    g, dt, C = gen(6), DT[kv], 310
    cfg = config(S=S, KH=KH, D=D, C=C, M=M, kv=kv)
    wide = [randn(g, S * M + 2, h, D, dtype=dt) for h in (H + 3, KH + 1, KH + 5)]
    q, kn, vn = wide[0][:S * M, 2:2 + H], wide[1][:S * M, 1:], wide[2][:S * M, 3:3 + KH]
    wq, wk = (randn(g, D, dtype=dt), randn(g, D, dtype=dt)) if norms else (None, None)
    out = randn(g, S * M + 1, H + 4, D, dtype=dt)
    before, q_out = out.clone(), out[:, 1:1 + H]
    k, v = (torch.zeros(S, 1, KH, C, D, dtype=dt, device="cuda") for _ in range(2))
    ws = B.new_workspace(cfg)
    first = [3 + s for s in range(S)]
    B.sirllm_append_kv(cfg, 0, q, kn, vn, wq, wk, 1e-6, 1e4, B.ROPE_HALF, i32(*first), None, q_out, k, v, ws)
    assert B.sirllm_status(ws) == 0
    for s in range(S):
        r, f = slice(s * M, s * M + M), first[s]
        pos = torch.arange(f, f + M, device="cuda")
        assert_turned(q_out[r], *ref_rope(q[r].double(), wq, pos, 1e-6, 1e4, B.ROPE_HALF))
        want, length = ref_rope(kn[r].double(), wk, pos, 1e-6, 1e4, B.ROPE_HALF)
        assert_turned(k[s, 0, :, f:f + M], want.transpose(0, 1), length.transpose(0, 1))
        assert same_bits(v[s, 0, :, f:f + M], vn[r].transpose(0, 1))
    assert same_bits(out[:, :1], before[:, :1]) and same_bits(out[:, 1 + H:], before[:, 1 + H:])
    assert same_bits(out[S * M:], before[S * M:])
    # in place, in rows that are wider than their heads
    turned, tail = q_out[:S * M].clone(), wide[0][S * M:].clone()
    B.sirllm_append_kv(cfg, 0, q, kn, vn, wq, wk, 1e-6, 1e4, B.ROPE_HALF, i32(*first), None, q, k, v, ws)
    assert same_bits(q, turned) and same_bits(wide[0][S * M:], tail)


@pytest.mark.parametrize("first,n", [(-1, 1), (61, 4), (64, 1), (2**31 - 1, 1)])
def test_append_that_does_not_fit_skips_the_stream_and_reports_it(first, n):
    g = gen(4)
    cfg = config(S=2, KH=2, D=32, C=64, M=4)
    ws = B.new_workspace(cfg)
    q, kn, vn = (randn(g, 8, h, 32, dtype=torch.bfloat16) for h in (4, 2, 2))
    k, v = (randn(g, 2, 1, 2, 64, 32, dtype=torch.bfloat16) for _ in range(2))
    out = randn(g, 8, 4, 32, dtype=torch.bfloat16)
    k0, v0, out0 = k.clone(), v.clone(), out.clone()
    B.sirllm_append_kv(cfg, 0, q, kn, vn, None, None, 1e-6, 1e4, B.ROPE_HALF, i32(first, 60), i32(n, 4), out, k, v, ws)
    assert B.sirllm_status(ws, clear=True) == B.STATUS_OVERFLOW
    assert same_bits(k[0], k0[0]) and same_bits(v[0], v0[0]) and same_bits(out[:4], out0[:4])
    assert same_bits(v[1, 0, :, 60:], vn[4:].transpose(0, 1)) and not same_bits(out[4:], out0[4:])
    # a stream without new tokens is not looked at
    B.sirllm_append_kv(cfg, 0, q, kn, vn, None, None, 1e-6, 1e4, B.ROPE_HALF, i32(first, 60), i32(0, 4), out, k, v, ws)
    assert B.sirllm_status(ws) == 0


@pytest.mark.parametrize("layout", [B.ROPE_HALF, B.ROPE_INTERLEAVED])
def test_append_angles_where_a_pair_nearly_cancels(layout):
    # a pair (sin, cos) of its own angle turns to (0, 1): what is left of the first element shows the
    # error of the angle, the sine and the cosine, far below the rounding of the 16-bit type.  Bound, of
    # the pair's length: hypot(2^-21.19, 2^-21.41) for the fast cosine and sine; for the angle 2^-26 of a
    # turn (its fraction in fp32), pi times the error of 2pi in fp32, half a step below 4 for their
    # product; 2^-25 for the one product that is rounded by itself (at most half the length).
    M, D = 49152, 128
    cfg = config(D=D, C=M, M=M, kv="f16")
    pos = torch.arange(M, device="cuda")
    i = torch.arange(D // 2, device="cuda")
    a, b = (i, i + D // 2) if layout == B.ROPE_HALF else (2 * i, 2 * i + 1)
    ang = pos.to(F64)[:, None] * torch.pow(torch.tensor(1e4, dtype=F64, device="cuda"), -2.0 * i.to(F64) / D)
    kn = torch.empty(M, 1, D, dtype=torch.float16, device="cuda")
    kn[:, 0, a], kn[:, 0, b] = torch.sin(ang).half(), torch.cos(ang).half()
    k, v = (torch.zeros(1, 1, 1, M, D, dtype=torch.float16, device="cuda") for _ in range(2))
    ws = B.new_workspace(cfg)
    B.sirllm_append_kv(cfg, 0, None, kn, kn, None, None, 0.0, 1e4, layout, i32(0), None, None, k, v, ws)
    want, length = ref_rope(kn.double(), None, pos, 0.0, 1e4, layout)
    got = k[0, 0, 0, :, a].double()
    want, length = want[:, 0, a], length[:, 0, a]
    turn = float(torch.tensor(2 * math.pi, dtype=torch.float32))
    angle = 2.0 ** -26 * 2 * math.pi + abs(turn / (2 * math.pi) - 1) * math.pi + 2.0 ** -23
    bound = math.hypot(2 ** -21.19, 2 ** -21.41) + angle + 2.0 ** -25
    tol = half_step(torch.float16) * want.abs() + bound * length + 2.0 ** -25
    d = (got - want).abs()
    assert (d <= tol).all(), f"worst {float((d / tol).max()):.3f} x tol"


def test_append_equals_the_rerotated_key_of_another_slot():
    # a key written at slot p and turned by sirllm_rerotate_keys to slot j is the key written at j,
    # up to the two extra roundings
    g = gen(5)
    D, C = 128, 4096
    cfg = config(KH=4, D=D, C=C, M=1, kv="f16")
    ws = B.new_workspace(cfg)
    kn = randn(g, 1, 4, D, dtype=torch.float16)
    k = torch.zeros(1, 1, 4, C, D, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    for layout in (B.ROPE_HALF, B.ROPE_INTERLEAVED):
        B.sirllm_append_kv(cfg, 0, None, kn, kn, None, None, 0.0, 1e4, layout, i32(7), None, None, k, v, ws)
        want = k[0, 0, :, 7].clone()
        B.sirllm_append_kv(cfg, 0, None, kn, kn, None, None, 0.0, 1e4, layout, i32(4000), None, None, k, v, ws)
        keep = torch.arange(C, dtype=torch.int32, device="cuda")
        keep[7] = 4000
        k[0, 0, :, 7] = k[0, 0, :, 4000]
        B.sirllm_rerotate_keys(cfg, k, keep, i32(8), 1e4, layout)
        pair = float(want.double().abs().max()) * math.sqrt(2)
        assert (k[0, 0, :, 7].double() - want.double()).abs().max() <= 3 * half_step(torch.float16) * pair


# --------------------------------------------------------------------------------------
# attend
# --------------------------------------------------------------------------------------

def ref_attend(q, k, v, n, scale):
    """One stream, fp64: q [H, D], k, v [KH, C, D] -> out, lse, tolerances of both."""
    H, D = q.shape
    KH = k.shape[0]
    u = half_step(q.dtype)
    if n == 0:
        return (torch.zeros(H, D, dtype=F64, device=q.device), torch.full((H,), -math.inf, dtype=F64, device=q.device),
                torch.zeros(H, D, dtype=F64, device=q.device), torch.zeros(H, dtype=F64, device=q.device))
    qd = q.double().view(KH, H // KH, D)
    kd, vd = k[:, :n].double(), v[:, :n].double()
    z = torch.einsum("ghd,gcd->ghc", qd, kd) * scale
    p = torch.softmax(z, -1)
    out = torch.einsum("ghc,gcd->ghd", p, vd)
    spread = torch.einsum("ghc,gcd->ghd", p, vd.abs())
    lse = torch.logsumexp(z, -1)
    dz = torch.einsum("ghd,gcd->ghc", qd.abs(), kd.abs()).amax(-1) * abs(scale) * D * 2.0 ** -23
    dz = dz + (z.abs().amax(-1) + 1) * 2.0 ** -22                       # scaling, exponent of two, its argument
    sums = (n / 16 + 64) * 2.0 ** -24
    tol = u * out.abs() + (u + 2 * dz + 2 * sums)[..., None] * spread + torch.finfo(q.dtype).smallest_normal * u
    return (out.reshape(H, D), lse.reshape(H), tol.reshape(H, D),
            (dz + sums + lse.abs() * 2.0 ** -22).reshape(H))


def check_attend(q, k, v, lens, scale, out, lse, layer=0):
    for s, n in enumerate(lens):
        o, l, to, tl = ref_attend(q[s], k[s, layer], v[s, layer], n, scale)
        if n == 0:
            assert (out[s] == 0).all() and (lse is None or (lse[s] == -math.inf).all())
            continue
        d = (out[s].double() - o).abs()
        assert (d <= to).all(), f"stream {s} ({n} slots): worst {float((d / to).max()):.2f} x tol"
        if lse is not None:
            d = (lse[s].double() - l).abs()
            assert (d <= tl).all(), f"stream {s} ({n} slots): lse off by {float(d.max()):.3g}"


def attend_case(S, H, KH, D, C, lens, kv="bf16", L=1, layer=0, seed=0, scale=None, q_scale=1.0, fill=None):
    g = gen(seed)
    dt = DT[kv]
    cfg = config(S=S, L=L, KH=KH, D=D, C=C, kv=kv)
    wide = randn(g, S, H + 3, D, dtype=dt, scale=q_scale)       # rows further apart than their heads
    q = wide[:, 1:1 + H]
    k, v = randn(g, S, L, KH, C, D, dtype=dt), randn(g, S, L, KH, C, D, dtype=dt)
    if fill is not None:                                        # what lies behind the live slots
        for s, n in enumerate(lens):
            k[s, :, :, n:] = fill
            v[s, :, :, n:] = fill
    o_wide = torch.full((S, H + 2, D), 7.0, dtype=dt, device="cuda")
    out = o_wide[:, 2:]
    lse = torch.full((S, H), 7.0, device="cuda")
    ws = B.new_attend_workspace(cfg)
    B.sirllm_attend(cfg, layer, q, k, v, i32(*lens), scale, out, lse, ws)
    assert B.sirllm_status(ws) == 0
    assert (o_wide[:, :2] == 7).all()
    check_attend(q, k, v, lens, D ** -0.5 if scale is None else scale, out, lse, layer)
    return cfg, q, k, v, out, lse, ws


LENS = [0, 1, 2, 15, 16, 17, 31, 127, 128, 129, 1000]


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("D", [8, 40, 64, 80, 96, 128, 200, 256])
@pytest.mark.parametrize("group", [1, 3, 8, 11, 16])
def test_attend_head_sizes_and_groups(kv, D, group):
    attend_case(len(LENS), 2 * group, 2, D, 1000, LENS, kv=kv, seed=D + group, fill=math.nan)


@pytest.mark.parametrize("H,KH", [(32, 8), (32, 32), (71, 1), (48, 8), (17, 1), (5, 5), (130, 2)])
def test_attend_head_layouts(H, KH):
    attend_case(2, H, KH, 128, 3000, [2999, 1234], L=2, layer=1, seed=H)


@pytest.mark.parametrize("n", [1, 16, 4096, 16383, 49152])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attend_one_long_stream(n, D):
    attend_case(1, 4, 1, D, 49152, [n], seed=n + D)


def test_attend_many_streams_of_all_lengths():
    g = torch.Generator()
    g.manual_seed(1)
    lens = torch.randint(0, 300, (700,), generator=g)
    lens[torch.randint(0, 700, (300,), generator=g)] = 0
    attend_case(700, 4, 2, 64, 300, lens.tolist(), seed=8, fill=math.inf)


@pytest.mark.parametrize("D,group", [(64, 1), (128, 1), (128, 4), (96, 8), (128, 11), (40, 3)])
@pytest.mark.parametrize("longest", [20, 300, 512])
def test_attend_many_short_units(D, group, longest):
    S, KH = 180, 8                                                      # more units than warps
    lens = [(37 * s) % (longest + 1) for s in range(S)]
    attend_case(S, KH * group, KH, D, longest, lens, kv="f16" if D == 96 else "bf16", seed=D + group, fill=math.nan)
    attend_case(S, KH * group, KH, D, longest, [longest] * S, seed=D)


def test_attend_only_the_last_stream_has_slots():
    attend_case(600, 2, 1, 64, 40, [0] * 599 + [33], seed=9)
    attend_case(5, 2, 1, 128, 40, [0] * 5, seed=9)


@pytest.mark.parametrize("S,KH", [(1, 1), (1, 8), (3, 5), (1, 16), (2, 15), (3, 11), (1, 34), (2, 30), (2, 37), (5, 15),
                                  (4, 37), (1, 149)])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_however_the_units_are_dealt_out(S, KH, D):
    # whole units per CTA, per cluster of 2, 4 or 8, or shares of the line: even and uneven lengths
    attend_case(S, 2 * KH, KH, D, 3100, [3100 - 3 * s for s in range(S)], seed=S * KH)
    attend_case(S, KH, KH, D, 3100, [[3000, 31, 0, 1500, 700][s % 5] for s in range(S)], seed=S + KH)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 30.0])
@pytest.mark.parametrize("kv", ["bf16", "f16"])
def test_attend_scales(scale, kv):
    attend_case(2, 8, 2, 64, 500, [500, 77], kv=kv, scale=scale, seed=11)


def test_attend_scores_that_keep_rising_and_falling():
    # keys ordered so that the running reference has to move at almost every tile, or never again
    g = gen(12)
    for order in (1, -1):
        S, H, KH, D, C = 1, 4, 1, 64, 4000
        cfg = config(S=S, KH=KH, D=D, C=C, kv="f16")
        q = torch.zeros(S, H, D, dtype=torch.float16, device="cuda")
        q[..., 0] = 1.0
        k = torch.zeros(S, 1, KH, C, D, dtype=torch.float16, device="cuda")
        k[..., 0] = torch.linspace(-2000, 2000, C, device="cuda") * order
        v = randn(g, S, 1, KH, C, D, dtype=torch.float16)
        out, lse = torch.empty_like(q), torch.empty(S, H, device="cuda")
        B.sirllm_attend(cfg, 0, q, k, v, i32(C), 1.0, out, lse, B.new_attend_workspace(cfg))
        check_attend(q, k, v, [C], 1.0, out, lse)


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("S,H,D,at", [(1, 1, 64, 0), (1, 4, 128, 49151), (1, 12, 128, 30000), (1, 2, 256, 17),
                                      (160, 1, 64, 0)])   # the last: thousands of slots per warp
@pytest.mark.parametrize("faint", [22.0, 25.5, 30.0])
def test_attend_one_dominant_slot_and_many_faint_ones(kv, S, H, D, at, faint):
    # The faint slots' weights are 2^-faint of the dominant one's, whose V row is zero.  Rounded to 16
    # bits relative to a reference 2^11 or more below the maximum, an fp16 weight is off by u or by half a
    # subnormal step, 2^-25: 2^-36 of the maximum per slot (bf16 has fp32's range).
    g = gen(17)
    C, dt = 49152, DT[kv]
    cfg = config(S=S, D=D, C=C, kv=kv)
    q = torch.zeros(S, H, D, dtype=dt, device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(S, 1, 1, C, D, dtype=dt, device="cuda")
    k[..., at, 0] = 1.0
    v = (1 + randn(g, 1, 1, 1, C, D, scale=0.2)).to(dt).expand(S, 1, 1, C, D).contiguous()
    v[..., at, :] = 0.0
    scale = faint * math.log(2)
    out, lse = torch.empty_like(q), torch.empty(S, H, device="cuda")
    B.sirllm_attend(cfg, 0, q, k, v, i32(*[C] * S), scale, out, lse, B.new_attend_workspace(cfg))
    want, l, tol, tol_l = ref_attend(q[0], k[0, 0], v[0, 0], C, scale)
    tol = tol + 2.0 ** -36 * v[0].double().abs().sum(-2).amax()
    d = (out.double() - want).abs()
    assert (d <= tol).all(), f"worst {float((d / tol).max()):.2f} x tol"
    assert ((lse.double() - l).abs() <= tol_l).all()


def test_attend_infinite_scores_follow_the_formula():
    cfg = config(D=64, C=64, kv="bf16")
    ws = B.new_attend_workspace(cfg)
    q = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 1, 1, 64, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.arange(64, device="cuda").view(1, 1, 1, 64, 1).expand(1, 1, 1, 64, 64).to(torch.bfloat16).contiguous()
    out, lse = torch.empty_like(q), torch.empty(1, 1, device="cuda")
    k[0, 0, 0, 5:, 0] = -math.inf          # slots 5.. weigh nothing
    B.sirllm_attend(cfg, 0, q, k, v, i32(64), 1.0, out, lse, ws)
    assert (out == 2.0).all() and abs(float(lse) - math.log(5)) < 1e-6
    k[0, 0, 0, 3, 0] = math.nan
    B.sirllm_attend(cfg, 0, q, k, v, i32(64), 1.0, out, lse, ws)
    assert out.isnan().all() and lse.isnan().all()
    B.sirllm_attend(cfg, 0, q, k, v, i32(3), 1.0, out, lse, ws)     # the NaN is not live any more
    assert (out == 1.0).all()


@pytest.mark.parametrize("bad", [-1, 101, 2**31 - 1, -2**31])
def test_attend_reports_a_length_outside_the_planes(bad):
    g = gen(13)
    cfg = config(S=3, KH=2, D=64, C=100)
    q = randn(g, 3, 4, 64, dtype=torch.bfloat16)
    k, v = (randn(g, 3, 1, 2, 100, 64, dtype=torch.bfloat16) for _ in range(2))
    out, lse = torch.full_like(q, 7.0), torch.full((3, 4), 7.0, device="cuda")
    ws = B.new_attend_workspace(cfg)
    B.sirllm_attend(cfg, 0, q, k, v, i32(100, bad, 60), None, out, lse, ws)
    assert B.sirllm_status(ws, clear=True) == B.STATUS_OVERFLOW
    assert (out[1] == 7).all() and (lse[1] == 7).all()
    for s, n in ((0, 100), (2, 60)):
        check_attend(q[s:s + 1], k[s:s + 1], v[s:s + 1], [n], 64 ** -0.5, out[s:s + 1], lse[s:s + 1])


def test_attend_offsets_past_32_bits():
    # 49152 slots x 128 elements x 8 heads x 48 layers: element offsets beyond 2^31
    S, L, KH, C, D = 1, 48, 8, 49152, 128
    if torch.cuda.mem_get_info()[0] < 14e9:
        pytest.skip("needs 14 GB of device memory")
    g = gen(14)
    cfg = config(S=S, L=L, KH=KH, D=D, C=C)
    k, v = (torch.zeros(S, L, KH, C, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[0, L - 1] = randn(g, KH, C, D, dtype=torch.bfloat16)
    v[0, L - 1] = randn(g, KH, C, D, dtype=torch.bfloat16)
    ws, wa = B.new_workspace(cfg), B.new_attend_workspace(cfg)
    q, kn, vn = (randn(g, 1, h, D, dtype=torch.bfloat16) for h in (16, KH, KH))
    B.sirllm_append_kv(cfg, L - 1, q, kn, vn, None, None, 0.0, 5e5, B.ROPE_HALF, i32(C - 1), None, q, k, v, ws)
    assert same_bits(v[0, L - 1, :, C - 1], vn[0])
    out, lse = torch.empty_like(q), torch.empty(1, 16, device="cuda")
    B.sirllm_attend(cfg, L - 1, q, k, v, i32(C), None, out, lse, wa)
    check_attend(q, k[:, L - 1:], v[:, L - 1:], [C], D ** -0.5, out, lse)


def test_attend_an_empty_stream_of_the_widest_row():
    # 2^28 - 1 heads of 8: 2147483640 elements, 8 below 2^31
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB of device memory")
    H, D = 2**28 - 1, 8
    cfg = config(D=D, C=1)
    q = torch.empty(1, H, D, dtype=torch.bfloat16, device="cuda")
    wide = torch.full((1, H + 64, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out, lse = wide[:, 32:32 + H], torch.full((1, H), 7.0, device="cuda")
    k, v = (torch.zeros(1, 1, 1, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = B.new_attend_workspace(cfg)
    B.sirllm_attend(cfg, 0, q, k, v, i32(0), None, out, lse, ws)
    assert B.sirllm_status(ws) == 0
    assert int(torch.count_nonzero(out)) == 0 and bool((lse == -math.inf).all())
    assert (wide[:, :32] == 7).all() and (wide[:, 32 + H:] == 7).all()


def test_attend_is_reproducible_and_leaves_its_workspace_ready():
    lens = [1, 800, 0, 3333, 64, 4095, 17]
    cfg, q, k, v, out, lse, ws = attend_case(7, 8, 2, 128, 4096, lens, seed=15)
    for _ in range(20):
        o2, l2 = torch.empty_like(q), torch.empty_like(lse)
        B.sirllm_attend(cfg, 0, q, k, v, i32(*lens), None, o2, l2, ws)
        assert same_bits(o2, out) and torch.equal(l2, lse)
    o3 = torch.empty_like(q)
    B.sirllm_attend(cfg, 0, q, k, v, i32(*lens), None, o3, None, ws)     # without the log-sums
    assert same_bits(o3, out)


def test_attend_in_two_graphs_sharing_a_workspace_and_on_another_stream():
    lens = [4000, 37, 512]
    cfg, q, k, v, out, lse, ws = attend_case(3, 16, 4, 128, 4096, lens, seed=16)
    n = i32(*lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], [torch.empty_like(q) for _ in range(2)]
    with torch.cuda.stream(side):
        for o in outs:
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=side):
                B.sirllm_attend(cfg, 0, q, k, v, n, None, o, None, ws)
            graphs.append(gr)
        for _ in range(3):
            for gr in graphs:
                gr.replay()
    side.synchronize()
    assert all(same_bits(o, out) for o in outs)
    n.copy_(i32(5, 0, 4096))                                  # lengths travel in device memory
    torch.cuda.synchronize()
    graphs[0].replay()
    torch.cuda.synchronize()
    check_attend(q, k, v, [5, 0, 4096], 128 ** -0.5, outs[0], None)


# --------------------------------------------------------------------------------------
# head
# --------------------------------------------------------------------------------------

def head_scores(cfg, hidden, weight, ids, n_new, ws=None, fill=7.0):
    ws = B.new_workspace(cfg) if ws is None else ws
    rows = cfg.n_streams * cfg.max_new
    tiles = B.sirllm_head_tiles(cfg, weight.shape[0])
    pairs = torch.full((rows, tiles, 2), fill, device="cuda")
    target = torch.full((rows,), fill, device="cuda")
    ent = torch.full((rows,), fill, device="cuda")
    B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, n_new, pairs, target, ws)
    B.sirllm_score_pairs(cfg, pairs, target, ids, n_new, ent, ws)
    return pairs, target, ent, ws


def ref_scores(hidden, weight, ids):
    """fp64 scores of [rows] and the bound on fp32 sums."""
    z = hidden.double() @ weight.double().T
    walk = (hidden.double().abs() @ weight.double().abs().T).amax(-1) * math.sqrt(hidden.shape[1]) * 2.0 ** -23
    e = torch.logsumexp(z, -1) - z.gather(1, ids.long().clamp(0, weight.shape[0] - 1)[:, None])[:, 0]
    return z, torch.where(ids < 0, 0.0, e), walk


def assert_scores(got, want, walk):
    tol = torch.clamp(1e-4 * want.abs(), min=1e-5) + 2 * walk
    d = (got.double() - want).abs()
    assert (d <= tol).all(), f"worst {float((d / tol).max()):.2f} x tol"


HEAD = [  # rows, width, vocabulary
    (1, 8, 1), (1, 64, 31), (3, 72, 33), (1, 4096, 32000), (5, 1000, 257), (127, 136, 500), (128, 64, 3000),
    (129, 200, 1000), (300, 64, 50257), (64, 512, 40001), (2, 7, 100), (33, 1, 50), (640, 256, 2049),
    (16, 72, 18944), (17, 264, 19000), (48, 128, 37889), (65, 64, 19000), (64, 2056, 777), (100, 1100, 20000),
]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocab", HEAD)
def test_head_scores_against_64_bits(dt, rows, width, vocab):
    g = gen(rows + width + vocab)
    cfg = config(C=max(rows, 1), M=rows, V=vocab)
    wide = (width + 7) // 8 * 8 + 8                                    # rows further apart than their width
    hidden = randn(g, rows, wide, dtype=DT[dt])[:, :width]
    weight = randn(g, vocab, wide, dtype=DT[dt], scale=2 / math.sqrt(width))[:, :width]
    ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[rows // 2] = -1
    pairs, target, ent, ws = head_scores(cfg, hidden, weight, ids, None)
    z, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(ent, want, walk)
    assert (pairs[..., 1] >= 1 - 1e-6).all()                           # a tile's largest logit counts exp(0)
    assert B.sirllm_status(ws) == 0
    known = ids >= 0
    tz = z.gather(1, ids.long().clamp(min=0)[:, None])[:, 0]
    assert ((target.double() - tz).abs()[known] <= (walk + tz.abs() * 2.0 ** -23)[known]).all()
    assert (target[~known] == 0).all()


@pytest.mark.parametrize("S,M,lens", [(3, 100, [0, 100, 1]), (40, 7, None), (2, 300, [130, 0]), (300, 1, None),
                                      (5, 64, [0, 0, 0, 0, 0]), (4, 9, [0, 9, 3, 1]), (64, 1, None), (2, 50, [3, 50])])
def test_head_ragged_rows_leave_the_rest_alone(S, M, lens):
    g = gen(S)
    W, V = 192, 777
    if lens is None:
        lens = [(7 * s) % (M + 1) for s in range(S)]
    cfg = config(S=S, C=M, M=M, V=V)
    hidden = randn(g, S * M, W, dtype=torch.bfloat16)
    used = torch.zeros(S * M, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        used[s * M:s * M + n] = True
    hidden[~used] = math.nan                                           # never looked at
    weight = randn(g, V, W, dtype=torch.bfloat16, scale=0.2)
    ids = torch.randint(0, V, (S * M,), generator=g, device="cuda", dtype=torch.int32)
    pairs, target, ent, ws = head_scores(cfg, hidden, weight, ids, i32(*lens))
    assert (pairs[~used] == 7).all() and (target[~used] == 7).all() and (ent[~used] == 7).all()
    if used.any():
        _, want, walk = ref_scores(hidden[used], weight, ids[used])
        assert_scores(ent[used], want, walk)
    assert B.sirllm_status(ws) == 0


def test_head_many_row_blocks_some_without_work():
    g = gen(25)
    S, M, W, V = 50, 300, 64, 300
    lens = [0 if s % 3 == 0 else (M if s % 3 == 1 else 17) for s in range(S)]
    cfg = config(S=S, C=M, M=M, V=V)
    hidden = randn(g, S * M, W, dtype=torch.bfloat16)
    weight = randn(g, V, W, dtype=torch.bfloat16, scale=0.2)
    ids = torch.randint(0, V, (S * M,), generator=g, device="cuda", dtype=torch.int32)
    used = torch.zeros(S * M, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        used[s * M:s * M + n] = True
    pairs, target, ent, ws = head_scores(cfg, hidden, weight, ids, i32(*lens))
    assert (ent[~used] == 7).all() and (pairs[~used] == 7).all()
    _, want, walk = ref_scores(hidden[used], weight, ids[used])
    assert_scores(ent[used], want, walk)


def test_head_more_rows_than_one_launch_takes():
    g = gen(26)
    S, M, W, V = 22, 49152, 8, 40                                      # 1,081,344 rows
    cfg = config(S=S, C=M, M=M, V=V)
    hidden = randn(g, S * M, W, dtype=torch.bfloat16)
    weight = randn(g, V, W, dtype=torch.bfloat16)
    ids = torch.randint(0, V, (S * M,), generator=g, device="cuda", dtype=torch.int32)
    _, _, ent, ws = head_scores(cfg, hidden, weight, ids, None)
    _, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(ent, want, walk)
    assert B.sirllm_status(ws) == 0


def test_head_launch_that_takes_longer_than_any_one_wait():
    # 3.4e15 operations in one launch: 2 s and more.  No wait inside may be bounded over the whole of it
    # (2^20 polls of a barrier at 1.5 us each are 1.55 s).
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB of device memory")
    g = gen(27)
    S, M, W, V = 32, 32768, 8192, 200000
    cfg = config(S=S, C=M, M=M, V=V)
    hidden = torch.empty(S * M, W, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    weight = torch.empty(V, W, dtype=torch.bfloat16, device="cuda").normal_(0, 2 / math.sqrt(W), generator=g)
    ids = torch.randint(0, V, (S * M,), generator=g, device="cuda", dtype=torch.int32)
    pairs, target, ent, ws = head_scores(cfg, hidden, weight, ids, None)
    assert B.sirllm_status(ws) == 0
    assert (pairs[..., 1] >= 1 - 1e-6).all()
    rows = torch.arange(0, S * M, S * M // 61, device="cuda")           # both CTAs' rows, first block to last
    rows[-1] = S * M - 1
    _, want, walk = ref_scores(hidden[rows], weight, ids[rows])
    assert_scores(ent[rows], want, walk)


@pytest.mark.parametrize("rows", [150, 100, 20])
def test_head_column_ranges_add_up_to_the_whole(rows):
    g = gen(21)
    W, V = 320, 5000
    cfg = config(C=rows, M=rows, V=V)
    ws = B.new_workspace(cfg)
    hidden = randn(g, rows, W, dtype=torch.bfloat16)
    weight = randn(g, V, W, dtype=torch.bfloat16, scale=0.15)
    ids = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[0], ids[1], ids[2] = -1, 0, V - 1
    cuts = [0, 1, 1800, 1900, V]
    parts, targets = [], []
    for a, b in zip(cuts, cuts[1:]):
        p = torch.empty(rows, B.sirllm_head_tiles(cfg, b - a), 2, device="cuda")
        t = torch.full((rows,), 7.0, device="cuda")
        B.sirllm_head_pairs(cfg, hidden, weight[a:b], a, ids, None, p, t, ws)
        parts.append(p)
        targets.append(t)
        inside = (ids >= a) & (ids < b)
        assert (t[~inside] == 0).all() and (t[inside] != 0).all()
    ent = torch.empty(rows, device="cuda")
    B.sirllm_score_pairs(cfg, torch.cat(parts, 1), sum(targets), ids, None, ent, ws)
    _, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(ent, want, walk)


@pytest.mark.parametrize("rows", [10, 70, 200])
def test_head_bad_ids_are_flagged_by_the_score_and_masked_columns_count_for_nothing(rows):
    g = gen(22)
    W, V = 64, 700
    cfg = config(C=rows, M=rows, V=V)
    hidden = randn(g, rows, W, dtype=torch.float16).abs()
    weight = randn(g, V, W, dtype=torch.float16, scale=0.2)
    weight[256:600, 0] = -math.inf                                     # one whole tile and more
    ids = torch.randint(0, 256, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ids[3], ids[4] = V, 2**31 - 1
    pairs, target, ent, ws = head_scores(cfg, hidden, weight, ids, None)
    assert B.sirllm_status(ws) == B.STATUS_TOKEN_RANGE
    assert (ent[3:5] == 0).all() and (target[3:5] == 0).all()
    live = torch.cat([weight[:256], weight[600:]])
    good = [i for i in range(rows) if i not in (3, 4)]
    _, want, walk = ref_scores(hidden[good], live, ids[good])
    assert_scores(ent[good], want, walk)
    assert not pairs.isnan().any()


@pytest.mark.parametrize("rows", [20, 120, 200])
def test_head_of_large_logits(rows):
    g = gen(23)
    W, V = 128, 2000
    cfg = config(C=rows, M=rows, V=V)
    hidden = randn(g, rows, W, dtype=torch.bfloat16, scale=30)
    weight = randn(g, V, W, dtype=torch.bfloat16, scale=3)             # logits of +-1000 and more
    ids = (hidden.float() @ weight.float().T).argmax(-1).to(torch.int32)
    _, _, ent, _ = head_scores(cfg, hidden, weight, ids, None)
    _, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(ent, want, walk)


@pytest.mark.parametrize("rows", [40, 100, 300])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_head_sums_lean_no_further_at_a_larger_width(rows, dt):
    # Terms of one sign, so that a truncated addition always errs the same way.  A chunk of 1024 elements
    # is 64 additions of 16 products each.  Addition j takes 17 terms in units of the sum so far's last
    # place and cuts each short by less than one of them, 2^-23 j/64 of the chunk's sum: over j = 1 .. 64
    # less than 17 * 65/2 * 2^-23 of it.  The chunks' rounded additions do not lean to a side, so the mean
    # error of a wider sum is that of a chunk; one chunk over 4096 or 8192 would lean 4 or 8 times as
    # far.  The mean over 40 rows is known to well within a quarter (one row scatters by that much).
    off = {}
    for width in (1024, 4096, 8192):
        g = gen(rows + width)
        V = 2000
        cfg = config(C=rows, M=rows, V=V)
        hidden = randn(g, rows, width).abs().to(DT[dt])
        weight = (randn(g, V, width).abs() / 64).to(DT[dt])
        ids = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
        _, target, _, _ = head_scores(cfg, hidden, weight, ids, None)
        z = (hidden.double() * weight.double()[ids.long()]).sum(-1)
        off[width] = float(((target.double() - z) / z).mean())
    assert abs(off[1024]) < 17 * 65 / 2 * 2.0 ** -23
    for width in (4096, 8192):
        assert abs(off[width] - off[1024]) < 0.25 * abs(off[1024]) + 2.0 ** -24, off


@pytest.mark.parametrize("rows", [7, 70, 300])
def test_head_replayed_from_a_graph_on_another_stream(rows):
    g = gen(24)
    W, V = 256, 4000
    cfg = config(C=rows, M=rows, V=V)
    hidden = randn(g, rows, W, dtype=torch.bfloat16)
    weight = randn(g, V, W, dtype=torch.bfloat16, scale=0.1)
    ids = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    _, _, first, ws = head_scores(cfg, hidden, weight, ids, None)
    pairs = torch.empty(rows, B.sirllm_head_tiles(cfg, V), 2, device="cuda")
    target, ent = torch.empty(rows, device="cuda"), torch.zeros(rows, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=side):
        B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, None, pairs, target, ws)
        B.sirllm_score_pairs(cfg, pairs, target, ids, None, ent, ws)
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(ent, first)
    hidden.copy_(randn(g, rows, W, dtype=torch.bfloat16))
    gr.replay()
    torch.cuda.synchronize()
    _, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(ent, want, walk)


# --------------------------------------------------------------------------------------
# a run of them together
# --------------------------------------------------------------------------------------

def test_dialogue_rounds_of_decode_steps():
    """Three rounds of generated tokens on two streams: every step writes a token's K/V rows into
    every layer and attends to the cache; the round's tokens are scored from the hidden states
    and the round ends with sirllm_step_pairs, which evicts.  Attention is checked at every
    step against a cache kept by the test: plain tensors, compacted by the oracle's rule of the
    kept slots (the call's own keep list applied row by row)."""
    g = gen(31)
    S, L, KH, H, D, C, M, V, W = 2, 2, 2, 6, 64, 96, 24, 900, 128
    dt = torch.bfloat16
    cfg = B.make_config(n_streams=S, n_layers=L, n_kv_heads=KH, head_dim=D, capacity=C, budget=40, n_sink=2,
                        n_recent=8, max_new=M, vocab=V, logits_dtype="f32", kv_dtype="bf16")
    token = B.make_config(n_streams=S, n_layers=L, n_kv_heads=KH, head_dim=D, capacity=C, budget=40, n_sink=2,
                          n_recent=8, max_new=1, vocab=V, logits_dtype="f32", kv_dtype="bf16")
    ws, ws1, wa = B.new_workspace(cfg), B.new_workspace(token), B.new_attend_workspace(cfg)
    k, v = (torch.zeros(S, L, KH, C, D, dtype=dt, device="cuda") for _ in range(2))
    mk, mv = k.clone(), v.clone()                      # the test's own cache
    weight = randn(g, V, W, dtype=dt, scale=0.2)
    wq, wk = randn(g, D, dtype=dt), randn(g, D, dtype=dt)
    scores = torch.zeros(S, C, device="cuda")
    live, decay = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.tensor([0.9, 0.8], device="cuda")
    keep = torch.zeros(S, cfg.threshold, dtype=torch.int32, device="cuda")
    n_keep = torch.zeros(S, dtype=torch.int32, device="cuda")
    ent = torch.zeros(S * M, device="cuda")
    pairs = torch.zeros(S * M, B.sirllm_head_tiles(cfg, V), 2, device="cuda")
    target = torch.zeros(S * M, device="cuda")
    evicted = False
    for rnd in range(3):
        turn = [M, M - 7 * rnd]                        # stream 1 falls silent earlier
        hidden = randn(g, S * M, W, dtype=dt)
        ids = torch.randint(0, V, (S * M,), generator=g, device="cuda", dtype=torch.int32)
        start = live.tolist()
        for t in range(M):
            n_new = i32(*[int(t < turn[s]) for s in range(S)])
            first = i32(*[start[s] + min(t, turn[s]) for s in range(S)])
            for layer in range(L):
                q, kn, vn = (randn(g, S, h, D, dtype=dt) for h in (H, KH, KH))
                q_out, out = torch.zeros_like(q), torch.empty_like(q)
                B.sirllm_append_kv(token, layer, q, kn, vn, wq, wk, 1e-6, 1e4, B.ROPE_HALF, first, n_new, q_out,
                                   k, v, ws1)
                lens = first + n_new
                B.sirllm_attend(token, layer, q_out, k, v, lens, None, out, None, wa)
                for s in range(S):
                    if t < turn[s]:
                        p = start[s] + t
                        turned, length = ref_rope(kn[s:s + 1].double(), wk, first[s:s + 1], 1e-6, 1e4, B.ROPE_HALF)
                        assert_turned(k[s, layer, :, p], turned[0], length[0])
                        mk[s, layer, :, p], mv[s, layer, :, p] = k[s, layer, :, p], vn[s]
                check_attend(q_out, mk, mv, lens.tolist(), D ** -0.5, out, None, layer)
        B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, i32(*turn), pairs, target, ws)
        B.sirllm_step_pairs(cfg, pairs, target, ids, i32(*turn), scores, None, live, decay, k, v, keep, n_keep, ent, ws)
        assert B.sirllm_status(ws) == 0 and B.sirllm_status(ws1) == 0 and B.sirllm_status(wa) == 0
        for s in range(S):
            r = slice(s * M, s * M + turn[s])
            _, want, walk = ref_scores(hidden[r], weight, ids[r])
            assert_scores(ent[r], want, walk)
            n = int(n_keep[s])
            assert int(live[s]) == n
            evicted |= n < start[s] + turn[s]
            rows = keep[s, :n].long()
            mk[s, :, :, :n], mv[s, :, :, :n] = mk[s, :, :, rows].clone(), mv[s, :, :, rows].clone()
            assert same_bits(k[s, :, :, :n], mk[s, :, :, :n]) and same_bits(v[s, :, :, :n], mv[s, :, :, :n])
    assert evicted


def test_decode_steps_back_to_back_and_replayed_equal_steps_one_by_one():
    """append -> attend -> head -> score for every token of a turn: launched without a wait between
    them, replayed from one graph, and with a synchronisation after every call."""
    g = gen(32)
    S, L, KH, H, D, C, M, V, W = 3, 2, 4, 8, 128, 700, 6, 3000, 256
    dt = torch.bfloat16
    cfg = B.make_config(n_streams=S, n_layers=L, n_kv_heads=KH, head_dim=D, capacity=C, budget=600, n_sink=2,
                        n_recent=8, max_new=1, vocab=V, logits_dtype="f32", kv_dtype="bf16")
    k0, v0 = (randn(g, S, L, KH, C, D, dtype=dt) for _ in range(2))
    qkv = randn(g, M, L, S, H + 2 * KH, D, dtype=dt)
    hidden, weight = randn(g, M, S, W, dtype=dt), randn(g, V, W, dtype=dt, scale=0.2)
    ids = torch.randint(0, V, (M, S), generator=g, device="cuda", dtype=torch.int32)
    start = torch.tensor([600, 0, 333], dtype=torch.int32, device="cuda")
    wq, wk = randn(g, D, dtype=dt), randn(g, D, dtype=dt)

    def buffers():
        return dict(k=k0.clone(), v=v0.clone(), q=torch.zeros(M, L, S, H, D, dtype=dt, device="cuda"),
                    out=torch.zeros(M, L, S, H, D, dtype=dt, device="cuda"), ent=torch.zeros(M, S, device="cuda"),
                    first=start.clone(), lens=start + 1, ws=B.new_workspace(cfg), wa=B.new_attend_workspace(cfg),
                    pairs=torch.zeros(S, B.sirllm_head_tiles(cfg, V), 2, device="cuda"),
                    target=torch.zeros(S, device="cuda"))

    def run(b, wait):
        for t in range(M):
            for layer in range(L):
                x = qkv[t, layer]
                B.sirllm_append_kv(cfg, layer, x[:, :H], x[:, H:H + KH], x[:, H + KH:], wq, wk, 1e-6, 1e4, B.ROPE_HALF,
                                   b["first"], None, b["q"][t, layer], b["k"], b["v"], b["ws"])
                wait()
                B.sirllm_attend(cfg, layer, b["q"][t, layer], b["k"], b["v"], b["lens"], None, b["out"][t, layer], None,
                                b["wa"])
                wait()
            B.sirllm_head_pairs(cfg, hidden[t], weight, 0, ids[t], None, b["pairs"], b["target"], b["ws"])
            wait()
            B.sirllm_score_pairs(cfg, b["pairs"], b["target"], ids[t], None, b["ent"][t], b["ws"])
            wait()
            b["first"] += 1
            b["lens"] += 1

    def same(x, y):
        return all(torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)) for n in ("k", "v", "q", "out", "ent"))

    one, loose, graphed = buffers(), buffers(), buffers()
    run(one, torch.cuda.synchronize)
    run(loose, lambda: None)
    torch.cuda.synchronize()
    assert same(one, loose)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=side):
        run(graphed, lambda: None)
    for _ in range(3):                               # the same turn again from the same start
        graphed["first"].copy_(start)
        graphed["lens"].copy_(start + 1)
        gr.replay()
        torch.cuda.synchronize()
        assert same(one, graphed)
    assert B.sirllm_status(graphed["ws"]) == 0 and B.sirllm_status(graphed["wa"]) == 0


def test_calls_at_once_on_two_streams():
    g = gen(33)
    dt = torch.bfloat16
    cfg = config(S=2, KH=8, D=128, C=4096, M=1, V=9000)
    k, v = (randn(g, 2, 1, 8, 4096, 128, dtype=dt) for _ in range(2))
    q, hidden = randn(g, 2, 32, 128, dtype=dt), randn(g, 2, 512, dtype=dt)
    weight = randn(g, 9000, 512, dtype=dt, scale=0.1)
    ids, lens = i32(5, 8999), i32(4096, 1777)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    torch.cuda.synchronize()
    for st in streams:                               # each stream has workspaces of its own
        with torch.cuda.stream(st):
            wa, ws = B.new_attend_workspace(cfg), B.new_workspace(cfg)
            out, pairs = torch.zeros_like(q), torch.zeros(2, B.sirllm_head_tiles(cfg, 9000), 2, device="cuda")
            target, ent = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
            got.append((out, ent, wa, ws, pairs, target))
    for _ in range(20):
        for st, (out, ent, wa, ws, pairs, target) in zip(streams, got):
            with torch.cuda.stream(st):
                B.sirllm_attend(cfg, 0, q, k, v, lens, None, out, None, wa)
                B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, None, pairs, target, ws)
                B.sirllm_score_pairs(cfg, pairs, target, ids, None, ent, ws)
    torch.cuda.synchronize()
    assert same_bits(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    check_attend(q, k, v, [4096, 1777], 128 ** -0.5, got[0][0], None)
    _, want, walk = ref_scores(hidden, weight, ids)
    assert_scores(got[0][1], want, walk)


def test_calls_behind_a_join_of_two_captured_streams():
    # each call's programmatic launch follows work of another stream, joined by an event
    g = gen(34)
    dt = torch.bfloat16
    cfg = config(S=1, KH=2, D=64, C=600, M=1, V=500)
    ws, wa = B.new_workspace(cfg), B.new_attend_workspace(cfg)
    k, v = (randn(g, 1, 1, 2, 600, 64, dtype=dt) for _ in range(2))
    q, kn, vn = (randn(g, 1, h, 64, dtype=dt) for h in (4, 2, 2))
    hidden, weight = torch.zeros(1, 128, dtype=dt, device="cuda"), randn(g, 500, 128, dtype=dt, scale=0.2)
    source = randn(g, 1, 128, dtype=dt)
    lens, first, ids = torch.zeros(1, dtype=torch.int32, device="cuda"), i32(0), i32(77)
    q_out, out = torch.zeros_like(q), torch.zeros_like(q)
    pairs, target = torch.zeros(1, B.sirllm_head_tiles(cfg, 500), 2, device="cuda"), torch.zeros(1, device="cuda")
    ent = torch.zeros(1, device="cuda")
    main, other = torch.cuda.Stream(), torch.cuda.Stream()
    gr = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(gr, stream=main):
        other.wait_stream(main)
        with torch.cuda.stream(other):
            first.fill_(410)
            lens.fill_(411)
        main.wait_stream(other)
        B.sirllm_append_kv(cfg, 0, q, kn, vn, None, None, 0.0, 1e4, B.ROPE_HALF, first, None, q_out, k, v, ws)
        other.wait_stream(main)
        with torch.cuda.stream(other):
            hidden.copy_(source)
        B.sirllm_attend(cfg, 0, q_out, k, v, lens, None, out, None, wa)
        main.wait_stream(other)
        B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, None, pairs, target, ws)
        B.sirllm_score_pairs(cfg, pairs, target, ids, None, ent, ws)
    for _ in range(3):
        first.zero_()
        lens.zero_()
        hidden.zero_()
        gr.replay()
        torch.cuda.synchronize()
        check_attend(q_out, k, v, [411], 64 ** -0.5, out, None)
        _, want, walk = ref_scores(source, weight, ids)
        assert_scores(ent, want, walk)


FIRST_CALL = """
import torch
from paper_2405_12528_b200 import binding as B
cfg = B.make_config(1, 1, 8, 128, 4096, 4096, 0, 0, {M}, 700, "f32", "bf16")
dt, M = torch.bfloat16, {M}
ws, wa = B.new_workspace(cfg), B.new_attend_workspace(cfg)
k, v = (torch.randn(1, 1, 8, 4096, 128, device="cuda").to(dt) for _ in range(2))
q, kn = torch.randn(M, 16, 128, device="cuda").to(dt), torch.randn(M, 8, 128, device="cuda").to(dt)
out, q_out = torch.zeros_like(q), torch.zeros_like(q)
hidden, weight = torch.randn(M, 64, device="cuda").to(dt), torch.randn(700, 64, device="cuda").to(dt)
pairs, target = torch.zeros(M, B.sirllm_head_tiles(cfg, 700), 2, device="cuda"), torch.zeros(M, device="cuda")
ids, first = torch.zeros(M, dtype=torch.int32, device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
lens = torch.full((1,), 4000, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    B.sirllm_append_kv(cfg, 0, q, kn, kn, None, None, 0.0, 1e4, 0, first, None, q_out, k, v, ws)
    B.sirllm_attend(cfg, 0, q_out, k, v, lens, None, out, None, wa)
    B.sirllm_head_pairs(cfg, hidden, weight, 0, ids, None, pairs, target, ws)
g.replay()
torch.cuda.synchronize()
assert float(out[0].abs().sum()) > 0 and float(pairs.abs().sum()) > 0 and B.sirllm_status(ws) == 0
print("captured")
"""


@pytest.mark.parametrize("M", [1, 200])
def test_the_process_first_call_may_be_a_captured_one(M):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST_CALL.format(M=M)], capture_output=True, text=True, cwd=root,
                         timeout=300)
    assert run.returncode == 0 and "captured" in run.stdout, run.stderr[-2000:]
