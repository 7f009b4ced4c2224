"""What the calls of a decode step refuse, on the host and before anything is enqueued (no GPU
needed): ``sirllm_append_kv``, ``sirllm_attend``, ``sirllm_head_pairs``."""
import ctypes
import math
import os
import socket

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2405_12528_b200 import binding as B
from paper_2405_12528_b200 import sharding


@pytest.fixture(scope="module")
def lib(cuda_library):
    return B.lib()


def cfg(**kw):
    base = dict(n_streams=2, n_layers=3, n_kv_heads=2, head_dim=64, capacity=128, budget=64, n_sink=4, n_recent=8,
                max_new=8, vocab=1000, logits_dtype="f32", kv_dtype="bf16")
    base.update(kw)
    return B.make_config(**base)


P, WS = 0x2000, 0x1000      # never dereferenced


def append(lib, c=None, **kw):
    a = dict(layer=0, q=P, n_heads=4, qs=256, k_new=P, ks=128, v_new=P, vs=128, wq=None, wk=None, eps=1e-6, base=1e4,
             layout=0, first=P, n_new=None, q_out=P, os=256, k=P, v=P, ws=WS)
    a.update(kw)
    return lib.sirllm_append_kv(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(k_new=None)), (B.ERR_NULL, dict(v_new=None)), (B.ERR_NULL, dict(first=None)),
    (B.ERR_NULL, dict(k=None)), (B.ERR_NULL, dict(v=None)), (B.ERR_NULL, dict(ws=None)),
    (B.ERR_NULL, dict(q=None)), (B.ERR_NULL, dict(q_out=None)),
    (B.ERR_BAD_CONFIG, dict(layer=-1)), (B.ERR_BAD_CONFIG, dict(layer=3)), (B.ERR_BAD_CONFIG, dict(n_heads=0)),
    (B.ERR_BAD_CONFIG, dict(n_heads=-4)), (B.ERR_BAD_CONFIG, dict(q=None, q_out=None)),
    (B.ERR_TOO_LARGE, dict(n_heads=0x3FFFFFFF)),
    (B.ERR_BAD_CONFIG, dict(base=0.0)), (B.ERR_BAD_CONFIG, dict(base=-1.0)), (B.ERR_BAD_CONFIG, dict(base=math.inf)),
    (B.ERR_BAD_CONFIG, dict(base=math.nan)), (B.ERR_BAD_CONFIG, dict(layout=2)), (B.ERR_BAD_CONFIG, dict(eps=-1e-6)),
    (B.ERR_BAD_CONFIG, dict(eps=math.nan)), (B.ERR_BAD_CONFIG, dict(qs=248)), (B.ERR_BAD_CONFIG, dict(os=248)),
    (B.ERR_BAD_CONFIG, dict(ks=120)), (B.ERR_BAD_CONFIG, dict(vs=120)),
    (B.ERR_ALIGN, dict(q=P + 8)), (B.ERR_ALIGN, dict(k=P + 2)), (B.ERR_ALIGN, dict(wk=P + 2)), (B.ERR_ALIGN, dict(qs=260)),
    (B.ERR_ALIGN, dict(vs=132)), (B.ERR_ALIGN, dict(ws=WS + 16)),
])
def test_append_refusals(lib, want, kw):
    assert append(lib, **kw) == want


def test_append_refuses_heads_of_half_vectors(lib):
    assert append(lib, cfg(head_dim=40), qs=160, os=160, ks=80, vs=80) == B.ERR_BAD_CONFIG
    assert append(lib, cfg(budget=5)) == B.ERR_BAD_CONFIG


def test_append_refuses_more_heads_than_it_counts(lib):
    big = cfg(n_streams=2**20, max_new=128, n_layers=1)
    assert append(lib, big, n_heads=16, qs=1024, os=1024) == B.ERR_TOO_LARGE


def attend(lib, c=None, **kw):
    a = dict(layer=0, q=P, n_heads=4, qs=256, k=P, v=P, kv_len=P, scale=0.1, out=P, os=256, lse=None, ws=WS)
    a.update(kw)
    return lib.sirllm_attend(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(q=None)), (B.ERR_NULL, dict(k=None)), (B.ERR_NULL, dict(v=None)), (B.ERR_NULL, dict(kv_len=None)),
    (B.ERR_NULL, dict(out=None)), (B.ERR_NULL, dict(ws=None)), (B.ERR_BAD_CONFIG, dict(layer=3)),
    (B.ERR_BAD_CONFIG, dict(layer=-1)), (B.ERR_BAD_CONFIG, dict(n_heads=0)), (B.ERR_BAD_CONFIG, dict(n_heads=3)),
    (B.ERR_BAD_CONFIG, dict(n_heads=-2)), (B.ERR_BAD_CONFIG, dict(scale=math.nan)),
    (B.ERR_BAD_CONFIG, dict(scale=math.inf)), (B.ERR_BAD_CONFIG, dict(qs=128)), (B.ERR_BAD_CONFIG, dict(os=128)),
    (B.ERR_ALIGN, dict(q=P + 2)), (B.ERR_ALIGN, dict(out=P + 8)), (B.ERR_ALIGN, dict(qs=258)), (B.ERR_ALIGN, dict(os=260)),
    (B.ERR_ALIGN, dict(ws=WS + 8)),
])
def test_attend_refusals(lib, want, kw):
    assert attend(lib, **kw) == want


@pytest.mark.parametrize("scale", [3e38, -2.4e38])
def test_attend_refuses_a_scale_that_overflows_in_units_of_log2(lib, scale):
    # scores are kept times log2 e: a score of 0 would become NaN
    assert attend(lib, scale=scale) == B.ERR_BAD_CONFIG


def test_attend_refuses_more_units_than_it_counts(lib):
    big = cfg(n_streams=2**24, n_layers=1, n_kv_heads=2, head_dim=8, capacity=1, budget=1, n_sink=0, n_recent=0, max_new=1)
    assert attend(lib, big, n_heads=2, qs=16, os=16) == B.ERR_TOO_LARGE


@pytest.mark.parametrize("streams,heads,dim,capacity", [
    (64, 196608, 8, 49152),         # 786432 units x (3072 tiles + 40): 2447376384 positions
    (1024, 10816, 8, 49152),        # 2154201088
    (1, 5600000, 256, 49152),       # wide heads: units of 8
    (2**18, 2032, 8, 400),          # 33.3 million units (below 2^25) of 25 tiles
])
def test_attend_refuses_more_positions_than_it_counts(lib, streams, heads, dim, capacity):
    # query heads that share a K/V head multiply the work without any memory for the cache
    big = cfg(n_streams=streams, n_layers=1, n_kv_heads=1, head_dim=dim, capacity=capacity, budget=capacity, n_sink=0,
              n_recent=0, max_new=1)
    units = streams * -(-heads // (16 if dim <= 128 else 8))
    wide = heads * dim
    refused = units * (-(-capacity // 16) + 40) > 2**31 - 1 - 256
    assert refused and attend(lib, big, n_heads=heads, qs=wide, os=wide) == B.ERR_TOO_LARGE


def test_attend_refuses_heads_wider_than_its_registers(lib):
    wide = cfg(head_dim=264)
    assert attend(lib, wide, qs=2048, os=2048) == B.ERR_TOO_LARGE
    assert B.sirllm_attend_workspace_bytes(wide) == 0
    assert lib.sirllm_attend_workspace_init(ctypes.byref(wide), WS, None) == B.ERR_TOO_LARGE
    n = B.sirllm_attend_workspace_bytes(cfg())
    assert n > 0 and n % 256 == 0 and n < B.sirllm_attend_workspace_bytes(cfg(head_dim=B.MAX_ATTEND_HEAD_DIM))
    assert B.sirllm_attend_workspace_bytes(cfg(budget=5)) == 0
    assert lib.sirllm_attend_workspace_init(ctypes.byref(cfg()), None, None) == B.ERR_NULL
    assert lib.sirllm_attend_workspace_init(ctypes.byref(cfg()), WS + 8, None) == B.ERR_ALIGN


def head(lib, c=None, **kw):
    a = dict(hidden=P, hs=64, weight=P, wst=64, d=64, dtype=B.BF16, col0=0, n_cols=1000, ids=P, n_new=None, pairs=P,
             ps=1000, target=P, ws=WS)
    a.update(kw)
    return lib.sirllm_head_pairs(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(hidden=None)), (B.ERR_NULL, dict(weight=None)), (B.ERR_NULL, dict(ids=None)),
    (B.ERR_NULL, dict(pairs=None)), (B.ERR_NULL, dict(target=None)), (B.ERR_NULL, dict(ws=None)),
    (B.ERR_BAD_CONFIG, dict(d=0)), (B.ERR_BAD_CONFIG, dict(dtype=B.F32)), (B.ERR_BAD_CONFIG, dict(n_cols=0)),
    (B.ERR_BAD_CONFIG, dict(n_cols=1001)), (B.ERR_BAD_CONFIG, dict(col0=1)), (B.ERR_BAD_CONFIG, dict(col0=-1)),
    (B.ERR_BAD_CONFIG, dict(hs=56)), (B.ERR_BAD_CONFIG, dict(wst=56)), (B.ERR_BAD_CONFIG, dict(ps=1)),
    (B.ERR_BAD_CONFIG, dict(wst=1 << 39)),
    (B.ERR_ALIGN, dict(hidden=P + 2)), (B.ERR_ALIGN, dict(weight=P + 8)), (B.ERR_ALIGN, dict(hs=68)),
    (B.ERR_ALIGN, dict(wst=66)), (B.ERR_ALIGN, dict(pairs=P + 4)), (B.ERR_ALIGN, dict(target=P + 2)),
    (B.ERR_ALIGN, dict(ws=WS + 4)),
])
def test_head_refusals(lib, want, kw):
    assert head(lib, **kw) == want


def test_head_tiles_cover_the_columns(lib):
    for rows in (1, 128, 129, 4096):
        for n in (1, 31, 32, 33, 255, 257, 32000, 50257, 128256):
            c = cfg(n_streams=1, capacity=max(rows, 64), max_new=rows, vocab=128256)
            t = B.sirllm_head_tiles(c, n)
            assert 1 <= t <= (n + 15) // 16 + 1 and t == B.sirllm_head_tiles(c, n)
    assert B.sirllm_head_tiles(cfg(), 0) == 0 and B.sirllm_head_tiles(cfg(), 1001) == 0
    assert B.sirllm_head_tiles(cfg(budget=5), 10) == 0


def test_binding_refuses_wrong_tensors_before_the_library(lib):
    c = cfg(head_dim=64)
    bf = torch.bfloat16
    z = lambda *s, dt=bf: torch.zeros(*s, dtype=dt)
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    kv = z(2, 3, 2, 128, 64)
    ws = torch.zeros(B.sirllm_workspace_bytes(c), dtype=torch.uint8)
    wa = torch.zeros(B.sirllm_attend_workspace_bytes(c), dtype=torch.uint8)

    def refused(fn, *a, needle):
        with pytest.raises(B.SirllmError) as err:
            fn(c, *a)
        assert needle in str(err.value), str(err.value)

    def app(needle, **kw):
        a = dict(layer=0, q=z(16, 4, 64), k_new=z(16, 2, 64), v_new=z(16, 2, 64), q_weight=z(64), k_weight=None,
                 eps=1e-6, rope_base=1e4, layout=0, first_slot=i(2), n_new=i(2), q_out=z(16, 4, 64), k=kv, v=kv, ws=ws)
        a.update(kw)
        refused(B.sirllm_append_kv, *a.values(), needle=needle)

    app("CUDA tensor")                                   # all sizes right: as far as residence
    app("q has shape", q=z(15, 4, 64), q_out=z(16, 4, 64))
    app("q_out has shape", q_out=z(16, 3, 64))
    app("k_new has shape", k_new=z(16, 3, 64))
    app("v_new has shape", v_new=z(16, 2, 32))
    app("dtype", q=z(16, 4, 64, dt=torch.float16))
    app("dtype", q_weight=z(64, dt=torch.float32))
    app("needs", k_weight=z(63))
    app("heads must be dense", k_new=z(16, 64, 2).transpose(1, 2))
    app("rows overlap", v_new=z(2, 64).as_strided((16, 2, 64), (0, 64, 1)))
    app("needs", first_slot=i(1))
    app("needs", k=kv[:, :2])
    app("needs", ws=ws[:-1])

    def att(needle, **kw):
        a = dict(layer=0, q=z(2, 4, 64), k=kv, v=kv, kv_len=i(2), scale=None, out=z(2, 4, 64), lse=None, ws=wa)
        a.update(kw)
        refused(B.sirllm_attend, *a.values(), needle=needle)

    att("CUDA tensor")
    att("q has shape", q=z(1, 4, 64))
    att("out has shape", out=z(2, 5, 64))
    att("dtype", out=z(2, 4, 64, dt=torch.float32))
    att("needs", kv_len=i(1))
    att("needs", lse=torch.zeros(7))
    att("needs", ws=wa[:-1])

    tiles = B.sirllm_head_tiles(c, 1000)
    pairs = torch.zeros(16, tiles, 2)

    def hd(needle, **kw):
        a = dict(hidden=z(16, 96), weight=z(1000, 96), col0=0, token_ids=i(16), n_new=None, pairs_out=pairs,
                 target_out=torch.zeros(16), ws=ws)
        a.update(kw)
        refused(B.sirllm_head_pairs, *a.values(), needle=needle)

    hd("CUDA tensor")
    hd("hidden has shape", hidden=z(15, 96))
    hd("do not match", weight=z(1000, 88))
    hd("do not match", weight=z(1000, 96, dt=torch.float16))
    hd("hidden has dtype", hidden=z(16, 96, dt=torch.float32), weight=z(1000, 96, dt=torch.float32))
    hd("tiles per row", pairs_out=torch.zeros(16, tiles + 1, 2))
    hd("tiles per row", weight=z(1001, 96))
    hd("rows must be dense", weight=z(96, 1000).t())
    hd("needs", token_ids=i(15))
    hd("needs", target_out=torch.zeros(15))


@pytest.mark.parametrize("call,arg", [(append, "first"), (append, "n_new"), (attend, "kv_len"), (attend, "lse"),
                                      (head, "ids"), (head, "n_new"), (head, "target")])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_words_off_their_4_bytes_are_refused(lib, call, arg, off):
    # the kernels would fault on them
    assert call(lib, **{arg: P + off}) == B.ERR_ALIGN


# ---- a vocabulary-parallel LM head: several tiles per rank through the exchange (gloo, two ranks) ----

def _tile_pairs(z, width):
    """(max, sum exp) of every ``width`` columns of fp64 logits, as sirllm_head_pairs hands them out."""
    parts = [(p.amax(-1), torch.exp(p - p.amax(-1, keepdim=True)).sum(-1)) for p in z.split(width, dim=1)]
    return torch.stack([torch.stack(p, -1) for p in parts], 1).float()


def _rank_of_a_parallel_head(rank, world, port, out):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        g = torch.Generator().manual_seed(4)
        z, ids = torch.randn(9, 101, generator=g, dtype=torch.float64) * 3, torch.randint(0, 101, (9,), generator=g)
        a, b = [(0, 70), (70, 101)][rank]                       # 5 and 3 tiles of 16 columns
        pairs = torch.zeros(9, 5, 2)
        mine = _tile_pairs(z[:, a:b], 16)
        pairs[:, :mine.shape[1]] = mine
        inside = (ids >= a) & (ids < b)
        target = torch.where(inside, z[torch.arange(9), ids], 0.0).float()
        got, tgt = sharding.exchange_vocab_partials(pairs, target)
        e = torch.log((got[..., 1].double() * torch.exp(got[..., 0].double())).sum(-1)) - tgt
        want = torch.logsumexp(z, -1) - z[torch.arange(9), ids]
        out.put((rank, tuple(got.shape), float((e - want).abs().max())))
    finally:
        dist.destroy_process_group()


def test_two_ranks_exchange_several_tiles_each():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    ctx = mp.get_context("spawn")
    out = ctx.Queue()
    procs = [ctx.Process(target=_rank_of_a_parallel_head, args=(r, 2, port, out)) for r in range(2)]
    for p in procs:
        p.start()
    results = sorted(out.get(timeout=120) for _ in procs)
    for p in procs:
        p.join(timeout=60)
        assert p.exitcode == 0
    # fp32 pairs and targets of logits below 16: each within 2^-21, their sums within a few of those
    assert all(shape == (9, 10, 2) and worst < 8 * 2.0 ** -21 for _, shape, worst in results)
    one, tgt = sharding.exchange_vocab_partials(torch.ones(4, 3, 2), torch.ones(4))   # a single process
    assert one.shape == (4, 3, 2) and tgt.shape == (4,)


def test_a_prepared_call_is_refused_on_another_device(monkeypatch):
    # its pointers are the first device's; the launch would go to the current one
    made = []

    class Call:
        argtypes = [ctypes.POINTER(B.Config), ctypes.c_int32, ctypes.c_void_p]

        def __call__(self, c, layer, stream):
            made.append((layer.value, stream.value))
            return B.OK

    device = [1]
    monkeypatch.setattr(B, "_current_device", lambda: device[0])
    monkeypatch.setattr(B, "_raw_stream", lambda d: 0x40 + d)
    call = B.Prepared(Call(), cfg(), (7, B._stream()))
    call()
    assert made == [(7, 0x41)]
    device[0] = 0
    with pytest.raises(B.SirllmError) as err:
        call()
    assert err.value.code == B.ERR_BAD_CONFIG and "cuda:1" in str(err.value) and made == [(7, 0x41)]
    device[0] = 1
    call()
    assert len(made) == 2
