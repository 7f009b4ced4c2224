"""What the calls for streams with a past in common refuse, on the host and before anything is enqueued
(no GPU needed): ``sirllm_beam_select``, ``sirllm_reorder_streams``, ``sirllm_attend_shared``."""
import ctypes
import math

import pytest
import torch

from paper_2405_12528_b200 import binding as B


@pytest.fixture(scope="module")
def lib(cuda_library):
    return B.lib()


def cfg(**kw):
    base = dict(n_streams=8, n_layers=3, n_kv_heads=2, head_dim=64, capacity=128, budget=64, n_sink=4, n_recent=8,
                max_new=8, vocab=1000, logits_dtype="f32", kv_dtype="bf16")
    base.update(kw)
    return B.make_config(**base)


P, WS = 0x2000, 0x1000      # never dereferenced


def select(lib, c=None, **kw):
    a = dict(logits=P, group=4, n_out=4, totals=P, ended=None, end=2, places=0, totals_out=P, source=P, tok=P, ent=P,
             fin=None, ws=WS)
    a.update(kw)
    return lib.sirllm_beam_select(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(logits=None)), (B.ERR_NULL, dict(totals=None)), (B.ERR_NULL, dict(totals_out=None)),
    (B.ERR_NULL, dict(source=None)), (B.ERR_NULL, dict(tok=None)), (B.ERR_NULL, dict(ws=None)),
    (B.ERR_BAD_CONFIG, dict(group=0)), (B.ERR_BAD_CONFIG, dict(group=-4)), (B.ERR_BAD_CONFIG, dict(group=3)),
    (B.ERR_BAD_CONFIG, dict(group=16)), (B.ERR_BAD_CONFIG, dict(n_out=0)), (B.ERR_BAD_CONFIG, dict(n_out=-1)),
    (B.ERR_BAD_CONFIG, dict(n_out=5, places=1, totals_out=2 * P)), (B.ERR_BAD_CONFIG, dict(end=-2)),
    (B.ERR_BAD_CONFIG, dict(end=1000)), (B.ERR_BAD_CONFIG, dict(n_out=5)),   # in place, of another size
    (B.ERR_BAD_CONFIG, dict(n_out=5, totals_out=2 * P, ended=P, fin=P)),
    (B.ERR_TOO_LARGE, dict(n_out=65, totals_out=2 * P)),
    (B.ERR_ALIGN, dict(logits=P + 2)), (B.ERR_ALIGN, dict(totals=P + 2)), (B.ERR_ALIGN, dict(ended=P + 1)),
    (B.ERR_ALIGN, dict(totals_out=P + 2)), (B.ERR_ALIGN, dict(source=P + 2)), (B.ERR_ALIGN, dict(tok=P + 3)),
    (B.ERR_ALIGN, dict(ent=P + 2)), (B.ERR_ALIGN, dict(fin=P + 2)), (B.ERR_ALIGN, dict(ws=WS + 128)),
])
def test_select_refusals(lib, want, kw):
    assert select(lib, **kw) == want


def test_select_refuses_large_groups_and_bad_configurations(lib):
    assert select(lib, cfg(n_streams=130), group=65, n_out=4, totals_out=2 * P) == B.ERR_TOO_LARGE
    assert select(lib, cfg(budget=5)) == B.ERR_BAD_CONFIG
    assert select(lib, cfg(vocab=2**26 + 1)) == B.ERR_TOO_LARGE
    assert select(lib, cfg(n_streams=2**24, n_layers=1, vocab=2**31 - 1), group=1, n_out=1) == B.ERR_TOO_LARGE


def test_beam_workspace(lib):
    assert B.sirllm_beam_workspace_bytes(cfg()) > 0
    assert B.sirllm_beam_workspace_bytes(cfg(budget=5)) == 0
    c = ctypes.byref(cfg())
    assert lib.sirllm_beam_workspace_init(c, None, None) == B.ERR_NULL
    assert lib.sirllm_beam_workspace_init(c, WS + 16, None) == B.ERR_ALIGN


def reorder(lib, c=None, **kw):
    a = dict(group=4, source=P, shared=None, scores=P, serial=P, live=P, k=P, v=P, ws=WS)
    a.update(kw)
    return lib.sirllm_reorder_streams(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(source=None)), (B.ERR_NULL, dict(live=None)), (B.ERR_NULL, dict(ws=None)),
    (B.ERR_BAD_CONFIG, dict(group=0)), (B.ERR_BAD_CONFIG, dict(group=-1)), (B.ERR_BAD_CONFIG, dict(group=3)),
    (B.ERR_ALIGN, dict(k=P + 8)), (B.ERR_ALIGN, dict(v=P + 2)), (B.ERR_ALIGN, dict(source=P + 2)),
    (B.ERR_ALIGN, dict(shared=P + 2)), (B.ERR_ALIGN, dict(scores=P + 2)), (B.ERR_ALIGN, dict(serial=P + 4)),
    (B.ERR_ALIGN, dict(live=P + 1)), (B.ERR_ALIGN, dict(ws=WS + 4)),
])
def test_reorder_refusals(lib, want, kw):
    assert reorder(lib, **kw) == want


def test_reorder_refuses_large_groups_and_bad_configurations(lib):
    assert reorder(lib, cfg(n_streams=514), group=257) == B.ERR_TOO_LARGE
    assert reorder(lib, cfg(head_dim=20)) == B.ERR_BAD_CONFIG


def attend(lib, c=None, **kw):
    a = dict(layer=0, group=4, shared=P, q=P, n_heads=4, qs=256, k=P, v=P, kv_len=P, scale=0.1, out=P, os=256, lse=None,
             ws=WS)
    a.update(kw)
    return lib.sirllm_attend_shared(ctypes.byref(c or cfg()), *a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (B.ERR_NULL, dict(shared=None)), (B.ERR_NULL, dict(q=None)), (B.ERR_NULL, dict(k=None)), (B.ERR_NULL, dict(v=None)),
    (B.ERR_NULL, dict(kv_len=None)), (B.ERR_NULL, dict(out=None)), (B.ERR_NULL, dict(ws=None)),
    (B.ERR_BAD_CONFIG, dict(layer=3)), (B.ERR_BAD_CONFIG, dict(group=0)), (B.ERR_BAD_CONFIG, dict(group=3)),
    (B.ERR_BAD_CONFIG, dict(group=16)), (B.ERR_BAD_CONFIG, dict(group=-8)),
    (B.ERR_BAD_CONFIG, dict(n_heads=0)), (B.ERR_BAD_CONFIG, dict(n_heads=3)), (B.ERR_BAD_CONFIG, dict(scale=math.nan)),
    (B.ERR_BAD_CONFIG, dict(scale=3e38)), (B.ERR_BAD_CONFIG, dict(qs=128)), (B.ERR_BAD_CONFIG, dict(os=128)),
    (B.ERR_ALIGN, dict(shared=P + 2)), (B.ERR_ALIGN, dict(q=P + 2)), (B.ERR_ALIGN, dict(out=P + 8)),
    (B.ERR_ALIGN, dict(k=P + 8)), (B.ERR_ALIGN, dict(qs=258)), (B.ERR_ALIGN, dict(kv_len=P + 2)),
    (B.ERR_ALIGN, dict(lse=P + 2)), (B.ERR_ALIGN, dict(ws=WS + 8)),
])
def test_attend_shared_refusals(lib, want, kw):
    assert attend(lib, **kw) == want


def test_attend_shared_refuses_sizes_and_configurations(lib):
    assert attend(lib, cfg(head_dim=264), qs=4 * 264, os=4 * 264) == B.ERR_TOO_LARGE
    assert attend(lib, cfg(budget=5)) == B.ERR_BAD_CONFIG
    assert lib.sirllm_attend_shared(None, 0, 4, P, P, 4, 256, P, P, P, 0.1, P, 256, None, WS, None) == B.ERR_NULL


def test_attend_shared_workspace(lib):
    size = B.sirllm_attend_shared_workspace_bytes
    assert size(cfg(), 4, 4) > 0
    for bad in (size(cfg(), 3, 4), size(cfg(), 0, 4), size(cfg(), 4, 3), size(cfg(), 4, 0), size(cfg(budget=5), 4, 4),
                size(cfg(head_dim=264), 4, 4)):
        assert bad == 0
    c = ctypes.byref(cfg())
    assert lib.sirllm_attend_shared_workspace_init(c, 4, 4, None, None) == B.ERR_NULL
    assert lib.sirllm_attend_shared_workspace_init(c, 4, 4, WS + 16, None) == B.ERR_ALIGN
    assert lib.sirllm_attend_shared_workspace_init(c, 3, 4, WS, None) == B.ERR_BAD_CONFIG
    assert lib.sirllm_attend_shared_workspace_init(c, 4, 3, WS, None) == B.ERR_BAD_CONFIG


# the binding: sizes, types and residence of every tensor
def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def bind_select(**kw):
    a = dict(logits=t(8, 1000), group=4, n_out=4, totals=t(8), ended=None, end=2, places=False, totals_out=t(8),
             source=t(8, dtype=torch.int32), tok=t(8, dtype=torch.int32), ent=None, fin=None,
             ws=t(1 << 20, dtype=torch.uint8))
    a.update(kw)
    B.sirllm_beam_select(cfg(), *a.values())


@pytest.mark.parametrize("kw", [
    dict(group=3), dict(group=0), dict(logits=t(7, 1000)), dict(logits=t(8, 999)),
    dict(logits=t(8, 1000, dtype=torch.bfloat16)), dict(totals=t(7)), dict(totals=t(8, dtype=torch.float64)),
    dict(ended=t(7, dtype=torch.int32)), dict(ended=t(8, dtype=torch.int64)), dict(totals_out=t(7)),
    dict(n_out=8), dict(source=t(8)), dict(tok=t(4, dtype=torch.int32)), dict(ent=t(7)), dict(fin=t(8)),
    dict(ws=t(64, dtype=torch.uint8)),
])
def test_select_binding_refuses_wrong_tensors(lib, kw):
    with pytest.raises(B.SirllmError) as e:
        bind_select(**kw)
    assert e.value.code == B.ERR_BAD_CONFIG


def bind_reorder(**kw):
    i = torch.int32
    kv = t(8, 3 * 2, 128, 64, dtype=torch.bfloat16)
    a = dict(group=4, source=t(8, dtype=i), shared=t(2, dtype=i), scores=t(8, 128), serial=t(8, 128, dtype=torch.int64),
             live=t(8, dtype=i), k=kv, v=kv, ws=t(1 << 20, dtype=torch.uint8))
    a.update(kw)
    B.sirllm_reorder_streams(cfg(), *a.values())


@pytest.mark.parametrize("kw", [
    dict(group=3), dict(source=t(7, dtype=torch.int32)), dict(source=t(8, dtype=torch.int64)),
    dict(shared=t(1, dtype=torch.int32)), dict(scores=t(8, 127)), dict(serial=t(8, 128)),
    dict(live=t(4, dtype=torch.int32)), dict(k=t(8, 6, 127, 64, dtype=torch.bfloat16)),
    dict(v=t(8, 6, 128, 64, dtype=torch.float16)), dict(ws=t(64, dtype=torch.uint8)),
])
def test_reorder_binding_refuses_wrong_tensors(lib, kw):
    with pytest.raises(B.SirllmError) as e:
        bind_reorder(**kw)
    assert e.value.code == B.ERR_BAD_CONFIG


def bind_attend(**kw):
    i = torch.int32
    kv, q = t(8, 6, 128, 64, dtype=torch.bfloat16), t(8, 4, 64, dtype=torch.bfloat16)
    a = dict(layer=0, group=4, shared=t(2, dtype=i), q=q, k=kv, v=kv, kv_len=t(8, dtype=i), scale=None, out=q, lse=None,
             ws=t(1 << 25, dtype=torch.uint8))
    a.update(kw)
    B.sirllm_attend_shared(cfg(), *a.values())


@pytest.mark.parametrize("kw", [
    dict(group=3), dict(shared=t(1, dtype=torch.int32)), dict(shared=t(2)), dict(q=t(7, 4, 64, dtype=torch.bfloat16)),
    dict(q=t(8, 4, 64)), dict(out=t(8, 2, 64, dtype=torch.bfloat16)), dict(k=t(8, 6, 128, 60, dtype=torch.bfloat16)),
    dict(kv_len=t(7, dtype=torch.int32)), dict(lse=t(8, 3)), dict(ws=t(64, dtype=torch.uint8)),
])
def test_attend_shared_binding_refuses_wrong_tensors(lib, kw):
    with pytest.raises(B.SirllmError) as e:
        bind_attend(**kw)
    assert e.value.code == B.ERR_BAD_CONFIG


def test_tensors_on_the_host_are_refused(lib):
    for call in (bind_select, bind_reorder, bind_attend):
        with pytest.raises(B.SirllmError) as e:
            call()
        assert e.value.code == B.ERR_NULL
