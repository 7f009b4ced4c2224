"""Numbers that do not fit the C side's 32 bits are refused by the binding (ctypes would cut them down to others
that do: an end token of 2^32 + 5 to 5, layer 2^32 to layer 0); no GPU needed."""
import pytest
import torch

from paper_2405_12528_b200 import binding as B

WIDE = [2**31, 2**32, 2**32 + 1, -2**31 - 1, -2**32]


@pytest.fixture(scope="module", autouse=True)
def lib(cuda_library):
    return B.lib()


def cfg():
    return B.make_config(n_streams=8, n_layers=3, n_kv_heads=2, head_dim=64, capacity=128, budget=64, n_sink=4,
                         n_recent=8, max_new=8, vocab=1000, logits_dtype="f32", kv_dtype="bf16")


def refused(call, *args):
    with pytest.raises(B.SirllmError) as e:
        call(cfg(), *args)
    assert e.value.code == B.ERR_BAD_CONFIG
    with pytest.raises(B.SirllmError) as e:
        B.prepared(call, cfg(), *args)
    assert e.value.code == B.ERR_BAD_CONFIG


@pytest.mark.parametrize("wide", WIDE)
def test_select(wide):
    refused(B.sirllm_beam_select, None, 4, 4, None, None, wide, False, None, None, None, None, None, None)
    refused(B.sirllm_beam_select, None, 4, wide, None, None, -1, False, None, None, None, None, None, None)
    refused(B.sirllm_beam_select, None, wide, 4, None, None, -1, False, None, None, None, None, None, None)


@pytest.mark.parametrize("wide", WIDE)
def test_attend_shared(wide):
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    refused(B.sirllm_attend_shared, wide, 4, None, q, None, None, None, None, q, None, None)
    refused(B.sirllm_attend_shared, 0, wide, None, q, None, None, None, None, q, None, None)
    for size in (lambda: B.sirllm_attend_shared_workspace_bytes(cfg(), wide + 4, 4),
                 lambda: B.sirllm_attend_shared_workspace_bytes(cfg(), 4, wide + 4)):
        assert size() == 0
    with pytest.raises(B.SirllmError):
        B.new_attend_shared_workspace(cfg(), 4, wide + 4)


@pytest.mark.parametrize("wide", WIDE)
def test_other_calls(wide):
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    refused(B.sirllm_attend, wide, q, None, None, None, None, q, None, None)
    refused(B.sirllm_keep_policy, wide, None, 1, 0, 0, None, None, None)
    refused(B.sirllm_reorder_streams, wide, None, None, None, None, None, None, None, None)


@pytest.mark.parametrize("n", [2**31 - 1, -2**31, -1, 0])
def test_numbers_that_fit_go_through(n):
    with pytest.raises(B.SirllmError) as e:   # as far as the tensors, of which one is not on a GPU
        B.sirllm_beam_select(cfg(), None, 4, 4, torch.zeros(8), None, n, False, None, None, None, None, None, None)
    assert e.value.code == B.ERR_NULL
