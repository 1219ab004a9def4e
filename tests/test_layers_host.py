"""More host-side checks of the linear layer, the embedding and AdamW. Nothing here launches a kernel, so
these tests run without a GPU; the addresses are never dereferenced."""
import ctypes
from unittest import mock

import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_layers_abi import INVALID, at, bwd, emb_bwd, emb_fwd, emb_shape, fwd, lib, linear_shape, tensor  # noqa: F401


def test_status_words_off_four_bytes_are_refused(lib):  # noqa: F811
    for off in (1, 2, 3):
        word = at(20) + off
        assert fwd(lib, linear_shape(in_=63), status=word) == INVALID
        assert fwd(lib, linear_shape(rows=3), status=word) == INVALID
        assert bwd(lib, linear_shape(act=2), status=word) == INVALID
        assert emb_fwd(lib, emb_shape(), status=word) == INVALID
        assert emb_bwd(lib, emb_shape(), status=word) == INVALID


def test_status_question_wants_an_answer_s_place(lib):  # noqa: F811
    assert lib.flarepp_layers_device_status(None, None) == INVALID


def test_only_8_bit_states_are_rounded_without_bias(lib):  # noqa: F811
    table = (flarepp.AdamwTensor * 1)(tensor())

    def step(n, bits, **over):
        h = flarepp.AdamwHyper(1e-3, 0.9, 0.999, 1e-8, 0.0, over.get("step", 1), bits)
        return lib.flarepp_adamw_step_unbiased(table, n, ctypes.byref(h), None)

    assert step(0, 8) == flarepp.OK
    assert step(0, 32) == step(0, 16) == step(0, 8, step=0) == INVALID
    table[0] = tensor(m_scale=0)
    assert step(1, 8) == INVALID
    assert lib.flarepp_adamw_step_unbiased(table, 0, None, None) == INVALID


def test_a_stream_of_another_device_is_refused():
    """The call would run on the current stream of its tensors' device, in no order with the given one."""
    stream = mock.Mock(spec=torch.cuda.Stream, device=torch.device("cuda", 1), cuda_stream=16)
    with pytest.raises(ValueError):
        flarepp._current(stream, torch.device("cuda", 0))


def test_buffers_that_a_step_writes_lie_apart():
    apart = flarepp._check_apart
    apart([])
    apart([(0, 16, True, "a"), (16, 32, True, "b"), (40, 44, False, "c"), (40, 60, False, "d")])
    apart([(8, 8, True, "empty"), (0, 16, True, "a")])
    for bad in ([(0, 16, True, "a"), (0, 16, True, "b")],                              # the same twice
                [(8, 20, False, "b"), (0, 16, True, "a")],                             # read where written
                [(0, 100, False, "a"), (10, 20, False, "b"), (30, 40, True, "c")],     # inside another
                [(0, 100, True, "a"), (10, 20, False, "b"), (30, 40, False, "c")]):
        with pytest.raises(flarepp.FlareppError) as e:
            apart(bad)
        assert e.value.status == INVALID
