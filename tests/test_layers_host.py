"""More host-side checks of the linear layer, the embedding and AdamW. Nothing here launches a kernel, so
these tests run without a GPU; the addresses are never dereferenced."""
from test_layers_abi import INVALID, at, bwd, emb_bwd, emb_fwd, emb_shape, fwd, lib, linear_shape  # noqa: F401


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
