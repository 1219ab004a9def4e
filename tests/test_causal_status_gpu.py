"""A status word keeps the worst of what was recorded in it: a wait that gave up (outputs are invalid) is not
hidden by an argument that was brought into its range (they are not)."""
import math

import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_decay_gpu import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    flarepp.layers_status()
    yield
    assert flarepp.layers_status() == flarepp.OK


def calls():
    q, k, v, ld, dy, S, _ = inputs(1, 2, 2, 700, 64, 64)
    ld[1] = 0.5  # counts as 0, and is recorded
    wrong = torch.tensor([0, 900, 700], dtype=torch.int32, device="cuda")
    S2 = torch.cat((S, S))
    X, n = torch.zeros(2, 30, 16, device="cuda"), torch.tensor([-1, 99], dtype=torch.int32, device="cuda")
    ids = torch.tensor([3, 99], dtype=torch.int32, device="cuda")
    table = torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda")
    return {
        "fwd": lambda s: flarepp.decay_attention_fwd(q, k, v, ld, state=S, status=s),
        "bwd": lambda s: flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, status=s),
        "offsets": lambda s: flarepp.decay_attention_fwd(q, k, v, ld.clamp(max=0), state=S2, offsets=wrong, status=s),
        "step": lambda s: flarepp.decay_attention_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], ld, S.clone(), status=s),
        "norm": lambda s: flarepp.group_norm_fwd(X, 2, lengths=n, status=s),
        "norm of few rows": lambda s: flarepp.group_norm_fwd(X[:, :3].contiguous(), 2, lengths=n, status=s),
        "embedding": lambda s: flarepp.embedding_fwd(ids, table, scale=1.0, status=s),
    }


@pytest.mark.parametrize("name", ["fwd", "bwd", "offsets", "step", "norm", "norm of few rows", "embedding"])
def test_a_worse_word_stays(name):
    call = calls()[name]
    for before, after in ((flarepp.OK, flarepp.ERR_INVALID_ARGUMENT), (flarepp.ERR_TIMEOUT, flarepp.ERR_TIMEOUT)):
        status = torch.full((1,), before, dtype=torch.int32, device="cuda")
        call(status)
        assert int(status) == after


@pytest.mark.parametrize("own", [True, False])
def test_a_wait_that_gave_up_early_in_a_backward(own):
    """Its first launches' waits run out; its later ones record the decay above 0 (with the word of the caller's and
    with the library's)."""
    q, k, v, ld, dy, S, _ = inputs(1, 2, 2, 700, 64, 64)
    ld[1] = 0.5
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if own else None
    lib = flarepp.load()
    lib.flarepp_test_wait_fault(19, 1, 20_000_000)
    try:
        flarepp.decay_attention_fwd(q, k, v, ld, state=S, status=status)
    finally:
        lib.flarepp_test_wait_fault(0, -1, 0)
    flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, status=status)
    torch.cuda.synchronize()
    assert (int(status) if own else flarepp.layers_status()) == flarepp.ERR_TIMEOUT
