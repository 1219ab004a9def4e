"""Going on from saved parameters and ``state_dict()`` alone gives the bits of the run that was never
interrupted, masters included."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_adamw_gpu import HYPER, _device  # noqa: F401

pytestmark = pytest.mark.gpu


def copied(state):
    return {k: [None if t is None else t.clone() for t in x] if isinstance(x, list) else x
            for k, x in state.items()}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("masters", [True, None])
def test_masters_are_part_of_the_state(bits, masters):
    g = torch.Generator(device="cuda").manual_seed(3)
    params = [torch.randn(n, generator=g, device="cuda").to(dt)
              for n, dt in ((700, torch.bfloat16), (300, torch.float32), (64, torch.bfloat16))]
    grads = [torch.zeros_like(p, dtype=torch.float32) for p in params]

    def steps(opt, n, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for _ in range(n):
            for x in grads:
                x.normal_(generator=gen)
            opt.step()

    whole = flarepp.AdamW(params, grads, state_bits=bits, masters=True, **dict(HYPER, lr=1e-4))
    steps(whole, 5, seed=1)
    half_p, saved = [p.clone() for p in params], copied(whole.state_dict())
    steps(whole, 5, seed=2)
    rest = flarepp.AdamW(half_p, grads, state_bits=bits, masters=masters, state=saved,
                         **dict(HYPER, lr=1e-4))
    steps(rest, 5, seed=2)
    assert rest.steps == whole.steps == 10 and rest.masters[1] is None
    for a, b in zip(params, half_p):
        assert torch.equal(a, b)
    for i in (0, 2):
        assert torch.equal(whole.masters[i], rest.masters[i])
        assert not torch.equal(whole.masters[i], params[i].float())  # the masters hold more than params


def test_a_state_without_masters_and_masters_refused():
    p, g = [torch.ones(8, device="cuda").bfloat16()], [torch.ones(8, device="cuda")]
    saved = flarepp.AdamW(p, g, masters=True, **HYPER).state_dict()
    assert flarepp.AdamW(p, g, masters=False, state=saved, **HYPER).masters == [None]
    given = [torch.zeros(8, device="cuda")]
    assert flarepp.AdamW(p, g, masters=given, state=saved, **HYPER).masters[0].data_ptr() == given[0].data_ptr()
    del saved["masters"]
    assert torch.equal(flarepp.AdamW(p, g, masters=True, state=saved, **HYPER).masters[0], p[0].float())
