"""Buffers that two tensors of an optimiser share: a step would write them from two blocks in no order, so
the optimiser is not made. (No step runs here.)"""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_adamw_gpu import HYPER, _device  # noqa: F401

pytestmark = pytest.mark.gpu


def test_refused():
    p, g = torch.ones(512, device="cuda"), torch.ones(512, device="cuda")
    q, h = p.clone(), g.clone()

    def refused(*args, **kw):
        with pytest.raises(flarepp.FlareppError) as e:
            flarepp.AdamW(*args, **kw, **HYPER)
        assert e.value.status == flarepp.ERR_INVALID_ARGUMENT

    refused([p, p], [g, h])                       # a tied weight given twice
    refused([p[:256], p[128:]], [g[:256], h[:384]])
    refused([p, q], [q, h])                       # a gradient that is another weight
    m = torch.zeros(512, device="cuda")
    refused([p, q], [g, h], state={"m": [m, m], "v": [g.clone(), g.clone()], "step": 0})
    low = p.bfloat16(), q.bfloat16()
    refused(low, [g, h], masters=[m, m])
    flarepp.AdamW([p, q], [g, g], **HYPER)        # a gradient may be read for two
    flarepp.AdamW([p[:256], p[256:]], [g[:256], g[256:]], **HYPER)
