"""Calls of the adapters' binding that the header allows."""
import pytest

from gpu_support import say
from lora_support import make, plan_of

pytestmark = pytest.mark.gpu


def test_backward_without_outputs_needs_no_workspace():
    import paper_2609_33977_amd as gm
    say("adapters: a backward that is asked for nothing; one that is asked for dA without a workspace")
    import torch
    c = make(20, 2, 64, (40,), 16)
    args = [t.cuda() for t in (c.dY, c.X, c.A, c.B, c.scale)]
    plan = plan_of(gm, c.ids, c.n)
    gm.gm_lora_bwd(*args, plan, None)
    dA = torch.full(c.A.shape, 3.0, device="cuda")
    with pytest.raises(ValueError, match="ws is required"):
        gm.gm_lora_bwd(*args, plan, None, dA=dA)
    torch.cuda.synchronize()
    assert bool((dA == 3.0).all())
