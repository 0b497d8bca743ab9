"""What the binding of the adapters and lists refuses, by name and before the library is called."""
import pytest

import paper_2609_33977_amd as gm


def test_lists_refuse_missing_tensors():
    import torch
    t, big = torch.zeros(4), torch.zeros(1 << 12, dtype=torch.uint8)
    with pytest.raises(ValueError, match="g is required"):
        gm.gm_tensor_list(None, big)
    with pytest.raises(ValueError, match=r"g\[1\] is required"):
        gm.gm_tensor_list([t, None], big)
    for name in ("p", "m", "v", "p16"):
        rest = {"p": [t], "m": [t], "v": [t], "p16": [t.bfloat16()], name: [None]}
        with pytest.raises(ValueError, match=f"{name} must hold a tensor"):
            gm.gm_tensor_list([t], big, **rest)
