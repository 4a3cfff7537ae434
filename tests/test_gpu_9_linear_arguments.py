"""The linear layer's binding: what is not a tensor is refused as every other wrong argument is."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wrong", [np.zeros((4, 40), np.float32), [0.0], 7, "x"], ids=["array", "list", "number", "text"])
def test_refuses_what_is_not_a_tensor(wrong):
    import torch
    import paper_2009_09271_amd as e
    x, w, y = (torch.zeros(*s, device="cuda") for s in ((4, 8), (40, 8), (4, 40)))
    q, s = e.ckpt_buffers(4, 8)
    calls = {"x": lambda: e.ef_linear_forward(wrong, w, y, None), "weight": lambda: e.ef_linear_forward(x, wrong, y, None),
             "y": lambda: e.ef_linear_forward(x, w, wrong, None), "bias": lambda: e.ef_linear_forward(x, w, y, None, bias=wrong),
             "res": lambda: e.ef_linear_forward(x, w, y, None, res=wrong), "ws": lambda: e.ef_linear_forward(x, w, y, wrong),
             "codes": lambda: e.ef_linear_forward(x, w, y, None, codes=wrong, scales=s), "dy": lambda: e.ef_linear_dgrad(wrong, w, x, None),
             "res ": lambda: e.ef_linear_dgrad(y, w, x, None, res=wrong), "ws ": lambda: e.ef_linear_dgrad(y, w, x, wrong),
             "scales": lambda: e.ef_linear_wgrad(y, q, wrong, 0, w, None), "dw": lambda: e.ef_linear_wgrad(y, q, s, 0, wrong, None),
             "db": lambda: e.ef_linear_wgrad(y, q, s, 0, w, None, db=wrong), "ws  ": lambda: e.ef_linear_wgrad(y, q, s, 0, w, wrong)}
    for name, call in calls.items():
        with pytest.raises(e.EfError) as ex:
            call()
        assert ex.value.code == e.EF_EINVAL and name.strip() in str(ex.value)
