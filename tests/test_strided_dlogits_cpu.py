"""dlogits that the binding allocates for logits that are a view of wider rows: the kernels step both by one row stride."""
import torch

import paper_2606_05597_amd as grpo


def test_gradients_of_strided_logits_get_their_stride():
    wide = torch.empty(4, 16)[:, :10]
    d = grpo._dlogits_arg(True, wide)
    assert d.shape == wide.shape and d.stride() == wide.stride()
