"""What the binding of the history block refuses before it looks at devices (nothing is launched)."""
import pytest
import torch

import paper_2403_00877_amd as dmt


def test_gradients_of_weights_need_the_experts_rows():
    dy, slot, weights, dweights = torch.ones(3, 4), torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, 2), torch.zeros(3, 2)
    for dz, source in ((None, None), (torch.zeros(6, 4), torch.zeros(6, dtype=torch.int32))):
        with pytest.raises(AssertionError, match="dweights"):
            dmt.dmt_expert_combine_bwd(dy, None, slot, source, weights, dz, dweights)
