"""What the binding of the history block refuses before it looks at devices (nothing is launched)."""
import pytest
import torch

import paper_2403_00877_amd as dmt


def test_gradients_of_weights_need_the_experts_rows():
    dy, slot, weights, dweights = torch.ones(3, 4), torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, 2), torch.zeros(3, 2)
    for dz, source in ((None, None), (torch.zeros(6, 4), torch.zeros(6, dtype=torch.int32))):
        with pytest.raises(AssertionError, match="dweights"):
            dmt.dmt_expert_combine_bwd(dy, None, slot, source, weights, dz, dweights)


def test_ids_need_the_number_of_sequences():
    x, ids, ws = torch.ones(4, 8), torch.zeros(4, dtype=torch.int32), torch.empty(256, dtype=torch.uint8)
    with pytest.raises(AssertionError, match="sequences"):
        dmt.dmt_gated_scan_fwd(x, x, x, ws, sequence_of=ids)
    with pytest.raises(AssertionError, match="sequences"):
        dmt.dmt_gated_scan_bwd(x, x, x, x, x, ws, ws, sequence_of=ids)
