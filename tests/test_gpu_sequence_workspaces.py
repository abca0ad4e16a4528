"""Workspaces that are no piece of GPU memory of their size are refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("make", [lambda n: torch.empty(n, dtype=torch.uint8),
                                  lambda n: torch.empty(n, dtype=torch.uint8).pin_memory(),
                                  lambda n: torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2],
                                  lambda n: torch.empty(1, dtype=torch.uint8, device="cuda").expand(n)],
                         ids=["host", "pinned", "strided", "expanded"])
def test_workspaces_that_are_refused(make):
    import paper_2403_00877_amd as dmt
    f32 = lambda *s: torch.full(s, 7.0, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    ws = make(1 << 20)
    x, out, stat, vec, norm, top = f32(600, 64), f32(600, 64), f32(600), f32(64), f32(1), i32(600, 3)
    lst = dmt.make_grad_list([x])
    calls = [lambda: dmt.dmt_embed_bwd(i32(600), x, out, ws),
             lambda: dmt.dmt_layer_norm_bwd(x, None, stat, stat, x, out, vec, vec, ws),
             lambda: dmt.dmt_token_logprob_fwd(x, i32(600), stat, stat, top, workspace=ws),
             lambda: dmt.dmt_grad_norm(lst, norm, ws),
             lambda: dmt.dmt_grad_clip(lst, 1.0, norm, ws)]
    for call in calls:
        with pytest.raises(AssertionError):
            call()
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((stat == 7).all()) and bool((vec == 7).all()) and float(norm) == 7
