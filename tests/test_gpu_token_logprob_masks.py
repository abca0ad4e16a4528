"""The gradient at masked scores: 0, whatever stands beside the mask and whatever gradient comes in."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [2, 300, 5003, 20_000])
def test_masked_scores_have_no_gradient(vocab, dt):
    import paper_2403_00877_amd as dmt
    rng = np.random.default_rng(vocab)
    nothing, plain, nan, inf, big = range(0, 4), range(4, 8), 8, 9, 10
    x = rng.normal(size=(11, vocab))
    masked = rng.random((11, vocab)) < 0.4
    masked[:, 0], masked[:, 1] = False, True
    masked[nothing] = True
    x[masked] = -np.inf
    x[nan, 0], x[inf, 0], x[big, 0] = np.nan, np.inf, 6e4
    x = torch.from_numpy(x).to(DT[dt]).cuda()
    # the rows' incoming gradients: 1, NaN, inf, -inf for those without a score and for ordinary ones; targets that are masked among them
    odd = [1.0, math.nan, math.inf, -math.inf]
    g = torch.tensor(odd + odd + [1.0, 1.0, 1.0], device="cuda")
    t = torch.tensor([0, 1, 1, 0, 1, 0, 1, 0, 1, 1, 1], dtype=torch.int32, device="cuda")
    lp, h, st = torch.empty(11, device="cuda"), torch.empty(11, device="cuda"), torch.empty(11, 2, device="cuda")
    ws = torch.empty(max(256, dmt.dmt_token_logprob_workspace_bytes(11, vocab, 0)), dtype=torch.uint8, device="cuda")
    dmt.dmt_token_logprob_fwd(x, t, lp, h, stats=st, workspace=ws)
    at = torch.from_numpy(masked).cuda()
    for a, b in ((g, None), (None, g), (g, g)):
        dx = torch.full_like(x, 7.0)
        dmt.dmt_token_logprob_bwd(x, t, st, h, a, b, dx)
        assert bool((dx[at] == 0).all()), (dx != 0).logical_and(at).any(1).nonzero().tolist()
        # what is not masked says that something is wrong with the row
        for r in (*plain[1:], nan, inf):
            assert not bool(dx[r, 0].isfinite()), r
        assert bool(dx[plain[0]].isfinite().all()) and bool(dx[big].isfinite().all())
    for large in (1e37, -3e38):
        g.fill_(large)
        for a, b in ((g, None), (None, g), (g, g)):
            dx = torch.full_like(x, 7.0)
            dmt.dmt_token_logprob_bwd(x, t, st, h, a, b, dx)
            assert bool((dx[at] == 0).all()), large
