"""What a row's kept sums say: { max_j x_j, sum_j exp(x_j - max) }, of which a caller makes log-sum-exp and probabilities of its own.

Tolerance, before any run: with u = 2^-24 the sum is 1050 u deep (1024 steps in one lane, then lanes, waves and blocks), and every term's
exponent is off by a handful of roundings relative to itself, weighted with the term's share at most 8 u (2 + H), H the entropy.
"""
import numpy as np
import pytest
import torch

from oracle import sequence as sq

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("k", [0, 10])
@pytest.mark.parametrize("rows,vocab", [(12, 1), (12, 300), (12, 5003), (12, 70_001), (4104, 700), (4104, 3001)])
def test_stats_are_the_maximum_and_the_sum(rows, vocab, k, dt):
    import paper_2403_00877_amd as dmt
    rng = np.random.default_rng(vocab)
    x = rng.normal(size=(12, vocab)) * 2.5
    # the rows lie at 0, some distance, and on both sides of where exponents are taken in another way
    x[1:11] += np.array([10, -100, 1000.7, -5000.3, 3e4, -6e4, 3e5, -1.0e6, 1.1e6, -3e8])[:, None]
    x[11, 1:] = -np.inf
    x = torch.from_numpy(x).to(DT[dt]).cuda()
    if dt == "f16":
        x[7:11].clamp_(-6e4, 6e4)
    big = x.repeat(rows // 12, 1)
    st = torch.full((rows, 2), 7.0, device="cuda")
    top = torch.empty(rows, k, dtype=torch.int32, device="cuda") if k else None
    ws = torch.empty(max(256, dmt.dmt_token_logprob_workspace_bytes(rows, vocab, k)), dtype=torch.uint8, device="cuda")
    dmt.dmt_token_logprob_fwd(big, top_ids=top, stats=st, workspace=ws)
    x64 = x.cpu().double().numpy()
    m = x64.max(1)
    s = np.exp(x64 - m[:, None]).sum(1)
    h = sq.token_logprob(x64, np.full(12, -1), 0)[1]
    got = st.cpu().double().numpy().reshape(-1, 12, 2)
    assert (got[:, :, 0] == m).all()
    off = abs(got[:, :, 1] - s) / s
    assert (off <= 1050 * U32 + 8 * U32 * (2 + h)).all(), (off.max(0) / U32).tolist()
