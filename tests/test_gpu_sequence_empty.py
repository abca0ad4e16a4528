"""Calls of no rows, ids or gradients, with workspaces of just the size that is asked for (an empty tensor has no address)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dmt():
    import paper_2403_00877_amd as d
    return d


def exactly(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def sevens(*shape):
    return torch.full(shape, 7.0, device="cuda")


@pytest.mark.parametrize("cols", [1, 16, 700, 8192, 9001, 20_000])
@pytest.mark.parametrize("given", ["both", "gamma", "beta"])
def test_layer_norm_bwd_of_no_rows(dmt, cols, given):
    x, mean = torch.empty(0, cols, device="cuda"), torch.empty(0, device="cuda")
    dg, db = (sevens(cols) if given in ("both", n) else None for n in ("gamma", "beta"))
    dmt.dmt_layer_norm_bwd(x, None, mean, mean, x, x, dg, db, exactly(dmt.dmt_layer_norm_bwd_workspace_bytes(0, cols)))
    assert all(bool((d == 0).all()) for d in (dg, db) if d is not None)
    dmt.dmt_layer_norm_bwd(x, None, mean, mean, x, x)


@pytest.mark.parametrize("rows", [1, 512, 513])
@pytest.mark.parametrize("cols", [16, 8193])
def test_layer_norm_bwd_with_just_its_workspace(dmt, rows, cols):
    x, dy = torch.ones(rows, cols, device="cuda"), torch.ones(rows, cols, device="cuda")
    mean, rstd, dx, dg, db = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), sevens(rows, cols), sevens(cols), sevens(cols)
    dmt.dmt_layer_norm_bwd(x, None, mean, rstd, dy, dx, dg, db, exactly(dmt.dmt_layer_norm_bwd_workspace_bytes(rows, cols)))
    assert bool((dg == rows).all()) and bool((db == rows).all())           # whole numbers: exact


def test_the_others_of_nothing(dmt):
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    table = sevens(300, 40)
    dmt.dmt_embed_fwd(table, ids, torch.empty(0, 40, device="cuda"))
    for accumulate, left in ((True, 7.0), (False, 0.0)):
        dmt.dmt_embed_bwd(ids, torch.empty(0, 40, device="cuda"), table, exactly(dmt.dmt_embed_bwd_workspace_bytes(0, 300, 40)),
                          accumulate=accumulate)
        assert bool((table == left).all())
    x, none = torch.empty(0, 9, device="cuda"), torch.empty(0, device="cuda")
    stats, top = torch.empty(0, 2, device="cuda"), torch.empty(0, 5, dtype=torch.int32, device="cuda")
    dmt.dmt_layer_norm_fwd(x, None, None, 1e-5, x, none, none)
    ws = exactly(dmt.dmt_token_logprob_workspace_bytes(0, 9, 5))
    dmt.dmt_token_logprob_fwd(x, ids, none, none, top, torch.empty(0, 5, device="cuda"), stats, ws)
    dmt.dmt_token_logprob_bwd(x, ids, stats, none, none, none, x)
    for grads in ([], [none]):
        lst, norm = dmt.make_grad_list(grads), sevens(1)
        dmt.dmt_grad_clip(lst, 1.0, norm, exactly(dmt.dmt_grad_norm_workspace_bytes(lst)))
        assert float(norm) == 0.0
