"""The example model with a history block, whole: every gradient of a training step against autograd in float64, and the states that
a server moves on item by item against the scan over the whole history."""
import os
import sys

import pytest
import torch

from oracle import history as hs

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _reference(m, history, target):
    """Loss and gradients of the same model in float64 on the CPU: the experts that were chosen and the masks of the dropouts given."""
    p = {n: v.detach().double().cpu().requires_grad_() for n, v in m.copies.items()}
    h, t = history.cpu().long(), target.cpu().long()
    B, L, D, n = m.batch, m.length, m.dim, m.n
    seed, step = m.rng.tolist()
    q = hs.dropout_threshold(m.p) / 65536
    keep = [torch.from_numpy(hs.dropout_keep(n, D, m.p, seed, step, site)).double() / (1 - q) for site in (0, 1)]

    def norm(x, which):
        mean, var = x.mean(-1, keepdim=True), x.var(-1, unbiased=False, keepdim=True)
        return (x - mean) / torch.sqrt(var + 1e-5) * p["gamma%d" % which] + p["beta%d" % which]

    e = torch.where((h >= 0)[..., None], p["table"][h.clamp(min=0)] * m.scale, 0.0)
    y1 = norm(e, 1)
    f, v = torch.sigmoid(y1 @ p["w_gate"].t() + p["b_gate"]), y1 @ p["w_value"].t()
    state, rows = torch.zeros(B, D, dtype=torch.float64), []
    for i in range(L):
        there = (h[:, i] >= 0)[:, None]
        state = torch.where(there, f[:, i] * state + (1 - f[:, i]) * v[:, i], state)
        rows.append(torch.where(there, state, 0.0))
    r1 = e.reshape(n, D) + torch.stack(rows, 1).reshape(n, D) * keep[0]
    y2 = norm(r1, 2)
    top, slot = m.top.cpu().long(), m.slot.cpu()
    route = (y2 @ p["w_route"].t()).gather(1, top.clamp(min=0))
    share = torch.softmax(route, 1)
    mixed = 0.0
    for x in range(m.experts):
        out = torch.relu(y2 @ p["w_exp%d" % x].t() + p["b_exp%d" % x])
        mixed = mixed + out * (share * ((top == x) & (slot >= 0))).sum(1, keepdim=True)
    r2 = r1 + mixed * keep[1]
    logp = torch.log_softmax(r2.view(B, L, D)[:, -1] @ p["table"].t(), 1)
    loss = -logp.gather(1, t[:, None]).mean()
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}


def _case(dtype, room, items=97, length=7, dim=32, batch=40):
    import history_block
    m = history_block.HistoryModel(items, length, dim, batch, experts=5, k=2, room=room, p=0.2, dtype=dtype, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    with torch.no_grad():
        for n, v in m.params.items():
            if v.dim() == 1:
                v.add_(0.1 * torch.randn(v.shape, generator=g, device="cuda"))
            m.copies[n].copy_(v)
    m.rng[1] = 11
    return m, *history_block.batch_of(g, items, length, batch)


@pytest.mark.parametrize("room", [0.5, 2.0])
def test_a_step_against_autograd(room):
    m, history, target = _case("f32", room)
    loss = float(m.backward(history, target))
    ref, grads = _reference(m, history, target)
    dropped = int(((m.slot < 0) & (m.top >= 0)).sum())
    assert (dropped > 0) == (room < 1)
    assert abs(loss - ref) <= 1e-5 * abs(ref)
    # float32 through ten layers: sums of up to 280 terms each, relative to the gradient's own size
    for n, g in m.grads.items():
        err = float((g.double().cpu() - grads[n]).norm() / grads[n].norm())
        assert err <= 2e-5, (n, err)
    assert int(m.bad) == -1


def test_states_moved_on_item_by_item_are_the_scans():
    m, history, _ = _case("f32", 5.0)
    m.capacity = m.n                                       # nothing is dropped, whatever the batch
    m.source = torch.zeros(m.experts * m.n, dtype=torch.int32, device="cuda")
    m.plan, m.towers = _wide_plan(m)
    query = m.forward(history, 0.0).clone()
    state = torch.zeros(m.batch, m.dim, device="cuda")
    users = torch.arange(m.batch, dtype=torch.int32, device="cuda")
    for i in range(m.length):
        items = history[:, i].contiguous()
        last = m.observe(state, torch.where(items >= 0, users, -1), items)
    # the same float32 steps in another order of sums: as the gradients above
    assert float((last - query).norm() / query.norm()) <= 2e-5
    assert int(m.bad) == -1


def _wide_plan(m):
    import paper_2403_00877_amd as dmt
    E, cap = m.experts, m.capacity
    plan = dmt.dmt_plan_create([1] * E, [m.dim] * E, "f32", E, list(range(E)), cap, 1)
    m.sent, m.answer = (torch.zeros(E * cap, m.dim, device="cuda") for _ in range(2))
    m.ws["tower"] = torch.empty(max(256, dmt.dmt_tm_workspace_bytes(plan, m.towers, cap)), dtype=torch.uint8, device="cuda")
    return plan, m.towers


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_example_runs(dtype, capsys):
    import history_block
    history_block.main(["--steps", "20", "--batch", "128", "--dtype", dtype])
    assert "next item found" in capsys.readouterr().out
