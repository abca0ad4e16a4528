"""The example model, whole: every gradient of a training step against autograd in float64, the clipped step, what it
recommends, and that it learns."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _reference(m, params, history, target):
    """Loss and gradients of the same model in float64 on the CPU."""
    p = {n: v.detach().double().cpu().requires_grad_() for n, v in params.items()}
    h, t = history.cpu().long(), target.cpu().long()
    emb = torch.where((h >= 0)[..., None], p["table"][h.clamp(min=0)] * m.scale, 0.0)
    mean, var = emb.mean(-1, keepdim=True), emb.var(-1, unbiased=False, keepdim=True)
    y = (emb - mean) / torch.sqrt(var + 1e-5) * p["gamma"] + p["beta"]
    q = torch.relu(y.reshape(m.batch, -1) @ p["w_proj"].t() + p["b_proj"])
    logp = torch.log_softmax(q @ p["table"].t(), 1)
    loss = -logp.gather(1, t[:, None]).mean()
    loss.backward()
    return float(loss.detach()), {n: v.grad for n, v in p.items()}, logp.detach()


def _case(dtype, items=301, length=5, dim=32, batch=48):
    import next_item
    m = next_item.NextItem(items, length, dim, batch, dtype, max_norm=0.05)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    with torch.no_grad():
        for n in ("gamma", "beta", "b_proj"):
            m.params[n].add_(0.1 * torch.randn(m.params[n].shape, generator=g, device="cuda"))
            m.copies[n].copy_(m.params[n])
    return m, *next_item.batch_of(g, items, length, batch)


def test_a_step_against_autograd():
    m, history, target = _case("f32")
    loss = float(m.backward(history, target))
    ref, grads, logp = _reference(m, m.copies, history, target)
    assert abs(loss - ref) <= 1e-5 * abs(ref)
    # float32 through five layers: sums of up to 301 terms each, relative to the gradient's own size
    for n, g in m.grads.items():
        err = float((g.double().cpu() - grads[n]).norm() / grads[n].norm())
        assert err <= 1e-5, (n, err)
    before = {n: p.clone() for n, p in m.params.items()}
    m.step(history, target)
    norm = float(torch.sqrt(sum((g ** 2).sum() for g in grads.values())))
    assert norm > m.max_norm and abs(float(m.norm) - norm) <= 1e-5 * norm
    for n, p in m.params.items():
        moved = before[n].double().cpu() - m.lr * (m.max_norm / norm) * grads[n]
        assert float((p.double().cpu() - moved).norm()) <= 1e-5 * float(moved.norm()), n
    assert int(m.bad) == -1


def test_recommendations_are_the_best_items():
    m, history, target = _case("f32")
    ids, logprobs = m.recommend(history)
    _, _, logp = _reference(m, m.copies, history, target)
    best = torch.topk(logp, ids.shape[1], dim=1)
    assert np.abs(logprobs.double().cpu().numpy() - best.values.numpy()).max() <= 1e-4
    # an item of another order only where two lie closer than the scores' own errors
    got = logp.gather(1, ids.cpu().long())
    assert float((got - best.values).abs().max()) <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_example_learns(dtype, capsys):
    import next_item
    hit = next_item.main(["--items", "500", "--steps", "300", "--dtype", dtype])
    assert hit > 0.9, capsys.readouterr().out
