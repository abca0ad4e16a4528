"""A next-item model on one GPU: the sequence branch's operators and a Tower Module, trained and asked.

    python examples/next_item.py [--steps N] [--dtype f32|bf16]

A user's history of L items (empty slots are -1) becomes L scaled embeddings, each normalised; side by side they are the
input of a Tower Module (linear + ReLU), whose output is scored against every item's embedding (the table is used twice):

    dmt_embed_fwd -> dmt_layer_norm_fwd -> dmt_tower_module_fwd -> scores -> dmt_token_logprob_fwd

and back through the same, the table's gradient summed over both uses, all gradients clipped to one global norm:

    dmt_token_logprob_bwd -> dmt_tower_module_bwd -> dmt_layer_norm_bwd -> dmt_embed_bwd -> dmt_grad_clip

The product with the table is a plain matrix product and left to the library for those.  Data: synthetic histories whose next item
follows from the last one.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2403_00877_amd as dmt  # noqa: E402

EPS = 1e-5


class NextItem:
    """Parameters in float32 with working copies in `dtype`, gradients in float32, buffers for one batch size."""

    def __init__(self, items: int, length: int, dim: int, batch: int, dtype: str = "f32", seed: int = 0,
                 lr: float = 0.5, max_norm: float = 1.0, top: int = 10):
        self.items, self.length, self.dim, self.batch = items, length, dim, batch
        self.lr, self.max_norm, self.scale = lr, max_norm, math.sqrt(dim)
        self.dtype = dt = dmt.binding.TORCH_DTYPE[dmt.binding.DTYPE_CODE[dtype]]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        wide = length * dim
        f32 = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device="cuda")
        work = lambda *shape: torch.empty(*shape, dtype=dt, device="cuda")
        draw = lambda bound, *shape: (torch.rand(*shape, generator=g, device="cuda") * 2 - 1) * bound
        self.params = dict(table=draw(1 / math.sqrt(dim), items, dim), gamma=f32(dim) + 1, beta=f32(dim),
                           w_proj=draw(1 / math.sqrt(wide), dim, wide), b_proj=f32(dim))
        self.copies = {n: p.to(dt, copy=True) for n, p in self.params.items()}
        self.grads = {n: torch.zeros_like(p) for n, p in self.params.items()}
        # one tower whose features are the history's slots
        self.plan = dmt.dmt_plan_create([1] * length, [dim] * length, dtype, 1, [0] * length, batch, 1)
        tower = dict(kind="linear_relu", out_dim=dim, w_proj=self.copies["w_proj"], b_proj=self.copies["b_proj"])
        self.tower = dmt.make_tm_params([tower])
        self.tower_grads = dmt.make_tm_grads([dict(dw_proj=self.grads["w_proj"], db_proj=self.grads["b_proj"])])
        self.grad_list = dmt.make_grad_list(list(self.grads.values()))
        n = batch * length
        self.emb, self.normed, self.query = work(n, dim), work(n, dim), work(batch, dim)
        self.mean, self.rstd = f32(n), f32(n)
        self.logprob, self.entropy, self.stats = f32(batch), f32(batch), f32(batch, 2)
        self.top_ids = torch.empty(batch, top, dtype=torch.int32, device="cuda")
        self.top_logprobs = f32(batch, top)
        self.weight = torch.full((batch,), -1.0 / batch, device="cuda")       # d(mean of -logprob) / d(logprob)
        self.grad_query, self.grad_normed, self.grad_emb = f32(batch, dim), f32(n, dim), f32(n, dim)
        self.norm = f32(1)
        self.bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
        scratch = lambda b: torch.empty(max(256, b), dtype=torch.uint8, device="cuda")
        self.ws = dict(tower=scratch(dmt.dmt_tm_workspace_bytes(self.plan, self.tower, batch)),
                       tower_bwd=scratch(dmt.dmt_tm_bwd_workspace_bytes(self.plan, self.tower, batch)),
                       norm_bwd=scratch(dmt.dmt_layer_norm_bwd_workspace_bytes(n, dim)),
                       embed_bwd=scratch(dmt.dmt_embed_bwd_workspace_bytes(n, items, dim)),
                       logprob=scratch(dmt.dmt_token_logprob_workspace_bytes(batch, items, top)),
                       clip=scratch(dmt.dmt_grad_norm_workspace_bytes(self.grad_list)))

    def scores(self, history: torch.Tensor) -> torch.Tensor:
        """[batch][items] from int32 [batch][length]."""
        c = self.copies
        dmt.dmt_embed_fwd(c["table"], history, self.emb, self.scale, self.bad)
        dmt.dmt_layer_norm_fwd(self.emb, c["gamma"], c["beta"], EPS, self.normed, self.mean, self.rstd)
        dmt.dmt_tower_module_fwd(self.plan, self.tower, self.normed, self.batch, self.query, self.ws["tower"])
        return self.query @ c["table"].t()

    def recommend(self, history: torch.Tensor):
        """The best items of every user and their log probabilities."""
        dmt.dmt_token_logprob_fwd(self.scores(history), top_ids=self.top_ids, top_logprobs=self.top_logprobs,
                                  workspace=self.ws["logprob"])
        return self.top_ids, self.top_logprobs

    def backward(self, history: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """The mean loss; its gradients, not yet clipped, in self.grads."""
        c, g = self.copies, self.grads
        x = self.scores(history)
        dmt.dmt_token_logprob_fwd(x, target, self.logprob, self.entropy, stats=self.stats, workspace=self.ws["logprob"],
                                  first_bad=self.bad)
        dmt.dmt_token_logprob_bwd(x, target, self.stats, None, self.weight, None, x)          # in place
        torch.matmul(x.t().float(), self.query.float(), out=g["table"])
        torch.matmul(x.float(), c["table"].float(), out=self.grad_query)
        dmt.dmt_tower_module_bwd(self.plan, self.tower, self.normed, self.query, self.batch, self.grad_query,
                                 self.grad_normed, self.tower_grads, self.ws["tower_bwd"])
        dmt.dmt_layer_norm_bwd(self.emb, c["gamma"], self.mean, self.rstd, self.grad_normed, self.grad_emb, g["gamma"],
                               g["beta"], self.ws["norm_bwd"])
        dmt.dmt_embed_bwd(history, self.grad_emb, g["table"], self.ws["embed_bwd"], self.scale, accumulate=True)
        return -self.logprob.mean()

    def step(self, history: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        loss = self.backward(history, target)
        dmt.dmt_grad_clip(self.grad_list, self.max_norm, self.norm, self.ws["clip"])
        for n, p in self.params.items():
            p.add_(self.grads[n], alpha=-self.lr)
            self.copies[n].copy_(p)
        return loss


def batch_of(g: torch.Generator, items: int, length: int, batch: int):
    """Histories of 1 ... length items, the empty slots in front; the next item is the last one's neighbour."""
    h = torch.randint(items, (batch, length), generator=g, device="cuda", dtype=torch.int32)
    empty = torch.randint(length, (batch, 1), generator=g, device="cuda")
    h.masked_fill_(torch.arange(length, device="cuda") < empty, -1)
    return h, (h[:, -1] + 1) % items


def main(argv=None) -> float:
    p = argparse.ArgumentParser()
    p.add_argument("--items", type=int, default=2000)
    p.add_argument("--length", type=int, default=8)
    p.add_argument("--dim", type=int, default=64)
    p.add_argument("--batch", type=int, default=512)
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = p.parse_args(argv)
    m = NextItem(a.items, a.length, a.dim, a.batch, a.dtype, lr=2.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for i in range(a.steps):
        loss = m.step(*batch_of(g, a.items, a.length, a.batch))
        if i % 50 == 0 or i == a.steps - 1:
            print("step %4d  loss %.4f  gradient norm %.4f" % (i, float(loss), float(m.norm)), flush=True)
    history, target = batch_of(g, a.items, a.length, a.batch)
    ids, _ = m.recommend(history)
    hit = float((ids == target[:, None]).any(1).float().mean())
    print("next item among the %d best: %.1f %%" % (ids.shape[1], 100 * hit))
    assert int(m.bad) == -1
    return hit


if __name__ == "__main__":
    main()
