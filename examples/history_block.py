"""A next-item model on one GPU whose history block mixes over time and by experts, trained, and served item by item.

    python examples/history_block.py [--steps N] [--dtype f32|bf16]

A user's history of up to L items (empty slots are -1, in front) becomes L embeddings e, and

    r1 = e + dropout(scan(norm(e) Wg + bg, norm(e) Wv))          dmt_layer_norm, dmt_gated_scan, dmt_dropout
    r2 = r1 + dropout(sum of w_j expert_j(norm(r1)))             dmt_token_logprob (the router's k best), dmt_expert_*,
                                                                 a Tower Module with one tower an expert

r2 of the last item is scored against every item's embedding.  The experts' room is a capacity, so that their rows are the
tower-major tensor that dmt_tower_module_fwd and _bwd take; what does not fit passes by on the residual path.  A server keeps a state a
user and sends each new item through dmt_gated_scan_step.  Plain matrix products are left to the library for those.
Data: synthetic histories; the next item follows from the last two.
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


class HistoryModel:
    """Parameters in float32 with working copies in `dtype`, gradients in float32, buffers for one batch size."""

    def __init__(self, items: int, length: int, dim: int, batch: int, experts: int = 4, k: int = 2, room: float = 1.5,
                 p: float = 0.1, dtype: str = "f32", seed: int = 0, lr: float = 0.5, max_norm: float = 1.0):
        self.items, self.length, self.dim, self.batch, self.experts, self.k = items, length, dim, batch, experts, k
        self.p, self.lr, self.max_norm, self.scale = p, lr, max_norm, math.sqrt(dim)
        self.dtype = dt = dmt.binding.TORCH_DTYPE[dmt.binding.DTYPE_CODE[dtype]]
        n = self.n = batch * length
        cap = self.capacity = max(8, math.ceil(n * k / experts * room / 8) * 8)
        rows = experts * cap
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        f32 = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device="cuda")
        i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
        work = lambda *shape: torch.zeros(*shape, dtype=dt, device="cuda")
        draw = lambda *shape: (torch.rand(*shape, generator=g, device="cuda") * 2 - 1) / math.sqrt(dim)
        self.params = dict(table=draw(items, dim), gamma1=f32(dim) + 1, beta1=f32(dim), w_gate=draw(dim, dim), b_gate=f32(dim) + 1,
                           w_value=draw(dim, dim), gamma2=f32(dim) + 1, beta2=f32(dim), w_route=draw(experts, dim))
        for e in range(experts):
            self.params["w_exp%d" % e], self.params["b_exp%d" % e] = draw(dim, dim), f32(dim)
        self.copies = {m: v.to(dt, copy=True) for m, v in self.params.items()}
        self.grads = {m: torch.zeros_like(v) for m, v in self.params.items()}
        c, d = self.copies, self.grads
        # a tower an expert, a batch as large as its room
        self.plan = dmt.dmt_plan_create([1] * experts, [dim] * experts, dtype, experts, list(range(experts)), cap, 1)
        self.towers = dmt.make_tm_params([dict(kind="linear_relu", out_dim=dim, w_proj=c["w_exp%d" % e], b_proj=c["b_exp%d" % e])
                                          for e in range(experts)])
        self.tower_grads = dmt.make_tm_grads([dict(dw_proj=d["w_exp%d" % e], db_proj=d["b_exp%d" % e]) for e in range(experts)])
        self.grad_list = dmt.make_grad_list(list(d.values()))
        self.e, self.y1, self.h, self.r1, self.y2, self.m, self.r2 = (work(n, dim) for _ in range(7))
        self.mean, self.rstd = [f32(n), f32(n)], [f32(n), f32(n)]
        self.top, self.top_lp = i32(n, k), f32(n, k)
        self.slot, self.source, self.sent, self.answer = i32(n, k), i32(rows), work(rows, dim), work(rows, dim)
        self.rng = torch.tensor([seed, 0], device="cuda")                     # the dropouts' seed and step
        self.bad = torch.full((1,), -1, dtype=torch.int64, device="cuda")
        self.logprob, self.stats, self.norm = f32(batch), f32(batch, 2), f32(1)
        self.weight = torch.full((batch,), -1.0 / batch, device="cuda")
        scratch = lambda b: torch.empty(max(256, b), dtype=torch.uint8, device="cuda")
        self.kept = scratch(dmt.dmt_gated_scan_kept_bytes(n, dim))
        self.ws = dict(scan=scratch(dmt.dmt_gated_scan_workspace_bytes(n, dim)),
                       route=scratch(dmt.dmt_token_logprob_workspace_bytes(n, experts, k)),
                       sort=scratch(dmt.dmt_expert_sort_workspace_bytes(n, k, experts)),
                       tower=scratch(dmt.dmt_tm_workspace_bytes(self.plan, self.towers, cap)),
                       tower_bwd=scratch(dmt.dmt_tm_bwd_workspace_bytes(self.plan, self.towers, cap)),
                       norm_bwd=scratch(dmt.dmt_layer_norm_bwd_workspace_bytes(n, dim)),
                       embed_bwd=scratch(dmt.dmt_embed_bwd_workspace_bytes(n, items, dim)),
                       logprob=scratch(dmt.dmt_token_logprob_workspace_bytes(batch, items, 0)),
                       clip=scratch(dmt.dmt_grad_norm_workspace_bytes(self.grad_list)))

    def _mix(self, rows: int, there: torch.Tensor, p: float) -> None:
        """r2[:rows] from r1[:rows]: the experts' half of the block."""
        c, cap = self.copies, self.capacity
        cut = lambda t: t[:rows]
        dmt.dmt_layer_norm_fwd(cut(self.r1), c["gamma2"], c["beta2"], EPS, cut(self.y2), cut(self.mean[1]), cut(self.rstd[1]))
        route = cut(self.y2) @ c["w_route"].t()
        dmt.dmt_token_logprob_fwd(route, top_ids=cut(self.top), top_logprobs=cut(self.top_lp), workspace=self.ws["route"])
        cut(self.top).masked_fill_(~there[:, None], -1)                       # empty slots are nobody's
        self.share = torch.softmax(cut(self.top_lp), 1)                       # over the k that were chosen
        dmt.dmt_expert_sort(cut(self.top), self.experts, cut(self.slot), self.source, None, None, self.ws["sort"], cap)
        dmt.dmt_expert_gather(cut(self.y2), cut(self.slot), self.source, self.sent)
        dmt.dmt_tower_module_fwd(self.plan, self.towers, self.sent, cap, self.answer, self.ws["tower"])
        dmt.dmt_expert_combine(self.answer, cut(self.slot), self.share, cut(self.m))
        dmt.dmt_dropout_fwd(cut(self.m), p, self.rng, cut(self.r2), residual=cut(self.r1), site=1)

    def forward(self, history: torch.Tensor, p: float) -> torch.Tensor:
        """Queries [batch][dim] from int32 [batch][length]."""
        c = self.copies
        self.there = (history >= 0).reshape(-1)
        user = torch.arange(self.batch, device="cuda", dtype=torch.int32)[:, None].expand(-1, self.length).reshape(-1)
        self.sequence_of = torch.where(self.there, user, -1)
        dmt.dmt_embed_fwd(c["table"], history, self.e, self.scale, self.bad)
        dmt.dmt_layer_norm_fwd(self.e, c["gamma1"], c["beta1"], EPS, self.y1, self.mean[0], self.rstd[0])
        self.gate = torch.addmm(c["b_gate"], self.y1, c["w_gate"].t())
        self.value = self.y1 @ c["w_value"].t()
        dmt.dmt_gated_scan_fwd(self.gate, self.value, self.h, self.ws["scan"], sequence_of=self.sequence_of,
                               sequences=self.batch, kept=self.kept)
        dmt.dmt_dropout_fwd(self.h, p, self.rng, self.r1, residual=self.e, site=0)
        self._mix(self.n, self.there, p)
        return self.r2.view(self.batch, self.length, self.dim)[:, -1].contiguous()

    def backward(self, history: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """The mean loss; its gradients, not yet clipped, in self.grads."""
        c, g, n, D = self.copies, self.grads, self.n, self.dim
        f32 = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device="cuda")
        query = self.forward(history, self.p)
        x = query @ c["table"].t()
        dmt.dmt_token_logprob_fwd(x, target, self.logprob, stats=self.stats, workspace=self.ws["logprob"], first_bad=self.bad)
        dmt.dmt_token_logprob_bwd(x, target, self.stats, None, self.weight, None, x)
        torch.matmul(x.t().float(), query.float(), out=g["table"])
        dr2 = f32(self.batch, self.length, D)
        dr2[:, -1] = x.float() @ c["table"].float()
        dr2 = dr2.view(n, D)
        # the experts' half
        dm, dsent, danswer = f32(n, D), f32(len(self.source), D), f32(len(self.source), D)
        dshare, dy2 = f32(n, self.k), f32(n, D)
        dmt.dmt_dropout_bwd(dr2, self.p, self.rng, dm, site=1)
        dmt.dmt_expert_combine_bwd(dm, self.answer, self.slot, self.source, self.share, danswer, dshare)
        dmt.dmt_tower_module_bwd(self.plan, self.towers, self.sent, self.answer, self.capacity, danswer, dsent, self.tower_grads,
                                 self.ws["tower_bwd"])
        dmt.dmt_expert_combine(dsent, self.slot, None, dy2)
        dtop = self.share * (dshare - (self.share * dshare).sum(1, keepdim=True))
        droute = f32(n, self.experts).scatter_(1, self.top.clamp(min=0).long(), torch.where(self.top >= 0, dtop, 0.0))
        torch.matmul(droute.t(), self.y2.float(), out=g["w_route"])
        dy2 += droute @ c["w_route"].float()
        dr1 = f32(n, D)
        dmt.dmt_layer_norm_bwd(self.r1, c["gamma2"], self.mean[1], self.rstd[1], dy2, dr1, g["gamma2"], g["beta2"], self.ws["norm_bwd"])
        dr1 += dr2
        # the half over time
        dh, dgate, dvalue, de = f32(n, D), f32(n, D), f32(n, D), f32(n, D)
        dmt.dmt_dropout_bwd(dr1, self.p, self.rng, dh, site=0)
        dmt.dmt_gated_scan_bwd(self.gate, self.value, dh, dgate, dvalue, self.kept, self.ws["scan"], sequence_of=self.sequence_of,
                               sequences=self.batch)
        y1 = self.y1.float()
        torch.matmul(dgate.t(), y1, out=g["w_gate"])
        torch.matmul(dvalue.t(), y1, out=g["w_value"])
        torch.sum(dgate, 0, out=g["b_gate"])
        dy1 = dgate @ c["w_gate"].float() + dvalue @ c["w_value"].float()
        dmt.dmt_layer_norm_bwd(self.e, c["gamma1"], self.mean[0], self.rstd[0], dy1, de, g["gamma1"], g["beta1"], self.ws["norm_bwd"])
        de += dr1
        dmt.dmt_embed_bwd(history, de, g["table"], self.ws["embed_bwd"], self.scale, accumulate=True)
        return -self.logprob.mean()

    def step(self, history: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        loss = self.backward(history, target)
        dmt.dmt_grad_clip(self.grad_list, self.max_norm, self.norm, self.ws["clip"])
        for m, v in self.params.items():
            v.add_(self.grads[m], alpha=-self.lr)
            self.copies[m].copy_(v)
        self.rng[1] += 1
        return loss

    def observe(self, state: torch.Tensor, users: torch.Tensor, items: torch.Tensor) -> torch.Tensor:
        """Each of `users` has seen one more item: its state (float32 [users][dim]) moves on; the queries of these users."""
        c, m = self.copies, len(users)
        e, y1 = self.e[:m], self.y1[:m]
        dmt.dmt_embed_fwd(c["table"], items, e, self.scale, self.bad)
        dmt.dmt_layer_norm_fwd(e, c["gamma1"], c["beta1"], EPS, y1)
        dmt.dmt_gated_scan_step(torch.addmm(c["b_gate"], y1, c["w_gate"].t()), y1 @ c["w_value"].t(), state, state, self.h[:m],
                                users, first_bad=self.bad)
        dmt.dmt_dropout_fwd(self.h[:m], 0.0, self.rng, self.r1[:m], residual=e)
        self._mix(m, items >= 0, 0.0)
        return self.r2[:m].clone()


def batch_of(g: torch.Generator, items: int, length: int, batch: int):
    """Histories of 2 ... length items, the empty slots in front; the next item is the sum of the last two."""
    h = torch.randint(items, (batch, length), generator=g, device="cuda", dtype=torch.int32)
    empty = torch.randint(length - 1, (batch, 1), generator=g, device="cuda")
    target = ((h[:, -1] + h[:, -2]) % items).to(torch.int32)
    return h.masked_fill_(torch.arange(length, device="cuda") < empty, -1), target


def main(argv=None) -> None:
    p = argparse.ArgumentParser()
    p.add_argument("--items", type=int, default=50)
    p.add_argument("--length", type=int, default=12)
    p.add_argument("--dim", type=int, default=64)
    p.add_argument("--batch", type=int, default=1024)
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = p.parse_args(argv)
    m = HistoryModel(a.items, a.length, a.dim, a.batch, dtype=a.dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for i in range(a.steps):
        loss = m.step(*batch_of(g, a.items, a.length, a.batch))
        if i % 50 == 0 or i == a.steps - 1:
            print("step %4d  loss %.4f  gradient norm %.4f" % (i, float(loss), float(m.norm)), flush=True)
    history, target = batch_of(g, a.items, a.length, a.batch)
    hit = float(((m.forward(history, 0.0) @ m.copies["table"].t()).argmax(1) == target).float().mean())
    print("next item found for %.1f %%" % (100 * hit))
    assert int(m.bad) == -1


if __name__ == "__main__":
    main()
