"""The operators of a sequence branch (a user's history of items, the next item) and what their time is measured on.

A case names one operator and direction ("op"):
  embed_fwd      a table's rows by id, scaled, one row per id
  embed_bwd      the table's gradient, dense float32, from the gradient of those rows
  norm_fwd       layer norm over the last axis, with the mean and 1/std that its backward reads
  norm_bwd       layer norm's gradients: of its input, its weight and its bias
  logprob_fwd    of a row of scores over items: log probability of a given item, entropy, the top k items
  logprob_train  the same without the top k, and the gradient of the scores
  clip           global 2-norm over many gradients, and the gradients scaled down to a largest norm
and its sizes, types and distributions.  `own` false computes the plain form in elementary torch operations in
float32; `own` true calls the library.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ELT = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5                       # layer norm
CLIP_EPS = 1e-6


# ------------------------------------------------------------------------------- the cases


def _embed(op, n, rows, cols, dtype, grad="f32", alpha=1.05, absent=0.0, name=None):
    c = dict(op=op, n=n, rows=rows, cols=cols, dtype=dtype, alpha=alpha, absent=absent)
    if op == "embed_bwd":
        c["dtype"] = grad                 # of the rows' gradient; the table's is float32
    return dict(c, name=name) if name else c


def _norm(op, rows, cols, dtype, grad="f32", pad=0, name=None):
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, pad=pad)
    if op == "norm_bwd":
        c["grad"] = grad
    return dict(c, name=name) if name else c


def _logprob(op, rows, vocab, dtype, k=0, masked=0.0, name=None):
    c = dict(op=op, rows=rows, vocab=vocab, dtype=dtype, masked=masked)
    if op == "logprob_fwd":
        c["k"] = k
    return dict(c, name=name) if name else c


def _clip(tensors, largest, dtype, share16, aligned, largest_norm, name=None):
    c = dict(op="clip", tensors=tensors, largest=largest, dtype=dtype, share16=share16, aligned=aligned,
             largest_norm=largest_norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's last item, served alone: nothing but latency
        _embed("embed_fwd", 1, 1_000_000, 128, "f16", name="embed_fwd_one"),
        # the histories of a batch of 8192 users, 32 items each, some slots empty, as they come (Zipf)
        _embed("embed_fwd", 262_144, 1_000_000, 128, "bf16", absent=0.1, name="embed_fwd_batch"),
        # a small catalogue with an odd width: a test or a debugging run
        _embed("embed_bwd", 1_003, 10_007, 100, "f32", grad="f32", name="embed_bwd_small"),
        # a training step's gradient of the item table: 8192 histories of 20, 1 M items
        _embed("embed_bwd", 163_840, 1_000_000, 128, "f32", grad="bf16", absent=0.1, name="embed_bwd_batch"),
        # one user's vector before the tower
        _norm("norm_fwd", 1, 1024, "bf16", name="norm_fwd_one"),
        # the input of a dot-product tower (28 terms and 8 x 128 features) of a large batch: rows of 2104 bytes
        _norm("norm_fwd", 65_536, 1052, "bf16", name="norm_fwd_odd"),
        # the widest towers' input, with the float32 gradients that a Tower Module's backward leaves
        _norm("norm_bwd", 8_192, 2048, "bf16", grad="f32", name="norm_bwd_wide"),
        # one user scored against a catalogue of 100 K, the ten best items asked for
        _logprob("logprob_fwd", 1, 100_000, "f32", k=10, name="logprob_one"),
        # a batch of users ranked over an odd catalogue, a tenth of it unavailable
        _logprob("logprob_fwd", 512, 100_003, "f16", k=20, masked=0.1, name="logprob_rank"),
        # a training step's loss over a batch of 8192
        _logprob("logprob_train", 8_192, 65_536, "bf16", name="logprob_train"),
        # the parameter gradients of eight dot-product towers
        _clip(16, 256 * 1052, "f32", 0.0, True, 1.0, name="clip_towers"),
        # a whole model's gradients, a table's among them, some held in 16 bits, packed as they come
        _clip(180, 1_000_000 * 128, "bf16", 0.3, False, 1.0, name="clip_model"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "logprob_fwd", "logprob_train", "clip"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op in ("embed_fwd", "embed_bwd"):
        rows = _log(rng, 10_000, 1_000_000)
        cols = min(_log(rng, 16, 1024), 128_000_000 // rows)
        if rng.random() < 0.5:
            cols = max(16, cols // 16 * 16)
        n = min(_log(rng, 1, 262_144), 2 ** 26 // cols)
        return _embed(op, n, rows, cols, dtype, grad=dtype, alpha=rng.choice([0.0, 1.05]), absent=rng.choice([0.0, 0.1]))
    if op in ("norm_fwd", "norm_bwd"):
        cols = _log(rng, 16, 8192)
        if rng.random() < 0.5:
            cols = max(16, cols // 16 * 16)
        rows = min(_log(rng, 1, 262_144), 2 ** 26 // cols)
        return _norm(op, rows, cols, dtype, grad=rng.choice(["f32", dtype]), pad=rng.choice([0, 0, 8, 5]))
    if op in ("logprob_fwd", "logprob_train"):
        vocab = _log(rng, 1_000, 262_144)
        rows = min(_log(rng, 1, 8192), 2 ** 26 // vocab)
        return _logprob(op, rows, vocab, dtype, k=rng.choice([0, 1, 5, 10, 20, 50]), masked=rng.choice([0.0, 0.1, 0.5]))
    return _clip(_log(rng, 1, 300), _log(rng, 1_000, 64_000_000), rng.choice(["f16", "bf16"]),
                 rng.choice([0.0, 0.3, 1.0]), rng.random() < 0.5, rng.choice([0.5, 1.0, 1e9]))


# ------------------------------------------------------------------------------- what a program has in hand


def _ids(g, n, rows, alpha, absent):
    """int32 ids: uniform (alpha 0) or Zipf over a seeded permutation of the rows; -1 where a slot is empty."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if alpha:
        p = torch.arange(1, rows + 1, device="cuda", dtype=torch.float64) ** -alpha
        cum = torch.cumsum(p, 0)
        rank = torch.searchsorted(cum, u * cum[-1]).clamp(max=rows - 1)
        ids = torch.randperm(rows, generator=g, device="cuda")[rank]
    else:
        ids = (u * rows).long().clamp(max=rows - 1)
    if absent:
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < absent, -1, ids)
    return ids.to(torch.int32)


def _randn(g, *shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(dtype)


def _padded(g, rows, cols, pad, dtype, scale, shift):
    """[rows][cols] inside rows of cols + pad elements."""
    return _randn(g, rows, cols + pad, dtype=dtype, scale=scale, shift=shift)[:, :cols]


def _sizes(case):
    """Element counts of a model's gradients: from vectors of 16 to the largest matrix, spread over the logarithm."""
    t, top = case["tensors"], case["largest"]
    if t == 1:
        return [top]
    lo = min(16, top)
    at = [math.exp(math.log(lo) + (math.log(top) - math.log(lo)) * (i / (t - 1)) ** 0.5) for i in range(t)]
    if top > 10_000_000:                  # one table; the other layers stay below a million elements
        at = [min(a, 1e6) for a in at[:-1]] + [top]
    sizes = [int(a) for a in at]
    sizes[-1] = top
    if case["aligned"]:
        sizes = [max(8, s // 8 * 8) for s in sizes]
    return sizes


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=dict(case))
    op = case["op"]
    if op == "embed_fwd":
        dt = TORCH_DTYPE[case["dtype"]]
        s["table"] = _randn(g, case["rows"], case["cols"], dtype=dt, scale=0.01)
        s["ids"] = _ids(g, case["n"], case["rows"], case["alpha"], case["absent"])
        s["out"] = torch.empty(case["n"], case["cols"], dtype=dt, device="cuda")
        s["scale"] = math.sqrt(case["cols"])
    elif op == "embed_bwd":
        dt = TORCH_DTYPE[case["dtype"]]
        s["ids"] = _ids(g, case["n"], case["rows"], case["alpha"], case["absent"])
        s["grad"] = _randn(g, case["n"], case["cols"], dtype=dt)
        s["out"] = torch.empty(case["rows"], case["cols"], dtype=torch.float32, device="cuda")
        s["scale"] = math.sqrt(case["cols"])
    elif op in ("norm_fwd", "norm_bwd"):
        dt, R, C = TORCH_DTYPE[case["dtype"]], case["rows"], case["cols"]
        s["x"] = _padded(g, R, C, case["pad"], dt, 1.5, 0.3)
        s["gamma"] = _randn(g, C, dtype=dt, scale=0.1, shift=1.0)
        s["beta"] = _randn(g, C, dtype=dt, scale=0.1)
        s["mean"] = torch.empty(R, dtype=torch.float32, device="cuda")
        s["rstd"] = torch.empty(R, dtype=torch.float32, device="cuda")
        if op == "norm_fwd":
            s["y"] = torch.empty(R, C, dtype=dt, device="cuda")
        else:
            gt = TORCH_DTYPE[case["grad"]]
            x = s["x"].float()            # the forward's statistics
            m = x.mean(1, keepdim=True)
            s["mean"].copy_(m[:, 0])
            s["rstd"].copy_((((x - m) ** 2).mean(1) + EPS) ** -0.5)
            s["dy"] = _randn(g, R, C, dtype=gt)
            s["dx"] = torch.empty(R, C, dtype=gt, device="cuda")
            s["dgamma"] = torch.empty(C, dtype=torch.float32, device="cuda")
            s["dbeta"] = torch.empty(C, dtype=torch.float32, device="cuda")
    elif op in ("logprob_fwd", "logprob_train"):
        dt, R, V = TORCH_DTYPE[case["dtype"]], case["rows"], case["vocab"]
        x = torch.randn(R, V, generator=g, device="cuda", dtype=torch.float32).mul_(2.5).to(dt)
        if case["masked"]:                # items that are not to be had: no part of the distribution
            x.masked_fill_(torch.rand(R, V, generator=g, device="cuda") < case["masked"], float("-inf"))
        t = torch.randint(V, (R,), generator=g, device="cuda")
        x.scatter_(1, t[:, None], _randn(g, R, 1, dtype=dt, scale=2.5, shift=4.0))
        s["x"], s["targets"] = x, t.to(torch.int32)
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device="cuda")
        s["logprob"], s["entropy"] = f32(R), f32(R)
        if op == "logprob_fwd":
            k = case["k"]
            s["top_ids"] = torch.empty(R, k, dtype=torch.int32, device="cuda") if k else None
            s["top_logprobs"] = f32(R, k) if k else None
        else:
            s["stats"] = f32(R, 2)
            s["g_lp"] = -(torch.rand(R, generator=g, device="cuda") + 0.5)      # a weight per sample, loss scale in it
            s["g_h"] = -0.05 * torch.rand(R, generator=g, device="cuda")        # a small reward for spread
            s["dx"] = torch.empty_like(x)
    else:
        sizes = _sizes(case)
        pick = random.Random(len(sizes))
        wide = [pick.random() >= case["share16"] for _ in sizes]
        if case["largest"] > 10_000_000 and case["share16"] < 1.0:
            wide[-1] = True
        flats, outs, s["grads"], s["clipped"] = [], [], [], []
        for dt, mine in ((torch.float32, wide), (TORCH_DTYPE[case["dtype"]], [not w for w in wide])):
            part = [n for n, w in zip(sizes, mine) if w]
            if not part:
                continue
            flat = _randn(g, sum(part), dtype=dt, scale=0.02)
            out = torch.empty_like(flat)
            flats.append(flat)
            outs.append(out)
            s["grads"] += list(torch.split(flat, part))
            s["clipped"] += list(torch.split(out, part))
        s["flats"], s["outs"] = flats, outs
        s["norm"] = torch.empty((), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------------------- one pass


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "embed_fwd":
        rows = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
        return torch.where((s["ids"] >= 0)[:, None], rows, 0.0).to(s["table"].dtype)
    if op == "embed_bwd":
        weight = torch.where(s["ids"] >= 0, s["scale"], 0.0)
        out = torch.zeros(c["rows"], c["cols"], dtype=torch.float32, device="cuda")
        return out.index_add_(0, s["ids"].clamp(min=0), s["grad"].float() * weight[:, None])
    if op == "norm_fwd":
        x = s["x"].float()
        m = x.mean(1, keepdim=True)
        d = x - m
        r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        y = d * r * s["gamma"].float() + s["beta"].float()
        return [y.to(s["x"].dtype), m[:, 0], r[:, 0]]
    if op == "norm_bwd":
        r = s["rstd"][:, None]
        h = (s["x"].float() - s["mean"][:, None]) * r
        dy = s["dy"].float()
        gr = dy * s["gamma"].float()
        dx = r * (gr - gr.mean(1, keepdim=True) - h * (gr * h).mean(1, keepdim=True))
        return [dx.to(s["dy"].dtype), (dy * h).sum(0), dy.sum(0)]
    if op in ("logprob_fwd", "logprob_train"):
        x = s["x"].float()
        at = s["targets"].long()[:, None]
        z = x - x.max(1, keepdim=True).values
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        lp = z - torch.log(total)
        p = e / total
        plp = torch.where(e > 0, p * lp, 0.0)
        entropy = -plp.sum(1)
        logprob = lp.gather(1, at)[:, 0]
        if op == "logprob_fwd":
            if not c["k"]:
                return [logprob, entropy]
            top = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :c["k"]]
            return [logprob, entropy, top.to(torch.int32), lp.gather(1, top)]
        g_lp, g_h = s["g_lp"][:, None], s["g_h"][:, None]
        dx = -g_lp * p - g_h * (plp + p * entropy[:, None])
        dx.scatter_add_(1, at, g_lp)
        return [logprob, entropy, dx.to(s["x"].dtype)]
    total = torch.stack([(g.float() * g.float()).sum() for g in s["grads"]]).sum()
    norm = torch.sqrt(total)
    coef = torch.clamp(c["largest_norm"] / (norm + CLIP_EPS), max=1.0)
    [o.copy_(g.float() * coef) for g, o in zip(s["grads"], s["clipped"])]
    return [norm, *s["outs"]]


def _workspace(s, dmt, nbytes):
    """The scratch memory that a program keeps beside its tensors."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(256, nbytes()), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _library(s):
    import paper_2403_00877_amd as dmt
    c = s["case"]
    op = c["op"]
    if op == "embed_fwd":
        dmt.dmt_embed_fwd(s["table"], s["ids"], s["out"], scale=s["scale"])
        return s["out"]
    if op == "embed_bwd":
        ws = _workspace(s, dmt, lambda: dmt.dmt_embed_bwd_workspace_bytes(c["n"], c["rows"], c["cols"]))
        dmt.dmt_embed_bwd(s["ids"], s["grad"], s["out"], ws, scale=s["scale"])
        return s["out"]
    if op == "norm_fwd":
        dmt.dmt_layer_norm_fwd(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        return [s["y"], s["mean"], s["rstd"]]
    if op == "norm_bwd":
        ws = _workspace(s, dmt, lambda: dmt.dmt_layer_norm_bwd_workspace_bytes(c["rows"], c["cols"]))
        dmt.dmt_layer_norm_bwd(s["x"], s["gamma"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dgamma"], s["dbeta"], ws)
        return [s["dx"], s["dgamma"], s["dbeta"]]
    if op in ("logprob_fwd", "logprob_train"):
        ws = _workspace(s, dmt, lambda: dmt.dmt_token_logprob_workspace_bytes(c["rows"], c["vocab"], c.get("k", 0)))
        if op == "logprob_fwd":
            dmt.dmt_token_logprob_fwd(s["x"], s["targets"], s["logprob"], s["entropy"], s["top_ids"], s["top_logprobs"],
                                      workspace=ws)
            return [s["logprob"], s["entropy"]] + ([s["top_ids"], s["top_logprobs"]] if c["k"] else [])
        dmt.dmt_token_logprob_fwd(s["x"], s["targets"], s["logprob"], s["entropy"], stats=s["stats"], workspace=ws)
        dmt.dmt_token_logprob_bwd(s["x"], s["targets"], s["stats"], s["entropy"], s["g_lp"], s["g_h"], s["dx"])
        return [s["logprob"], s["entropy"], s["dx"]]
    if "list" not in s:                   # the gradients' addresses and sizes, as a program hands them over
        s["list"] = dmt.make_grad_list(s["grads"], s["clipped"])
    ws = _workspace(s, dmt, lambda: dmt.dmt_grad_norm_workspace_bytes(s["list"]))
    dmt.dmt_grad_clip(s["list"], c["largest_norm"], s["norm"], ws)
    return [s["norm"], *s["outs"]]


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed_fwd":
        out = s["table"].double()[s["ids"].clamp(min=0).long()] * s["scale"]
        out[s["ids"] < 0] = 0
        return out
    if op == "embed_bwd":
        keep = s["ids"] >= 0
        out = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device="cuda")
        out.index_put_((s["ids"][keep].long(),), s["grad"].double()[keep] * s["scale"], accumulate=True)
        return out
    if op == "norm_fwd":
        x = s["x"].double()
        m, v = x.mean(1), x.var(1, unbiased=False)
        y = (x - m[:, None]) / torch.sqrt(v + EPS)[:, None] * s["gamma"].double() + s["beta"].double()
        return [y, m, 1 / torch.sqrt(v + EPS)]
    if op == "norm_bwd":
        m, r = s["mean"].double()[:, None], s["rstd"].double()[:, None]
        h, dy = (s["x"].double() - m) * r, s["dy"].double()
        gr = dy * s["gamma"].double()
        n = case["cols"]
        dx = r / n * (n * gr - gr.sum(1, keepdim=True) - h * (gr * h).sum(1, keepdim=True))
        return [dx, (dy * h).sum(0), dy.sum(0)]
    if op in ("logprob_fwd", "logprob_train"):
        out = []
        step = max(1, 2 ** 26 // case["vocab"])
        for a in range(0, case["rows"], step):
            b = min(case["rows"], a + step)
            x = s["x"][a:b].double()
            lp = x - torch.logsumexp(x, 1, keepdim=True)
            at = s["targets"][a:b].long()[:, None]
            p = torch.exp(lp)
            plp = torch.nan_to_num(p * lp, nan=0.0)
            h = -plp.sum(1, keepdim=True)
            part = [lp.gather(1, at)[:, 0], h[:, 0]]
            if op == "logprob_fwd":
                if case["k"]:
                    part.append(torch.topk(lp, case["k"], dim=1).values)
            else:
                hot = torch.zeros_like(p).scatter_(1, at, 1.0)
                part.append(s["g_lp"].double()[a:b, None] * (hot - p) - s["g_h"].double()[a:b, None] * (plp + p * h))
            out.append(part)
        out = [torch.cat(v) for v in zip(*out)]
        if op == "logprob_fwd" and case["k"]:
            out.insert(2, None)
        return out
    norm = math.sqrt(sum(float((f.double() ** 2).sum()) for f in s["flats"]))
    coef = min(1.0, case["largest_norm"] / (norm + CLIP_EPS))
    return [torch.tensor(norm, dtype=torch.float64), *[f.double() * coef for f in s["flats"]]]


# ------------------------------------------------------------------------------- what a pass cannot do without


def _distinct(rows, alpha, n):
    """Expected number of different rows among n ids."""
    if not alpha:
        return rows * -math.expm1(n * math.log1p(-1.0 / rows))
    p = np.arange(1, rows + 1, dtype=np.float64) ** -alpha
    p /= p.sum()
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    op = case["op"]
    if op in ("embed_fwd", "embed_bwd"):
        n, C, e = case["n"], case["cols"], ELT[case["dtype"]]
        there = n * (1 - case["absent"])
        if op == "embed_fwd":
            return {"bytes": 4 * n + _distinct(case["rows"], case["alpha"], there) * C * e + n * C * e, "flops": there * C}
        return {"bytes": 4 * n + there * C * e + case["rows"] * C * 4, "flops": 2 * there * C}
    if op in ("norm_fwd", "norm_bwd"):
        R, C, e = case["rows"], case["cols"], ELT[case["dtype"]]
        if op == "norm_fwd":
            return {"bytes": 2 * R * C * e + 8 * R + 2 * C * e, "flops": 8 * R * C}
        eg = ELT[case["grad"]]
        return {"bytes": R * C * (e + 2 * eg) + 8 * R + C * (e + 8), "flops": 14 * R * C}
    if op in ("logprob_fwd", "logprob_train"):
        R, V, e = case["rows"], case["vocab"], ELT[case["dtype"]]
        if op == "logprob_fwd":
            return {"bytes": R * V * e + R * (12 + 8 * case["k"]), "flops": 5 * R * V}
        return {"bytes": 2 * R * V * e + R * 28, "flops": 11 * R * V}
    sizes = _sizes(case)
    e = case["share16"] * 2 + (1 - case["share16"]) * 4
    if case["largest"] > 10_000_000 and case["share16"] < 1.0:
        total = sum(sizes[:-1]) * e + sizes[-1] * 4
    else:
        total = sum(sizes) * e
    return {"bytes": 2 * total + 4, "flops": 3 * sum(sizes)}
