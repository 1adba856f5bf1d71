"""The operators of a language-model client's local step, as a user calls them through paper_2402_03770_amd.cvlc.

A client's update is what its local step leaves in one flat fp32 vector: the gradient of the embedding table (by
far its largest part, mostly rows that nothing touched), the gradients of the norms' weights, and, at the start of
the backward pass, the gradient of the loss.  The loss is distillation from a teacher's top logits: what clients and
server send each other where whole logits would be too much.

`op` is the call:
  embed        out[i] = scale * table[id_i], zeros for a negative id (padding)
  embed_grad   dtable[v] = scale * sum of dout[i] over the i with id_i = v, every row of the table written
  norm         layer norm of rows, with the rows' (mean, 1/deviation) kept for the backward pass
  norm_grad    dx, and dgamma, dbeta summed over all rows
  distill      mode "loss": the rows' losses and (max, sum) kept for the backward pass; "grad": losses and the logits'
               gradient in one call; "back": the gradient from what "loss" kept

Sizes: models of 10 to 262 144 classes or tokens (100 classes are the paper's image task), widths of 8 to 16 384,
one token to 131 072 of them.  `own` is set by whoever measures: False computes the plain form.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
MOST_BYTES = 2_000_000_000     # of a drawn case; the largest listed one moves somewhat more
MOST_VALUES = 1 << 29          # of a drawn case's table or logits


def listed():
    return [
        # one short text of a few tokens: nothing but latency
        dict(name="embed_16x512", op="embed", n=16, dim=512, vocab=8192, type="f32", pad=0.0),
        # a full local batch of a large model, with padding at the texts' ends
        dict(name="embed_65536x2048", op="embed", n=65536, dim=2048, vocab=50000, type="bf16", pad=0.1),
        # a small model on a small client: 20 texts of 32 tokens
        dict(name="embed_grad_640x96_1000", op="embed_grad", n=640, dim=96, vocab=1000, type="f32", pad=0.1),
        # a medium model
        dict(name="embed_grad_16384x768_32000", op="embed_grad", n=16384, dim=768, vocab=32000, type="bf16", pad=0.0),
        # the largest table: most of its rows are touched by no token
        dict(name="embed_grad_131072x2048_131072", op="embed_grad", n=131072, dim=2048, vocab=131072, type="bf16", pad=0.05),
        # a few rows, as at the end of a classifier
        dict(name="norm_20x512", op="norm", n=20, dim=512, type="f32", pad=0),
        # a full local batch of a large model
        dict(name="norm_65536x4096", op="norm", n=65536, dim=4096, type="bf16", pad=0),
        # a width that is a multiple of nothing
        dict(name="norm_grad_2007x1003", op="norm_grad", n=2007, dim=1003, type="f32", pad=0),
        # a full local batch of a large model
        dict(name="norm_grad_32768x4096", op="norm_grad", n=32768, dim=4096, type="bf16", pad=0),
        # 100 classes, one local batch of images
        dict(name="distill_64x100", op="distill", mode="grad", n=64, vocab=100, k=10, type="f32", T=4.0, masked=0.0, pad=0),
        # a language model's vocabulary, a local batch of texts whose prompts carry no loss
        dict(name="distill_4096x131072", op="distill", mode="grad", n=4096, vocab=131072, k=64, type="bf16", T=2.0, masked=0.1, pad=0),
        # one short text: few rows of a large, odd vocabulary; the loss alone
        dict(name="distill_loss_24x200003", op="distill", mode="loss", n=24, vocab=200003, k=20, type="f16", T=1.0, masked=0.0, pad=5),
    ]


def draw(rng):
    def size(low, high):
        v = int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))
        v = max(low, min(high, v))
        if rng.random() < 0.4 and v >= 64:          # some sizes are round
            v -= v % (64 if v < 4096 else 1024)
        return v

    op = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "distill", "distill", "distill"])
    while True:
        case = dict(op=op, type=rng.choice(["f32", "bf16", "bf16", "f16"]))
        if op in ("embed", "embed_grad"):
            case |= dict(n=size(1, 131072), dim=size(16, 8192), vocab=size(64, 262144), pad=rng.choice([0.0, 0.05, 0.3]))
            values = case["vocab"] * case["dim"]
        elif op in ("norm", "norm_grad"):
            case |= dict(n=size(1, 131072), dim=size(8, 16384), pad=rng.choice([0, 0, 8, 3]))
            values = 0
        else:
            vocab = size(10, 262144)
            case |= dict(mode=rng.choice(["loss", "grad", "grad", "back"]), n=size(1, 65536), vocab=vocab,
                         k=min(vocab, size(1, 256)), T=rng.choice([1.0, 2.0, 4.0, 0.5]), masked=rng.choice([0.0, 0.0, 0.2]),
                         pad=rng.choice([0, 0, 8, 5]))
            values = case["n"] * vocab
        if values <= MOST_VALUES and work(case)["bytes"] <= MOST_BYTES:
            return case


def _distinct(case):
    """How many different tokens a case's texts are expected to hold."""
    r = torch.arange(case["vocab"], dtype=torch.float64)
    share = torch.log((r + 2.0) / (r + 1.0)) / math.log(case["vocab"] + 1.0)
    return float(-torch.expm1(case["n"] * (1.0 - case["pad"]) * torch.log1p(-share)).sum())


def work(case):
    op, n = case["op"], case["n"]
    e = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
    if op == "embed":
        values = n * case["dim"]
        return {"bytes": _distinct(case) * case["dim"] * e + values * e + 8 * n, "flops": values}
    if op == "embed_grad":
        values = n * case["dim"] * (1.0 - case["pad"])
        return {"bytes": values * e + 8 * n + 4 * case["vocab"] * case["dim"], "flops": values}
    if op == "norm":
        values = n * case["dim"]
        return {"bytes": 2 * values * e + 8 * case["dim"] + 8 * n, "flops": 8 * values}
    if op == "norm_grad":
        values = n * case["dim"]
        return {"bytes": 3 * values * e + 12 * case["dim"] + 8 * n, "flops": 14 * values}
    values, lists = n * case["vocab"], 8 * n * case["k"]
    live = 1.0 - case["masked"]
    passes = live if case["mode"] == "loss" else live + 1.0      # masked rows are not read, their gradient is written
    return {"bytes": values * e * passes + lists + 16 * n, "flops": 6 * values * live}


# ----------------------------------------------------------------------------- inputs
def _rows(n, width, extra, dtype):
    """An uninitialised matrix whose rows lie `extra` values further apart than they are long."""
    return torch.empty(n, width + extra, dtype=dtype, device=DEV)[:, :width]


def _tokens(case, gen):
    """Tokens of texts: low numbers are frequent (a rank's share falls as one over the rank); -1 is padding."""
    n, vocab = case["n"], case["vocab"]
    u = torch.rand(n, dtype=torch.float64, device=DEV, generator=gen)
    ids = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
    if case["pad"]:
        ids[torch.rand(n, device=DEV, generator=gen) < case["pad"]] = -1
    return ids


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, n, dtype = case["op"], case["n"], TYPES[case["type"]]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, dtype=dtype, device=DEV, generator=gen)

    state = dict(case=case)
    if op == "embed":
        state |= dict(ids=_tokens(case, gen), table=normal(case["vocab"], case["dim"], dtype=dtype).mul_(0.02),
                      scale=math.sqrt(case["dim"]))
    elif op == "embed_grad":
        state |= dict(ids=_tokens(case, gen), dout=normal(n, case["dim"], dtype=dtype).mul_(0.01), scale=math.sqrt(case["dim"]))
    elif op in ("norm", "norm_grad"):
        dim = case["dim"]
        x = _rows(n, dim, case["pad"], dtype)
        # channels with scales of their own, rows with an offset
        x.copy_(normal(n, dim, dtype=dtype) * torch.exp(0.5 * normal(dim)).to(dtype) + 0.5 * normal(n, 1).to(dtype))
        state |= dict(x=x, gamma=1.0 + 0.2 * normal(dim), beta=0.1 * normal(dim))
        if op == "norm_grad":
            dy = _rows(n, dim, case["pad"], dtype)
            dy.copy_(normal(n, dim, dtype=dtype).mul_(0.01))
            xf = x.float()
            mean = xf.mean(1)
            rstd = torch.rsqrt((xf - mean[:, None]).square().mean(1) + EPS)
            state |= dict(dy=dy, stats=torch.stack([mean, rstd], 1).contiguous())
    else:
        vocab, k = case["vocab"], case["k"]
        logits = _rows(n, vocab, case["pad"], dtype)
        logits.copy_(normal(n, vocab, dtype=dtype).mul_(2.0))
        # the teacher's list, best first: spread over the vocabulary; the student has learnt part of it
        first = torch.randint(vocab, (n, 1), device=DEV, generator=gen)
        ids = (first + torch.arange(k, device=DEV) * (vocab // k)) % vocab
        values = 12.0 - torch.cumsum(torch.rand(n, k, device=DEV, generator=gen), 1)
        logits.scatter_add_(1, ids, (values * torch.rand(n, 1, device=DEV, generator=gen)).to(dtype))
        weights = None
        if case["masked"]:
            weights = torch.full((n,), 1.0 / n, device=DEV)
            weights[torch.rand(n, device=DEV, generator=gen) < case["masked"]] = 0.0
        state |= dict(logits=logits, ids=ids.int(), values=values, weights=weights)
        if case["mode"] == "back":
            zf = logits.float()
            top = zf.amax(1)
            state["stats"] = torch.stack([top, torch.exp((zf - top[:, None]) / case["T"]).sum(1)], 1).contiguous()
    return state


# ----------------------------------------------------------------------------- one pass
def run(state):
    return _calls(state) if own else PLAIN[state["case"]["op"]](state)


def _calls(state):
    import paper_2402_03770_amd.cvlc as cv

    case, op = state["case"], state["case"]["op"]
    kept = state.get("kept")
    if kept is None:                                # output buffers and workspace of a program's own, made once
        kept = state["kept"] = _buffers(case, cv)
    if op == "embed":
        cv.embed(state["ids"], state["table"], kept["out"], scale=state["scale"])
        return kept["out"]
    if op == "embed_grad":
        cv.embed_grad(state["ids"], state["dout"], kept["dtable"], kept["workspace"], scale=state["scale"])
        return kept["dtable"]
    if op == "norm":
        cv.layer_norm(state["x"], state["gamma"], state["beta"], kept["y"], kept["stats"], eps=EPS)
        return {"y": kept["y"], "stats": kept["stats"]}
    if op == "norm_grad":
        cv.layer_norm_grad(state["dy"], state["x"], state["stats"], state["gamma"], kept["dx"], kept["dgamma"],
                           kept["dbeta"], kept["workspace"])
        return {"dx": kept["dx"], "dgamma": kept["dgamma"], "dbeta": kept["dbeta"]}
    if case["mode"] == "back":
        cv.distill_grad(state["logits"], state["ids"], state["values"], state["stats"], kept["dlogits"],
                        temperature=case["T"], weights=state["weights"])
        return kept["dlogits"]
    if case["mode"] == "loss":
        cv.distill(state["logits"], state["ids"], state["values"], kept["loss"], kept["workspace"], temperature=case["T"],
                   weights=state["weights"], stats_out=kept["stats"])
        return {"loss": kept["loss"], "stats": kept["stats"]}
    cv.distill(state["logits"], state["ids"], state["values"], kept["loss"], kept["workspace"], temperature=case["T"],
               weights=state["weights"], dlogits=kept["dlogits"])
    return {"loss": kept["loss"], "dlogits": kept["dlogits"]}


def _buffers(case, cv):
    op, n, dtype = case["op"], case["n"], TYPES[case["type"]]

    def new(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if op == "embed":
        return dict(out=new(n, case["dim"], dtype=dtype))
    if op == "embed_grad":
        need = cv.embed_grad_workspace_bytes(n, case["vocab"], case["dim"])
        return dict(dtable=new(case["vocab"], case["dim"]), workspace=cv.new_workspace(need, DEV))
    if op == "norm":
        return dict(y=new(n, case["dim"], dtype=dtype), stats=new(n, 2))
    if op == "norm_grad":
        return dict(dx=new(n, case["dim"], dtype=dtype), dgamma=new(case["dim"]), dbeta=new(case["dim"]),
                    workspace=cv.new_workspace(cv.layer_norm_grad_workspace_bytes(n, case["dim"]), DEV))
    if case["mode"] == "back":
        return dict(dlogits=new(n, case["vocab"], dtype=dtype))
    kept = dict(loss=new(n), workspace=cv.new_workspace(cv.distill_workspace_bytes(n, case["vocab"]), DEV))
    if case["mode"] == "loss":
        return kept | dict(stats=new(n, 2))
    return kept | dict(dlogits=new(n, case["vocab"], dtype=dtype))


def _plain_embed(s):
    rows = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
    return rows.masked_fill_((s["ids"] < 0)[:, None], 0.0).to(s["table"].dtype)


def _plain_embed_grad(s):
    case = s["case"]
    terms = s["dout"].float().masked_fill_((s["ids"] < 0)[:, None], 0.0) if case["pad"] else s["dout"].float()
    return torch.zeros(case["vocab"], case["dim"], device=DEV).index_add_(0, s["ids"].clamp(min=0), terms).mul_(s["scale"])


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    y = (x * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype)
    return {"y": y, "stats": torch.cat([mean, rstd], 1)}


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["stats"][:, 1:]
    h = (s["x"].float() - s["stats"][:, :1]) * rstd
    g = dy * s["gamma"]
    dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * rstd
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}


def _plain_distill(s):
    case, T = s["case"], s["case"]["T"]
    z, ids = s["logits"].float(), s["ids"].long()
    if case["mode"] == "back":
        top, total = s["stats"][:, :1], s["stats"][:, 1:]
        e = torch.exp((z - top) / T)
    else:
        top = z.amax(1, keepdim=True)
        e = torch.exp((z - top) / T)
        total = e.sum(1, keepdim=True)
    t = (s["values"] - s["values"].amax(1, keepdim=True)) / T
    pe = torch.exp(t)
    ptotal = pe.sum(1, keepdim=True)
    p, logp = pe / ptotal, t - torch.log(ptotal)
    w = s["weights"][:, None] if s["weights"] is not None else 1.0
    out = {}
    if case["mode"] != "back":
        logq = (z.gather(1, ids) - top) / T - torch.log(total)
        out["loss"] = (w * (p * (logp - logq))).sum(1) * (T * T)
    if case["mode"] == "loss":
        stats = torch.cat([top, total], 1)
        if s["weights"] is not None:                # a row without weight is not looked at: it keeps zeros
            stats = stats.masked_fill(w == 0, 0.0)
        out["stats"] = stats
        return out
    g = e.mul_(1.0 / total).scatter_add_(1, ids, -p).mul_(w * T if s["weights"] is not None else T)
    out["dlogits"] = g.to(s["logits"].dtype)
    return out if case["mode"] == "grad" else out["dlogits"]


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
         "distill": _plain_distill}


# ----------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, n, f64 = case["op"], case["n"], torch.float64
    step = max(1, (1 << 26) // case.get("dim", case.get("vocab")))     # rows at a time
    if op == "embed":
        out = torch.zeros(n, case["dim"], dtype=f64, device=DEV)
        at = torch.nonzero(s["ids"] >= 0)[:, 0]
        out[at] = s["table"][s["ids"][at]].to(f64) * s["scale"]
        return out
    if op == "embed_grad":
        order = torch.argsort(s["ids"], stable=True)
        order = order[s["ids"][order] >= 0]
        out = torch.zeros(case["vocab"], case["dim"], dtype=f64, device=DEV)
        for b in range(0, order.numel(), step):
            part = order[b:b + step]
            rows, where = torch.unique_consecutive(s["ids"][part], return_inverse=True)
            sums = torch.zeros(rows.numel(), case["dim"], dtype=f64, device=DEV)
            out[rows] += sums.index_add_(0, where, s["dout"][part].to(f64))
        return out * s["scale"]
    if op == "norm":
        y, stats = [], []
        for b in range(0, n, step):
            x = s["x"][b:b + step].to(f64)
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            inv = 1.0 / torch.sqrt(var + EPS)
            y.append((x - mean) * inv * s["gamma"].to(f64) + s["beta"].to(f64))
            stats.append(torch.cat([mean, inv], 1))
        return {"y": torch.cat(y), "stats": torch.cat(stats)}
    if op == "norm_grad":
        dx, dim = [], case["dim"]
        dgamma, dbeta = torch.zeros(dim, dtype=f64, device=DEV), torch.zeros(dim, dtype=f64, device=DEV)
        for b in range(0, n, step):
            stats = s["stats"][b:b + step].to(f64)
            dy, inv = s["dy"][b:b + step].to(f64), stats[:, 1:]
            h = (s["x"][b:b + step].to(f64) - stats[:, :1]) * inv
            dgamma += (dy * h).sum(0)
            dbeta += dy.sum(0)
            g = dy * s["gamma"].to(f64)
            dx.append(inv * (g - g.sum(1, keepdim=True) / dim - h * ((g * h).sum(1, keepdim=True) / dim)))
        return {"dx": torch.cat(dx), "dgamma": dgamma, "dbeta": dbeta}
    T, mode = case["T"], case["mode"]
    loss, stats, grads = [], [], []
    for b in range(0, n, step):
        z = s["logits"][b:b + step].to(f64)
        ids, w = s["ids"][b:b + step].long(), torch.ones(z.shape[0], dtype=f64, device=DEV)
        if s["weights"] is not None:
            w = s["weights"][b:b + step].to(f64)
        logp = torch.log_softmax(s["values"][b:b + step].to(f64) / T, 1)
        p = logp.exp()
        if mode == "back":
            kept = s["stats"][b:b + step].to(f64)
            logq = (z - kept[:, :1]) / T - torch.log(kept[:, 1:])
        else:
            logq = torch.log_softmax(z / T, 1)
            loss.append(w * T * T * (p * (logp - torch.gather(logq, 1, ids))).sum(1))
        if mode == "loss":
            top = z.max(1).values
            lost = (w == 0)[:, None]
            stats.append(torch.stack([top, ((z - top[:, None]) / T).exp().sum(1)], 1).masked_fill_(lost, 0.0))
        else:
            dz = logq.exp()
            dz.scatter_add_(1, ids, -p)
            grads.append(dz.mul_((w * T)[:, None]))
    if mode == "loss":
        return {"loss": torch.cat(loss), "stats": torch.cat(stats)}
    grads = torch.cat(grads)
    return grads if mode == "back" else {"loss": torch.cat(loss), "dlogits": grads}
