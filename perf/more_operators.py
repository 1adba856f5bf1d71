"""The operators of a client that trains a language model on its own texts, as a user calls them through paper_2402_03770_amd.cvlc.

Beside the embedding and the norms such a local step needs something that lets a token see those before it, the loss
against the texts' own next tokens, and the optimiser of its local iterations:

  xent         softmax cross entropy of logits = scale * hidden @ table.T over the vocabulary, without the logits in memory;
               mode "loss": the rows' losses and (max, sum); "grad": losses, the hidden rows' gradient and the table's
  scan         a gated linear recurrence: f = sigmoid(gate), h_t = f_t h_(t-1) + (1 - f_t) x_t, channel by channel, over
               sequences that lie one after the other; mode "forward", "backward" (from the kept h), "step" (one token
               of every sequence, states in slots)
  adamw        one AdamW step over all tensors of a model, its two averages in 32 bits or in 8

Sizes: vocabularies of 10 to 262 144 tokens, widths of 16 to 8192, one token to 131 072, models of ten thousand weights to
some hundred million.  `own` is set by whoever measures: False computes the plain form.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256                    # values of an 8-bit state that share a scale
TOP = 448.0                    # largest value of float8_e4m3fn
TINY = 2.0 ** -100             # a block whose largest value is below it is held as zeros
BETAS, EPS, RATE, DECAY, SEED = (0.9, 0.95), 1e-8, 1e-3, 0.1, 1234
MOST_FLOPS = 2.0e12            # of a drawn loss; the largest listed one computes somewhat more
MOST_LOGITS = 1 << 28          # the plain form holds them all
MOST_BYTES = {"scan": 1_200_000_000, "adamw": 4_000_000_000}   # of a drawn one


def listed():
    return [
        # one local batch of a small model: latency
        dict(name="xent_grad_64x64_1000", op="xent", mode="grad", n=64, dim=64, vocab=1000, type="f32", dtable="f32", padding=0.1, pad=0),
        # a medium model that is trained in fp32
        dict(name="xent_grad_2048x768_32000", op="xent", mode="grad", n=2048, dim=768, vocab=32000, type="f32", dtable="f32", padding=0.1, pad=0),
        # a full local batch of a large model, the table's gradient straight into the update vector
        dict(name="xent_grad_4096x2048_50000", op="xent", mode="grad", n=4096, dim=2048, vocab=50000, type="bf16", dtable="f32", padding=0.1, pad=0),
        # sizes that are multiples of nothing, rows with a gap, the table's gradient in its own type
        dict(name="xent_grad_1003x1001_32003", op="xent", mode="grad", n=1003, dim=1001, vocab=32003, type="f16", dtable="same", padding=0.0, pad=3),
        # scoring one short text: few rows, the largest vocabulary
        dict(name="xent_loss_24x2048_200003", op="xent", mode="loss", n=24, dim=2048, vocab=200003, type="bf16", dtable="same", padding=0.0, pad=0),
        # one short text through a small model
        dict(name="scan_forward_32x96", op="scan", mode="forward", n=32, dim=96, sequences=1, ragged=False, type="f32", states=False, pad=0),
        # a full local batch of a large model: texts of 4096 tokens
        dict(name="scan_forward_65536x2048", op="scan", mode="forward", n=65536, dim=2048, sequences=16, ragged=False, type="bf16", states=True, pad=0),
        # one long document and the texts behind it, of any lengths
        dict(name="scan_backward_100003x1000", op="scan", mode="backward", n=100003, dim=1000, sequences=7, ragged=True, type="bf16", states=True, pad=0),
        # serving: one token of each of 256 sequences
        dict(name="scan_step_256x2048", op="scan", mode="step", n=256, dim=2048, sequences=1024, ragged=False, type="bf16", states=True, pad=0),
        # a small model, averages in 32 bits
        dict(name="adamw_f32_1000x96x2", op="adamw", vocab=1000, dim=96, layers=2, type="f32", bits=32, copy="none"),
        # many tensors of odd sizes, averages in 8 bits
        dict(name="adamw_8bit_5003x251x96", op="adamw", vocab=5003, dim=251, layers=96, type="f32", bits=8, copy="none"),
        # a large model: 16-bit gradients and working copy, averages in 8 bits
        dict(name="adamw_8bit_131072x2048x8", op="adamw", vocab=131072, dim=2048, layers=8, type="bf16", bits=8, copy="bf16"),
    ]


def draw(rng):
    def size(low, high):
        v = int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))
        v = max(low, min(high, v))
        if rng.random() < 0.5 and v >= 64:          # some sizes are round
            v -= v % (64 if v < 4096 else 1024)
        return v

    op = rng.choice(["xent", "xent", "xent", "scan", "scan", "scan", "adamw", "adamw"])
    while True:
        case = dict(op=op, type=rng.choice(["f32", "bf16", "bf16", "f16"]))
        if op == "xent":
            case |= dict(mode=rng.choice(["loss", "grad", "grad"]), n=size(1, 16384), dim=size(16, 8192), vocab=size(10, 262144),
                         dtable=rng.choice(["f32", "same"]), padding=rng.choice([0.0, 0.1, 0.5]), pad=rng.choice([0, 0, 8, 3]))
            fits = case["n"] * case["vocab"] <= MOST_LOGITS and work(case)["flops"] <= MOST_FLOPS
        elif op == "scan":
            case |= dict(mode=rng.choice(["forward", "backward", "backward", "step"]), dim=size(16, 8192), states=rng.random() < 0.5,
                         pad=rng.choice([0, 0, 8, 3]))
            if case["mode"] == "step":
                n = size(1, 4096)
                case |= dict(n=n, sequences=n + size(1, 1024), ragged=False, states=True)
            elif rng.random() < 0.5:
                n = size(1, 131072)
                case |= dict(n=n, sequences=min(n, size(1, 64)), ragged=True)
            else:
                sequences = size(1, 64)
                case |= dict(n=sequences * size(1, 131072 // sequences), sequences=sequences, ragged=False)
            fits = work(case)["bytes"] <= MOST_BYTES[op]
        else:
            case |= dict(vocab=size(64, 131072), dim=size(16, 2048), layers=size(1, 128), bits=rng.choice([8, 8, 32]),
                         copy=rng.choice(["none", "bf16", "f16"]))
            fits = work(case)["bytes"] <= MOST_BYTES[op]
        if fits:
            return case


def _shapes(case):
    """The tensors of a model: the table, then every layer's gate and candidate matrices, and its norm's two vectors.
    Rows and columns; the vectors, of one row, do not decay."""
    dim = case["dim"]
    return [(case["vocab"], dim)] + [(dim, dim), (dim, dim), (1, dim), (1, dim)] * case["layers"]


def _bytes_of(name):
    return {"none": 0, "f32": 4, "bf16": 2, "f16": 2}[name]


def work(case):
    e = _bytes_of(case["type"])
    if case["op"] == "xent":
        n, dim, vocab = case["n"], case["dim"], case["vocab"]
        product = 2.0 * n * (1.0 - case["padding"]) * dim * vocab
        if case["mode"] == "loss":
            return {"bytes": e * (n + vocab) * dim + 20 * n, "flops": product}
        out = 4 if case["dtable"] == "f32" else e
        return {"bytes": e * (2 * n + vocab) * dim + out * vocab * dim + 16 * n, "flops": 3 * product}
    if case["op"] == "scan":
        values, states = case["n"] * case["dim"], 4 * case["sequences"] * case["dim"]
        if case["mode"] == "step":
            return {"bytes": (3 * e + 8) * values + 8 * case["n"], "flops": 6 * values}
        streams, kept = (3, 2) if case["mode"] == "forward" else (6, 3)
        return {"bytes": streams * e * values + (kept * states if case["states"] else 0), "flops": (6 if streams == 3 else 12) * values}
    shapes = _shapes(case)
    n = sum(r * c for r, c in shapes)
    blocks = sum(-(-r * c // BLOCK) for r, c in shapes)
    held = 16 * n if case["bits"] == 32 else 4 * n + 16 * blocks
    return {"bytes": (8 + e + _bytes_of(case["copy"])) * n + held, "flops": 16 * n}


# ----------------------------------------------------------------------------- inputs
def _rows(n, width, extra, dtype):
    """An uninitialised matrix whose rows lie `extra` values further apart than they are long."""
    return torch.empty(n, width + extra, dtype=dtype, device=DEV)[:, :width]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = TYPES[case["type"]]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, dtype=dtype, device=DEV, generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device=DEV, generator=gen)

    state = dict(case=case)
    if case["op"] == "xent":
        n, dim, vocab = case["n"], case["dim"], case["vocab"]
        # next tokens of texts: low numbers are frequent; -1 where a text has none
        labels = (torch.exp(uniform(n).double() * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
        table = _rows(vocab, dim, case["pad"], dtype)
        table.copy_(normal(vocab, dim, dtype=dtype).mul_(1.5 * dim ** -0.5))
        hidden = _rows(n, dim, case["pad"], dtype)                       # rows as a norm leaves them, some of which know the answer
        hidden.copy_(normal(n, dim) + 4.0 * uniform(n, 1) * table[labels].float())
        if case["padding"]:
            labels[uniform(n) < case["padding"]] = -1
        live = labels >= 0
        state |= dict(hidden=hidden, table=table, labels=labels, scale=1.0,
                      weights=(live / live.sum().clamp(min=1)).float() if case["mode"] == "grad" else None)
    elif case["op"] == "scan":
        n, dim, sequences = case["n"], case["dim"], case["sequences"]
        x, gate = _rows(n, dim, case["pad"], dtype), _rows(n, dim, case["pad"], dtype)
        x.copy_(normal(n, dim, dtype=dtype))
        # channels that forget at once and channels that remember for thousands of tokens
        gate.copy_(normal(n, dim, dtype=dtype) + torch.linspace(-1.0, 7.0, dim, device=DEV).to(dtype))
        state |= dict(x=x, gate=gate)
        if case["mode"] == "step":
            slots = torch.randperm(sequences, device=DEV, generator=gen)[:n]
            return state | dict(states=normal(sequences, dim), slots=slots)
        starts = torch.arange(sequences + 1, device=DEV) * (n // sequences)
        if case["ragged"]:                          # cuts anywhere: one text is long, some are short, some are empty
            cuts = (uniform(max(sequences - 1, 1)).square() * (n + 1)).long().clamp_(0, n)[:sequences - 1]
            starts = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), cuts.sort().values, torch.full((1,), n, dtype=torch.long, device=DEV)])
        state |= dict(starts=starts, h0=normal(sequences, dim) if case["states"] else None)
        if case["mode"] == "backward":
            dy = _rows(n, dim, case["pad"], dtype)
            dy.copy_(normal(n, dim, dtype=dtype))
            h = _rows(n, dim, case["pad"], dtype)
            h.copy_(_plain_forward(state)["h"])
            state |= dict(dy=dy, h=h, dlast=normal(sequences, dim) if case["states"] else None)
    else:
        shapes = _shapes(case)
        sizes = [r * c for r, c in shapes]
        n, copy = sum(sizes), TYPES.get(case["copy"])
        # a model some hundred steps into its training, and a new gradient; matrices' rows have scales of their own
        spread = torch.exp(1.5 * normal(sum(r for r, _ in shapes)))
        spread = torch.repeat_interleave(spread, torch.tensor([c for r, c in shapes for _ in range(r)], device=DEV), output_size=n) * 1e-3
        grad = normal(n).mul_(spread).to(dtype)
        param = normal(n).mul_(0.02)
        m, v = normal(n).mul_(spread).mul_(0.3), uniform(n).add_(0.5).mul_(spread).square_()
        state |= dict(sizes=sizes, decays=[DECAY if r > 1 else 0.0 for r, _ in shapes], param=param, grad=grad, step=300,
                      copy=param.to(copy) if copy is not None else None)
        if case["bits"] == 32:
            state |= dict(m=m, v=v)
        else:
            spans = _spans(state)
            m, ms = _held(m, spans, None)
            v, vs = _held(v.sqrt_(), spans, torch.full((n,), 1 << 15, dtype=torch.int64, device=DEV))
            state |= dict(m=m, v=v, scales=torch.stack([ms, vs], 1).contiguous())
    return state


# ----------------------------------------------------------------------------- one pass
def run(state):
    return _calls(state) if own else PLAIN[state["case"]["op"]](state)


def _calls(state):
    import paper_2402_03770_amd.cvlc as cv

    case = state["case"]
    kept = state.get("kept")
    if kept is None:                                # output buffers, workspaces and plans of a program's own, made once
        kept = state["kept"] = _buffers(state, cv)
    if case["op"] == "xent":
        cv.linear_xent(state["hidden"], state["table"], state["labels"], kept["loss"], kept["workspace"], scale=state["scale"],
                       weights=state["weights"], stats_out=kept["stats"])
        if case["mode"] == "loss":
            return {"loss": kept["loss"], "stats": kept["stats"]}
        cv.linear_xent_grad(state["hidden"], state["table"], state["labels"], kept["stats"], kept["dhidden"], kept["dtable"],
                            kept["workspace"], scale=state["scale"], weights=state["weights"])
        return {"loss": kept["loss"], "dhidden": kept["dhidden"], "dtable": kept["dtable"]}
    if case["op"] == "scan":
        if case["mode"] == "step":
            cv.gated_scan_step(state["x"], state["gate"], state["states"], kept["h"], slots=state["slots"])
            return {"h": kept["h"], "states": state["states"]}
        cut = dict(starts=state["starts"]) if case["ragged"] else dict(sequences=case["sequences"])
        if case["mode"] == "forward":
            cv.gated_scan(state["x"], state["gate"], kept["h"], kept["workspace"], h0=state["h0"], last_out=kept["last"], **cut)
            return {"h": kept["h"], "last": kept["last"]}
        cv.gated_scan_grad(state["dy"], state["x"], state["gate"], state["h"], kept["dx"], kept["dgate"], kept["workspace"],
                           h0=state["h0"], dlast=state["dlast"], dh0_out=kept["dh0"], **cut)
        return {"dx": kept["dx"], "dgate": kept["dgate"], "dh0": kept["dh0"]}
    cv.adamw(kept["plan"], state["step"], RATE, betas=BETAS, eps=EPS, seed=SEED)
    out = {"param": state["param"], "m": state["m"], "v": state["v"]}
    if case["bits"] == 8:
        out["scales"] = state["scales"]
    if state["copy"] is not None:
        out["copy"] = state["copy"]
    return out


def _buffers(state, cv):
    case, dtype = state["case"], TYPES[state["case"]["type"]]

    def new(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if case["op"] == "xent":
        n, dim, vocab = case["n"], case["dim"], case["vocab"]
        kept = dict(loss=new(n), stats=new(n, 2))
        need = cv.linear_xent_workspace_bytes(n, vocab, dim, dtype)
        if case["mode"] == "grad":
            dtable = torch.float32 if case["dtable"] == "f32" else dtype
            kept |= dict(dhidden=new(n, dim, dtype=dtype), dtable=new(vocab, dim, dtype=dtable))
            need = max(need, cv.linear_xent_grad_workspace_bytes(n, vocab, dim, dtype, dtable))
        return kept | dict(workspace=cv.new_workspace(need, DEV))
    if case["op"] == "scan":
        n, dim, sequences = case["n"], case["dim"], case["sequences"]
        if case["mode"] == "step":
            return dict(h=new(n, dim, dtype=dtype))
        states = new(sequences, dim) if case["states"] else None
        need = cv.gated_scan_workspace_bytes(n, dim, sequences)
        kept = dict(workspace=cv.new_workspace(need, DEV))
        if case["mode"] == "forward":
            return kept | dict(h=new(n, dim, dtype=dtype), last=states)
        return kept | dict(dx=new(n, dim, dtype=dtype), dgate=new(n, dim, dtype=dtype), dh0=states)
    sizes = state["sizes"]

    def parts(flat):
        return list(torch.split(flat, sizes)) if flat is not None else None

    scales = None
    if case["bits"] == 8:
        scales = list(torch.split(state["scales"], [-(-s // BLOCK) for s in sizes]))
    return dict(plan=cv.AdamwPlan(parts(state["param"]), parts(state["grad"]), parts(state["m"]), parts(state["v"]), scales=scales,
                                  copies=parts(state["copy"]), weight_decays=state["decays"]))


def _plain_xent(s):
    case = s["case"]
    h, table = s["hidden"].float(), s["table"].float()
    z = torch.mm(h, table.t()).mul_(s["scale"])
    live = s["labels"] >= 0
    at = s["labels"].clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    answer = z.gather(1, at)
    e = torch.exp(z.sub_(top))
    total = e.sum(1, keepdim=True)
    w = live.float() if s["weights"] is None else s["weights"] * live
    loss = (torch.log(total) + (top - answer))[:, 0] * w
    if case["mode"] == "loss":
        return {"loss": loss, "stats": torch.cat([top, total], 1) * live[:, None]}
    g = e.div_(total).scatter_add_(1, at, torch.full_like(total, -1.0)).mul_((w * s["scale"])[:, None])
    dtable = torch.mm(g.t(), h)
    return {"loss": loss, "dhidden": torch.mm(g, table).to(s["hidden"].dtype),
            "dtable": dtable if case["dtable"] == "f32" else dtable.to(s["table"].dtype)}


def _running(a, b):
    """h_t = a_t h_(t-1) + b_t from h = 0 on, down the rows: every round joins each row with the one `far` above it."""
    n, far = a.shape[0], 1
    while far < n:
        b = torch.cat([b[:far], b[far:] + a[far:] * b[:-far]])
        a = torch.cat([a[:far], a[far:] * a[:-far]])
        far *= 2
    return b


def _ends(s):
    """First and last rows of the sequences that have any, and which these are."""
    first, last = s["starts"][:-1], s["starts"][1:] - 1
    some = torch.nonzero(last >= first)[:, 0]
    return first[some], last[some], some


def _plain_forward(s):
    x, gate = s["x"].float(), s["gate"].float()
    f = 1.0 / (1.0 + torch.exp(-gate))
    b = x * (1.0 / (1.0 + torch.exp(gate)))
    first, last, some = _ends(s)
    if s["h0"] is not None:
        b.index_add_(0, first, f[first] * s["h0"][some])
    f[first] = 0.0
    h = _running(f, b)
    ends = None
    if s["h0"] is not None:
        ends = s["h0"].clone()
        ends[some] = h[last]
    return {"h": h.to(s["x"].dtype), "last": ends}


def _plain_scan(s):
    mode = s["case"]["mode"]
    if mode == "forward":
        return _plain_forward(s)
    x, gate = s["x"].float(), s["gate"].float()
    f, rest = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    if mode == "step":
        h = f * s["states"][s["slots"]] + rest * x
        s["states"][s["slots"]] = h
        return {"h": h.to(s["x"].dtype), "states": s["states"]}
    first, last, some = _ends(s)
    b = s["dy"].float()
    if s["dlast"] is not None:
        b = b.index_add(0, last, s["dlast"][some])
    a = torch.cat([f[1:], f[:1]])                   # row t's factor is the next row's gate
    a[last] = 0.0
    d = _running(a.flip(0), b.flip(0)).flip(0)
    before = torch.cat([s["h"][:1], s["h"][:-1]]).float()
    before[first] = s["h0"][some] if s["h0"] is not None else 0.0
    dh0 = None
    if s["dlast"] is not None:
        dh0 = s["dlast"].clone()
        dh0[some] = f[first] * d[first]
    return {"dx": (rest * d).to(s["x"].dtype),
            "dgate": (d * (before - x) * (f * rest)).to(s["x"].dtype), "dh0": dh0}


def _spans(s):
    """For every weight its place where each tensor begins a new block of 256; and how many blocks there are."""
    counts = torch.tensor([-(-n // BLOCK) for n in s["sizes"]], device=DEV)
    sizes = torch.tensor(s["sizes"], device=DEV)
    ahead = (counts.cumsum(0) - counts) * BLOCK - (sizes.cumsum(0) - sizes)
    n = sum(s["sizes"])
    return torch.repeat_interleave(ahead, sizes, output_size=n).add_(torch.arange(n, device=DEV)), sum(-(-k // BLOCK) for k in s["sizes"])


def _held(x, spans, chance):
    """x in 8 bits: codes and the blocks' scales.  To nearest, or, with 16 bits of `chance` for every value (>= 0), up or
    down by them and never down to zero."""
    place, blocks = spans
    laid = torch.zeros(blocks * BLOCK, device=DEV)
    laid[place] = x.abs()
    top, block = laid.view(blocks, BLOCK).amax(1), place // BLOCK
    top = torch.where(top >= TINY, top, 0.0)
    y = (x * torch.where(top > 0, TOP / top, 0.0)[block]).clamp_(-TOP, TOP)
    if chance is not None:
        # eight values to an octave from 2^-6 on, steps of 2^-9 below
        normal = ((y.view(torch.int32) + (chance << 4).int()) & -(1 << 20)).view(torch.float32)
        small = torch.floor(y * 512.0 + chance * 2.0 ** -16) * 2.0 ** -9
        y = torch.where(y >= 2.0 ** -6, normal, torch.where(y > 0, small.clamp(min=2.0 ** -9), 0.0)).clamp_(max=TOP)
    return y.to(torch.float8_e4m3fn), top * (1.0 / TOP)


def _chance(s):
    """16 bits for every weight: Philox4x32-10 with the seed as its key, of (number in the tensor / 8, step, tensor); the
    eight halves of its words, low ones first."""
    low = 0xFFFFFFFF
    sizes = s["sizes"]
    eighths = [-(-n // 8) for n in sizes]
    total = sum(eighths)
    lengths = torch.tensor(eighths, device=DEV)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), lengths, output_size=total)
    at = torch.arange(total, device=DEV) - (lengths.cumsum(0) - lengths)[tensor]
    c = [at, torch.zeros_like(at), torch.full_like(at, s["step"]), tensor]
    k = [SEED & low, SEED >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((q >> 32) & low) ^ c[1] ^ k[0], q & low, ((p >> 32) & low) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    halves = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], 1)
    return halves[torch.arange(8, device=DEV) < (torch.tensor(sizes, device=DEV)[tensor] - at * 8)[:, None]]


def _plain_adamw(s):
    case = s["case"]
    n, (b1, b2), t = sum(s["sizes"]), BETAS, s["step"]
    rate, root = RATE / (1.0 - b1 ** t), math.sqrt(1.0 - b2 ** t)
    keep = torch.repeat_interleave(torch.tensor([1.0 - RATE * d for d in s["decays"]], device=DEV),
                                   torch.tensor(s["sizes"], device=DEV), output_size=n)
    g = s["grad"].float()
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        spans = _spans(s)
        scales = s["scales"][spans[0] // BLOCK]
        m = s["m"].float() * scales[:, 0]
        v = (s["v"].float() * scales[:, 1]).square()
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * g * (1.0 - b2)
    r = torch.sqrt(v)
    s["param"].copy_(s["param"] * keep - rate * (m / (r / root + EPS)))
    out = {"param": s["param"], "m": s["m"], "v": s["v"]}
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        mc, ms = _held(m, spans, None)
        vc, vs = _held(r, spans, _chance(s))
        s["m"].copy_(mc)
        s["v"].copy_(vc)
        s["scales"].copy_(torch.stack([ms, vs], 1))
        out["scales"] = s["scales"]
    if s["copy"] is not None:
        s["copy"].copy_(s["param"])
        out["copy"] = s["copy"]
    return out


PLAIN = {"xent": _plain_xent, "scan": _plain_scan, "adamw": _plain_adamw}


# ----------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"xent": _exact_xent, "scan": _exact_scan, "adamw": _exact_adamw}[case["op"]](case, s)


def _exact_xent(case, s):
    f64 = torch.float64
    n, vocab = case["n"], case["vocab"]
    table = s["table"].to(f64)
    step = max(1, (1 << 27) // vocab)                # rows at a time
    loss, stats, dhidden = [], [], []
    dtable = torch.zeros(vocab, case["dim"], dtype=f64, device=DEV) if case["mode"] == "grad" else None
    for i in range(0, n, step):
        h, labels = s["hidden"][i:i + step].to(f64), s["labels"][i:i + step]
        w = (labels >= 0).to(f64)
        if s["weights"] is not None:
            w = w * s["weights"][i:i + step].to(f64)
        z = torch.matmul(h, table.mT) * s["scale"]
        logq = torch.log_softmax(z, 1)
        loss.append(-w * logq[torch.arange(len(labels), device=DEV), labels.clamp(min=0)])
        if case["mode"] == "loss":
            top = z.max(1).values
            stats.append(torch.stack([top, torch.exp(torch.logsumexp(z, 1) - top)], 1) * (labels >= 0)[:, None])
            continue
        dz = torch.exp(logq)
        dz[torch.arange(len(labels), device=DEV), labels.clamp(min=0)] -= 1.0
        dz *= (w * s["scale"])[:, None]
        dhidden.append(torch.matmul(dz, table))
        dtable += torch.matmul(dz.mT, h)
    if case["mode"] == "loss":
        return {"loss": torch.cat(loss), "stats": torch.cat(stats)}
    return {"loss": torch.cat(loss), "dhidden": torch.cat(dhidden), "dtable": dtable}


def _exact_walk(decay, add):
    """The recurrence in pieces of rows that all walk at once, then from piece to piece."""
    n, dim = add.shape
    long = max(1, math.isqrt(n))
    pieces = -(-n // long)
    spare = pieces * long - n
    decay = torch.nn.functional.pad(decay, (0, 0, 0, spare)).view(pieces, long, dim)
    out = torch.nn.functional.pad(add, (0, 0, 0, spare)).view(pieces, long, dim)
    reach = decay.clone()
    for t in range(1, long):
        out[:, t] += decay[:, t] * out[:, t - 1]
        reach[:, t] *= reach[:, t - 1]
    for p in range(1, pieces):
        out[p] += reach[p] * out[p - 1, -1]
    return out.view(-1, dim)[:n]


def _exact_scan(case, s):
    f64 = torch.float64
    x, gate = s["x"].to(f64), s["gate"].to(f64)
    f, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    if case["mode"] == "step":
        h = torch.lerp(x, s["states"][s["slots"]].to(f64), f)
        states = s["states"].to(f64)
        states[s["slots"]] = h
        return {"h": h, "states": states}
    length = s["starts"].diff()
    some = length > 0
    first, last = s["starts"][:-1][some], s["starts"][1:][some] - 1
    if case["mode"] == "forward":
        add, decay = rest * x, f.clone()
        if s["h0"] is not None:
            add[first] += f[first] * s["h0"][some].to(f64)
        decay[first] = 0.0
        h = _exact_walk(decay, add)
        ends = None
        if s["h0"] is not None:
            ends = s["h0"].to(f64)
            ends[some] = h[last]
        return {"h": h, "last": ends}
    add, decay = s["dy"].to(f64), torch.roll(f, -1, 0)
    decay[last] = 0.0
    if s["dlast"] is not None:
        add[last] += s["dlast"][some].to(f64)
    d = _exact_walk(decay.flip(0), add.flip(0)).flip(0)
    del add, decay
    held = torch.roll(s["h"], 1, 0).to(f64)
    held[first] = s["h0"][some].to(f64) if s["h0"] is not None else 0.0
    dh0 = None
    if s["dlast"] is not None:
        dh0 = s["dlast"].to(f64)
        dh0[some] = d[first] * f[first]
    return {"dx": d * rest, "dgate": d * f * rest * (held - x), "dh0": dh0}


def _exact_adamw(case, s):
    """Weights and averages from what the states stand for.  Codes of 8 bits have none: a value next to a border may go
    either way."""
    f64 = torch.float64
    (b1, b2), t = BETAS, s["step"]
    param, m, v, scales, at, block = [], [], [], [], 0, 0
    for n, decay in zip(s["sizes"], s["decays"]):
        part = slice(at, at + n)
        g = s["grad"][part].to(f64)
        old_m, old_v = s["m"][part].to(f64), s["v"][part].to(f64)
        if case["bits"] == 8:
            count = -(-n // BLOCK)
            held = torch.repeat_interleave(s["scales"][block:block + count].to(f64), BLOCK, 0)[:n]
            old_m, old_v = old_m * held[:, 0], (old_v * held[:, 1]) ** 2
        new_m, new_v = torch.lerp(g, old_m, b1), torch.lerp(g * g, old_v, b2)
        move = (new_m / (1.0 - b1 ** t)) / (torch.sqrt(new_v / (1.0 - b2 ** t)) + EPS)
        p = s["param"][part].to(f64)
        param.append(p - RATE * decay * p - RATE * move)
        if case["bits"] == 32:
            m.append(new_m)
            v.append(new_v)
        else:
            tops = [torch.nn.functional.pad(u, (0, count * BLOCK - n)).view(count, BLOCK).abs().amax(1) / TOP
                    for u in (new_m, torch.sqrt(new_v))]
            scales.append(torch.stack(tops, 1))
            block += count
        at += n
    param = torch.cat(param)
    out = {"param": param, "m": torch.cat(m) if m else None, "v": torch.cat(v) if v else None}
    if case["bits"] == 8:
        out["scales"] = torch.cat(scales)
    if s["copy"] is not None:
        out["copy"] = param
    return out
