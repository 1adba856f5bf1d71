"""What a client trains with, on inputs and sizes beside the ordinary: values that are not finite, sequences without rows, averages
over thousands of steps, calls that the caches do not hold.  Oracles as in test_training.py."""
import ctypes as C
import warnings

import numpy as np
import pytest
import torch

import paper_2402_03770_amd.cvlc as cv
from oracle import training as ref
from test_local_step import BF16, DEV, F16, F32, assert_near, f64
from test_training import Scan, Tensors, Xent, check_adamw, cuts

gpu = pytest.mark.gpu


# ----------------------------------------------------------------------------- the gated scan
# lengths, width: all rows in one iteration of a workgroup, in several, in ranges of a thread's each, and enough channels for every
# CU to go over all rows
FLAT = {"one": ([3, 5, 0, 40, 2, 30], 24), "several": ([200, 1, 0, 310, 7, 2, 60], 20), "ranges": ([900, 3, 0, 1200, 17, 8, 700], 40),
        "wide": ([200, 1, 0, 310, 7, 60], 8200)}


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("lengths,dim", FLAT.values(), ids=FLAT)
def test_gated_scan_keeps_what_is_not_finite_to_its_sequence(dtype, bad, lengths, dim):
    """A value that is not finite, in every sequence in turn: the other sequences, and the other channels, come out bit by bit as
    without it; so do the sequence's rows that the walk comes to before it."""
    starts, bounds = cuts(lengths)
    n, at = int(starts[-1]), torch.from_numpy(starts).to(DEV)
    s = Scan(n, dim, dtype, len(lengths))
    s.forward(starts=at)
    s.backward(starts=at)
    clean = [t.clone() for t in (s.h, s.last, s.dx, s.dgate, s.dh0)]
    for j, (low, high) in enumerate(bounds):
        if low == high:
            continue
        row, c = low + (high - low) // 3, dim // 2
        other_rows, other_states = [k for k in range(n) if not low <= k < high], [k for k in range(len(lengths)) if k != j]
        others = [k for k in range(dim) if k != c]

        def apart(got, want, inside, still):
            """`got` is `want` but in the channel, where of the sequence's rows the `still` are too and the rest are not finite."""
            rows = other_rows if inside else other_states
            assert torch.equal(got[:, others], want[:, others]) and torch.equal(got[rows][:, c], want[rows][:, c])
            own = got[low:high, c] if inside else got[j:j + 1, c]
            was = want[low:high, c] if inside else want[j:j + 1, c]
            assert torch.equal(own[still], was[still]) and not bool(torch.isfinite(own[~still]).any())

        none, k = torch.zeros(1, dtype=torch.bool, device=DEV), torch.arange(low, high, device=DEV)
        for name, place, first in (("x", s.x[row], row), ("gate", s.gate[row], row), ("h0", s.h0[j], low)):
            if name == "gate" and np.isinf(bad):
                continue                                               # a gate that keeps everything, and as good as any
            kept = place[c].clone()
            place[c] = bad
            s.forward(starts=at)
            place[c] = kept
            apart(s.h, clean[0], True, k < first)
            apart(s.last, clean[1], False, none)
        s.h.copy_(clean[0])
        for place, first in ((s.dy[row], row), (s.dlast[j], high)):
            kept = place[c].clone()
            place[c] = bad
            s.backward(starts=at)
            place[c] = kept
            apart(s.dx, clean[2], True, k > first)
            apart(s.dgate, clean[3], True, k > first)
            apart(s.dh0, clean[4], False, none)


@gpu
@pytest.mark.parametrize("lengths,dim", FLAT.values(), ids=FLAT)
def test_gated_scan_whose_gates_forget_everything_keeps_a_nan(lengths, dim):
    """Products of gates that are too small for fp32 are not taken for a sequence's beginning."""
    starts, bounds = cuts(lengths)
    n, at = int(starts[-1]), torch.from_numpy(starts).to(DEV)
    s = Scan(n, dim, F32, len(lengths))
    s.gate.fill_(-60.0)
    j = int(np.argmax(lengths))
    low, high = bounds[j]
    s.x[low + 2] = float("nan")
    s.forward(starts=at)
    bad = np.isnan(f64(s.h))
    assert bad[low + 2:high].all() and bad.sum() == (high - low - 2) * dim and bool(torch.isnan(s.last[j]).all())


@gpu
@pytest.mark.parametrize("dim", [1, 3, 33, 64, 65, 512, 513, 2304, 8192])
@pytest.mark.parametrize("sequences,every,rows", [(43, 3, 2), (4096, 50, 1), (4097, 50, 1), (9001, 400, 30), (70, 1000, 0)])
def test_gated_scan_states_of_sequences_without_rows(sequences, every, rows, dim):
    """Of `sequences` one in `every` has `rows` rows; the others hand their states on, forward and back, at any width."""
    if sequences * dim > 1 << 23:
        dim = (1 << 23) // sequences
    lengths = [rows if j % every == every - 1 else 0 for j in range(sequences)]
    starts, _ = cuts(lengths)
    n, at = int(starts[-1]), torch.from_numpy(starts).to(DEV)
    empty = torch.tensor([k == 0 for k in lengths], device=DEV)
    s, status = Scan(n, dim, F32, sequences), torch.zeros(1, dtype=torch.int32, device=DEV)
    s.forward(starts=at, status=status)
    s.backward(starts=at, status=status)
    assert status.item() == 0
    assert torch.equal(s.last[empty], s.h0[empty]) and torch.equal(s.dh0[empty], s.dlast[empty])
    full = [k for k, x in enumerate(lengths) if x]
    assert torch.equal(s.last[full], s.h[starts[1:][full] - 1])
    s.h0 = s.dlast = None
    s.forward(starts=at)
    s.backward(starts=at)
    assert not bool(s.last[empty].any()) and not bool(s.dh0[empty].any())
    if n:                                                              # without states that are handed on, offsets are looked at all the same
        at[sequences // 2] = n + 1
        cv.gated_scan(s.x, s.gate, s.h, s.ws, starts=at, status=status)
        assert status.item() == cv.DEV_INDEX


# ----------------------------------------------------------------------------- AdamW
@gpu
@pytest.mark.parametrize("grad,copy", [(F32, None), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("sizes", [[1], [255, 256, 257], [7, 0, 513, 1, 2048, 30], [8193, 20000]], ids=str)
def test_adamw_m_by_chance(grad, copy, sizes):
    """m's codes are those that its chances say; everything else is, bit by bit, what it is without."""
    t, same = (Tensors(sizes, 8, grad, copy, offset=3, seed=len(sizes)) for _ in range(2))
    decays, seed, betas = [0.1 * (i % 3) for i in range(len(sizes))], 2 ** 40 + 5, (0.9, 0.999)
    plans = [cv.AdamwPlan(x.param, x.grad, x.m, x.v, scales=x.scales, copies=x.copy, weight_decays=decays, m_by_chance=on)
             for x, on in ((t, True), (same, False))]
    for step in (1, 2, 1000):
        for a, b in zip(same.m, t.m):
            a.copy_(b)
        before = [t.read(i) for i in range(len(sizes))]
        for plan in plans:
            cv.adamw(plan, step, 1e-2, betas=betas, grad_scale=0.7, seed=seed)
        check_adamw(same, before, decays, step, 1e-2, betas, 1e-8, 0.7, seed, copy)
        for a, b in zip((*t.param, *t.v, *t.scales, *(t.copy or [])), (*same.param, *same.v, *same.scales, *(same.copy or []))):
            assert torch.equal(a, b)
        for i, (old, decay) in enumerate(zip(before, decays)):
            _, _, m, off, *_ = ref.adamw(*old, step, 1e-2, betas, 1e-8, decay, 0.7, True)
            top = ref.spread(f64(t.scales[i])[:, :1], m.size)[:, 0]
            rel = np.where(m != 0, off / np.maximum(np.abs(m), 1e-300), 0.0) + 6 * ref.U
            with np.errstate(divide="ignore", invalid="ignore"):
                y = np.where(top > 0, np.abs(m) / top, 0.0)
            # beyond the values' own error a step of 2^-9 and its chance have a rounding in the sum of up to 8
            chance = ref.chances(m.size, seed, step, i, word=1)
            low, high = (ref.by_chance(np.minimum(y * (1 + s * rel), 448.0), np.clip(chance + s * 2.0 ** -4, 0, 65535.9375), least=0) for s in (-1, 1))
            codes = t.m[i].cpu().numpy().astype(np.int64)
            assert np.all((low <= codes & 127) & (codes & 127 <= high)) and np.sum(low != high) <= 1 + 0.02 * m.size
            assert np.all((codes & 127 == 0) | ((codes >= 128) == (m < 0)))


@gpu
@pytest.mark.parametrize("betas", [(0.9, 0.95), (0.95, 0.99), (0.99, 0.999)], ids=str)
@pytest.mark.parametrize("dim", [64, 251])
def test_adamw_8bit_weights_whose_gradient_ends_come_to_rest(dim, betas):
    """Of every four rows of a table one keeps getting gradients, three do not after step 20, beside it in a block.  The mean of a
    code that is rounded by chance goes as the average itself does, by beta1 a step, from 448 at most; a code that is not zero is
    2^-9 at least, so one that lasts for k steps has a probability of 448 * 512 * beta1^k, and as many times more as its block's
    scale has become smaller by: less than 2^-36 after `still` of them where that is less than 16.  In blocks without a row that goes
    on the scales vanish with what they hold.  From there on the weights are where they are, to the last bit."""
    rows, n = 64, 64 * dim
    still = int(np.ceil(-np.log(448.0 * 512 * 2.0 ** 40 * n) / np.log(betas[0])))
    gen = torch.Generator().manual_seed(dim)
    param, grad = torch.randn(n, generator=gen).to(DEV), torch.empty(n, device=DEV)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    plan = cv.AdamwPlan([param], [grad], [m], [v], scales=[torch.zeros(-(-n // 256), 2, device=DEV)], m_by_chance=True)
    ended = (torch.arange(rows, device=DEV) % 4 != 0).repeat_interleave(dim)
    blocks = torch.nn.functional.pad(~ended, (0, -n % 256)).view(-1, 256).any(1)      # with a row that goes on
    beside = ended & blocks.repeat_interleave(256)[:n]
    gen = torch.Generator(DEV).manual_seed(1)
    start = param.clone()
    for step in range(1, 20 + still + 400):
        grad.normal_(generator=gen)
        if step > 20:
            grad[ended] = 0.0
        cv.adamw(plan, step, 1e-3, betas=betas, seed=5)
        if step == 20:
            assert bool((m[beside] & 127).any())
        if step == 20 + still:
            assert not bool((m[beside] & 127).any())
            rest = param.clone()
    assert torch.equal(param[ended], rest[ended])
    assert (param[~ended] != rest[~ended]).float().mean() > 0.99 and (param[ended] != start[ended]).float().mean() > 0.99


@gpu
def test_adamw_8bit_m_moves_on_average():
    """A gradient that is 0.7 of the average: m must come down to it, by less than half a code a step."""
    n, held, b1 = 256 * 64, 64.0, 0.9
    t = Tensors([n], 8, F32, None, offset=0, seed=1)
    t.m[0].fill_(int(ref.nearest(np.array([held]))[0]))
    t.m[0][::256] = 0x7E                                               # the blocks' largest, which holds the scale where it is
    t.v[0].zero_()
    t.scales[0].fill_(1.0)
    t.grad[0].fill_(0.7 * held)
    t.grad[0][::256] = 448.0
    plan = cv.AdamwPlan(t.param, t.grad, t.m, t.v, scales=t.scales, m_by_chance=True)
    for k, want in ((3, 0.7 * held + 0.3 * held * b1 ** 3), (100, 0.7 * held)):
        for step in range(1, k + 1):
            cv.adamw(plan, step + 100 * k, 0.0, betas=(b1, 0.99), seed=3)
        got = (ref.values(t.m[0].cpu()) * ref.spread(f64(t.scales[0]), n)[:, 0]).reshape(-1, 256)[:, 1:]
        # Between 32 and 64 codes are 4 apart: a rounding's variance is 4 at most, and what is left of all before it adds up to
        # 4 / (1 - b1^2); 6 deviations of the mean, a chance's step of 2^-16 of 4 for each of 1 / (1 - b1) roundings, what is left
        # of the start after the steps, and fp32's roundings.
        tol = 6 * np.sqrt(4 / (1 - b1 ** 2) / got.size) + 4 * 2.0 ** -16 / (1 - b1) + (0.3 * held * b1 ** 103 if k == 100 else 0) + 1e-4
        assert abs(got.mean() - want) <= tol


@gpu
def test_adamw_m_by_chance_is_a_choice():
    """A warning where averages in 8 bits come without it; flags that are not there are refused."""
    t = Tensors([300], 8, F32, None, offset=0, seed=1)
    lists, other = (t.param, t.grad, t.m, t.v), Tensors([300], 32, F32, None, offset=0, seed=1)
    with pytest.warns(UserWarning, match="m_by_chance"):
        cv.AdamwPlan(*lists, scales=t.scales)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        for on in (True, False):
            cv.AdamwPlan(*lists, scales=t.scales, m_by_chance=on)
        for on in (None, True):
            cv.AdamwPlan(other.param, other.grad, other.m, other.v, m_by_chance=on)


def test_adamw_flags_that_are_not_there():
    ok, data = 1 << 20, cv.AdamwPlanData()
    for flags, want in ((2, cv.ERR_ARG), (1 << 8, cv.ERR_ARG), (3, cv.ERR_ARG)):
        t = (cv.AdamwTensor * 1)(cv.AdamwTensor(100, ok, ok + 4096, ok + 8192, ok + 16384, ok + 32768, None, 1, 0, 8, 0.0, flags))
        assert cv.lib().cvlc_adamw_plan(1, t, ok + (1 << 20), 1 << 20, C.byref(data), None) == want


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_keeps_weights_from_what_is_not_finite(bits):
    """Rates from the device that are no numbers, averages and weights that are none, steps beyond fp32: told of, and such elements
    stay; the others go on."""
    t = Tensors([600], bits, F32, None, offset=0, seed=2)
    plan = cv.AdamwPlan(t.param, t.grad, t.m, t.v, scales=t.scales, m_by_chance=True)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    start = t.param[0].clone()
    for now in ((5.0, float("nan"), 1.0), (5.0, float("inf"), 1.0), (5.0, 1e-3, float("nan")), (1.0, 3e38, 1.0)):       # the last: a rate of 3e38 / (1 - 0.9)
        cv.adamw(plan, 0, 0.0, now=torch.tensor(now, device=DEV), status=status)
        assert status.item() == cv.DEV_NONFINITE
        assert torch.equal(t.param[0], start)
        status.zero_()
    t.param[0][7] = float("inf")
    if bits == 32:
        t.m[0][9], t.m[0][11], t.v[0][13] = float("nan"), -float("inf"), float("nan")
    else:
        t.m[0][9] = t.v[0][13] = 0x7F
        t.m[0][11] = 0xFF
    odd = [7, 9, 11, 13]
    start = t.param[0].clone()
    cv.adamw(plan, 5, 1e-3, status=status)
    others = [i for i in range(600) if i not in odd]
    assert status.item() == cv.DEV_NONFINITE and torch.equal(t.param[0][odd], start[odd])
    assert bool(torch.isfinite(t.param[0][others]).all()) and (t.param[0][others] != start[others]).float().mean() > 0.9
    t.param[0][7] = 1.0
    status.zero_()
    if bits == 8:                                                      # codes that stood for nothing do no longer
        cv.adamw(plan, 6, 1e-3, status=status)
        assert status.item() == 0


# ----------------------------------------------------------------------------- the loss over a vocabulary
@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n", [20, 80])
@pytest.mark.parametrize("weight,scale", [(1e32, 1.0), (3e36, -0.5), (1e-32, 1.0), (1e-36, -0.5), (1e-39, 1.0), (1e-44, 1.0)])
def test_linear_xent_of_weights_at_the_ends_of_fp32(dtype, n, weight, scale):
    """Whatever finite weights are, fp32 results are where fp32 has them; in fp16 dhidden of large ones is beyond the type."""
    x = Xent(n, 64, 300, dtype, F32, padding=0.0)
    x.weights = torch.full((n,), weight, device=DEV)
    x.weights[::3] *= 1e-3
    x.forward(scale)
    with_hidden = dtype != F16 or weight < 1
    x.backward(scale, dhidden=with_hidden)
    x.check(scale, dhidden=with_hidden)


@gpu
@pytest.mark.parametrize("dtype,dtable,n,dim,vocab,extra", [(BF16, F32, 70_001, 40, 300, 3), (F16, F16, 70_001, 40, 300, 0), (F32, F32, 66_000, 24, 130, 1),
                                                            (BF16, F32, 20_001, 1030, 2100, 0)])
def test_linear_xent_of_very_many_tokens(dtype, dtable, n, dim, vocab, extra):
    x = Xent(n, dim, vocab, dtype, dtable, extra)
    x.forward()
    x.backward()
    x.check()


PLANES = {("bf16", "bf16"): 2.0 ** -17, ("bf16", "f32"): 2.0 ** -17, ("f16", "f16"): 2.0 ** -23, ("f16", "f32"): 2.0 ** -23}


@gpu
@pytest.mark.parametrize("dtype,dtable", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("n,dim,vocab", [(18, 24, 57), (40, 24, 20_000), (263, 16, 9000), (4100, 16, 30)])
@pytest.mark.parametrize("alone", [False, True])
def test_linear_xent_dtable_of_entries_that_cancel(dtype, dtable, n, dim, vocab, alone):
    """A few words are most of the labels, and the hidden rows know them: a row of dtable is the difference of sums of many times
    its size.  Two planes round an entry of G by half a step of half a step of 16 bits."""
    x = Xent(n, dim, vocab, dtype, dtable, padding=0.0, weights=False)
    x.labels %= 3
    x.hidden.copy_((x.hidden.float() * 0.5 + 2.0 * x.table[x.labels].float()).to(dtype))
    x.forward()
    x.backward(dhidden=not alone)
    _, _, _, _, G, off_G, h, t = ref.linear_xent(f64(x.hidden), f64(x.table), x.labels.cpu().numpy())
    name = {F32: "f32", BF16: "bf16", F16: "f16"}
    _, _, want, off = ref.linear_xent_grad(G, off_G, h, t, 0.0, PLANES[name[dtype], name[dtable]])
    assert_near(x.dtable, want, off, dtable, "dtable")


@gpu
@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("vocab", [300, 7777, 20_001])
def test_linear_xent_dtable_in_fp32_of_few_bfloat16_rows(n, vocab):
    """Equal logits: an entry of G is 1 / vocab, whose bits two planes of bfloat16 do not hold, off by the division's rounding, the
    label's subtraction and the planes' 2^-26; a sum of 3 n products adds a rounding for each, and its scale one."""
    x = Xent(n, 40, vocab, BF16, F32, padding=0.0, weights=False)
    x.table.zero_()
    x.forward()
    x.backward(dhidden=False)
    G = np.full((n, vocab), 1.0 / vocab)
    G[np.arange(n), x.labels.cpu().numpy()] -= 1.0
    h = f64(x.hidden)
    tol = (8 + 3 * n) * ref.U * (np.abs(G).T @ np.abs(h))
    assert_near(x.dtable, G.T @ h, tol, F32, "dtable")
    two = torch.tensor(8192.0 / vocab, dtype=torch.float32)
    rest = two - two.bfloat16().float()
    assert abs((rest - rest.bfloat16().float()).item()) > 15 * ref.U * two.item()      # what two planes would have left


# ----------------------------------------------------------------------------- more than the caches hold
@gpu
@pytest.mark.parametrize("bits,grad,copy,by_chance,n", [(32, F32, None, False, 5_500_001), (32, BF16, F16, False, 6_500_003), (8, F32, BF16, True, 9_500_001),
                                                        (8, BF16, None, False, 11_000_007)])
def test_adamw_of_more_than_the_caches_hold(bits, grad, copy, by_chance, n):
    """Three tensors at odd addresses whose step goes past the caches' order, bit by bit as each of them by itself, where it does not."""
    g = torch.Generator(DEV).manual_seed(n)

    def new(dtype, make):
        flat = torch.zeros(n + 3, dtype=dtype, device=DEV)
        flat[3:] = make.to(dtype)
        return flat[3:]

    def averages():
        if bits == 32:
            return [new(F32, torch.randn(n, device=DEV, generator=g)), new(F32, torch.rand(n, device=DEV, generator=g) + 0.3), None]
        codes = [new(torch.uint8, torch.randint(0, 127, (n,), device=DEV, generator=g)) for _ in range(2)]
        return codes + [torch.rand(-(-n // 256), 2, device=DEV, generator=g) * 1e-2]

    def tensors():
        return [new(F32, torch.randn(n, device=DEV, generator=g)), new(grad, torch.randn(n, device=DEV, generator=g)), *averages(),
                new(copy, torch.zeros(n, device=DEV)) if copy is not None else None]

    def step(parts):
        lists = [list(x) for x in zip(*parts)]
        plan = cv.AdamwPlan(*lists[:4], scales=lists[4], copies=lists[5], weight_decays=[0.1] * len(parts), m_by_chance=by_chance)
        for t in (1, 2):
            cv.adamw(plan, t, 1e-2, seed=77)
        return plan.data.moved

    together = [tensors() for _ in range(3)]
    alone = [[None if t is None else t.clone() for t in x] for x in together]
    empty = [None if t is None else t[:0].clone() for t in alone[0]]   # keep the others' numbers, which their chances go by
    assert step(together) > 256_000_000
    for i, x in enumerate(alone):
        assert step([empty] * i + [x]) < 256_000_000
        for a, b in zip(together[i], x):
            assert a is None or torch.equal(a, b)


@gpu
@pytest.mark.parametrize("dtype,sequences,length,starts", [(BF16, 16, 2810, False), (F32, 8, 2750, False), (F16, 7, 45_000, True), (F32, 5, 22_000, True)])
def test_gated_scan_of_more_than_the_caches_hold(dtype, sequences, length, starts):
    """Every row once, and ranges, past the caches' order, rows at odd addresses: some channels against the formulas, no byte beside them."""
    dim = 1001
    rng = np.random.default_rng(3)
    lengths = [length] * sequences if not starts else np.diff([0, *np.sort(rng.integers(0, length, sequences - 1)), length]).tolist()
    at, bounds = cuts(lengths)
    n = int(at[-1])
    s = Scan(n, dim, dtype, sequences, extra=2, offset=1)
    assert n * dim * s.x.element_size() * 3 > 256_000_000
    cut = dict(starts=torch.from_numpy(at).to(DEV)) if starts else dict(sequences=sequences)
    s.forward(**cut)
    s.backward(**cut)
    some = [0, 1, 7, 8, 500, 993, 999, 1000]
    x, gate, dy, h = (f64(t[:, some]) for t in (s.x, s.gate, s.dy, s.h))
    h0, dlast = f64(s.h0[:, some]), f64(s.dlast[:, some])
    want, off, last, off_last = ref.gated_scan(x, gate, bounds, h0)
    assert_near(s.h[:, some], want, off, dtype, "h")
    assert_near(s.last[:, some], last, off_last, F32, "last")
    dx, off_x, dgate, off_g, dh0, off_0 = ref.gated_scan_grad(dy, x, gate, h, bounds, h0, dlast)
    assert_near(s.dx[:, some], dx, off_x, dtype, "dx")
    assert_near(s.dgate[:, some], dgate, off_g, dtype, "dgate")
    assert_near(s.dh0[:, some], dh0, off_0, F32, "dh0")
    for m, flat in ((s.h, s.h_flat), (s.dx, s.dx_flat), (s.dgate, s.dgate_flat)):
        assert bool(torch.isfinite(m).all()) and (m == 5.0).float().mean() < 1e-2      # every entry was written
        m[:] = 5.0
        assert bool((flat == 5.0).all())
