"""What a client trains its own model with: the AdamW step, the gated scan, the loss over a large vocabulary.

Against the same formulas in 64 bits (oracle/training.py, which also says how far fp32 arithmetic may be off), with half a
step of the output's type on top.
"""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2402_03770_amd.cvlc as cv
from oracle import training as ref
from test_local_step import BF16, DEV, F16, F32, assert_near, f64, matrix, random_matrix, tokens, untouched  # noqa: F401

gpu = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def refused(call, *args, **kw):
    with pytest.raises(cv.CvlcError) as e:
        call(*args, **kw)
    return e.value.code == cv.ERR_ARG


# ----------------------------------------------------------------------------- AdamW
class Tensors:
    """Tensors of some sizes, cut from flat buffers that begin `offset` elements in, with room behind that must stay as it is."""

    def __init__(self, sizes, bits, grad, copy, offset, seed, device=DEV):
        g = torch.Generator().manual_seed(seed)
        n, self.sizes, self.bits, self.flats = sum(sizes), sizes, bits, []
        spread = torch.exp(2.0 * torch.randn(n, generator=g))
        held = F32 if bits == 32 else torch.uint8

        def cut(dtype, make):
            flat = torch.zeros(offset + n + 16, dtype=dtype, device=device)
            flat[offset:offset + n] = make.to(dtype).to(device)
            self.flats.append((flat, offset + n))
            parts, at = [], offset
            for s in sizes:
                parts.append(flat[at:at + s])
                at += s
            return parts

        self.param = cut(F32, torch.randn(n, generator=g))
        self.grad = cut(grad, torch.randn(n, generator=g) * spread * 1e-2)
        self.scales = None
        if bits == 32:
            self.m = cut(F32, torch.randn(n, generator=g) * spread * 1e-2)
            self.v = cut(F32, (torch.rand(n, generator=g) + 0.3) * (spread * 1e-2) ** 2)
        else:
            self.m = cut(held, torch.randint(0, 127, (n,), generator=g) + 128 * torch.randint(0, 2, (n,), generator=g))
            self.v = cut(held, torch.randint(0, 127, (n,), generator=g))
            self.scales = [(torch.rand(-(-s // 256), 2, generator=g) * 1e-4).to(device) for s in sizes]
        self.copy = cut(copy, torch.zeros(n)) if copy is not None else None

    def plan(self, decays):
        return cv.AdamwPlan(self.param, self.grad, self.m, self.v, scales=self.scales, copies=self.copy, weight_decays=decays)

    def read(self, i):
        """A tensor's weights, gradient and averages in 64 bits."""
        m, v = self.m[i], self.v[i]
        if self.bits == 32:
            return f64(self.param[i]), f64(self.grad[i]), f64(m), f64(v)
        scale = ref.spread(f64(self.scales[i]), m.numel())
        return f64(self.param[i]), f64(self.grad[i]), ref.values(m.cpu()) * scale[:, 0], (ref.values(v.cpu()) * scale[:, 1]) ** 2


def check_adamw(t, before, decays, step, lr, betas, eps, grad_scale=1.0, seed=0, copy=None):
    for i, (old, decay) in enumerate(zip(before, decays)):
        p, off_p, m, off_m, v, off_v, root, off_root, fine = ref.adamw(*old, step, lr, betas, eps, decay, grad_scale, t.bits == 8)
        assert_near(t.param[i], p, off_p, F32, f"weights {i}")
        if t.copy is not None:
            assert torch.equal(t.copy[i], t.param[i].to(copy)), f"copy {i}"
        if t.bits == 32:
            assert_near(t.m[i], m, off_m, F32, f"m {i}")
            assert_near(t.v[i], v, off_v, F32, f"v {i}")
            continue
        scales = f64(t.scales[i])
        for k, (x, off) in enumerate(((m, off_m), (root, off_root))):
            want, tol = ref.scales_of(x, off)
            assert np.all(np.abs(scales[:, k] - want) <= tol + 2.0 ** -149), f"scales {i}"
            top = np.repeat(scales[:, k], ref.BLOCK)[:x.size]
            rel = np.where(np.abs(x) > 0, off / np.maximum(np.abs(x), 1e-300), 0.0) + 6 * ref.U
            with np.errstate(divide="ignore", invalid="ignore"):
                y = np.where(top > 0, np.abs(x) / top, 0.0)
            codes = (t.m if k == 0 else t.v)[i].view(torch.uint8).cpu().numpy().astype(np.int64)
            if k == 0:
                low, high = (ref.nearest(np.minimum(y * (1 + s * rel), 448.0)) for s in (-1, 1))
                assert np.all((codes & 127 == 0) | ((codes >= 128) == (x < 0))), f"signs of m {i}"
            else:
                chance = ref.chances(x.size, seed, step, i)
                # beyond the values' own error a step of 2^-9 and its chance have a rounding in the sum of up to 8
                low, high = (ref.by_chance(np.minimum(y * (1 + s * rel), 448.0), np.clip(chance + s * 2.0 ** -4, 0, 65535.9375)) for s in (-1, 1))
                assert np.all(codes < 128)
            assert np.all((low <= codes & 127) & (codes & 127 <= high)), f"codes {k} of {i}"
            assert np.sum(low != high) <= 1 + 0.02 * x.size                 # the borders leave nearly all of them no choice


SIZES = [[1], [255, 256, 257], [7, 0, 513, 1, 2048, 30], [8192, 8193, 20000]]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad,copy", [(F32, None), (BF16, BF16), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_adamw(bits, grad, copy, sizes):
    t = Tensors(sizes, bits, grad, copy, offset=3, seed=len(sizes) + bits)
    decays = [0.1 * (i % 3) for i in range(len(sizes))]
    plan = t.plan(decays)
    for step in (1, 2, 1000):                                          # one after the other, on what the one before left
        before = [t.read(i) for i in range(len(sizes))]
        cv.adamw(plan, step, 1e-2, betas=(0.9, 0.999), eps=1e-8, grad_scale=0.7, seed=2 ** 40 + 5)
        check_adamw(t, before, decays, step, 1e-2, (0.9, 0.999), 1e-8, 0.7, 2 ** 40 + 5, copy)
    for flat, end in t.flats:
        assert not bool(flat[:3].float().any()) and not bool(flat[end:].float().any())


@gpu
def test_adamw_of_many_tensors_and_both_widths():
    """More tensors than one launch lays out; averages of 8 and of 32 bits, gradients of all types in one step."""
    kinds = [Tensors([1 + 37 * (i % 11)] * 30, bits, grad, copy, offset=i, seed=i)
             for i, (bits, grad, copy) in enumerate([(8, F32, None), (32, BF16, F16), (8, F16, BF16), (32, F32, None), (8, BF16, None)])]
    lists = [[], [], [], [], [], []]
    for t in kinds:
        for out, part in zip(lists, (t.param, t.grad, t.m, t.v, t.scales or [None] * 30, t.copy or [None] * 30)):
            out += part
    decays = [0.01 * i for i in range(150)]
    plan = cv.AdamwPlan(*lists[:4], scales=lists[4], copies=lists[5], weight_decays=decays)
    before = [[t.read(i) for i in range(30)] for t in kinds]
    cv.adamw(plan, 3, 1e-3, seed=9)
    for k, t in enumerate(kinds):
        if t.bits == 32:
            check_adamw(t, before[k], decays[30 * k:30 * k + 30], 3, 1e-3, (0.9, 0.999), 1e-8, copy=F16)
        else:                                                          # the counter holds the tensor's number in the plan
            chances = ref.chances
            try:
                ref.chances = lambda n, seed, step, tensor, k=k: chances(n, seed, step, 30 * k + tensor)
                check_adamw(t, before[k], decays[30 * k:30 * k + 30], 3, 1e-3, (0.9, 0.999), 1e-8, seed=9, copy=BF16)
            finally:
                ref.chances = chances


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zeros_and_gradients_that_are_not_numbers(bits):
    """All averages zero, half of the gradients too; NaN, infinities and squares beyond fp32 leave their elements alone."""
    t = Tensors([700, 300], bits, F32, None, offset=0, seed=4)
    for part in (*t.m, *t.v, *(t.scales or [])):
        part.zero_()
    t.grad[0][::2] = 0.0
    t.grad[1].zero_()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30], device=DEV)
    t.grad[0][40:44] = bad
    before, status = [t.read(i) for i in range(2)], torch.zeros(1, dtype=torch.int32, device=DEV)
    cv.adamw(t.plan([0.0, 0.1]), 1, 0.1, status=status)
    assert status.item() == cv.DEV_NONFINITE
    check_adamw(t, before, [0.0, 0.1], 1, 0.1, (0.9, 0.999), 1e-8)
    assert np.array_equal(f64(t.param[0])[40:44], before[0][0][40:44]) and not t.m[1].view(torch.uint8).any()
    status.zero_()
    t.grad[0][40:44] = 1.0
    cv.adamw(t.plan([0.0, 0.1]), 2, 0.1, status=status)
    assert status.item() == 0


@gpu
def test_adamw_8bit_roots_move_on_average():
    """A gradient that is a third smaller than the average remembers: sqrt v must come down, by less than a code a step."""
    n = 256 * 64
    t = Tensors([n], 8, F32, None, offset=0, seed=1)
    t.m[0].zero_()
    t.v[0].fill_(0x60)
    t.v[0][::256] = 0x7E                                               # the blocks' largest, which holds the scale where it is
    t.scales[0].fill_(1.0)
    held = float(ref.values([0x60])[0])
    t.grad[0].fill_(held * 2 / 3)
    t.grad[0][::256] = 448.0
    plan, want = t.plan([0.0]), held ** 2
    for step in range(100, 200):
        cv.adamw(plan, step, 0.0, betas=(0.9, 0.99), seed=3)
        want = 0.99 * want + 0.01 * (held * 2 / 3) ** 2
    scale = ref.spread(f64(t.scales[0]), n)[:, 1]
    got = (ref.values(t.v[0].cpu()) * scale).reshape(-1, 256)[:, 1:]
    # A step takes r at most (1 - 0.99) / 2 (r^2 - g^2) / r < 0.0028 of `held` away from a code, so it jumps by a gap (an eighth
    # of `held` at most) with the probability of that over the gap: 100 steps add a variance of at most 0.28 / 8 = 0.035.
    # v is the mean of r^2, so the mean of r may be off its root by 0.035 / (2 * 0.8) either way, and 6 deviations of the
    # mean of 16 320 values.
    assert abs(got.mean() - np.sqrt(want)) <= held * (0.022 + 6 * np.sqrt(0.035 / got.size))
    assert got.mean() < held * 0.95


@gpu
def test_adamw_replayed_reads_its_rates():
    """Captured with rates on the device, replayed three times with others between eager work, against the eager step."""
    t, same = (Tensors([1000, 24], 8, BF16, BF16, offset=1, seed=6) for _ in range(2))
    plan, other = t.plan([0.1, 0.0]), same.plan([0.1, 0.0])
    now = torch.tensor([1.0, 1e-2, 1.0], device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cv.adamw(plan, 0, 0.0, now=now, seed=7)
    torch.cuda.current_stream().wait_stream(side)
    cv.adamw(other, 1, 1e-2, seed=7)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cv.adamw(plan, 0, 0.0, now=now, seed=7)
        assert refused(t.plan, [0.1, 0.0])                             # plans are made before
    for step, lr, scale in ((2, 1e-2, 1.0), (3, 5e-3, 0.5), (4, 2e-3, 2.0)):
        now.copy_(torch.tensor([step, lr, scale]))
        graph.replay()
        cv.adamw(other, step, float(np.float32(lr)), grad_scale=scale, seed=7)
        torch.cuda.synchronize()
        for a, b in zip((*t.param, *t.m, *t.v, *t.scales, *t.copy), (*same.param, *same.m, *same.v, *same.scales, *same.copy)):
            assert torch.equal(a, b)


def test_adamw_refusals_on_the_host():
    """Through the C entry points; nothing is launched."""
    lib, ok = cv.lib(), 1 << 20

    def tensor(**kw):
        base = dict(n=100, param=ok, grad=ok + 4096, m=ok + 8192, v=ok + 16384, scales=ok + 32768, copy=None, grad_type=1, copy_type=0,
                    state_bits=8, weight_decay=0.0)
        return cv.AdamwTensor(*(base | kw).values())

    def plan(*tensors, ws=ok + (1 << 20), size=1 << 20, out=True):
        data = cv.AdamwPlanData()
        table = (cv.AdamwTensor * max(len(tensors), 1))(*tensors)
        return lib.cvlc_adamw_plan(len(tensors), table, ws, size, C.byref(data) if out else None, None)

    for kw in (dict(grad_type=3), dict(state_bits=16), dict(param=None), dict(param=ok + 2), dict(grad=ok + 4097), dict(m=None),
               dict(scales=None), dict(scales=ok + 32772), dict(copy=ok + 65536, copy_type=0), dict(weight_decay=float("nan")),
               dict(state_bits=32, m=ok + 8193), dict(n=(1 << 35) + 1), dict(grad=ok + 200), dict(v=ok + 8191 + 100), dict(copy=ok + 8100, copy_type=1)):
        assert plan(tensor(**kw)) == cv.ERR_ARG, kw
    assert plan(tensor(), tensor()) == cv.ERR_ARG                        # the same weights twice
    assert plan(tensor(), ws=None) == plan(tensor(), ws=ok + 128) == plan(tensor(), out=False) == cv.ERR_ARG
    assert plan(tensor(), size=256) == -4
    need = lib.cvlc_adamw_workspace_bytes(1, (cv.AdamwTensor * 1)(tensor()))
    assert plan(tensor(), size=need - 1) == -4
    empty = cv.AdamwPlanData()
    assert lib.cvlc_adamw_plan(0, None, ok, 1 << 20, C.byref(empty), None) == 0

    def step(data=None, now=None, status=None, **kw):
        rates = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0, step=1) | kw
        return lib.cvlc_adamw(C.byref(data or cv.AdamwPlanData(ok, 1, 0, 0)), C.byref(cv.AdamwRates(*rates.values())), now, 0, status, None)

    assert step() == 0                                                   # nothing to do
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=0.0), dict(eps=1e-60), dict(eps=float("inf")),
               dict(step=0), dict(lr=float("inf")), dict(grad_scale=float("nan")), dict(now=ok + 2), dict(status=ok + 1),
               dict(data=cv.AdamwPlanData(ok + 1, 1, 0, 0)), dict(data=cv.AdamwPlanData(ok, 1, 1 << 24, 0))):
        assert step(**kw) == cv.ERR_ARG, kw


def test_adamw_plans_are_refused():
    def t(n, dtype=F32):
        return torch.zeros(n, dtype=dtype)

    for args in (([t(4)], [t(4)], [t(4)], []), ([], [], [], []), ([t(4, BF16)], [t(4)], [t(4)], [t(4)]), ([t(4)], [t(5)], [t(4)], [t(4)]),
                 ([t(4)], [t(4)], [t(4, E4M3)], [t(4)]), ([t(4)], [t(4)], [t(4, E4M3)], [t(4, E4M3)]), ([t(8)[::2]], [t(4)], [t(4)], [t(4)]),
                 ([t(4)], [t(4)], [t(4)], [t(4)])):                         # the last: on no GPU
        assert refused(cv.AdamwPlan, *args)
    assert refused(cv.AdamwPlan, [t(4)], [t(4)], [t(4)], [t(4)], copies=[t(4)])
    assert refused(cv.AdamwPlan, [t(4)], [t(4)], [t(4)], [t(4)], scales=[t(2).view(1, 2)])


# ----------------------------------------------------------------------------- the gated scan
def cuts(lengths, before=0):
    starts = np.concatenate([[0], np.cumsum(lengths)]) + before
    return starts, list(zip(starts[:-1].tolist(), starts[1:].tolist()))


class Scan:
    def __init__(self, n, dim, dtype, sequences, extra=0, offset=0, seed=1, states=True):
        self.n, self.dim, self.dtype, self.extra, self.offset = n, dim, dtype, extra, offset
        self.x = random_matrix(n, dim, dtype, seed, extra, offset)
        self.gate = random_matrix(n, dim, dtype, seed + 1, extra, offset, scale=4.0, shift=1.0)
        self.dy = random_matrix(n, dim, dtype, seed + 2, extra, offset)
        g = torch.Generator().manual_seed(seed + 3)
        self.h0, self.dlast = (torch.randn(sequences, dim, generator=g).to(DEV) if states else None for _ in range(2))
        self.last, self.dh0 = (torch.full((sequences, dim), 7.0, device=DEV) if states else None for _ in range(2))
        self.h, self.h_flat = matrix(n, dim, dtype, extra, offset, fill=5.0)
        self.dx, self.dx_flat = matrix(n, dim, dtype, extra, offset, fill=5.0)
        self.dgate, self.dgate_flat = matrix(n, dim, dtype, extra, offset, fill=5.0)
        self.ws = cv.new_workspace(cv.gated_scan_workspace_bytes(n, dim, sequences), DEV)
        self.ws.fill_(0xFF)

    def forward(self, **cut):
        cv.gated_scan(self.x, self.gate, self.h, self.ws, h0=self.h0, last_out=self.last, **cut)

    def backward(self, **cut):
        cv.gated_scan_grad(self.dy, self.x, self.gate, self.h, self.dx, self.dgate, self.ws, h0=self.h0, dlast=self.dlast,
                           dh0_out=self.dh0, **cut)

    def check(self, bounds):
        opt = lambda t: None if t is None else f64(t)  # noqa: E731
        low, high = bounds[0][0], bounds[-1][1]
        h, off, last, off_last = ref.gated_scan(f64(self.x), f64(self.gate), bounds, opt(self.h0))
        assert_near(self.h[low:high], h[low:high], off[low:high], self.dtype, "h")
        dx, off_x, dgate, off_g, dh0, off_0 = ref.gated_scan_grad(f64(self.dy), f64(self.x), f64(self.gate), f64(self.h), bounds,
                                                                  opt(self.h0), opt(self.dlast))
        assert_near(self.dx[low:high], dx[low:high], off_x[low:high], self.dtype, "dx")
        assert_near(self.dgate[low:high], dgate[low:high], off_g[low:high], self.dtype, "dgate")
        if self.h0 is not None:
            assert_near(self.last, last, off_last, F32, "last")
            assert_near(self.dh0, dh0, off_0, F32, "dh0")
        for m, flat in ((self.h, self.h_flat), (self.dx, self.dx_flat), (self.dgate, self.dgate_flat)):
            m[low:high] = 5.0
            assert bool((flat == 5.0).all()), "something else was written"


LENGTHS = [[1], [0, 1, 0, 5, 0], [2, 3, 300, 1], [257, 0, 0, 256], [1] * 600, [0] * 700 + [40, 3], [1500]]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim,extra,offset", [(1, 0, 0), (7, 1, 1), (130, 3, 1), (64, 0, 0)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: f"{len(v)}of{sum(v)}")
def test_gated_scan(dtype, dim, extra, offset, lengths):
    """Sequences of any lengths, rows before and behind them that hold NaN and stay as they are."""
    n = sum(lengths) + 5
    starts, bounds = cuts(lengths, before=2)
    s = Scan(n, dim, dtype, len(lengths), extra, offset, states=dim != 64)
    for m in (s.x, s.gate, s.dy):
        m[:2] = float("nan")
        m[n - 3:] = float("nan")
    cut = dict(starts=torch.from_numpy(starts).to(torch.int32 if dim % 2 else torch.int64).to(DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    s.forward(**cut)
    s.backward(**cut)
    assert cut["status"].item() == 0
    s.check(bounds)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sequences,length,dim", [(1, 1, 5), (3, 1, 40), (1, 2500, 130), (2, 700, 1000), (300, 4, 16), (40, 300, 64), (1, 9000, 8), (5, 1025, 260)])
def test_gated_scan_of_equal_lengths(dtype, sequences, length, dim):
    s = Scan(sequences * length, dim, dtype, sequences, extra=2)
    s.forward(sequences=sequences)
    s.backward(sequences=sequences)
    _, bounds = cuts([length] * sequences)
    s.check(bounds)


@gpu
def test_gated_scan_cut_both_ways_agrees():
    """Offsets of equal lengths against the lengths alone: the same values up to the order of joining."""
    a, b = (Scan(8 * 600, 200, F32, 8) for _ in range(2))
    starts, bounds = cuts([600] * 8)
    a.forward(sequences=8)
    a.backward(sequences=8)
    b.forward(starts=torch.from_numpy(starts).to(DEV))
    b.backward(starts=torch.from_numpy(starts).to(DEV))
    a.check(bounds)
    b.check(bounds)


@gpu
def test_gated_scan_of_far_gates():
    """Gates that keep or replace everything, infinite ones too; a NaN reaches the rows behind it in its channel and sequence only."""
    n, dim = 600, 24
    s = Scan(2 * n, dim, F32, 2)
    s.gate[:, :8] = torch.linspace(-150.0, 150.0, 2 * n, device=DEV)[:, None]
    s.gate[:, 8], s.gate[:, 9] = float("inf"), -float("inf")
    s.x[100, 20] = float("nan")
    s.forward(sequences=2)
    h = s.h.clone()
    want, off, last, off_last = ref.gated_scan(f64(s.x), f64(s.gate), [(0, n), (n, 2 * n)], f64(s.h0))
    assert np.isnan(f64(h)[100:n, 20]).all() and np.isnan(want[100:n, 20]).all() and np.isnan(f64(h)).sum() == n - 100
    some = [c for c in range(dim) if c != 20]
    assert_near(h[:, some], want[:, some], off[:, some])
    assert_near(s.last[:, some], last[:, some], off_last[:, some])
    assert torch.equal(h[:n, 8], s.h0[0, 8].expand(n)) and torch.equal(h[:, 9], s.x[:, 9])


@gpu
def test_gated_scan_grad_against_differences():
    """The gradient of a random projection of all results, in the oracle's 64 bits, against central differences."""
    n, dim, bounds = 23, 3, [(0, 9), (9, 9), (9, 23)]
    s = Scan(n, dim, F32, 3)
    starts = torch.tensor([0, 9, 9, 23], device=DEV)
    s.forward(starts=starts)
    s.backward(starts=starts)
    x, gate, h0, dy, dlast = (f64(t) for t in (s.x, s.gate, s.h0, s.dy, s.dlast))

    def value(x, gate, h0):
        h, _, last, _ = ref.gated_scan(x, gate, bounds, h0)
        return (h * dy).sum() + (last * dlast).sum()

    rng = np.random.default_rng(3)
    for k, got in enumerate((s.dx, s.dgate, s.dh0)):
        way = rng.standard_normal(f64(got).shape)
        step, args = 1e-5, [x, gate, h0]
        ends = [value(*(a + sign * step * way if i == k else a for i, a in enumerate(args))) for sign in (1, -1)]
        want = (ends[0] - ends[1]) / (2 * step)
        # third derivatives of some tens times step^2, and fp32's error of every entry (h's rounding in dgate among it)
        assert abs((f64(got) * way).sum() - want) <= 1e-7 + 2e-6 * np.abs(f64(got) * way).sum()


@gpu
def test_gated_scan_offsets_that_do_not_go():
    """Descending, negative or too large ones are told of, and nothing outside the matrices is written."""
    for bad in ([0, 50, 40, 100], [-3, 50, 60, 100], [0, 50, 60, 1000], [2 ** 40, 0, 0, 0]):
        s = Scan(100, 20, BF16, 3)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        s.forward(starts=torch.tensor(bad, device=DEV), status=status)
        assert status.item() == cv.DEV_INDEX
        status.zero_()
        s.backward(starts=torch.tensor(bad, device=DEV), status=status)
        assert status.item() == cv.DEV_INDEX
        for m, flat in ((s.h, s.h_flat), (s.dx, s.dx_flat), (s.dgate, s.dgate_flat)):
            assert untouched(flat, m, 5.0)


@gpu
def test_gated_scan_without_rows():
    s = Scan(0, 12, F32, 4)
    s.forward(sequences=4)
    s.backward(starts=torch.zeros(5, dtype=torch.int64, device=DEV))
    assert torch.equal(s.last, s.h0) and torch.equal(s.dh0, s.dlast)
    s.h0 = s.dlast = None
    s.forward(starts=torch.zeros(5, dtype=torch.int64, device=DEV))
    s.backward(sequences=4)
    assert not s.last.any() and not s.dh0.any()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,dim,slots,extra", [(1, 1, 1, 0), (5, 7, 5, 1), (64, 130, 200, 3), (300, 2049, 301, 0)])
def test_gated_scan_step(dtype, n, dim, slots, extra):
    x, gate = random_matrix(n, dim, dtype, 1, extra, 1), random_matrix(n, dim, dtype, 2, extra, 1, scale=3.0)
    h, flat = matrix(n, dim, dtype, extra, 1, fill=5.0)
    g = torch.Generator().manual_seed(3)
    states, at = torch.randn(slots, dim, generator=g).to(DEV), torch.randperm(slots, generator=g)[:n]
    at[n // 2] = -1 if n > 1 else at[0]
    before, status = f64(states), torch.zeros(1, dtype=torch.int32, device=DEV)
    cv.gated_scan_step(x, gate, states, h, slots=at.to(torch.int32 if n % 2 else torch.int64).to(DEV), status=status)
    want_h, off_h, want, off = np.zeros((n, dim)), np.zeros((n, dim)), before.copy(), np.zeros((slots, dim))
    for i, slot in enumerate(at.tolist()):
        if slot >= 0:
            want_h[i:i + 1], off_h[i:i + 1], want[slot:slot + 1], off[slot:slot + 1] = ref.gated_scan(f64(x)[i:i + 1], f64(gate)[i:i + 1], [(0, 1)], before[slot:slot + 1])
    assert_near(h, want_h, off_h, dtype)
    assert_near(states, want, off)
    assert status.item() == 0 and untouched(flat, h, 5.0)


@gpu
def test_gated_scan_step_of_slots_that_do_not_go():
    """One that is not there and one that two rows name: zeros and a status; the first row that names a slot has it."""
    n, dim = 600, 20
    x, gate = random_matrix(n, dim, F32, 1), random_matrix(n, dim, F32, 2)
    at = torch.arange(n)
    at[3], at[599], at[400], at[401] = 1000, 7, 2 ** 40, -5
    states, h = torch.ones(1000, dim, device=DEV), torch.empty(n, dim, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    cv.gated_scan_step(x, gate, states, h, slots=at.to(DEV), status=status)
    assert status.item() == cv.DEV_INDEX
    live = [i for i in range(n) if i not in (3, 599, 400, 401)]
    want, off, _, _ = ref.gated_scan(f64(x[live]), f64(gate[live]), [(i, i + 1) for i in range(len(live))], np.ones((len(live), dim)))
    assert_near(h[live], want, off)
    assert not h[[3, 599, 400, 401]].any() and torch.equal(states[live], h[live])
    assert bool((states[[3, 400, 401, *range(600, 1000)]] == 1.0).all())
    cv.gated_scan_step(x, gate, states, h)                              # without slots: a row each, nothing told


@gpu
@pytest.mark.parametrize("dtype,n,dim", [(F32, 4097, 6), (BF16, 5003, 17), (F16, 70001, 3)])
def test_gated_scan_step_of_many_slots(dtype, n, dim):
    """Rows enough for their slots to be looked at several at a time; some named twice, near by and far off, some not there."""
    x, gate = random_matrix(n, dim, dtype, 1, 1, 1), random_matrix(n, dim, dtype, 2, 1, 1)
    at = torch.randperm(n, generator=torch.Generator().manual_seed(3))
    wrong = [4, 17, 31, 33, n - 2, n - 1]
    at[4], at[17], at[31], at[33], at[n - 2], at[n - 1], at[40] = at[3], at[16], n, at[0], at[n - 3], at[5], -1
    g = torch.Generator().manual_seed(4)
    states, status = torch.randn(n, dim, generator=g).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    before = f64(states)
    h, flat = matrix(n, dim, dtype, 1, 1, fill=5.0)
    cv.gated_scan_step(x, gate, states, h, slots=at.to(torch.int32 if dim == 6 else torch.int64).to(DEV), status=status)
    live = np.array([i for i in range(n) if i not in (*wrong, 40)])
    slots = at.numpy()[live]
    f, rest = ref.sigmoid(f64(gate)[live])
    want_h, off_h, want, off = np.zeros((n, dim)), np.zeros((n, dim)), before.copy(), np.zeros((n, dim))
    want_h[live] = f * before[slots] + rest * f64(x)[live]
    off_h[live] = 16 * ref.U * (f * np.abs(before[slots]) + rest * np.abs(f64(x)[live])) + 2.0 ** -126   # as a step of the scan
    want[slots], off[slots] = want_h[live], off_h[live]
    assert_near(h, want_h, off_h, dtype)
    assert_near(states, want, off)
    assert status.item() == cv.DEV_INDEX and untouched(flat, h, 5.0)


@gpu
def test_gated_scan_steps_walk_as_the_scan_does():
    n, dim = 40, 33
    s = Scan(3 * n, dim, F32, 3)
    s.forward(sequences=3)
    states, h = s.h0.clone(), torch.empty(3, dim, device=DEV)
    rows = torch.empty(3 * n, dim, device=DEV)
    for t in range(n):
        at = [t, n + t, 2 * n + t]
        cv.gated_scan_step(s.x[at], s.gate[at], states, h)
        rows[at] = h
    want, off, last, off_last = ref.gated_scan(f64(s.x), f64(s.gate), [(0, n), (n, 2 * n), (2 * n, 3 * n)], f64(s.h0))
    assert_near(rows, want, off)
    assert_near(states, last, off_last)


def test_gated_scan_refusals():
    def t(*shape, dtype=F32):
        return torch.zeros(*shape, dtype=dtype)

    x, ws = t(6, 4), torch.zeros(1 << 20, dtype=torch.uint8)
    good = dict(x=x, gate=x, h=x, workspace=ws)
    for kw in (dict(), dict(sequences=2, starts=t(3, dtype=torch.int64)), dict(sequences=4), dict(sequences=0), dict(sequences=-1), dict(starts=t(3)),
               dict(starts=t(0, dtype=torch.int32)), dict(sequences=2, gate=t(6, 5)), dict(sequences=2, h=t(6, 4, dtype=BF16)),
               dict(sequences=2, x=t(4, 6).t()), dict(sequences=2, h0=t(3, 4)), dict(sequences=2, last_out=t(2, 4, dtype=BF16)),
               dict(sequences=2, status=t(1)), dict(sequences=2)):           # the last: on no GPU
        assert refused(cv.gated_scan, **(good | kw)), kw
    good = dict(dy=x, x=x, gate=x, h=x, dx=x, dgate=x, workspace=ws)
    for kw in (dict(), dict(sequences=2, dgate=t(6, 4, dtype=F16)), dict(sequences=2, dlast=t(2, 5)), dict(sequences=2, dh0_out=t(6, 4)), dict(sequences=2)):
        assert refused(cv.gated_scan_grad, **(good | kw)), kw
    good = dict(x=x, gate=x, states=t(9, 4), h=x)
    for kw in (dict(states=t(9, 5)), dict(states=t(4)), dict(slots=t(5, dtype=torch.int64)), dict(slots=t(6)), dict(states=t(9, 4, dtype=BF16)), dict()):
        assert refused(cv.gated_scan_step, **(good | kw)), kw


def test_gated_scan_refusals_on_the_host():
    lib, ok = cv.lib(), 1 << 20
    need = lib.cvlc_gated_scan_workspace_bytes(6, 4, 2)

    def forward(**kw):
        a = dict(n=6, dim=4, x=ok, xs=4, gate=ok, gs=4, kind=0, count=2, starts=None, size=0, h0=None, h=ok, hs=4, last=None, ws=ok, bytes=need,
                 status=None) | kw
        return lib.cvlc_gated_scan(*a.values(), None)

    for kw in (dict(dim=0), dict(n=1 << 31), dict(kind=3), dict(xs=3), dict(gs=3), dict(hs=3), dict(x=None), dict(gate=ok + 2), dict(h=None), dict(count=4),
               dict(count=0), dict(starts=ok, size=2), dict(starts=ok + 4, size=8), dict(h0=ok + 2), dict(last=ok + 1), dict(ws=None), dict(ws=ok + 8),
               dict(status=ok + 2)):
        assert forward(**kw) == cv.ERR_ARG, kw
    assert forward(bytes=need - 1) == -4

    def backward(**kw):
        a = dict(n=6, dim=4, dy=ok, ys=4, x=ok, xs=4, gate=ok, gs=4, h=ok, hs=4, kind=1, count=2, starts=None, size=0, h0=None, dlast=None, dx=ok, dxs=4,
                 dgate=ok, dgs=4, dh0=None, ws=ok, bytes=need, status=None) | kw
        return lib.cvlc_gated_scan_grad(*a.values(), None)

    for kw in (dict(ys=3), dict(dxs=0), dict(dgs=3), dict(dy=None), dict(dx=ok + 1), dict(dgate=None), dict(dlast=ok + 2), dict(dh0=ok + 3), dict(kind=9)):
        assert backward(**kw) == cv.ERR_ARG, kw

    def step(**kw):
        a = dict(n=6, dim=4, x=ok, xs=4, gate=ok, gs=4, kind=0, slots=None, size=0, count=6, states=ok, h=ok, hs=4, status=None) | kw
        return lib.cvlc_gated_scan_step(*a.values(), None)

    for kw in (dict(dim=0), dict(count=5), dict(slots=ok, size=1), dict(slots=ok + 4, size=8), dict(states=None), dict(states=ok + 2), dict(x=None), dict(hs=2),
               dict(status=ok + 1)):
        assert step(**kw) == cv.ERR_ARG, kw
    assert step(n=0, x=None, gate=None, h=None, states=None) == 0


# ----------------------------------------------------------------------------- the loss over a vocabulary
NAMES = {F32: "f32", BF16: "bf16", F16: "f16"}


class Xent:
    def __init__(self, n, dim, vocab, dtype, dtable=None, extra=0, offset=0, weights=True, padding=0.2, seed=1, spread=2.0, kind=torch.int64):
        self.n, self.dim, self.vocab, self.dtype, self.dtable_type = n, dim, vocab, dtype, dtable or dtype
        self.hidden = random_matrix(n, dim, dtype, seed, extra, offset)
        self.table = random_matrix(vocab, dim, dtype, seed + 1, extra, offset, scale=spread * dim ** -0.5)
        self.labels = tokens(n, vocab, seed + 2, padding, kind).to(DEV)
        g = torch.Generator().manual_seed(seed + 3)
        self.weights = None
        if weights:
            self.weights = (torch.rand(n, generator=g) / n).to(DEV)
            self.weights[::7] = 0.0
        self.loss, self.stats = torch.full((n,), 7.0, device=DEV), torch.full((n, 2), 7.0, device=DEV)
        self.dhidden, self.dhidden_flat = matrix(n, dim, dtype, extra, offset, fill=5.0)
        self.dtable, self.dtable_flat = matrix(vocab, dim, self.dtable_type, extra, offset, fill=5.0)
        need = max(cv.linear_xent_workspace_bytes(n, vocab, dim, dtype), cv.linear_xent_grad_workspace_bytes(n, vocab, dim, dtype, self.dtable_type))
        self.ws = cv.new_workspace(need, DEV)
        self.ws.fill_(0xFF)                                            # NaN in every type
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def forward(self, scale=1.0):
        cv.linear_xent(self.hidden, self.table, self.labels, self.loss, self.ws, scale=scale, weights=self.weights, stats_out=self.stats, status=self.status)

    def backward(self, scale=1.0, accumulate=False, dhidden=True, dtable=True):
        cv.linear_xent_grad(self.hidden, self.table, self.labels, self.stats, self.dhidden if dhidden else None, self.dtable if dtable else None, self.ws,
                            scale=scale, weights=self.weights, accumulate=accumulate, status=self.status)

    def check(self, scale=1.0, start=None, dhidden=True, dtable=True):
        name, out = NAMES[self.dtype], NAMES[self.dtable_type]
        cut = 2.0 ** -22 if self.dtype == F32 else 0.0
        hidden = np.nan_to_num(f64(self.hidden)) * (self.labels.cpu().numpy() >= 0)[:, None]
        loss, tol, stats, stats_tol, G, off_G, h, t = ref.linear_xent(hidden, f64(self.table), self.labels.cpu().numpy(), scale,
                                                                      None if self.weights is None else f64(self.weights), cut)
        assert_near(self.loss, loss, tol, F32, "loss")
        assert_near(self.stats, stats, stats_tol, F32, "stats")
        dh, off_h, dt, off_t = ref.linear_xent_grad(G, off_G, h, t, ref.ROUNDS[name, name], ref.ROUNDS[name, out], cut, start)
        for on, m, flat, want, off, kind, what in ((dhidden, self.dhidden, self.dhidden_flat, dh, off_h, self.dtype, "dhidden"),
                                                   (dtable, self.dtable, self.dtable_flat, dt, off_t, self.dtable_type, "dtable")):
            if on:
                assert_near(m, want, off, kind, what)
                assert untouched(flat, m, 5.0), what
            else:
                assert bool((flat == 5.0).all()), what


XENT_TYPES = [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)]


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
@pytest.mark.parametrize("n,dim,vocab,extra,offset", [(1, 1, 1, 0, 0), (3, 5, 7, 1, 1), (64, 64, 1000, 0, 0), (33, 100, 300, 3, 1), (130, 128, 257, 8, 8),
                                                      (32, 65, 2049, 0, 0), (257, 192, 1030, 1, 1)])
def test_linear_xent(dtype, dtable, n, dim, vocab, extra, offset):
    x = Xent(n, dim, vocab, dtype, dtable, extra, offset, weights=n != 64, kind=torch.int32 if n % 2 else torch.int64)
    if n > 1:
        x.hidden[x.labels < 0] = float("nan")                          # padded rows may hold anything
    x.forward(0.7)
    x.backward(0.7)
    x.check(0.7)
    assert x.status.item() == 0


@gpu
@pytest.mark.parametrize("dtype,dtable,n,dim,vocab", [(BF16, F32, 2100, 128, 8000), (F16, F16, 100, 1536, 8200), (BF16, BF16, 3200, 4096, 300),
                                                      (F32, F32, 2000, 64, 20000), (F32, F32, 700, 300, 3000)])
def test_linear_xent_of_large_tiles_and_pieces(dtype, dtable, n, dim, vocab):
    """Sizes at which every product takes the large tiles, and at which the vocabulary goes in several pieces."""
    x = Xent(n, dim, vocab, dtype, dtable, weights=False)
    x.forward()
    x.backward()
    x.check()


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
def test_linear_xent_gradients_alone_and_added(dtype, dtable):
    x = Xent(90, 72, 500, dtype, dtable)
    x.forward()
    x.backward(dtable=False)
    x.check(dtable=False)
    x = Xent(90, 72, 500, dtype, dtable)
    x.forward()
    x.backward(dhidden=False)
    x.check(dhidden=False)
    start = f64(random_matrix(500, 72, dtable, 9, scale=1e-3))
    x.dtable.copy_(torch.from_numpy(start))
    x.dhidden.fill_(5.0)
    x.backward(accumulate=True, dhidden=False)
    x.check(dhidden=False, start=start)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("weight", [1e-30, 1e-6, 1e6, 1e25])
def test_linear_xent_of_far_weights(dtype, weight):
    """Weights far from 1, among them rows a millionth of the others: G is scaled, so all keep their bits."""
    x = Xent(80, 64, 300, dtype, F32, padding=0.0)
    x.weights = torch.full((80,), weight, device=DEV)
    x.weights[::3] *= 1e-6
    if dtype == F16:                                                   # dhidden of such weights is beyond its type
        x.weights *= min(1.0, 1e3 / weight) if weight > 1 else 1.0
    x.forward()
    x.backward()
    x.check()


@gpu
@pytest.mark.parametrize("n", [20, 150])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("what", ["no hidden", "no table", "scale 0", "scale -1.5", "no weight", "weights below 0", "far", "one label"])
def test_linear_xent_at_the_ends_of_what_is_allowed(n, dtype, what):
    x, scale = Xent(n, 64, 300, dtype, F32), {"scale 0": 0.0, "scale -1.5": -1.5}.get(what, 1.0)
    if what == "no hidden":
        x.hidden.zero_()
    elif what == "no table":
        x.table.zero_()
    elif what == "no weight":
        x.weights.zero_()
    elif what == "weights below 0":
        x.weights.neg_()
    elif what == "far":                                                # powers of two, and what the types hold
        far = 2.0 ** (10 if dtype == F16 else 90)
        x.hidden.mul_(far)
        x.table.mul_(1 / far if dtype != F16 else 2.0 ** -4)
        scale = 1.0 if dtype != F16 else 2.0 ** -6
    elif what == "one label":
        x.labels.fill_(7)
    x.forward(scale)
    x.backward(scale)
    if what == "no weight":
        assert not x.loss.any() and not x.dhidden.any() and not x.dtable.any()
    x.check(scale)


@gpu
def test_linear_xent_without_rows_or_loss():
    x = Xent(0, 16, 30, F32)
    x.forward()
    x.backward()
    assert not x.dtable.any() and untouched(x.dtable_flat, x.dtable, 5.0)
    x.dtable.fill_(3.0)
    x.backward(accumulate=True)
    assert bool((x.dtable == 3.0).all())
    x = Xent(20, 16, 30, BF16, F32)
    x.labels.fill_(-1)
    x.hidden.fill_(float("nan"))
    x.forward()
    x.backward()
    assert not x.loss.any() and not x.stats.any() and not x.dhidden.any() and not x.dtable.any()


@gpu
def test_linear_xent_labels_beyond_the_vocabulary():
    x = Xent(40, 24, 100, F32, weights=False)
    x.labels[3], x.labels[5] = 100, 2 ** 40
    x.forward()
    assert x.status.item() == cv.DEV_INDEX
    x.status.zero_()
    x.backward()
    assert x.status.item() == cv.DEV_INDEX
    x.labels[[3, 5]] = -1
    x.check()


@gpu
def test_linear_xent_grad_against_differences():
    """Gradients along a random way against central differences of the oracle's loss in 64 bits."""
    x = Xent(20, 12, 50, F32)
    x.forward()
    x.backward()
    rng = np.random.default_rng(5)
    args = [f64(x.hidden), f64(x.table)]
    for k, got in enumerate((x.dhidden, x.dtable)):
        way, step = rng.standard_normal(args[k].shape), 1e-4
        ends = [ref.linear_xent(*(a + sign * step * way if i == k else a for i, a in enumerate(args)), x.labels.cpu().numpy(), 1.0, f64(x.weights))[0].sum()
                for sign in (1, -1)]
        want = (ends[0] - ends[1]) / (2 * step)
        # a third derivative of some tens of logits cubed (weights add up to 1 at most) times step^2, and fp32's roundings
        assert abs((f64(got) * way).sum() - want) <= 1e-6 + 1e-5 * np.abs(f64(got) * way).sum()


@gpu
def test_linear_xent_repeats_its_bits():
    x = Xent(500, 200, 3001, BF16, F32)
    x.forward()
    x.backward()
    kept = [t.clone() for t in (x.loss, x.stats, x.dhidden, x.dtable)]
    for _ in range(3):
        x.ws.fill_(0xFF)
        x.forward()
        x.backward()
        assert all(torch.equal(a, b) for a, b in zip(kept, (x.loss, x.stats, x.dhidden, x.dtable)))


def test_linear_xent_refusals():
    def t(*shape, dtype=F32):
        return torch.zeros(*shape, dtype=dtype)

    h, table, labels, ws = t(6, 4), t(9, 4), t(6, dtype=torch.int64), torch.zeros(1 << 20, dtype=torch.uint8)
    good = dict(hidden=h, table=table, labels=labels, loss_out=t(6), workspace=ws)
    for kw in (dict(hidden=t(6)), dict(table=t(9, 5)), dict(table=t(9, 4, dtype=BF16)), dict(labels=t(6)), dict(labels=labels[:5]), dict(loss_out=t(5)),
               dict(weights=t(6, dtype=BF16)), dict(stats_out=t(6)), dict(status=t(1)), dict(hidden=t(4, 6).t()), dict()):   # the last: on no GPU
        assert refused(cv.linear_xent, **(good | kw)), kw
    good = dict(hidden=h, table=table, labels=labels, stats=t(6, 2), dhidden=t(6, 4), dtable=t(9, 4), workspace=ws)
    for kw in (dict(stats=t(6)), dict(dhidden=t(6, 4, dtype=F16)), dict(dtable=t(8, 4)), dict(dtable=t(9, 4, dtype=torch.float64)), dict()):
        assert refused(cv.linear_xent_grad, **(good | kw)), kw
    assert refused(cv.linear_xent_workspace_bytes, 6, 9, 4, torch.float64)


def test_linear_xent_refusals_on_the_host():
    lib, ok = cv.lib(), 1 << 20
    need = lib.cvlc_linear_xent_workspace_bytes(6, 9, 4, 1)

    def loss(**kw):
        a = dict(n=6, vocab=9, dim=4, h=ok, hs=4, t=ok, ts=4, kind=1, labels=ok, size=8, scale=1.0, w=None, loss=ok, stats=None, ws=ok, bytes=need, status=None) | kw
        return lib.cvlc_linear_xent(*a.values(), None)

    for kw in (dict(vocab=0), dict(dim=0), dict(dim=(1 << 20) + 1, hs=1 << 21, ts=1 << 21), dict(n=(1 << 22) + 1), dict(h=None), dict(h=ok + 1), dict(hs=3), dict(t=ok + 1),
               dict(ts=3), dict(kind=3), dict(labels=None), dict(labels=ok + 4), dict(size=2), dict(scale=float("nan")), dict(w=ok + 2), dict(loss=None),
               dict(loss=ok + 2), dict(stats=ok + 4), dict(ws=None), dict(ws=ok + 4), dict(status=ok + 2), dict(n=1 << 22, vocab=1 << 20)):
        assert loss(**kw) == cv.ERR_ARG, kw
    assert loss(bytes=need - 1) == -4
    assert loss(n=0, h=None, t=None, labels=None, loss=None) == 0
    need = lib.cvlc_linear_xent_grad_workspace_bytes(6, 9, 4, 1, 0)

    def grad(**kw):
        a = dict(n=6, vocab=9, dim=4, h=ok, hs=4, t=ok, ts=4, kind=1, labels=ok, size=4, scale=1.0, w=None, stats=ok, dh=ok, dhs=4, dt=ok, dtt=0, dts=4, flags=0,
                 ws=ok, bytes=need, status=None) | kw
        return lib.cvlc_linear_xent_grad(*a.values(), None)

    for kw in (dict(stats=None), dict(stats=ok + 4), dict(dh=None, dt=None), dict(dh=ok + 1), dict(dhs=3), dict(dt=ok + 2), dict(dtt=2), dict(dts=3), dict(flags=2),
               dict(kind=0, dtt=1)):
        assert grad(**kw) == cv.ERR_ARG, kw
    assert grad(bytes=need - 1) == -4
    assert grad(n=0, h=None, t=None, labels=None, stats=None, dt=None) == 0


@gpu
@pytest.mark.parametrize("dtype,dtable,n,dim,vocab", [(BF16, F32, 100, 4096, 40000), (F32, F32, 20, 2048, 40000), (F16, F16, 300, 6000, 30001)])
def test_linear_xent_of_several_pieces(dtype, dtable, n, dim, vocab):
    """Tables whose planes and gradients go through the workspace in several pieces, the last of them smaller."""
    each = dim * 2 * (2 if dtype == F32 else 1) + -(-n // 64) * 64 * 2 * (2 if dtable == F32 else 1)
    assert each * vocab > 320 << 20, "one piece"
    x = Xent(n, dim, vocab, dtype, dtable)
    x.forward()
    x.backward()
    x.check()


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
@pytest.mark.parametrize("n,dim,vocab,extra", [(3000, 40, 11, 1), (5001, 130, 300, 0), (4100, 24, 2000, 8)])
def test_linear_xent_of_many_tokens_and_few_words(dtype, dtable, n, dim, vocab, extra):
    """Where tokens are shared out among the table's gradients' workgroups, also added to what is there."""
    x = Xent(n, dim, vocab, dtype, dtable, extra)
    x.forward()
    x.backward()
    x.check()
    start = f64(random_matrix(vocab, dim, dtable, 9, scale=1e-3))
    x.dtable.copy_(torch.from_numpy(start))
    x.dhidden.fill_(5.0)
    x.backward(accumulate=True, dhidden=False)
    x.check(dhidden=False, start=start)


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
@pytest.mark.parametrize("n", [15, 16, 17, 32, 48, 64, 65])
@pytest.mark.parametrize("dim,vocab,extra,offset", [(577, 65, 2, 0), (1030, 191, 1, 1), (32, 64, 0, 0), (31, 63, 5, 3)])
def test_linear_xent_of_few_tokens(dtype, dtable, n, dim, vocab, extra, offset):
    """Up to 64 tokens and one more; K that ends inside a line, vocabularies that end inside 64 rows, rows at any address."""
    x = Xent(n, dim, vocab, dtype, dtable, extra, offset)
    x.hidden[x.labels < 0] = float("nan")
    x.forward(0.5)
    x.backward(0.5)
    x.check(0.5)


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
@pytest.mark.parametrize("n,vocab", [(128, 700), (129, 63), (128, 2048), (200, 1025), (256, 1024), (256, 1025), (257, 200)])
def test_linear_xent_of_a_few_times_64_tokens(dtype, dtable, n, vocab):
    x = Xent(n, 300, vocab, dtype, dtable, 1, 1)
    x.hidden[x.labels < 0] = float("nan")
    x.forward()
    x.backward()
    x.check()


@gpu
@pytest.mark.parametrize("dtype,dtable", XENT_TYPES)
@pytest.mark.parametrize("n", [32, 33, 64])
@pytest.mark.parametrize("dim,extra", [(128, 0), (128, 1)])
def test_linear_xent_of_few_tokens_and_many_words(dtype, dtable, n, dim, extra):
    """Where tables that tiles can read as they are, and others, go different ways."""
    x = Xent(n, dim, 16500, dtype, dtable, extra)
    x.forward()
    x.backward()
    x.check()


# ----------------------------------------------------------------------------- streams, graphs, together
@gpu
def test_training_on_a_side_stream_and_in_a_graph():
    """A step's forward and backward behind the kernels that make its inputs, on a stream of its own; then captured and
    replayed on fresh inputs, with the same step eager on the same buffers and workspaces in between."""
    n, dim, vocab = 300, 96, 2001
    starts = torch.tensor([0, 100, 100, 101, 300], dtype=torch.int32, device=DEV)
    x, gate, h, dh, dx, dgate = (torch.randn(n, dim, device=DEV, dtype=BF16) for _ in range(6))
    table, labels = random_matrix(vocab, dim, BF16, 5, scale=0.1), tokens(n, vocab, 6).to(DEV)
    loss, stats, dtable = torch.empty(n, device=DEV), torch.empty(n, 2, device=DEV), torch.empty(vocab, dim, device=DEV)
    h0, last, dh0 = torch.randn(4, dim, device=DEV), torch.empty(4, dim, device=DEV), torch.empty(4, dim, device=DEV)
    ws = cv.new_workspace(max(cv.gated_scan_workspace_bytes(n, dim, 4), cv.linear_xent_workspace_bytes(n, vocab, dim, BF16),
                              cv.linear_xent_grad_workspace_bytes(n, vocab, dim, BF16, F32)), DEV)   # calls in turn share it

    def step():
        cv.gated_scan(x, gate, h, ws, starts=starts, h0=h0, last_out=last)
        cv.linear_xent(h, table, labels, loss, ws, stats_out=stats)
        cv.linear_xent_grad(h, table, labels, stats, dh, dtable, ws)
        cv.gated_scan_grad(dh, x, gate, h, dx, dgate, ws, starts=starts, h0=h0, dlast=last, dh0_out=dh0)

    outs = (h, last, loss, stats, dh, dtable, dx, dgate, dh0)

    def wiped(call):
        for t in outs:
            t.fill_(3.0)
        ws.fill_(0xFF)
        call()
        torch.cuda.synchronize()
        return [t.clone() for t in outs]

    def equal(a, b):
        return all(torch.equal(p, q) for p, q in zip(a, b))

    want = wiped(step)

    def aside():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            table.mul_(2.0).mul_(0.5)
            step()
        torch.cuda.current_stream().wait_stream(side)

    assert equal(wiped(aside), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn(n, dim, generator=g))
        labels.copy_(tokens(n, vocab, 20 + seed))
        starts.copy_(torch.tensor([0, 7 * seed, 50, 299 - seed, 300], dtype=torch.int32))
        assert equal(wiped(graph.replay), wiped(step))


@gpu
def test_local_training_example():
    """The example's gradients against automatic differentiation of its loss in 64 bits, its single tokens against its
    scan, one step of AdamW from its gradients; then that it runs."""
    import math

    from examples import local_training as ex

    g = torch.Generator().manual_seed(3)
    vocab, dim, lengths = 150, 24, [20, 1, 33, 6]
    starts = torch.tensor([0, *np.cumsum(lengths)], dtype=torch.int32)
    n = sum(lengths)
    model = ex.Model(vocab, dim, DEV)
    flat = torch.randn(model.flat.numel(), generator=g) * 0.5
    model.flat.copy_(flat)
    ids = torch.randint(vocab, (n,), generator=g)
    ids[-2:] = -1
    client = ex.Client(model, ids.to(DEV), starts.to(DEV))
    client.model.flat.copy_(model.flat)
    loss = client.gradient()

    p = flat.double().requires_grad_()
    table, inp, gate, gamma, beta = ex.Model.parts(model, p)
    x = table[ids.clamp(min=0)] * math.sqrt(dim) * (ids >= 0).double()[:, None]
    c = x - x.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * gamma + beta
    u, f, rows = y @ inp, torch.sigmoid(y @ gate), []
    for low, high in zip(starts[:-1].tolist(), starts[1:].tolist()):
        state = torch.zeros(dim, dtype=torch.float64)
        for t in range(low, high):
            state = f[t] * state + (1 - f[t]) * u[t]
            rows.append(state)
    h = torch.stack(rows)
    labels = client.labels.cpu()
    want = torch.nn.functional.cross_entropy((h @ table.t())[labels >= 0], labels[labels >= 0])
    want.backward()
    # seven sums in a row, of 150 terms at most, each off by no more than its length times a rounding of its terms, which
    # cancel to a tenth of their size at worst
    slack = 7 * 150 * ref.U * 10
    assert loss.item() == pytest.approx(want.item(), rel=slack)
    assert torch.linalg.norm(client.grad.cpu().double() - p.grad) <= slack * torch.linalg.norm(p.grad)
    assert client.status.item() == 0

    # the first text again, a token at a time
    states, got = torch.zeros(1, dim, device=DEV), torch.empty(1, dim, device=DEV)
    for t in range(lengths[0]):
        cv.gated_scan_step(client.u[t:t + 1], client.f[t:t + 1], states, got)
        assert torch.linalg.norm(got - client.h[t:t + 1]) <= 20 * 16 * ref.U * torch.linalg.norm(client.u[:t + 1])

    # from no averages AdamW's first step is by the gradient's sign, almost: m / (1 - b1) over the root of v / (1 - b2), each
    # within a step of their 8 bits (which the step itself does not see: it takes the averages before they are rounded)
    before, grad = client.model.flat.clone(), client.grad.clone()
    cv.adamw(client.plan, 1, 1e-3, seed=5)
    decay = torch.cat([torch.full((q.numel(),), w) for q, w in zip(client.model.parts(before), [0.01] * 3 + [0.0] * 2)]).to(DEV)
    want = before.double() * (1 - 1e-3 * decay.double()) - 1e-3 * grad.double() / (grad.double().abs() + 1e-8)
    # an AdamW step's roundings: 16 of the move (b1, b2 and what they leave are fp32: 1 - 0.999 is off by 2^-14 of itself, but
    # v and its correction by the same), and two of the weight
    assert bool(((client.model.flat.double() - want).abs() <= 1e-3 * 2.0 ** -13 + 2 * ref.U * want.abs() + 2.0 ** -126).all())

    losses, text = ex.run(rounds=3, clients=2, steps=2, texts=4, length=20, vocab=300, dim=32, say=lambda line: None)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    assert text.shape == (8, 4) and bool(((text >= 0) & (text < 300)).all())
