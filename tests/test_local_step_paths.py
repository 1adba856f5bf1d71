"""The local step's operators where one kernel takes over from another: bits of the smallest results, the largest calls,
places of one call in another's buffers.  Against the same formulas in 64 bits, as tests/test_local_step.py.
"""
import re

import numpy as np
import pytest
import torch

import paper_2402_03770_amd.cvlc as cv
from oracle import local_step as ref

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
gpu = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def uniform(rows, width, low, high, seed, dtype=F32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (low + (high - low) * torch.rand(rows, width, generator=g, device=DEV)).to(dtype)


def workspace(n, vocab):
    return cv.new_workspace(cv.distill_workspace_bytes(n, vocab), DEV)


# a wavefront per row, several, a row that the registers do not hold, one of few that is cut into parts
ROWS = [(300, 100), (40, 3001), (600, 20001), (520, 70001), (3, 100000)]


def both_gradients(logits, ids, values, T, weights=None, **more):
    """The gradient in the loss's pass, and alone from the kept statistics."""
    n, vocab = logits.shape
    fused, alone, stats, loss = torch.empty_like(logits), torch.empty_like(logits), torch.empty(n, 2, device=DEV), torch.empty(n, device=DEV)
    cv.distill(logits, ids, values, loss, workspace(n, vocab), temperature=T, weights=weights, dlogits=fused, stats_out=stats, **more)
    cv.distill_grad(logits, ids, values, stats, alone, temperature=T, weights=weights, **more)
    return fused, alone


@gpu
@pytest.mark.parametrize("n,vocab", ROWS)
@pytest.mark.parametrize("T,spread", [(1.0, 0.25), (2.0, 0.25), (0.5, 110.0)])
def test_distill_gradient_keeps_the_bits_of_fp32(n, vocab, T, spread):
    """Two unlisted places of a row differ by exp((z - z') / T) alone, whatever the row's sum: next to the maximum, and down
    to the smallest results."""
    logits = uniform(n, vocab, 0.0, spread * T, 1)
    logits[:, 0] = spread * T                                # the row's maximum
    ids, values = torch.full((n, 1), vocab - 1, dtype=torch.int32, device=DEV), torch.zeros(n, 1, device=DEV)
    some = [0, n // 2, n - 1]
    z = f64(logits[some])
    arg = (z - z[:, :1]) / T
    for got in both_gradients(logits, ids, values, T):
        g = f64(got[some])
        want = g[:, :1] * np.exp(arg)
        # (z - m), 1 / T and their product rounded, 1 ulp of the exponential, the product with the row's scale; the maximum's
        # own entry has the last two; a result below the normal ones is rounded to half the smallest
        tol = (3 * np.abs(arg) + 7) * ref.U * want + 2.0 ** -150
        assert np.all(np.abs(g - want)[:, :-1] <= tol[:, :-1]), float(((np.abs(g - want) - 2.0 ** -150) / want / ref.U)[:, :-1].max())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab", ROWS)
@pytest.mark.parametrize("weight", [1e-28, -1e-33, 3e-37])
def test_distill_gradient_of_tiny_weights(n, vocab, dtype, weight):
    """A weight scales the gradient and costs none of its bits, as long as the results are normal numbers."""
    logits = uniform(n, vocab, -2.0, 2.0, 2, dtype)
    ids = torch.tensor([[1, vocab - 1, 1]], dtype=torch.int64, device=DEV).expand(n, 3).contiguous()
    values = uniform(n, 3, 0.0, 2.0, 3)
    some = [0, n - 1]
    w = np.full(2, float(np.float32(weight)))
    want, tol = ref.distill(f64(logits[some]), ids[some].cpu().numpy(), f64(values[some]), T=1.0, weights=w)[4:]
    tol = tol + ref.half_step(np.abs(want) + tol, torch.finfo(dtype).eps, 2.0 ** -149 if dtype == F32 else 2.0 ** -133) + 2.0 ** -149
    # (a row's scale may lie below the normal numbers itself, and so may its product)
    for got in both_gradients(logits, ids, values, 1.0, weights=torch.full((n,), weight, device=DEV)):
        err = np.abs(f64(got[some]) - want)
        assert np.all(err <= tol), float((err / np.abs(want)).max())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab", ROWS)
def test_distill_gradient_of_a_tiny_share(n, vocab, dtype):
    """Log-probabilities whose sum P is tiny: P q keeps its bits at listed places and at the others."""
    logits = uniform(n, vocab, -2.0, 2.0, 4, dtype)
    ids = torch.tensor([[1, vocab - 1]], dtype=torch.int32, device=DEV).expand(n, 2).contiguous()
    values = torch.full((n, 2), -70.0, device=DEV)
    values[:, 1] = -80.0                                      # P is 4e-31: 1 / S and 2^-32 more would leave the normal range
    some = [0, n - 1]
    want, tol = ref.distill(f64(logits[some]), ids[some].cpu().numpy(), f64(values[some]), T=1.0, logprobs=True)[4:]
    tol = tol + ref.half_step(np.abs(want) + tol, torch.finfo(dtype).eps, 2.0 ** -149 if dtype == F32 else 2.0 ** -133)
    for got in both_gradients(logits, ids, values, 1.0, logprobs=True):
        err = np.abs(f64(got[some]) - want)
        assert np.all(err <= tol), float((err / np.abs(want)).max())


@gpu
@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("n,vocab", ROWS)
def test_distill_grad_in_place(n, vocab, dtype):
    """The gradient alone may take the logits' place: the same bits as beside them; rows without weight are zeros."""
    logits = uniform(n, vocab, -3.0, 3.0, 5, dtype)
    g = torch.Generator(device=DEV).manual_seed(6)
    # every part of a row has listed places, some of them listed twice
    ids = torch.randint(vocab, (n, 33), generator=g, device=DEV)
    ids[:, 20:] = ids[:, :13]
    values, weights = uniform(n, 33, 0.0, 3.0, 7), uniform(n, 1, 0.5, 1.0, 8)[:, 0].contiguous()
    weights[1] = 0.0
    stats, loss, beside = torch.empty(n, 2, device=DEV), torch.empty(n, device=DEV), torch.empty_like(logits)
    cv.distill(logits, ids, values, loss, workspace(n, vocab), temperature=1.5, weights=weights, stats_out=stats)
    cv.distill_grad(logits, ids, values, stats, beside, temperature=1.5, weights=weights)
    some = [0, 1, n - 1]
    want, tol = ref.distill(f64(logits[some]), ids[some].cpu().numpy(), f64(values[some]), T=1.5, weights=f64(weights[some]))[4:]
    cv.distill_grad(logits, ids, values, stats, logits, temperature=1.5, weights=weights)
    assert torch.equal(logits, beside)
    tol = tol + ref.half_step(np.abs(want) + tol, torch.finfo(dtype).eps, 2.0 ** -149 if dtype == F32 else 2.0 ** -24)
    assert np.all(np.abs(f64(logits[some]) - want) <= tol)
    assert not bool(logits[1].any())


def near(got, want, tol, dtype=F32):
    """Within `tol` and half a step of the type; equal where the value is infinite."""
    got = f64(got)
    fine = np.isfinite(want)
    assert got.shape == want.shape and np.array_equal(got[~fine], want[~fine], equal_nan=True)
    smallest = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}[dtype]
    tol = tol[fine] + ref.half_step(np.abs(want[fine]) + tol[fine], torch.finfo(dtype).eps, smallest)
    assert np.all(np.abs(got[fine] - want[fine]) <= tol), float((np.abs(got[fine] - want[fine]) - tol).max())


def spread_lists(n, vocab, k, seed):
    """Lists over the whole vocabulary, an eighth of whose entries repeat others."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(vocab, (n, k), generator=g, device=DEV, dtype=torch.int32)
    if k >= 8:
        ids[:, -(k // 8):] = ids[:, :k // 8]
    return ids, 3.0 * torch.randn(n, k, generator=g, device=DEV)


def check_all(logits, ids, values, T, some, weights=None):
    """Loss alone, gradient alone, both together, and both in place, at sampled rows."""
    n, vocab = logits.shape
    w = None if weights is None else f64(weights[some])
    loss, loss_tol, stats, stats_tol, grad, grad_tol = ref.distill(f64(logits[some]), ids[some].cpu().numpy(), f64(values[some]), T=T, weights=w)
    ws, got_loss, got_stats = workspace(n, vocab), torch.full((n,), 11.0, device=DEV), torch.full((n, 2), 11.0, device=DEV)
    ws.fill_(0xA5)
    cv.distill(logits, ids, values, got_loss, ws, temperature=T, weights=weights, stats_out=got_stats)
    near(got_loss[some], loss, loss_tol)
    near(got_stats[some], stats, stats_tol)
    d = torch.full_like(logits, 13.0)
    cv.distill_grad(logits, ids, values, got_stats, d, temperature=T, weights=weights)
    near(d[some], grad, grad_tol, logits.dtype)
    d.fill_(13.0)
    got_loss.fill_(11.0)
    cv.distill(logits, ids, values, got_loss, ws, temperature=T, weights=weights, dlogits=d)
    near(got_loss[some], loss, loss_tol)
    near(d[some], grad, grad_tol, logits.dtype)
    again = torch.empty_like(got_loss)
    cv.distill(logits, ids, values, again, ws, temperature=T, weights=weights, dlogits=logits)
    assert torch.equal(again, got_loss) and torch.equal(logits, d)


@gpu
@pytest.mark.parametrize("n,vocab,dtype", [(520, 70001, F32), (513, 262144, BF16), (1100, 140001, F16)])
def test_distill_of_many_rows_beyond_the_registers(n, vocab, dtype):
    """Rows that one workgroup goes over in passes; the larger two of them past the caches' order."""
    logits = uniform(n, vocab, -4.0, 4.0, 10, dtype)
    logits[:, vocab // 3] = float("-inf")
    ids, values = spread_lists(n, vocab, 70, 11)
    check_all(logits, ids, values, 1.5, [0, 1, n // 2, n - 1])


@gpu
@pytest.mark.parametrize("n,vocab,dtype", [(9000, 15003, BF16), (700_000, 100, F32), (70_000, 1000, F32), (1000, 66001, F32)])
def test_distill_of_more_than_the_caches_hold(n, vocab, dtype):
    """Short rows and long ones, read and written past the caches' order."""
    logits = uniform(n, vocab, -4.0, 4.0, 12, dtype)
    ids, values = spread_lists(n, vocab, 9, 13)
    check_all(logits, ids, values, 2.0, [0, 1, 4095, n // 2, n - 2, n - 1] if n > 4095 else [0, 1, n - 1])


@gpu
@pytest.mark.parametrize("k", [681, 682, 683, 1000, 1024])
@pytest.mark.parametrize("n,vocab", [(700, 62), (300, 900), (2000, 1030), (30, 5000)])
def test_distill_of_long_lists_on_short_rows(n, vocab, k):
    """Four rows' lists to a workgroup, in up to 96 KB of LDS."""
    logits = uniform(n, vocab, -4.0, 4.0, 14, BF16)
    ids, values = spread_lists(n, vocab, k, 15)
    check_all(logits, ids, values, 2.0, [0, 1, 2, 3, n - 2, n - 1])


@gpu
@pytest.mark.parametrize("n,vocab", ROWS)
def test_distill_reads_nothing_of_rows_without_weight(n, vocab):
    """Logits, lists and statistics of such rows hold NaN and numbers beyond the vocabulary: zeros, and no bit of the status."""
    logits = uniform(n, vocab, -4.0, 4.0, 16, BF16)
    ids, values = spread_lists(n, vocab, 12, 17)
    weights = torch.ones(n, device=DEV)
    weights[::3] = 0.0
    lost = weights == 0.0
    logits[lost], values[lost], ids[lost] = float("nan"), float("nan"), 1 << 30
    status, ws = torch.zeros(1, dtype=torch.int32, device=DEV), workspace(n, vocab)
    loss, stats = torch.full((n,), 11.0, device=DEV), torch.full((n, 2), 11.0, device=DEV)
    cv.distill(logits, ids, values, loss, ws, weights=weights, stats_out=stats, status=status)
    stats_lost = stats[lost].clone()
    stats[lost] = float("nan")
    alone, fused, loss2 = torch.full_like(logits, 13.0), torch.full_like(logits, 13.0), torch.full((n,), 11.0, device=DEV)
    cv.distill_grad(logits, ids, values, stats, alone, weights=weights, status=status)
    cv.distill(logits, ids, values, loss2, ws, weights=weights, dlogits=fused, status=status)
    for zeros in (loss[lost], loss2[lost], stats_lost, alone[lost], fused[lost]):
        assert not bool(zeros.any())
    assert status.item() == 0
    some = [1, 2] + ([n - 2] if (n - 2) % 3 else [])
    want = ref.distill(f64(logits[some]), ids[some].cpu().numpy(), f64(values[some]))
    near(loss[some], want[0], want[1])
    near(loss2[some], want[0], want[1])
    near(alone[some], want[4], want[5], BF16)
    near(fused[some], want[4], want[5], BF16)


# ----------------------------------------------------------------------------- embedding
def text(n, vocab, seed, beyond=0):
    """Tokens of which the low ones are frequent, a tenth padding, `beyond` of them beyond the vocabulary."""
    rng = np.random.default_rng(seed)
    ids = np.minimum((np.exp(rng.random(n) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1)
    ids[rng.random(n) < 0.1] = -1
    ids[rng.choice(n, beyond, replace=False)] = vocab
    ids[0] = ids[n // 2] = ids[n - 1] = vocab - 1             # the last digit's largest value, from several tiles
    return torch.from_numpy(ids).to(DEV)


def check_embed_grad(ids, dout, vocab, scale, status, start=None):
    """Against sums in 64 bits on the GPU; twice, bit for bit."""
    n, dim = dout.shape
    ws = cv.new_workspace(cv.embed_grad_workspace_bytes(n, vocab, dim), DEV)
    got = []
    for _ in range(2):
        ws.fill_(0xA5)
        dtable = torch.full((vocab, dim), 5.0, device=DEV) if start is None else start.clone()
        cv.embed_grad(ids, dout, dtable, ws, scale=scale, accumulate=start is not None)
        assert cv.device_status(ws) == status
        got.append(dtable)
    assert torch.equal(*got)
    del got
    there = (ids >= 0) & (ids < vocab)
    rows, where = torch.unique(ids[there], return_inverse=True)
    want, size = torch.zeros(2, rows.numel(), dim, dtype=torch.float64, device=DEV)
    part = max(1, (1 << 26) // dim)                           # rows at a time
    places = torch.nonzero(there)[:, 0]
    for b in range(0, places.numel(), part):
        d = dout[places[b:b + part]].double()
        want.index_add_(0, where[b:b + part], d)
        size.index_add_(0, where[b:b + part], d.abs())
    count = torch.bincount(where, minlength=rows.numel())[:, None]
    want, tol = want * scale, (count + 3) * ref.U * size * abs(scale)
    if start is not None:
        want += start[rows].double()
        tol += want.abs() * ref.U
    assert bool(((dtable[rows].double() - want).abs() <= tol + 2.0 ** -149).all())
    rest = torch.ones(vocab, dtype=torch.bool, device=DEV)
    rest[rows] = False
    untouched = dtable[rest]
    assert torch.equal(untouched, start[rest]) if start is not None else not bool(untouched.any())


@gpu
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,dim,vocab", [(20_000, 3, 5_000_000), (40_000, 9, 4_194_303), (40_000, 9, 4_194_304), (300_000, 7, 50_000),
                                         (270_000, 2, 6_000_000), (17_000, 40, 2_000)])
def test_embed_grad_by_every_number_of_digits(n, dim, vocab, add):
    """One, two and three passes of the sort over several tiles; tiles counted by every workgroup for itself and, more than
    64 of them, by a scan between the passes."""
    g = torch.Generator(device=DEV).manual_seed(20)
    dout = torch.randn(n, dim, generator=g, device=DEV).to(BF16)
    start = torch.randn(vocab, dim, generator=g, device=DEV) if add else None
    check_embed_grad(text(n, vocab, 21, beyond=5), dout, vocab, 0.5, cv.DEV_INDEX, start)


@gpu
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,dim,dtype", [(70_000, 1000, F32), (100_001, 1300, BF16), (33_000, 4099, F16)])
def test_embed_grad_of_more_than_the_caches_hold(n, dim, dtype, add):
    """Rows read past the caches' order."""
    g = torch.Generator(device=DEV).manual_seed(22)
    dout = torch.randn(n, dim, generator=g, device=DEV).to(dtype)
    vocab = 9000
    start = torch.randn(vocab, dim, generator=g, device=DEV) if add else None
    check_embed_grad(text(n, vocab, 23), dout, vocab, 2.0, 0, start)


@gpu
@pytest.mark.parametrize("n", [4096, 16384, 16385])
@pytest.mark.parametrize("share", [0.5, 1.0])
@pytest.mark.parametrize("add", [False, True])
def test_embed_grad_of_one_token_above_all(n, share, add):
    """A padding or separator token that is a row like any other, for half of the places and for all of them."""
    g = torch.Generator(device=DEV).manual_seed(24)
    vocab, dim = 3000, 256
    dout = torch.randn(n, dim, generator=g, device=DEV).to(BF16)
    ids = text(n, vocab, 25)
    ids[torch.rand(n, generator=g, device=DEV) < share] = 11
    start = torch.randn(vocab, dim, generator=g, device=DEV) if add else None
    check_embed_grad(ids, dout, vocab, 1.0, 0, start)


@gpu
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("n,dim", [(300_001, 100), (70_001, 240), (2_200_003, 5)])
def test_embed_of_four_rows_to_a_thread(types, n, dim):
    """More than 8192 workgroups of several rows each; the last ones have fewer."""
    tt, to = types
    vocab, scale = 500, 1.5
    g = torch.Generator(device=DEV).manual_seed(26)
    table = torch.randn(vocab, dim, generator=g, device=DEV).to(tt)
    ids = text(n, vocab, 27, beyond=3)
    flat = torch.full((n * (dim + 1) + 8,), 3.0, dtype=to, device=DEV)
    out = flat[:n * (dim + 1)].view(n, dim + 1)[:, :dim]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    cv.embed(ids.int(), table, out, scale=scale, status=status)
    there = (ids >= 0) & (ids < vocab)
    want = torch.where(there[:, None], table[ids.clamp(0, vocab - 1)].float() * scale, 0.0).to(to)
    assert torch.equal(out, want) and status.item() == cv.DEV_INDEX
    out.fill_(3.0)
    assert bool((flat == 3.0).all())


# ----------------------------------------------------------------------------- layer norm
def test_norm_shapes_are_those_that_calls_reach():
    """Rows of 16384 values are the longest in registers: 4 accesses for each of 1024 threads where an access holds four
    values.  Where it holds eight (both types of 16 bits) no call takes that shape, so the library holds no kernel of it."""
    with open(cv.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"norm_(?:grad_)?rows_kernelI\w+?RowShapeILj16ELj4E", f.read()))
    assert any(b"kernelIff" in n for n in names)
    assert not [n for n in names if not n.split(b"kernelI")[1].startswith(b"f")], names


@gpu
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("n", [8191, 8192, 16383, 16384])
def test_layer_norm_by_one_wavefront_and_by_more(types, n):
    """One side and the other of the numbers of rows from which a wavefront has a row to itself; sampled rows, all of y."""
    tx, ty = types
    dim = 1301 if tx == F32 else 2603                        # 326 accesses; half of it has 163
    for width in (dim, dim // 2):
        x = 3.0 + 2.0 * uniform(n, width, -1.0, 1.0, 30).to(tx)
        gamma, beta = uniform(2, width, 0.5, 1.5, 31)
        y, stats = torch.full((n, width), 7.0, dtype=ty, device=DEV), torch.empty(n, 2, device=DEV)
        cv.layer_norm(x, gamma, beta, y, stats)
        some = [0, 1, 2, 3, n // 2, n - 2, n - 1]
        want, tol, s, s_tol = ref.layer_norm(f64(x[some]), f64(gamma), f64(beta), 1e-5)
        near(stats[some], s, s_tol)
        near(y[some], want, tol, ty)
        h = (x.double() - stats[:, :1].double()) * stats[:, 1:].double() * gamma.double() + beta.double()
        # from the statistics as they are: the difference, two products and a sum rounded, then the type
        tol = 4 * ref.U * (h.abs() + beta.abs().double()) + h.abs() * (torch.finfo(ty).eps / 2) * 1.001 + 2.0 ** -149
        assert bool(((y.double() - h).abs() <= tol).all())
