"""The local step's operators where one kernel takes over from another: bits of the smallest results, the largest calls,
places of one call in another's buffers.  Against the same formulas in 64 bits, as tests/test_local_step.py.
"""
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
