"""What a client trains with, on inputs and sizes beside the ordinary: values that are not finite, sequences without rows, averages
over thousands of steps, calls that the caches do not hold.  Oracles as in test_training.py."""
import numpy as np
import pytest
import torch

import paper_2402_03770_amd.cvlc as cv
from test_local_step import BF16, DEV, F16, F32, f64
from test_training import Scan, cuts

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
