"""The bounds that the decays' gradient is held to on the GPU (test_gpu_attend_decays.py), looked at on the host: the way it is put together gives the
gradient, and what a mistake in it would give lies far outside."""
import numpy as np
import pytest

import decay_ref as D
import mixer_ref as R

CASES = [([2300], True, True), ([2300], False, True), ([37, 2100, 1100], True, False), ([1100, 1100], False, False), ([70, 5, 200], True, True)]


@pytest.mark.parametrize("lengths,rows,slow", CASES)
def test_mistakes_lie_outside(lengths, rows, slow):
    H = 2
    q, k, v, decay, h0, dy, dlast, off = D.inputs(lengths, H, 1, 8, 12, rows, 3, slow)
    N = q.shape[0]
    args = (q, k, v, np.broadcast_to(decay, (N, H)), R.spans(N, len(lengths), off), h0, 0.25, dy, dlast)
    want = R.attend(*args)["dg"]
    row, total = D.bounds(*args)
    assert (np.abs(D.assembled(*args) - want) <= 1e-3 * row + 1e-300).all()
    chunks = -(-max(lengths) // D.CHUNK)
    # what a call with a mistake would give in place of the gradient; a sum over all rows may hide part of it, not all
    wrong = [np.zeros_like(want)] + [D.assembled(*args, lost=(n,)) for n in {0, 1, chunks // 2, chunks - 1, "end"}]
    for i, w in enumerate(wrong):
        off_by = np.abs(w - want)
        assert off_by.max() > 100 * row[np.unravel_index(off_by.argmax(), row.shape)], i
        assert (np.abs((w - want).sum(0)) > 2 * total).any(), i
    assert (np.abs(want.sum(0)) > 5 * total).all()
    few = np.abs(want) <= row                       # zeros pass for few rows alone (that forget everything)
    assert few.mean() < 0.02
