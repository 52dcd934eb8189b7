"""The bounds that hold the documented precision of linear attention (64-bit sums of log decays, three BF16 parts of what stays
in the state) pass it and fail less, in the oracle."""
import numpy as np
import pytest

from tests import linear_chunks as L
from tests import linear_ref as R


def _frobenius(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("n", [1, 64, 65, 200])
def test_chunks_agree_with_the_definition(n):
    q, k, v, g, start = L.inputs(n, 2, n, L.mild(n, 2))
    ref, s, oa, sa = R.linear(q, k, v, g, start, 0.1)
    out, state = L.linear(q, k, v, g, start, 0.1)
    R.check_out(out, ref, oa, n, g, "outputs")
    R.check_state(state, s, sa, n, g, "state")


def test_sums_of_decays():
    """A chunk that clears the state and then keeps it tells 64-bit sums from 32-bit ones."""
    q, k, v, g, start = L.inputs(64, 1, 1, L.cleared, start=False)
    ref, s, oa, sa = R.linear(q, k, v, g, start, 0.1)
    out, state = L.linear(q, k, v, g, start, 0.1)
    R.check_out(out, ref, oa, 64, g, "outputs")
    R.check_state(state, s, sa, 64, g, "state")
    _, state = L.linear(q, k, v, g, start, 0.1, sums=np.float32)
    with pytest.raises(AssertionError, match="state"):
        R.check_state(state, s, sa, 64, g, "state")


@pytest.mark.parametrize("n", [64, 130, 300])
def test_parts_of_the_state(n):
    """Three BF16 parts keep the state's norm to FP32's own error, two do not."""
    q, k, v, g, start = L.inputs(n, 2, n, L.mild(n, 2), start=False)
    s = R.linear(q, k, v, g, start, 0.1)[1]
    assert _frobenius(L.linear(q, k, v, g, start, 0.1)[1], s) < L.FROBENIUS
    assert _frobenius(L.linear(q, k, v, g, start, 0.1, parts=2)[1], s) > 2 * L.FROBENIUS
