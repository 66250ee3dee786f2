"""8-bit inputs of the token operators start at any byte: what the argument checks let through (no GPU needed)."""
import pytest

import test_token_refusals as R
from test_token_refusals import P  # noqa: F401  (a fixture)


@pytest.mark.parametrize("off", range(1, 5))
def test_an_8_bit_input_may_start_at_any_byte(P, off):
    x = dict(x=R.AT + off, x_scales=R.AT + off)
    assert P.linear_workspace(R.linear(P, ldxs=1, **x)) >= 4 * 16 * 2                 # room for the rows that it is read back into
    assert P.linear_workspace(R.linear(P, ldxs=1, **x), True) >= 4 * 16 * 2
    assert P.ffn_workspace(R.ffn(P, ldxs=1, **x)) >= 4 * 16 * 2
    assert P.ffn_workspace(R.ffn(P, ldxs=1, **x), True) >= 4 * 16 * 2
    for bad in (dict(x=0), dict(ldx=15), dict(ldxs=0)):                               # the other checks stand
        R.refused(P, P.linear_forward, R.linear(P, **{**dict(ldxs=1), **x, **bad}))
        R.refused(P, P.ffn_backward, R.ffn(P, **{**dict(ldxs=1), **x, **bad}))
