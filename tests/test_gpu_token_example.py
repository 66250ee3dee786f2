"""The example that runs the token operators together: it learns, and one token at a time gives what it learned."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_token_stage_learns_a_permutation():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_stage as T
    model, behind, losses = T.train(verbose=False)
    assert 5.5 < losses[0] < 9.0 and losses[-1] < 0.1, (losses[0], losses[-1])       # ln 512 = 6.2 and the spread of untrained logits
    got, at = T.follow(model, 3, 20), 3
    for t in got:
        at = int(behind[at])
        assert t == at
