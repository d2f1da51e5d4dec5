"""The example that runs the recurrent block's operators together: it learns, and the samplers' 8-bit steps
answer as the trained network does. The cues have 6 standard normal columns, so answering zeros is off by 6
in the mean square; a network that cannot remember does no better."""
import pytest

from .helpers import log

pytestmark = pytest.mark.gpu


def test_history_policy_learns_and_serves():
    from examples import history_policy
    first, last, served = history_policy.run(steps=150, log=log)
    assert first > 6.0 * 0.5
    assert last < 2.0, last
    assert served < 2.0, served
