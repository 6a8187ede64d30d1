"""The operators together, as the learning explorer of examples/ uses them."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
from examples import policy_explorer  # noqa: E402


def test_policy_explorer_learns_and_repeats():
    """The draws' mean measurement rises from that of the accepted pool (about
    -1.3) towards 0, and the same seed gives the same rounds."""
    a = policy_explorer.run(rounds=40)
    assert sum(a[-5:]) / 5 > sum(a[:5]) / 5 + 0.3
    assert policy_explorer.run(rounds=40) == a
