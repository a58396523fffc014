"""The streaming example refuses, before it needs a GPU, more steps than its sequences have positions."""
import os
import sys

import pytest

pytest.importorskip("torch")


def test_more_steps_than_positions_are_refused():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import streaming
    with pytest.raises(ValueError):
        streaming.generate(steps=streaming.CONTEXT - streaming.PROMPT + 1)
