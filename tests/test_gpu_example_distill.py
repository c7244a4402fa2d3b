"""The distillation example learns: its loss falls below two thirds of the first one's."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def test_the_student_learns():
    import distill_student
    history = distill_student.train()
    assert history[-1][0] < history[0][0] * 2 / 3
    assert history[-1][1] > history[0][1] + 0.1
