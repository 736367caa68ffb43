"""The distillation example: lists, loss and gradient, sparsified update and
verification run together, and the student gets better at both measures."""
import importlib.util
import os

import pytest

from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "distill_draft.py")


def test_student_learns_and_drafts_are_accepted():
    need_gpu()
    spec = importlib.util.spec_from_file_location("distill_draft", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    announce("distill_draft example")
    losses, accepted = example.train(steps=100, rows=512, words=2048, report=lambda *_: None)
    assert losses[-1] < 0.5 * losses[0]
    assert accepted[-1] > accepted[0] + 0.5
