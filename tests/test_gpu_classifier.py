"""The classifier example: trained with the operators, it learns, and its answers in
8-bit integers are its answers."""

import math

import pytest

from .gpu_run import note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [{}, {"steps": 25, "batch": 333, "inputs": 129, "hidden": 77, "classes": 5, "seed": 3}])
def test_classifier_learns_and_answers(kw):
    from paper_1902_06714_amd import classifier
    note(f"classifier {kw}")
    r = classifier.run(**kw)
    classes = kw.get("classes", 10)
    # no weights at first: every class is as likely
    assert abs(r["first_loss"] - math.log(classes)) < 1e-4
    assert r["last_loss"] < 0.5 * r["first_loss"]
    assert r["accuracy"] > 0.8
    # 8 bits move a logit by about a hundredth of its spread
    assert abs(r["accuracy_8bit"] - r["accuracy"]) < 0.02
    assert 0.0 < r["entropy"] < math.log(classes)
