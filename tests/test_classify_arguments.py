"""Arguments of the classifier that are refused before anything is computed; no
GPU."""
from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import pytest

from paper_2410_23244_amd.bart import BartError
from paper_2410_23244_amd.classify import Classifier


@pytest.mark.parametrize("n,p,ny,nt,pt,kw", [
    (8, 2, 7, 3, 2, {}),                # fewer classes than observations: one would be dropped
    (8, 2, 9, 3, 2, {}), (8, 2, 8, 3, 1, {}), (8, 2, 8, 3, 3, {}),
    (8, 2, 8, 3, 2, dict(n_keep=0)),    # a mean over no sweep
    (8, 2, 8, 3, 2, dict(n_keep=-1)), (8, 2, 8, 3, 2, dict(n_burn=-1))])
def test_observations_that_do_not_fit_together(n, p, ny, nt, pt, kw):
    with pytest.raises(BartError):
        Classifier().fit(np.zeros((n, p)), np.arange(ny) % 2, np.zeros((nt, pt)), **kw)


@pytest.mark.parametrize("X,X_test", [(np.zeros(4), np.zeros((1, 1))),
                                      (np.zeros((4, 1)), np.zeros(1)),
                                      (np.zeros((4, 1, 1)), np.zeros((1, 1, 1)))])
def test_observations_that_are_no_matrix(X, X_test):
    with pytest.raises(BartError):
        Classifier().fit(X, np.arange(4) % 2, X_test)


@pytest.mark.parametrize("y", [[0.0, 1.7, 2.0], [0, 1], [[0, 1, 2]]])
def test_classes_to_score_that_are_none(y):
    """A class of 1.7 would become 1."""
    f = Classifier()
    f.n_class, f.scores = 3, SimpleNamespace(shape=(1, 3, 3), device="cpu")
    f.calibration = SimpleNamespace(answer=lambda *a, **k: None)
    with pytest.raises(BartError):
        f.answer(y)
    assert f.answer([0, -1, 3]) is None     # no class, and one that was not fitted
