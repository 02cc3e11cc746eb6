"""The sequence operators together with the regression, as a user's program has them: examples/sequence_regression.py."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_layer_regression_and_single_tokens(lib):
    spec = importlib.util.spec_from_file_location("sequence_regression", os.path.join(ROOT, "examples", "sequence_regression.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    out = m.main()
    assert out["losses"][-1] < 0.25 * out["losses"][0]           # the gradients lead downhill
    assert np.isfinite(out["nll"]).all() and out["nll"][-1] < out["nll"][0]
    assert out["rmse"][1] < 0.5 * out["spread"]                  # the prediction says something about unseen sequences
    assert out["apart"] < 64 * 2.0 ** -24                        # single tokens give what the whole prompt gives
