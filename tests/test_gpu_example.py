"""The example that runs look-up, first layer, backward, clipping and row writes together."""
import importlib.util
import os

import numpy as np
import pytest

from tests import lowbit_reference as ref

pytestmark = pytest.mark.gpu


def test_finetuning_example_learns_and_serves_what_it_learnt():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "finetune_step.py")
    spec = importlib.util.spec_from_file_location("finetune_step", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses, norms, master, served = ex.main(steps=8, verbose=False)
    assert np.isfinite(losses).all() and losses[-1] < 0.9 * losses[0]
    for t, q in zip(master, served):  # the served rows are the quantised master rows, bit for bit
        assert np.array_equal(q.cpu().numpy(), ref.mx4_rows(t.double().cpu().numpy()))
