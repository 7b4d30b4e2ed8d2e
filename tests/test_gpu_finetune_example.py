"""The operators together, as the example uses them: a coded layer's adapter and weights learn, and requests with
different adapters are served in one call."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_adapter_learns_and_serves():
    import finetune_coded_layer as ex
    losses, A, B = ex.train_adapter()
    assert losses[-1] < 0.5 * losses[0]
    base, y, ids = ex.serve(A, B)
    changed = (y != base).any(dim=1)
    assert torch.equal(changed, ids == 0)                 # the trained adapter acts; the zero one and none leave the product alone


def test_weights_learn():
    import finetune_coded_layer as ex
    losses = ex.train_weights()
    assert losses[-1] < 0.1 * losses[0]
