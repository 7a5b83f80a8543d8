"""The example that trains and serves bags of attending rows."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def test_trains_and_serves():
    import sequence_bags as ex
    gen = torch.Generator().manual_seed(3)
    model = ex.Model("cuda", gen)
    losses = ex.train(model, 256, 40, gen)
    # a prediction that knows nothing has log(16); the class of the newest item tells all
    assert all(math.isfinite(x) for x in losses)
    assert losses[-1] < losses[0] and losses[-1] < math.log(ex.CLASSES)
    assert float(model.bias.abs().max()) > 0
    # both ways are fp32 over the same keys; scores of up to S err by (DIM + 2) 2^-23 S each, so
    # the weights by twice that relatively: 9e-5 for scores up to 20
    diff, size = ex.serve(model, 64, 5, gen)
    assert diff <= 1e-4 * size
