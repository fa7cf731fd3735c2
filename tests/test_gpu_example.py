"""The operators together as a model uses them: examples/hybrid_layers.py learns, and serves what it computes as a whole."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_hybrid_layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_layers.py")
    spec = importlib.util.spec_from_file_location("hybrid_layers", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, off, apart = m.main()
    assert losses[-1] < 0.8 * losses[0]
    # bf16 activations: each of the two layers rounds at every operator (2^-9 of a value, about ten of them in a row)
    assert off < 2e-2 and apart < 2e-2
