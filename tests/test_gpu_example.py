"""The training-and-serving example runs, learns, and serves what it learned."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_train_and_serve():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_serve.py")
    spec = importlib.util.spec_from_file_location("train_and_serve", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, one, few = example.main(60)
    assert losses[-1] < 0.7 * losses[0], losses
    # the batch path rounds its hidden activations to bf16, the one for few tokens keeps more
    assert one <= 1e-2 and few <= 1e-2, (one, few)
