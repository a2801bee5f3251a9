"""GPU: the example that fits output layers to given embeddings learns. Targets
have unit mean square, so a map that knows nothing of them errs by about 1 (and
the random initial one by about 2); 40 steps of the fit must at least halve the
first error, in either dtype, and give the same numbers again."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "fit_output_layers.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("fit_output_layers", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fit_learns(example, dtype):
    losses = example.fit(steps=40, dtype=dtype)
    assert len(losses) == 41
    assert losses[-1] < 0.5 * losses[0], losses
    if dtype == torch.float32:
        assert example.fit(steps=3, dtype=dtype)[:1] == losses[:1]
