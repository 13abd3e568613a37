"""The example that trains through the codes runs and learns."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_finetune_quantized():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("finetune_quantized", os.path.join(ROOT, "examples", "finetune_quantized.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(steps=30)
    assert losses[-1] < 0.7 * losses[0]
