"""The routed products together, as a program uses them: the example's training step against autograd, its decoding step, its sparse product."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("sizes", [(), (33, 72, 40, 5, 3), (700, 128, 130, 16, 4)])
def test_example(sizes):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("experts_block", os.path.join(ROOT, "examples", "experts_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # three products one after the other in single precision, each off by at most (c + 1) * 2^-24 of its magnitudes, both sides: relative to the
    # norm about sqrt(c) * 2^-24 each, under 2e-6 for c up to 700
    assert example.main(*sizes) < 1e-5
