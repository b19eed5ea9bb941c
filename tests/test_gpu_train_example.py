"""The training example: the distance transforms and the training operators in one loop."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_loss_falls():
    import torch
    spec = importlib.util.spec_from_file_location("train_marks", os.path.join(ROOT, "examples", "train_marks.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    history, right, network = module.main(["--steps", "40", "--batch", "4", "--size", "64", "--quiet"])
    # a fair coin's loss is 0.693; both tables have learned something
    assert history[0] > 0.5
    assert sum(history[-5:]) / 5 < 0.35
    assert right > 0.9
    for table in (network.position, network.prior):
        assert torch.isfinite(table).all() and float(table.detach().abs().max()) > 0.01
