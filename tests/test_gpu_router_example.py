"""The router's training loop (examples/train_router.py): balance loss, compressed exchange, norm and AdamW together."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("train_router", os.path.join(ROOT, "examples", "train_router.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def mean_of_last(history, column):
    return sum(h[column] for h in history[-10:]) / 10


@pytest.mark.parametrize("bits", [8, 32])
def test_the_balance_loss_spreads_the_load(example, bits):
    with_loss, without = (example.train(steps=60, alpha=alpha, state_bits=bits) for alpha in (1.0, 0.0))
    assert all(0.99 < h[0] for h in with_loss)                               # 1 where the load is balanced, more elsewhere
    assert mean_of_last(with_loss, 0) < mean_of_last(without, 0) - 0.1
    assert mean_of_last(with_loss, 1) < mean_of_last(without, 1)
    assert mean_of_last(without, 2) < without[0][2]                          # and the task is learnt: its gradient falls


def test_states_in_8_bits_train_as_those_in_32(example):
    a, b = (example.train(steps=60, alpha=0.5, state_bits=bits) for bits in (8, 32))
    assert abs(mean_of_last(a, 0) - mean_of_last(b, 0)) < 0.05 * mean_of_last(b, 0)


def test_the_same_seed_gives_the_same_run(example):
    assert example.train(steps=5, seed=3) == example.train(steps=5, seed=3)
