"""The example that samples, scores, and learns by the library's calls alone."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("kind", ["policy", "pref"])
def test_rewards_rise(example, kind):
    model = example.Model(seed=1)
    rounds = [example.learn(model, kind) for _ in range(30)]
    first = rounds[0]
    # The model that sampled and the model that is scored are one: what is left are the roundings of hidden states and
    # logits to bf16 (logits of standard deviation 1, up to about 5: 2^-9 of it each, a few of them together).
    assert all(r["drift"] < 0.1 for r in rounds)
    # before the first update the model is its reference
    assert abs(first["losses"][0] - math.log(2)) < 1e-3 if kind == "pref" else abs(first["losses"][0]) < 1.0
    assert all(math.isfinite(x) for r in rounds for x in r["losses"] + [r["norm"]])
    # the second update's loss, on the same answers: a step descends while the model is near its reference (further out
    # the divergence's exponential of a rare token may rise more than the rest falls)
    assert all(r["losses"][1] < r["losses"][0] for r in rounds[:5])
    mean = [sum(r["reward"] for r in part) / 5 for part in (rounds[:5], rounds[-5:])]
    assert mean[1] > mean[0] + 0.02
