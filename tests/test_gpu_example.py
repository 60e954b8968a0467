"""The example trains, and gives the same a token at a time as over a whole sequence.

Tolerances: logits are sums of bfloat16 products through two layers, each of whose some ten roundings of 2^-9 the two ways take
differently: 5e-2 of their 2-norm.  A state is a sum of products of such inputs: the same.  The loss of guessing is log 64 = 4.2; a
model that has learned which four tokens may come next is at log 4 = 1.4, below half of it."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_gated_linear_attention():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_linear_attention.py")
    spec = importlib.util.spec_from_file_location("gated_linear_attention", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, apart, states_apart = example.main(steps=150, say=lambda line: print(line, flush=True))
    assert losses[0] > 3.5 and losses[-1] < 2.1, losses[::10]
    assert apart < 5e-2 and states_apart < 5e-2
